// Row operators over logits: log probabilities of given columns with the
// row's entropy and its best columns, and the distillation loss with its
// gradient (the training paragraph of Section 2 follows labels; these follow
// scores).
//
// Both rest on one row statistic.  With c = log2(e) / tau and a reference b, a
// whole number near max(x) c, e_v = 2^(x_v c - b): a fused multiply-add whose
// only rounding is that of the small exponent, so rows far from 0 lose
// nothing, and sums with different references join by exact powers of two.
// Then S = sum e_v, log2 q_v = x_v c - b - log2 S, and the entropy is
// log S - (sum e_v (x_v c - b)) ln 2 / S: every term has one sign.  Where
// max(x) c passes 1e37 (rows masked throughout with the lowest value) two
// different logits lie so far apart that e_v is 1 at the maximum, else 0.
//
// A workgroup holds its piece of a row in registers, so a row is read once
// whatever is computed from it: maximum, sums, the best columns, and in the
// distillation's fused form the gradient.  A thread adds at most 128 powers
// in fp32; everything across threads is fp64 in a fixed order.  Rows longer
// than a workgroup holds, and rows too few to fill the GPU, are cut into at
// most 64 chunks whose results a second launch joins.
#include <algorithm>
#include <cmath>

#include "rows_device.h"

namespace ifvs {

namespace {

constexpr double kLn2 = 0.69314718055994530942;
constexpr float kExpFloor = -200.0f;            // 2^-200 is 0 in fp32
constexpr float kHuge = 1e37f;
constexpr int kMaxChunks = 64;                  // one per lane of the joining wavefront
constexpr int64_t kMaxGrid = 1 << 22;           // workgroups of one launch
constexpr int kListCap = 1024;                  // candidate columns a workgroup collects for its best
constexpr int kGroups = 64;                     // thread groups whose maxima give the collecting threshold
static_assert(kGroups >= 32, "the threshold is the n_top-th largest group maximum");

__device__ __forceinline__ float exp2_fast(float z) { return __builtin_amdgcn_exp2f(z); }

__device__ __forceinline__ double times_pow2(double v, double e) {
  return ldexp(v, static_cast<int>(fmax(fmin(e, 4000.0), -4000.0)));
}

__device__ __forceinline__ int row_cols(const int32_t* n_valid, int64_t i, int64_t cols) {
  if (!n_valid) return static_cast<int>(cols);
  const int64_t v = n_valid[i];
  return static_cast<int>(v < 0 ? 0 : (v < cols ? v : cols));
}

// Sums relative to 2^origin.  sum is NaN where the row has no finite
// distribution (a NaN or +inf logit), 0 where nothing lies above -inf.
struct Stat {
  double origin, sum, wsum;
};

__device__ __forceinline__ Stat join(const Stat& a, const Stat& b) {
  if (b.sum == 0.0) return a;
  if (a.sum == 0.0) return b;
  const double o = fmax(a.origin, b.origin);
  const double da = a.origin - o, db = b.origin - o;
  const double sa = times_pow2(a.sum, da), sb = times_pow2(b.sum, db);
  // sum e (z + d) = wsum + d sum; a vanished part adds nothing
  const double wa = sa == 0.0 ? 0.0 : times_pow2(a.wsum, da) + da * sa;
  const double wb = sb == 0.0 ? 0.0 : times_pow2(b.wsum, db) + db * sb;
  return {o, sa + sb, wa + wb};
}

// The sums of a wavefront's elements, in every lane.
template <bool kEntropy, typename T, int kThreads, int kVecs>
__device__ __forceinline__ Stat wave_stat(RowTile<T, kThreads, kVecs>& tile, float mx, float c) {
  constexpr int kE = Elem<T>::kPerVec;
  tile.forget_unpacked();
  float sum = 0.0f, wsum = 0.0f;
  double origin = 0.0;
  const float b = mx == -INFINITY ? 0.0f : rintf(mx * c);
  if (fabsf(b) < kHuge) {
    origin = b;
    auto add = [&](float x) {
      const float z = __fmaf_rn(x, c, -b);
      const float e = exp2_fast(z);
      sum += e;
      if constexpr (kEntropy) wsum = __fmaf_rn(e, fmaxf(z, kExpFloor), wsum);
    };
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (tile.has(i)) {
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
#pragma unroll
        for (int j = 0; j < kE; ++j) add(f[j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    add(tile.tail);
  } else {
    origin = static_cast<double>(mx) * c;
    auto add = [&](float x) { sum += x == mx ? 1.0f : (isnan(x) || x == INFINITY ? NAN : 0.0f); };
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (tile.has(i)) {
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
#pragma unroll
        for (int j = 0; j < kE; ++j) add(f[j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    add(tile.tail);
    if (mx == INFINITY) sum = NAN;
  }
  return {origin, wave_add(static_cast<double>(sum)), kEntropy ? wave_add(static_cast<double>(wsum)) : 0.0};
}

// ------------------------------------------------------------ best columns
// A column as a whole number: larger is better, ties to the lower column; 0 is
// none.  +0 and -0 are equal.
__device__ __forceinline__ uint64_t column_key(float x, int column) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  const uint32_t ordered = (b >> 31) ? ~b : (b | 0x80000000u);
  return (static_cast<uint64_t>(ordered) << 32) | static_cast<uint32_t>(~column);
}
__device__ __forceinline__ int key_column(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t o = static_cast<uint32_t>(key >> 32);
  return __uint_as_float((o >> 31) ? (o & 0x7FFFFFFFu) : ~o);
}

template <int kCtrl>
__device__ __forceinline__ uint64_t key_perm(uint64_t v) {
  const uint32_t lo = __builtin_amdgcn_mov_dpp(static_cast<int>(v), kCtrl, 0xF, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp(static_cast<int>(v >> 32), kCtrl, 0xF, 0xF, true);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
__device__ __forceinline__ uint64_t key_lane(uint64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
__device__ __forceinline__ uint64_t key_max(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t wave_key_max(uint64_t v) {
  v = key_max(v, key_perm<kPermXor1>(v));
  v = key_max(v, key_perm<kPermXor2>(v));
  v = key_max(v, key_perm<kPermHalfMirror>(v));
  v = key_max(v, key_perm<kPermMirror>(v));
  return key_max(key_max(key_lane(v, 0), key_lane(v, 16)), key_max(key_lane(v, 32), key_lane(v, 48)));
}

// The nth largest (1-based) of a wavefront's 64 values.
__device__ __forceinline__ float nth_largest(float v, int nth) {
  int greater = 0;
#pragma unroll
  for (int s = 0; s < 64; ++s) greater += lane_of(v, s) > v ? 1 : 0;
  return -wave_max(greater < nth ? -v : -INFINITY);
}

// Shared memory of best_columns.
struct BestLds {
  uint64_t list[kListCap];
  uint64_t round[16];
  float group[kGroups];
  float threshold;
  int count;
};

// The tile's n_top best columns (plus first_column) as keys in descending
// order, 0 past the last: emit(rank, key) once per rank, by some thread.
// Every element at least as large as the n_top-th largest of the 64 group
// maxima is collected (n_top of them at least, few more unless the row is
// full of ties) and ranked by counting.  More than the list holds: one round
// over the tile's len elements at x per rank.
template <typename T, int kThreads, int kVecs, typename Emit>
__device__ __forceinline__ void best_columns(RowTile<T, kThreads, kVecs>& tile, float thread_max,
                                             const T* x, int len, int first_column, int n_top, BestLds& s, Emit emit) {
  const int tid = threadIdx.x;
  constexpr int kPer = kThreads / kGroups;
  float g = thread_max;
  if constexpr (kPer == 4) g = quad_max(g);
  if constexpr (kPer == 16) g = sixteen_max(g);
  static_assert(kPer == 1 || kPer == 4 || kPer == 16, "group of lanes");
  if (tid % kPer == 0) s.group[tid / kPer] = g;
  if (tid == 0) s.count = 0;
  group_sync<kThreads>();
  if (tid < 64) {
    const float t = nth_largest(s.group[tid], n_top);
    if (tid == 0) s.threshold = t;
  }
  group_sync<kThreads>();
  const float threshold = s.threshold;
  constexpr int kE = Elem<T>::kPerVec;
  if (thread_max >= threshold && thread_max > -INFINITY) {
    auto keep = [&](float x, int column) {
      if (x > -INFINITY) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kListCap) s.list[at] = column_key(x, first_column + column);
      }
    };
    tile.forget_unpacked();
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (tile.has(i)) {
        // a vector's hits as a mask, walked only where there are any
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < kE; ++j) hits |= f[j] >= threshold ? 1u << j : 0u;
        while (hits != 0) {
          const int j = __builtin_ctz(hits);
          hits &= hits - 1;
          float y = f[0];
#pragma unroll
          for (int o = 1; o < kE; ++o) y = j == o ? f[o] : y;
          keep(y, tile.column(i, j));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    if (tile.tail >= threshold) keep(tile.tail, tile.tail_column());
  }
  group_sync<kThreads>();
  const int m = s.count;
  if (m <= kListCap) {
    for (int e = tid; e < m; e += kThreads) {
      const uint64_t key = s.list[e];
      int rank = 0;
      for (int o = 0; o < m; ++o) rank += s.list[o] > key ? 1 : 0;
      if (rank < n_top) emit(rank, key);
    }
    for (int r = m + tid; r < n_top; r += kThreads) emit(r, 0);
  } else {
    uint64_t last = ~uint64_t{0};
    for (int r = 0; r < n_top; ++r) {
      uint64_t best = 0;
      for (int v = tid; v < len; v += kThreads) {
        const float f = elem_load(x + v);
        const uint64_t key = column_key(f, first_column + v);
        if (f > -INFINITY && key < last && key > best) best = key;
      }
      best = wave_key_max(best);
      if ((tid & 63) == 0) s.round[tid >> 6] = best;
      group_sync<kThreads>();
      for (int w = 0; w < kThreads / 64; ++w) best = key_max(best, s.round[w]);
      group_sync<kThreads>();
      if (tid == 0) emit(r, best);
      last = best;
    }
  }
  group_sync<kThreads>();
}

// -------------------------------------------------------- log probabilities
// What a row's outputs are computed from.
struct RowProb {
  double origin, log2_sum;      // kept apart: the origin may be 1e38
  double c;                     // the fp32 constant of the sums: x c is exact in 64 bits
  bool nan, empty;
  __device__ __forceinline__ RowProb(const Stat& st, float cc) {
    nan = isnan(st.sum);
    empty = st.sum == 0.0;
    origin = st.origin;
    log2_sum = log2(st.sum);
    c = cc;
  }
  __device__ __forceinline__ float logp(float x) const {
    if (nan) return NAN;
    if (empty) return -INFINITY;
    return static_cast<float>((static_cast<double>(x) * c - origin - log2_sum) * kLn2);
  }
  __device__ __forceinline__ float entropy(const Stat& st) const {
    if (nan) return NAN;
    if (empty) return 0.0f;
    return static_cast<float>((log2_sum - st.wsum / st.sum) * kLn2);
  }
};

template <typename T>
__device__ __forceinline__ void write_given(const LogProbArgs& a, int64_t row, const T* x, int len, const RowProb& p,
                                            int tid, int threads) {
  for (int g = tid; g < a.n_given; g += threads) {
    const int64_t v = a.given[row * a.n_given + g];
    a.given_out[row * a.n_given + g] = v >= 0 && v < len ? p.logp(elem_load(x + v)) : -INFINITY;
  }
}

// One workgroup per (row, chunk of `chunk` columns), items from item0 on.
// kWhole: chunks is 1 and the workgroup writes the row's outputs, else its
// statistics and best columns go to the workspace.
template <typename T, int kThreads, int kVecs, bool kWhole>
__global__ __launch_bounds__(kThreads, 4) void log_probs_tile_kernel(const LogProbArgs a, int64_t item0, int chunk,
                                                                     int chunks, Stat* stats, uint64_t* keys) {
  constexpr int kWaves = kThreads / 64;
  __shared__ BestLds s_best;
  __shared__ Stat s_stat[kWaves];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int64_t item = item0 + blockIdx.x;
  const int64_t row = kWhole ? item : item / chunks;
  const int first = kWhole ? 0 : static_cast<int>(item - row * chunks) * chunk;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  const int len = row_cols(a.n_valid, row, a.cols);
  const int mine = kWhole ? len : max(0, min(chunk, len - first));
  RowTile<T, kThreads, kVecs> tile;
  tile.load(x + first, mine);
  const float tmax = tile.thread_max();
  Stat st = wave_stat<true>(tile, wave_max(tmax), static_cast<float>(a.c));
  if constexpr (kWaves > 1) {
    if ((tid & 63) == 0) s_stat[wave] = st;
    __syncthreads();
    st = s_stat[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) st = join(st, s_stat[w]);
  }
  if constexpr (!kWhole) {
    if (tid == 0) stats[item] = st;
    if (a.n_top > 0) {
      uint64_t* out = keys + item * a.n_top;
      best_columns(tile, tmax, x + first, mine, first, a.n_top, s_best, [&](int r, uint64_t key) { out[r] = key; });
    }
  } else {
    const RowProb p(st, static_cast<float>(a.c));
    if (tid == 0 && a.entropy_out) a.entropy_out[row] = p.entropy(st);
    write_given(a, row, x, len, p, tid, kThreads);
    if (a.n_top > 0) {
      int32_t* ids = a.top_ids_out + row * a.n_top;
      float* top = a.top_out + row * a.n_top;
      if (p.nan) {
        for (int r = tid; r < a.n_top; r += kThreads) {
          ids[r] = -1;
          top[r] = NAN;
        }
      } else {
        best_columns(tile, tmax, x, mine, 0, a.n_top, s_best, [&](int r, uint64_t key) {
          ids[r] = key ? key_column(key) : -1;
          top[r] = key ? p.logp(key_logit(key)) : -INFINITY;
        });
      }
    }
  }
}

// One wavefront per row joins its chunks (a lane each).
template <typename T>
__global__ __launch_bounds__(64) void log_probs_join_kernel(const LogProbArgs a, int64_t row0, int chunks,
                                                            const Stat* stats, const uint64_t* keys) {
  const int lane = threadIdx.x;
  const int64_t row = row0 + blockIdx.x;
  const Stat mine = lane < chunks ? stats[row * chunks + lane] : Stat{0.0, 0.0, 0.0};
  uint64_t head = 0;
  const uint64_t* list = keys + (row * chunks + (lane < chunks ? lane : 0)) * a.n_top;
  if (a.n_top > 0 && lane < chunks) head = list[0];
  Stat st{lane_of(mine.origin, 0), lane_of(mine.sum, 0), lane_of(mine.wsum, 0)};
  for (int j = 1; j < chunks; ++j)
    st = join(st, Stat{lane_of(mine.origin, j), lane_of(mine.sum, j), lane_of(mine.wsum, j)});
  const RowProb p(st, static_cast<float>(a.c));
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  if (lane == 0 && a.entropy_out) a.entropy_out[row] = p.entropy(st);
  write_given(a, row, x, row_cols(a.n_valid, row, a.cols), p, lane, 64);
  int at = 0;
  uint64_t won = 0;                                   // lane r: the key of rank r
  for (int r = 0; r < a.n_top; ++r) {
    const uint64_t best = p.nan ? 0 : wave_key_max(head);
    if (best != 0 && head == best) {
      ++at;
      head = at < a.n_top ? list[at] : 0;
    }
    if (lane == r) won = best;
  }
  if (lane < a.n_top) {
    a.top_ids_out[row * a.n_top + lane] = won ? key_column(won) : -1;
    a.top_out[row * a.n_top + lane] = won ? p.logp(key_logit(won)) : (p.nan ? NAN : -INFINITY);
  }
}

// ------------------------------------------------------------- distillation
// One workgroup per row.  The teacher's probabilities are held in LDS; a
// column's teacher probability is looked up among the slots.
constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;

struct RowRef {
  float c;       // log2(e) / tau
  float shift;   // subtracted before the product (0, or the maximum)
  float b;       // subtracted after it
  __device__ __forceinline__ float exponent(float x) const { return __fmaf_rn(x - shift, c, -b); }
  __device__ __forceinline__ double exponent64(float x) const {
    return (static_cast<double>(x) - shift) * c - b;
  }
  // What an exponent is relative to: x c = exponent + origin.
  __device__ __forceinline__ double origin() const { return static_cast<double>(shift) * c + b; }
};

__device__ __forceinline__ RowRef row_ref(float mx, float c) {
  const float b = mx * c;
  if (fabsf(b) < 1e37f) return {c, 0.0f, b};
  return {c, mx, 0.0f};
}

template <int kWaves>
__device__ __forceinline__ double block_add(double v, double* s) {
  v = wave_add(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v += s[w];
  __syncthreads();
  return v;
}

template <int kWaves>
__device__ __forceinline__ float block_max(float v, double* s) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v = fmaxf(v, static_cast<float>(s[w]));
  __syncthreads();
  return v;
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void distill_kernel(const DistillArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  double* s_red = reinterpret_cast<double*>(smem);          // [kRowWaves]
  double* s_p = s_red + kRowWaves;                            // [n_teacher]
  int* s_id = reinterpret_cast<int*>(s_p + a.n_teacher);      // [n_teacher], -1 absent
  const int tid = threadIdx.x;
  const int64_t i = blockIdx.x;
  const T* x = static_cast<const T*>(a.logits) + i * a.ld;
  T* grad = a.grad_out ? static_cast<T*>(a.grad_out) + i * a.grad_ld : nullptr;
  const int cols = static_cast<int>(a.cols);
  const float weight = a.row_weight ? a.row_weight[i] : 1.0f;
  const int len = row_cols(a.n_valid, i, a.cols);
  auto skip = [&](float loss, float g) {
    if (tid == 0) a.loss_out[i] = loss;
    if (grad)
      for (int v = tid; v < cols; v += kRowThreads) grad[v] = elem_round<T>(v < len ? g : 0.0f);
  };
  if (weight == 0.0f) return skip(0.0f, 0.0f);

  // The teacher.
  const double inv_tau = 1.0 / static_cast<double>(a.tau);
  float tmax = -INFINITY;
  double bad = 0.0, present = 0.0;
  for (int k = tid; k < a.n_teacher; k += kRowThreads) {
    const int id = a.teacher_ids[i * a.n_teacher + k];
    const float t = a.teacher_logits[i * a.n_teacher + k];
    const bool there = id >= 0 && id < len;
    s_id[k] = there ? id : -1;
    if (!there) continue;
    present += 1.0;
    if (isnan(t) || t == INFINITY) bad = 1.0;
    tmax = fmaxf(tmax, t);
  }
  present = block_add<kRowWaves>(present, s_red);
  const bool rest = a.teacher_lse != nullptr;
  double lse;
  if (rest) {
    lse = a.teacher_lse[i];
  } else {
    tmax = block_max<kRowWaves>(tmax, s_red);
    double sum = 0.0;
    for (int k = tid; k < a.n_teacher; k += kRowThreads)
      if (s_id[k] >= 0) sum += exp((static_cast<double>(a.teacher_logits[i * a.n_teacher + k]) - tmax) * inv_tau);
    sum = block_add<kRowWaves>(sum, s_red);
    lse = static_cast<double>(tmax) * inv_tau + log(sum);
    if (present > 0.0 && tmax == -INFINITY) bad = 1.0;
  }
  double psum = 0.0;
  for (int k = tid; k < a.n_teacher; k += kRowThreads) {
    const double p =
        s_id[k] < 0 ? 0.0 : exp(static_cast<double>(a.teacher_logits[i * a.n_teacher + k]) * inv_tau - lse);
    s_p[k] = p;
    psum += p;
  }
  psum = block_add<kRowWaves>(psum, s_red);
  const double p_rest = rest ? fmax(0.0, 1.0 - psum) : 0.0;

  // The student: all columns, and those that no slot names.
  auto named = [&](int v) {
    for (int k = 0; k < a.n_teacher; ++k)
      if (s_id[k] == v) return true;
    return false;
  };
  float mx = -INFINITY, mx_rest = -INFINITY;
  for (int v = tid; v < len; v += kRowThreads) {
    const float f = elem_load(x + v);
    if (isnan(f) || f == INFINITY) bad = 1.0;
    mx = fmaxf(mx, f);
    if (rest && !named(v)) mx_rest = fmaxf(mx_rest, f);
  }
  bad = block_add<kRowWaves>(bad, s_red);
  mx = block_max<kRowWaves>(mx, s_red);
  mx_rest = block_max<kRowWaves>(mx_rest, s_red);
  if (bad > 0.0) return skip(NAN, NAN);
  if (mx == -INFINITY || (!rest && present == 0.0)) return skip(0.0f, 0.0f);
  const RowRef ref = row_ref(mx, static_cast<float>(a.c)), ref_rest = row_ref(mx_rest, static_cast<float>(a.c));
  float sum = 0.0f, sum_rest = 0.0f;
  for (int v = tid; v < len; v += kRowThreads) {
    const float f = elem_load(x + v);
    sum += exp2f(ref.exponent(f));
    if (rest && mx_rest > -INFINITY && !named(v)) sum_rest += exp2f(ref_rest.exponent(f));
  }
  const double S = block_add<kRowWaves>(sum, s_red);
  const double S_rest = block_add<kRowWaves>(sum_rest, s_red);
  const double log2S = log2(S);

  double loss = 0.0;
  for (int k = tid; k < a.n_teacher; k += kRowThreads)
    if (s_id[k] >= 0 && s_p[k] > 0.0)
      loss += s_p[k] * (log(s_p[k]) - (ref.exponent64(elem_load(x + s_id[k])) - log2S) * kLn2);
  loss = block_add<kRowWaves>(loss, s_red);
  // log Q of the rest, relative to the row's own sum.
  const double logQ = S_rest > 0.0 ? (ref_rest.origin() - ref.origin() + log2(S_rest) - log2S) * kLn2 : -INFINITY;
  if (p_rest > 0.0 && S_rest > 0.0) loss += p_rest * (log(p_rest) - logQ);
  if (tid == 0) a.loss_out[i] = static_cast<float>(loss * (static_cast<double>(a.tau) * a.tau));
  if (!grad) return;
  __syncthreads();                       // the listed logits are read: in place from here on
  const double up = static_cast<double>(weight) * a.tau;
  const double keep = rest && S_rest > 0.0 ? 1.0 - p_rest * exp(-logQ) : 1.0;
  for (int v = tid; v < cols; v += kRowThreads) {
    double g = 0.0;
    if (v < len) {
      const double q = exp2(ref.exponent64(elem_load(x + v)) - log2S);
      double p = 0.0;
      bool is_named = false;
      for (int k = 0; k < a.n_teacher; ++k)
        if (s_id[k] == v) {
          p += s_p[k];
          is_named = true;
        }
      g = up * (rest && !is_named ? q * keep : q - p);
    }
    grad[v] = elem_round<T>(static_cast<float>(g));
  }
}

}  // namespace

// How a row's columns go over workgroups: threads and vectors per thread of a
// workgroup, columns per chunk, chunks per row.
struct RowPlan {
  int threads, vecs, chunk, chunks;
};

// A row goes to the smallest workgroup that holds it, a wavefront up to 512
// vectors; longer rows, and rows too few to give every CU a workgroup, to
// chunks of 256-thread workgroups.  A chunk of fewer than 256 vectors would
// leave threads idle.
RowPlan log_probs_plan(int64_t n, int64_t cols, int per_vec) {
  constexpr int64_t kFill = 512;               // workgroups: two per CU
  const int64_t vecs = (cols + per_vec - 1) / per_vec;
  if (vecs <= 128) return {64, 2, static_cast<int>(cols), 1};
  if (vecs <= 512) return {64, 8, static_cast<int>(cols), 1};
  int64_t chunks = (vecs + 4095) / 4096;
  if (n * chunks < kFill) chunks = std::min<int64_t>({(kFill + n - 1) / n, (vecs + 255) / 256, kMaxChunks});
  if (chunks == 1) return {256, vecs <= 2048 ? 8 : 16, static_cast<int>(cols), 1};
  const int64_t chunk = (vecs + chunks - 1) / chunks;
  return {256, chunk <= 2048 ? 8 : 16, static_cast<int>(chunk * per_vec),
          static_cast<int>((vecs + chunk - 1) / chunk)};
}

int64_t log_probs_workspace_bytes(int64_t n, int64_t cols, int n_top) {
  int64_t most = 0;                            // the element type is not known here
  for (int per_vec : {4, 8}) {
    const RowPlan p = log_probs_plan(n, cols, per_vec);
    if (n > 0 && p.chunks > 1) most = std::max<int64_t>(most, n * p.chunks);
  }
  return most * static_cast<int64_t>(sizeof(Stat) + 8 * n_top);
}
int64_t distill_workspace_bytes(int64_t, int64_t) { return 0; }

// Launches fn(first item, items) over slices that a grid can count.
template <typename F>
hipError_t in_slices(int64_t items, F&& fn) {
  for (int64_t at = 0; at < items; at += kMaxGrid) {
    fn(at, static_cast<unsigned>(std::min(items - at, kMaxGrid)));
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t log_probs_typed(const LogProbArgs& a, hipStream_t s) {
  const RowPlan p = log_probs_plan(a.n, a.cols, Elem<T>::kPerVec);
  const int64_t items = a.n * p.chunks;
  Stat* stats = static_cast<Stat*>(a.workspace);
  uint64_t* keys = reinterpret_cast<uint64_t*>(stats + items);
  const hipError_t e = in_slices(items, [&](int64_t at, unsigned grid) {
    if (p.chunks > 1) {
      if (p.vecs == 8) log_probs_tile_kernel<T, 256, 8, false><<<grid, 256, 0, s>>>(a, at, p.chunk, p.chunks, stats, keys);
      else log_probs_tile_kernel<T, 256, 16, false><<<grid, 256, 0, s>>>(a, at, p.chunk, p.chunks, stats, keys);
    } else if (p.threads == 64) {
      if (p.vecs == 2) log_probs_tile_kernel<T, 64, 2, true><<<grid, 64, 0, s>>>(a, at, p.chunk, 1, stats, keys);
      else log_probs_tile_kernel<T, 64, 8, true><<<grid, 64, 0, s>>>(a, at, p.chunk, 1, stats, keys);
    } else {
      if (p.vecs == 8) log_probs_tile_kernel<T, 256, 8, true><<<grid, 256, 0, s>>>(a, at, p.chunk, 1, stats, keys);
      else log_probs_tile_kernel<T, 256, 16, true><<<grid, 256, 0, s>>>(a, at, p.chunk, 1, stats, keys);
    }
  });
  if (e != hipSuccess || p.chunks == 1) return e;
  return in_slices(a.n, [&](int64_t at, unsigned grid) {
    log_probs_join_kernel<T><<<grid, 64, 0, s>>>(a, at, p.chunks, stats, keys);
  });
}

hipError_t launch_log_probs(const LogProbArgs& a, hipStream_t s) {
  switch (a.n == 0 ? -1 : a.dtype) {
    case -1: return hipSuccess;
    case kElemF32: return log_probs_typed<float>(a, s);
    case kElemF16: return log_probs_typed<_Float16>(a, s);
    default: return log_probs_typed<__bf16>(a, s);
  }
}

hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(a.n)), block(kRowThreads);
  const size_t lds = sizeof(double) * kRowWaves + (sizeof(double) + sizeof(int)) * a.n_teacher;
  switch (a.dtype) {
    case kElemF32: distill_kernel<float><<<grid, block, lds, s>>>(a); break;
    case kElemF16: distill_kernel<_Float16><<<grid, block, lds, s>>>(a); break;
    default: distill_kernel<__bf16><<<grid, block, lds, s>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace ifvs
