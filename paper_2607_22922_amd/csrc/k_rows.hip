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
// log S - (sum e_v (x_v c - b)) ln 2 / S: every term has one sign.  From
// |max(x) c| = 2^24 on (columns masked throughout with a finite value, a small
// tau) fp32 does not hold every whole number: b and the exponents are computed
// in 64 bits there, which a wavefront decides for its columns.
//
// A workgroup holds its piece of a row in registers, so a row is read once
// whatever is computed from it: maximum, sums, the best columns, and in the
// distillation's fused form the gradient.  A thread adds at most 128 powers
// in fp32; everything across threads is fp64 in a fixed order.  Rows longer
// than a workgroup holds, and rows too few to fill the GPU, are cut into at
// most 64 chunks whose results a second launch joins.
#include <algorithm>
#include <cmath>

#include "ifvs.h"
#include "rows_device.h"

namespace ifvs {

namespace {

constexpr double kLn2 = 0.69314718055994530942;
constexpr float kExpFloor = -200.0f;            // 2^-200 is 0 in fp32
constexpr float kFar = 16777216.0f;             // 2^24: fp32 holds every whole number below
constexpr int kMaxChunks = 64;                  // one per lane of the joining wavefront; 2^20 fp32 columns are 64
static_assert(IFVS_MAX_COLS / 4 <= kMaxChunks * 4096, "chunks of 4096 vectors");
constexpr int64_t kMaxGrid = 1 << 22;           // workgroups of one launch
constexpr int kListCap = 1024;                  // candidate columns a workgroup collects for its best
constexpr int kGroups = 64;                     // thread groups whose maxima give the collecting threshold
static_assert(kGroups >= 32, "the threshold is the n_top-th largest group maximum");

__device__ __forceinline__ float exp2_fast(float z) { return __builtin_amdgcn_exp2f(z); }

__device__ __forceinline__ double times_pow2(double v, double e) {
  return ldexp(v, static_cast<int>(fmax(fmin(e, 4000.0), -4000.0)));
}

// x c - origin for a whole origin near the maximum's x c, far from 0.  (Equal
// logits have equal products; where a product is rounded, past 2^53, others
// lie thousands of powers of two apart.)
__device__ __forceinline__ float far_exponent(float x, double c, double origin) {
  return static_cast<float>(static_cast<double>(x) * c - origin);
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

// Joins the sums that a wavefront's lanes hold (sum 0: none), in every lane.
__device__ __forceinline__ Stat join_lanes(const Stat& mine) {
  const bool any = mine.sum != 0.0;
  const double o = wave_max(any ? mine.origin : -INFINITY);
  const double d = any ? mine.origin - o : 0.0;
  const double sum = any ? times_pow2(mine.sum, d) : 0.0;
  const double wsum = sum == 0.0 ? 0.0 : times_pow2(mine.wsum, d) + d * sum;
  return {o, wave_add(sum), wave_add(wsum)};
}

// The sums of a wavefront's elements, in every lane.
template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ Stat wave_stat(RowTile<T, kThreads, kVecs>& tile, float mx, float c) {
  constexpr int kE = Elem<T>::kPerVec;
  tile.forget_unpacked();
  float sum = 0.0f, wsum = 0.0f;
  const float b = mx == -INFINITY ? 0.0f : rintf(mx * c);
  double origin = b;
  auto add = [&](float z) {
    const float e = exp2_fast(z);
    sum += e;
    wsum = __fmaf_rn(e, fmaxf(z, kExpFloor), wsum);
  };
  if (fabsf(b) < kFar) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (tile.has(i)) {
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
#pragma unroll
        for (int j = 0; j < kE; ++j) add(__fmaf_rn(f[j], c, -b));
        __builtin_amdgcn_sched_barrier(0);
      }
    add(__fmaf_rn(tile.edge, c, -b));
  } else {
    const double wide = c;                          // its products with a logit are exact
    origin = rint(mx * wide);
    tile.each([&](float v, int) { add(far_exponent(v, wide, origin)); });
  }
  return {origin, wave_add(static_cast<double>(sum)), wave_add(static_cast<double>(wsum))};
}

// ------------------------------------------------------------ best columns
// Whole numbers in the order of the logits (+0 and -0 equal).
__device__ __forceinline__ uint32_t ordered_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return __uint_as_float((o >> 31) ? (o & 0x7FFFFFFFu) : ~o);
}

// A column as a whole number: larger is better, ties to the lower column; 0 is
// none.
__device__ __forceinline__ uint64_t column_key(float x, int column) {
  return (static_cast<uint64_t>(ordered_bits(x)) << 32) | static_cast<uint32_t>(~column);
}
__device__ __forceinline__ int key_column(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }
__device__ __forceinline__ float key_logit(uint64_t key) {
  return from_ordered(static_cast<uint32_t>(key >> 32));
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

// The nth largest (1-based) of a wavefront's 64 values, for 16-bit elements a
// value just below it.  A bisection over the bits that an element has, a
// comparison and a count of lanes each (64 comparisons with every lane's value
// cost three times the vector instructions; fewer bits than the element's
// would let rows far from 0 pass whole).
template <int kLowBit>
__device__ __forceinline__ float reached_by(float v, int nth) {
  const uint32_t key = ordered_bits(v);
  uint32_t cut = 0;
#pragma unroll
  for (int b = 31; b >= kLowBit; --b) {
    const uint32_t t = cut | (1u << b);
    if (__popcll(__ballot(key >= t)) >= nth) cut = t;
  }
  // below the keys of all numbers: everything reaches it
  return cut <= ordered_bits(-INFINITY) ? -INFINITY : from_ordered(cut);
}

// Shared memory of best_columns.
constexpr int kStaged = 8;                 // threads whose elements a wavefront lays out
template <int kThreads, int kVecs>
struct BestLds {
  Word4 stage[kThreads / 64][kStaged][kVecs];
  uint64_t list[kListCap];
  uint64_t round[kThreads / 64];
  float group[kGroups];
  int count;
};

// The tile's n_top best columns (plus first_column) as keys in descending
// order, 0 past the last: emit(rank, key) once per rank, by some thread.
// Every element at least as large as the n_top-th largest of the 64 group
// maxima is collected (n_top of them at least, few more unless the row is
// full of ties) and ranked by counting.  Few threads hold such an element: they
// lay their vectors out in LDS and their wavefront looks at them an element a
// lane (2048 rows of 50001 fp16 logits, 10 alternatives: 48 us, each thread
// looking at its own 54), except that in short tiles many holders look at their
// own each (4096 rows of 1000, 32 alternatives: 11 us against 18).  More than the
// list holds: collected again by key from memory, and where that is too much too,
// one round over the tile's len elements at x per rank.
template <typename T, int kThreads, int kVecs, typename Emit>
__device__ __forceinline__ void best_columns(RowTile<T, kThreads, kVecs>& tile, float thread_max,
                                             const T* x, int len, int first_column, int n_top,
                                             BestLds<kThreads, kVecs>& s, Emit emit) {
  constexpr int kE = Elem<T>::kPerVec;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int kPer = kThreads / kGroups;
  float g = thread_max;
  if constexpr (kPer == 4) g = quad_max(g);
  if constexpr (kPer == 16) g = sixteen_max(g);
  static_assert(kPer == 1 || kPer == 4 || kPer == 16, "group of lanes");
  if (tid % kPer == 0) s.group[tid / kPer] = g;
  if (tid == 0) s.count = 0;
  group_sync<kThreads>();
  const float threshold = reached_by<Elem<T>::kLowBit>(s.group[lane], n_top);
  auto keep = [&](float f, int column) {
    if (f >= threshold && f > -INFINITY) {
      const int at = atomicAdd(&s.count, 1);
      if (at < kListCap) s.list[at] = column_key(f, first_column + column);
    }
  };
  keep(tile.edge, tile.edge_column());
  uint64_t holders = __ballot(thread_max >= threshold && thread_max > -INFINITY);
  tile.forget_unpacked();
  if (kVecs > 8 || __popcll(holders) <= kStaged) {
    while (holders != 0) {
      const int mine = __popcll(holders & ((1ull << lane) - 1));
      if (((holders >> lane) & 1u) && mine < kStaged) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) s.stage[wave][mine][i] = tile.v[i];
      }
      group_sync<64>();
      for (int h = 0; h < kStaged && holders != 0; ++h, holders &= holders - 1) {
        const int owner = (tid & ~63) + __builtin_ctzll(holders);
        const T* staged = reinterpret_cast<const T*>(&s.stage[wave][h][0]);
#pragma unroll
        for (int e0 = 0; e0 < kVecs * kE; e0 += 64) {
          const int e = e0 + lane;
          if (kVecs * kE >= 64 || e < kVecs * kE)
            keep(static_cast<float>(staged[e]), tile.head + (e / kE * kThreads + owner) * kE + e % kE);
        }
      }
      group_sync<64>();
    }
  } else if ((holders >> lane) & 1u) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (tile.has(i)) {
        // a vector's elements are looked at only where its maximum is enough
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
        float most = f[0];
#pragma unroll
        for (int j = 1; j < kE; ++j) most = fmaxf(most, f[j]);
        if (most >= threshold) {
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
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  group_sync<kThreads>();
  int m = s.count;
  if (m > kListCap) {
    // A row full of equal logits: the same with keys, in which no two columns
    // are equal, from memory (the tile would cost every row registers).
    group_sync<kThreads>();
    uint64_t key = 0;
    if (thread_max > -INFINITY) {
      int lowest = 0x7FFFFFFF;
      tile.each_vector_from_memory(x, [&](float f, int column) {
        if (f == thread_max) lowest = min(lowest, column);
        return lowest == 0x7FFFFFFF;
      });
      key = column_key(thread_max, first_column + lowest);
    }
    s.list[tid] = key;
    if (tid == 0) s.count = 0;
    group_sync<kThreads>();
    uint64_t group = 0;
#pragma unroll
    for (int r = 0; r < kPer; ++r) group = key_max(group, s.list[lane * kPer + r]);
    int greater = 0;
    for (int o = 0; o < 64; ++o) greater += key_lane(group, o) > group ? 1 : 0;
    // fewer than n_top groups with a key: every element
    const uint64_t at = __ballot(greater == n_top - 1 && group != 0);
    const uint64_t cut = at != 0 ? key_lane(group, __builtin_ctzll(at)) : 1;
    group_sync<kThreads>();
    if (key >= cut)
      tile.each_vector_from_memory(x, [&](float f, int column) {
        if (f > -INFINITY && column_key(f, first_column + column) >= cut) {
          const int to = atomicAdd(&s.count, 1);
          if (to < kListCap) s.list[to] = column_key(f, first_column + column);
        }
        return true;
      });
    group_sync<kThreads>();
    m = s.count;
  }
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
  __shared__ BestLds<kThreads, kVecs> s_best;
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
  Stat st = wave_stat(tile, wave_max(tmax), static_cast<float>(a.c));
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
  const Stat st = join_lanes(mine);
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
// A row's columns are those that teacher slots name ("named", at most
// n_teacher) and the others.  The others' sum comes from the tile, with the
// named columns taken out of it before (a bit per column in LDS); the named
// ones are computed one by one in 64 bits.  So the rest's share is summed by
// itself, never as a difference, and a teacher that takes nearly everything
// loses no bits.  With R the others' log2 sum and L the row's, an other
// column's gradient is
//   weight tau (q - P q / Q) = [weight tau (2^(R - L) - P)] 2^(x c - R):
// one exponential and one product a column, for both forms of the loss (P = 0
// without teacher_lse).
//
// The loss is a difference of logarithms that may be 1e-3 of them, so the
// exponents are computed with c in two parts (log2(e) / tau rounded to fp32
// alone moves the temperature by 2^-25).  c_lo > 0, so that -inf stays -inf; from
// tau = 1e37 on it may lie below the smallest fp32 number, which then stands for
// it (and changes no exponent by more than 2^-21).
struct SplitC {
  float hi, lo;
};

__device__ __forceinline__ SplitC split_c(double c) {
  float hi = static_cast<float>(c);
  if (hi >= c) hi = __uint_as_float(__float_as_uint(hi) - 1);
  return {hi, fmaxf(static_cast<float>(c - hi), 0x1p-149f)};
}

// A chunk's sums: the others', relative to 2^other_origin, and the named
// columns', relative to 2^named_origin; over the named slots sum p (log p -
// ln 2 (x c - named_origin)) and sum p.  named_sum is NaN where the row has no
// finite distribution or no finite teacher.
struct DistillStat {
  double other_origin, other_sum, named_origin, named_sum, loss, psum;
};

// What the others' gradient needs, cheap to compute while the tile is held: an
// other column has coef 2^(x c - origin).
constexpr int kRowNan = 1, kRowFinite = 2;        // 0: loss and gradient 0
struct DistillRow {
  double origin, hi, all;      // all columns' sum is 2^hi all
  float coef;
  int mode;
};

// What takes logarithms: a named column has weight tau (2^(x c - hi - log2_all) - p).
struct DistillEnd {
  double log2_all;
  float loss;
};

// Dynamic LDS of the distillation: per slot the probability, the logit and the
// column relative to the chunk (-1 elsewhere); a hash table of the columns;
// then a bit per column.
struct TeacherLds {
  double* p;
  float* x;
  int* column;
  int* hash;
  int hash_bits;
  unsigned char* bits;
};

// At least twice as many entries as slots, so a probe always ends.
__host__ __device__ constexpr int teacher_hash_bits(int n_teacher) {
  int b = 6;
  while ((1 << b) < 2 * n_teacher) ++b;
  return b;
}
__host__ __device__ constexpr size_t teacher_slot_bytes(int n_teacher) {
  return (static_cast<size_t>(n_teacher) * 16 + 15) & ~size_t{15};
}
__host__ __device__ constexpr size_t teacher_lds_bytes(int n_teacher) {
  return teacher_slot_bytes(n_teacher) + (size_t{4} << teacher_hash_bits(n_teacher));
}

__device__ __forceinline__ TeacherLds teacher_lds(unsigned char* smem, int n_teacher) {
  TeacherLds t;
  t.p = reinterpret_cast<double*>(smem);
  t.x = reinterpret_cast<float*>(t.p + n_teacher);
  t.column = reinterpret_cast<int*>(t.x + n_teacher);
  t.hash = reinterpret_cast<int*>(smem + teacher_slot_bytes(n_teacher));
  t.hash_bits = teacher_hash_bits(n_teacher);
  t.bits = smem + teacher_lds_bytes(n_teacher);
  return t;
}

// What one wavefront finds out about the teacher.
struct Teacher {
  double top, lse;     // log p = (t - top) / tau - lse: the largest logit apart, which may be 1e38
  double rest;         // P
  bool bad, present;   // a NaN or +inf among the present slots; any
  bool undefined;      // its sum has no logarithm (rows left out do not look at it)
  bool repeats;        // two slots name one column of the chunk
};

// One wavefront reads the slots; columns in [first, first + mine) are named.
__device__ __forceinline__ Teacher read_teacher(const DistillArgs& a, int64_t row, int len, int first, int mine,
                                                const TeacherLds& t) {
  const int lane = threadIdx.x & 63;
  const int32_t* ids = a.teacher_ids + row * a.n_teacher;
  const float* logits = a.teacher_logits + row * a.n_teacher;
  const double inv_tau = 1.0 / static_cast<double>(a.tau);
  float mx = -INFINITY;
  bool bad = false, present = false;
  for (int k = lane; k < a.n_teacher; k += 64) {
    const int id = ids[k];
    const float v = logits[k];
    if (id >= 0 && id < len) {
      present = true;
      if (isnan(v) || v == INFINITY) bad = true;
      mx = fmaxf(mx, v);
    }
    t.column[k] = id >= first && id < first + mine ? id - first : -1;
  }
  // Columns that several slots name are rare and cost comparing every pair
  // (256 rows of 4096 columns, 128 slots: 28 us); a hash table says whether
  // there are any.
  Teacher out;
  for (int h = lane; h < (1 << t.hash_bits); h += 64) t.hash[h] = -1;
  group_sync<64>();
  bool repeats = false;
  for (int k = lane; k < a.n_teacher; k += 64) {
    const int column = t.column[k];
    if (column < 0) continue;
    for (uint32_t h = (static_cast<uint32_t>(column) * 2654435761u) >> (32 - t.hash_bits);; ++h) {
      const int was = atomicCAS(&t.hash[h & ((1u << t.hash_bits) - 1)], -1, column);
      repeats = repeats || was == column;
      if (was == -1 || was == column) break;
    }
  }
  out.repeats = __any(repeats);
  out.present = __any(present);
  mx = wave_max(mx);
  if (a.teacher_lse) {
    out.top = 0.0;
    out.lse = a.teacher_lse[row];
    out.undefined = !isfinite(out.lse);
  } else {
    out.undefined = out.present && mx == -INFINITY;
    double sum = 0.0;
    for (int k = lane; k < a.n_teacher; k += 64)
      if (ids[k] >= 0 && ids[k] < len) sum += exp((static_cast<double>(logits[k]) - mx) * inv_tau);
    out.top = mx;
    out.lse = log(wave_add(sum));
  }
  double psum = 0.0;
  for (int k = lane; k < a.n_teacher; k += 64) {
    const double p = ids[k] >= 0 && ids[k] < len ? exp((logits[k] - out.top) * inv_tau - out.lse) : 0.0;
    t.p[k] = p;
    psum += p;
  }
  out.rest = a.teacher_lse ? fmax(0.0, 1.0 - wave_add(psum)) : 0.0;
  out.bad = __any(bad);
  return out;
}

// 2^d of a difference of exponents.
__device__ __forceinline__ double pow2(double d) { return d < -4000.0 ? 0.0 : exp2(d); }

// The named columns' part of a chunk's sums, by one wavefront.  A column that
// several slots name counts once in the student's sum.
__device__ __forceinline__ DistillStat named_stat(const DistillArgs& a, int64_t row, const TeacherLds& t,
                                                  const Teacher& teacher) {
  const int lane = threadIdx.x & 63;
  const double inv_tau = 1.0 / static_cast<double>(a.tau);
  const float* logits = a.teacher_logits + row * a.n_teacher;
  double mx = -INFINITY;
  bool bad = teacher.bad;
  for (int k = lane; k < a.n_teacher; k += 64)
    if (t.column[k] >= 0) {
      const float x = t.x[k];
      if (isnan(x) || x == INFINITY) bad = true;
      mx = fmax(mx, x * a.c);
    }
  mx = wave_max(mx);
  mx = mx == -INFINITY ? 0.0 : rint(mx);           // whole: sums join by exact powers of two
  double sum = 0.0, loss = 0.0, psum = 0.0;
  for (int k = lane; k < a.n_teacher; k += 64) {
    const int column = t.column[k];
    if (column < 0) continue;
    const double z = t.x[k] * a.c - mx, p = t.p[k];
    bool again = false;
    if (teacher.repeats)
      for (int o = 0; o < k; ++o) again |= t.column[o] == column;
    if (!again) sum += pow2(z);
    if (p > 0.0) {
      loss += p * ((logits[k] - teacher.top) * inv_tau - teacher.lse - z * kLn2);
      psum += p;
    }
  }
  sum = wave_add(sum);
  return {0.0, 0.0, mx, __any(bad) ? NAN : sum, wave_add(loss), wave_add(psum)};
}

// Joins the statistics that a wavefront's lanes hold, in every lane.
__device__ __forceinline__ DistillStat join_lanes(const DistillStat& mine) {
  const Stat other = join_lanes(Stat{mine.other_origin, mine.other_sum, 0.0});
  DistillStat st{other.origin, other.sum, 0.0, 0.0, 0.0, 0.0};
  const bool named = mine.named_sum != 0.0 || mine.psum != 0.0;
  const double m = wave_max(named ? mine.named_origin : -INFINITY);
  const double d = named ? mine.named_origin - m : 0.0;
  st.named_origin = m;
  st.named_sum = wave_add(named ? times_pow2(mine.named_sum, d) : 0.0);
  // sum p (log p - ln 2 (x c - m)) from the chunk's own origin
  st.loss = wave_add(mine.psum == 0.0 ? 0.0 : mine.loss - mine.psum * d * kLn2);
  st.psum = wave_add(mine.psum);
  return st;
}

// From the whole row's sums.
__device__ __forceinline__ DistillRow distill_row(const DistillArgs& a, const DistillStat& st, const Teacher& teacher,
                                                  float weight) {
  DistillRow r{};
  if (!a.teacher_lse && !teacher.present) return r;                   // nothing to follow
  const bool other = st.other_sum != 0.0, named = st.named_sum != 0.0;
  if (teacher.bad || isnan(st.other_sum) || isnan(st.named_sum)) {
    r.mode = kRowNan;
    return r;
  }
  if (!other && !named) return r;                                     // no distribution
  if (teacher.undefined) {
    r.mode = kRowNan;
    return r;
  }
  r.hi = fmax(other ? st.other_origin : -INFINITY, named ? st.named_origin : -INFINITY);
  const double others = other ? times_pow2(st.other_sum, st.other_origin - r.hi) : 0.0;
  r.all = others + (named ? times_pow2(st.named_sum, st.named_origin - r.hi) : 0.0);
  r.mode = kRowFinite;
  r.origin = other ? st.other_origin : r.hi;
  // Q = others / all
  if (other)
    r.coef = static_cast<float>(static_cast<double>(weight) * a.tau * (others / r.all - teacher.rest) / st.other_sum);
  return r;
}

__device__ __forceinline__ DistillEnd distill_end(const DistillArgs& a, const DistillRow& r, const DistillStat& st,
                                                  const Teacher& teacher) {
  if (r.mode != kRowFinite) return {0.0, r.mode == kRowNan ? NAN : 0.0f};
  DistillEnd e;
  e.log2_all = log2(r.all);
  double loss = st.psum > 0.0 ? st.loss + st.psum * ((r.hi - st.named_origin) + e.log2_all) * kLn2 : 0.0;
  if (st.other_sum != 0.0 && teacher.rest > 0.0)
    loss += teacher.rest *
            (log(teacher.rest) - ((st.other_origin - r.hi) + (log2(st.other_sum) - e.log2_all)) * kLn2);
  e.loss = static_cast<float>(loss * (static_cast<double>(a.tau) * a.tau));
  return e;
}

// The other columns' sum in a wavefront's registers, in every lane.
template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ Stat other_stat(RowTile<T, kThreads, kVecs>& tile, float mx, const DistillArgs& a) {
  constexpr int kE = Elem<T>::kPerVec;
  const SplitC c = split_c(a.c);
  const float b = mx == -INFINITY ? 0.0f : rintf(mx * c.hi);
  float sum = 0.0f;
  double origin = b;
  tile.forget_unpacked();
  if (fabsf(b) < kFar) {
    auto add = [&](float v) { sum += exp2_fast(__fmaf_rn(v, c.lo, __fmaf_rn(v, c.hi, -b))); };
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (tile.has(i)) {
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
#pragma unroll
        for (int j = 0; j < kE; ++j) add(f[j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    add(tile.edge);
  } else {
    origin = rint(mx * a.c);
    tile.each([&](float v, int) { sum += exp2_fast(far_exponent(v, a.c, origin)); });
  }
  return {origin, wave_add(static_cast<double>(sum)), 0.0};
}

// n elements of g at p.
template <typename T>
__device__ __forceinline__ void fill_range(T* p, int n, float g, int tid, int threads) {
  constexpr int kE = Elem<T>::kPerVec;
  float f[kE];
#pragma unroll
  for (int j = 0; j < kE; ++j) f[j] = g;
  const Word4 w = Elem<T>::pack(f);
  const int head = head_of(p, max(n, 0)), nvec = (n - head) / kE;
  for (int v = tid; v < nvec; v += threads) store_words(p + head + v * kE, w);
  if (tid < n - nvec * kE) p[tid < head ? tid : nvec * kE + tid] = elem_round<T>(g);
}

// The gradient of the tile's columns, every one as an other one.
template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ void write_others(RowTile<T, kThreads, kVecs>& tile, const DistillArgs& a,
                                             const DistillRow& r, const T* x, T* grad) {
  constexpr int kE = Elem<T>::kPerVec;
  const int tid = threadIdx.x;
  const SplitC c = split_c(a.c);
  const float coef = r.coef;
  tile.forget_unpacked();
  if (!(fabs(r.origin) < kFar)) {
    tile.each_from_memory(x, [&](float v, int column) {
      grad[column] = elem_round<T>(coef * exp2_fast(far_exponent(v, a.c, r.origin)));
    });
    return;
  }
  const float b = static_cast<float>(r.origin);
  auto gradient = [&](float v) { return coef * exp2_fast(__fmaf_rn(v, c.lo, __fmaf_rn(v, c.hi, -b))); };
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
    if (tile.has(i)) {
      if (tid < tile.nvec - i * kThreads) {
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
#pragma unroll
        for (int j = 0; j < kE; ++j) f[j] = gradient(f[j]);
        char* to = reinterpret_cast<char*>(grad + tile.head) + static_cast<int64_t>(i) * kThreads * 16;
        store_words(to + tid * 16u, Elem<T>::pack(f));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  if (tid < tile.nedge) grad[tile.edge_column()] = elem_round<T>(gradient(tile.edge));
}

// After the tile: the loss, and the named columns' gradient over what
// write_others has put there (the workgroup's stores have left when the
// barrier opens, so these come last).  grad may be null.
template <typename T, int kThreads>
__device__ __forceinline__ void finish_named(const DistillArgs& a, int64_t row, const DistillRow& r,
                                             const DistillStat& st, const Teacher& teacher, float weight,
                                             const TeacherLds& t, bool write_loss, T* grad, DistillEnd& s_end) {
  const int tid = threadIdx.x;
  if (tid < 64) {
    const DistillEnd e = distill_end(a, r, st, teacher);
    if (tid == 0) {
      s_end = e;
      if (write_loss) a.loss_out[row] = e.loss;
    }
  }
  if (!grad || r.mode != kRowFinite) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  group_sync<kThreads>();
  const double log2_all = s_end.log2_all;
  for (int k = tid; k < a.n_teacher; k += kThreads) {
    const int column = t.column[k];
    if (column < 0) continue;
    double p = t.p[k];
    if (teacher.repeats) {
      p = 0.0;
      for (int o = 0; o < a.n_teacher; ++o) p += t.column[o] == column ? t.p[o] : 0.0;
    }
    const double q = pow2(t.x[k] * a.c - r.hi - log2_all);
    grad[column] = elem_round<T>(static_cast<float>(static_cast<double>(weight) * a.tau * (q - p)));
  }
}

// Columns without a gradient: those past the row's length, and all of a row
// that is left out or undefined (false: there is nothing else to write).
template <typename T, int kThreads>
__device__ __forceinline__ bool write_rest(const DistillRow& r, T* grad, int mine, int cols) {
  const int tid = threadIdx.x;
  fill_range(grad + mine, cols - mine, 0.0f, tid, kThreads);
  if (r.mode == kRowFinite) return true;
  fill_range(grad, mine, r.mode == kRowNan ? NAN : 0.0f, tid, kThreads);
  return false;
}

// The named columns' logits, by the wavefront that read the teacher.
template <typename T>
__device__ __forceinline__ void gather_named(const DistillArgs& a, const T* x, const TeacherLds& t) {
  for (int k = threadIdx.x & 63; k < a.n_teacher; k += 64) {
    const int column = t.column[k];
    t.x[k] = column >= 0 ? elem_load(x + column) : -INFINITY;
  }
}

// A bit for every named column of [first, first + columns), by one wavefront.
template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ void mark_named(const RowTile<T, kThreads, kVecs>& tile, const DistillArgs& a,
                                           const TeacherLds& t, int first, int columns) {
  constexpr int kBitWords = (RowTile<T, kThreads, kVecs>::kBitBytes + 15) / 16;
  const int lane = threadIdx.x & 63;
  for (int w = lane; w < kBitWords; w += 64) reinterpret_cast<Word4*>(t.bits)[w] = Word4{0, 0, 0, 0};
  group_sync<64>();
  for (int k = lane; k < a.n_teacher; k += 64) {
    const int column = t.column[k] - first;
    if (t.column[k] >= 0 && column >= 0 && column < columns) {
      const int bit = tile.bit_of(column);
      atomicOr(reinterpret_cast<unsigned*>(t.bits) + (bit >> 5), 1u << (bit & 31));
    }
  }
}

// Takes the named columns out of the tile.
template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ void drop_named(RowTile<T, kThreads, kVecs>& tile, const unsigned char* bits) {
  constexpr int kE = Elem<T>::kPerVec;
  const int tid = threadIdx.x;
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
    if (tile.has(i)) {
      const uint32_t hit = bits[i * kThreads + tid];
      if (hit != 0) {
        float f[kE];
        Elem<T>::unpack(tile.v[i], f);
#pragma unroll
        for (int j = 0; j < kE; ++j) f[j] = (hit >> j) & 1u ? -INFINITY : f[j];
        tile.v[i] = Elem<T>::pack(f);
      }
    }
  if (tid < tile.nedge && ((bits[kThreads * kVecs + (tid >> 3)] >> (tid & 7)) & 1u)) tile.edge = -INFINITY;
}

// What the wavefront that reads the teacher leaves for the workgroup.
struct TeacherState {
  Teacher teacher;
  DistillStat named;
};

template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ void teacher_state(const DistillArgs& a, int64_t row, const T* x, int len, int first,
                                              int mine, const TeacherLds& t, TeacherState& s) {
  const Teacher teacher = read_teacher(a, row, len, first, mine, t);
  gather_named(a, x, t);
  const DistillStat named = named_stat(a, row, t, teacher);
  if ((threadIdx.x & 63) == 0) s = {teacher, named};
}

// Joins the wavefronts' sums of the others to the named columns' in
// s.named, and leaves the row's gradient data in s_row (whole rows).  Two
// barriers.
template <int kThreads>
__device__ __forceinline__ void join_row(const DistillArgs& a, float weight, const Stat& other, Stat* s_stat,
                                         TeacherState& s, DistillRow* s_row) {
  constexpr int kWaves = kThreads / 64;
  const int tid = threadIdx.x;
  if (kWaves > 1 && (tid & 63) == 0) s_stat[tid >> 6] = other;
  group_sync<kThreads>();
  if (tid < 64) {
    DistillStat st = s.named;
    const Stat all = kWaves > 1 ? join_lanes(tid < kWaves ? s_stat[tid] : Stat{0.0, 0.0, 0.0}) : other;
    st.other_origin = all.origin;
    st.other_sum = all.sum;
    if (tid == 0) s.named = st;
    if (s_row) {
      const DistillRow r = distill_row(a, st, s.teacher, weight);
      if (tid == 0) *s_row = r;
    }
  }
  group_sync<kThreads>();
}

// One workgroup per row (kWhole: chunks is 1, loss and gradient are written)
// or per (row, chunk), whose sums go to the workspace.
template <typename T, int kThreads, int kVecs, bool kWhole>
__global__ __launch_bounds__(kThreads, 4) void distill_tile_kernel(const DistillArgs a, int64_t item0, int chunk,
                                                                   int chunks, DistillStat* stats) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Stat s_stat[kThreads / 64];
  __shared__ DistillRow s_row;
  __shared__ DistillEnd s_end;
  __shared__ TeacherState s_teacher;
  const int tid = threadIdx.x;
  const int64_t item = item0 + blockIdx.x;
  const int64_t row = kWhole ? item : item / chunks;
  const int first = kWhole ? 0 : static_cast<int>(item - row * chunks) * chunk;
  const float weight = a.row_weight ? a.row_weight[row] : 1.0f;
  const int cols = static_cast<int>(a.cols);
  if (weight == 0.0f) {
    if constexpr (kWhole) {
      if (tid == 0) a.loss_out[row] = 0.0f;
      if (a.grad_out) fill_range(static_cast<T*>(a.grad_out) + row * a.grad_ld, cols, 0.0f, tid, kThreads);
    }
    return;
  }
  const T* x = static_cast<const T*>(a.logits) + row * a.ld + first;
  const int len = row_cols(a.n_valid, row, a.cols);
  const int mine = kWhole ? len : max(0, min(chunk, len - first));
  const TeacherLds t = teacher_lds(smem, a.n_teacher);
  RowTile<T, kThreads, kVecs> tile;
  // The teacher's wavefront has no registers for its mathematics beside a
  // large tile: it reads its part of the row afterwards.
  constexpr bool kTeacherFirst = kVecs > 8;
  tile.place(x, mine);
  if (!kTeacherFirst) tile.load(x, mine);
  if (tid < 64) {
    teacher_state<T, kThreads, kVecs>(a, row, x, len, first, mine, t, s_teacher);
    mark_named(tile, a, t, 0, mine);
  }
  if (kTeacherFirst) tile.load(x, mine);
  group_sync<kThreads>();
  drop_named(tile, t.bits);
  const Stat other = other_stat(tile, wave_max(tile.thread_max()), a);
  join_row<kThreads>(a, weight, other, s_stat, s_teacher, kWhole ? &s_row : nullptr);
  if constexpr (kWhole) {
    const DistillRow r = s_row;
    T* grad = a.grad_out ? static_cast<T*>(a.grad_out) + row * a.grad_ld : nullptr;
    if (grad && write_rest<T, kThreads>(r, grad, mine, cols)) write_others(tile, a, r, x, grad);
    finish_named<T, kThreads>(a, row, r, s_teacher.named, s_teacher.teacher, weight, t, true, grad, s_end);
  } else if (tid == 0) {
    stats[item] = s_teacher.named;
  }
}

// A workgroup per row longer than its tile: the row's segments pass through
// the tile from the last to the first, which stays; the others are read again
// for the gradient (from the last-level cache: the rows in flight fit it).
template <typename T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads) void distill_long_kernel(const DistillArgs a, int64_t row0) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Stat s_stat[kThreads / 64];
  __shared__ DistillRow s_row;
  __shared__ DistillEnd s_end;
  __shared__ TeacherState s_teacher;
  using Tile = RowTile<T, kThreads, kVecs>;
  const int tid = threadIdx.x;
  const int64_t row = row0 + blockIdx.x;
  const float weight = a.row_weight ? a.row_weight[row] : 1.0f;
  const int cols = static_cast<int>(a.cols);
  T* grad = a.grad_out ? static_cast<T*>(a.grad_out) + row * a.grad_ld : nullptr;
  if (weight == 0.0f) {
    if (tid == 0) a.loss_out[row] = 0.0f;
    if (grad) fill_range(grad, cols, 0.0f, tid, kThreads);
    return;
  }
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  const int mine = row_cols(a.n_valid, row, a.cols);
  const TeacherLds t = teacher_lds(smem, a.n_teacher);
  if (tid < 64) teacher_state<T, kThreads, kVecs>(a, row, x, mine, 0, mine, t, s_teacher);
  Tile tile;
  Stat other{0.0, 0.0, 0.0};
  int at = mine > 0 ? (mine - 1) / Tile::kCapacity * Tile::kCapacity : 0;
  for (;; at -= Tile::kCapacity) {
    const int n = min(mine - at, Tile::kCapacity);
    if (at > 0 && grad) tile.template load<false>(x + at, n);
    else tile.load(x + at, n);
    if (tid < 64) mark_named(tile, a, t, at, n);
    __syncthreads();
    drop_named(tile, t.bits);
    other = join(other, other_stat(tile, wave_max(tile.thread_max()), a));
    if (at == 0) break;
    __syncthreads();                                   // the segment's bits have been read
  }
  join_row<kThreads>(a, weight, other, s_stat, s_teacher, &s_row);
  const DistillRow r = s_row;
  if (grad && write_rest<T, kThreads>(r, grad, mine, cols)) {
    write_others(tile, a, r, x, grad);
    for (at = Tile::kCapacity; at < mine; at += Tile::kCapacity) {
      tile.load(x + at, min(mine - at, Tile::kCapacity));
      write_others(tile, a, r, x + at, grad + at);
    }
  }
  finish_named<T, kThreads>(a, row, r, s_teacher.named, s_teacher.teacher, weight, t, true, grad, s_end);
}

// The second launch of rows in chunks: every workgroup joins its row's sums
// and writes its chunk's gradient, the first chunk's also the loss.  Without a
// gradient one wavefront per row (chunks_grid 1).
template <typename T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(const DistillArgs a, int64_t item0, int chunk,
                                                                int chunks, int chunks_grid,
                                                                const DistillStat* stats) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ DistillRow s_row;
  __shared__ DistillEnd s_end;
  __shared__ TeacherState s_teacher;
  const int tid = threadIdx.x;
  const int64_t item = item0 + blockIdx.x;
  const int64_t row = item / chunks_grid;
  const int first = static_cast<int>(item - row * chunks_grid) * chunk;
  const float weight = a.row_weight ? a.row_weight[row] : 1.0f;
  const int cols = min(chunk, static_cast<int>(a.cols) - first);
  T* grad = a.grad_out ? static_cast<T*>(a.grad_out) + row * a.grad_ld + first : nullptr;
  if (weight == 0.0f) {
    if (first == 0 && tid == 0) a.loss_out[row] = 0.0f;
    if (grad) fill_range(grad, cols, 0.0f, tid, kThreads);
    return;
  }
  const T* x = static_cast<const T*>(a.logits) + row * a.ld + first;
  const int len = row_cols(a.n_valid, row, a.cols);
  const int mine = max(0, min(chunk, len - first));
  const TeacherLds t = teacher_lds(smem, a.n_teacher);
  RowTile<T, kThreads, kVecs> tile;
  if (tid < 64) {
    const DistillStat own = tid < chunks ? stats[row * chunks + tid] : DistillStat{};
    const Teacher teacher = read_teacher(a, row, len, first, mine, t);
    if (grad) gather_named(a, x, t);
    const DistillStat st = join_lanes(own);
    const DistillRow r = distill_row(a, st, teacher, weight);
    if (tid == 0) {
      s_teacher = {teacher, st};
      s_row = r;
    }
  }
  if (grad) tile.load(x, mine);
  group_sync<kThreads>();
  const DistillRow r = s_row;
  if (grad && write_rest<T, kThreads>(r, grad, mine, cols)) write_others(tile, a, r, x, grad);
  finish_named<T, kThreads>(a, row, r, s_teacher.named, s_teacher.teacher, weight, t, first == 0, grad, s_end);
}

}  // namespace

// How a row's columns go over workgroups: threads and vectors per thread of a
// workgroup, columns per chunk, chunks per row.
struct RowPlan {
  int threads, vecs, chunk, chunks;
};

// A row of up to 4096 vectors goes to the smallest workgroup that holds it (a
// wavefront up to 512 vectors), longer rows to chunks of 256-thread
// workgroups: enough of them to give every CU two, none of fewer than 256
// vectors.  (One launch of few workgroups beats two launches that fill the
// GPU: 256 rows of 28000 fp16 logits 17 us against 23.)  n > 0.
RowPlan log_probs_plan(int64_t n, int64_t cols, int per_vec) {
  constexpr int64_t kFill = 512;
  const int64_t vecs = (cols + per_vec - 1) / per_vec;
  if (vecs <= 128) return {64, 2, static_cast<int>(cols), 1};
  if (vecs <= 512) return {64, 8, static_cast<int>(cols), 1};
  if (vecs <= 4096) return {256, vecs <= 2048 ? 8 : 16, static_cast<int>(cols), 1};
  int64_t chunks = (vecs + 4095) / 4096;
  if (n * chunks < kFill)
    chunks = std::max(chunks, std::min<int64_t>({(kFill + n - 1) / n, (vecs + 255) / 256, kMaxChunks}));
  const int64_t chunk = (vecs + chunks - 1) / chunks;
  return {256, chunk <= 2048 ? 8 : 16, static_cast<int>(chunk * per_vec),
          static_cast<int>((vecs + chunk - 1) / chunk)};
}

int64_t log_probs_workspace_bytes(int64_t n, int64_t cols, int n_top) {
  if (n == 0) return 0;
  int64_t most = 0;                            // the element type is not known here
  for (int per_vec : {4, 8}) {
    const RowPlan p = log_probs_plan(n, cols, per_vec);
    if (p.chunks > 1) most = std::max<int64_t>(most, n * p.chunks);
  }
  return most * static_cast<int64_t>(sizeof(Stat) + 8 * n_top);
}
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

// As log_probs_plan, but where there is a row for every other CU a workgroup
// takes a whole long row: it reads part of the logits once, where two launches
// read all of them twice (131072 bf16 columns, 512 rows: 69 us against 98; 128
// rows 36 and 35, 64 rows 33 and 23).  Few rows of up to 4096 vectors go to the
// same workgroups of 512 threads (256 rows of 28000 columns 17 us, in 256
// threads 23), many to smaller ones (800 rows: 38 us against 31).
constexpr int kLongThreads = 512, kLongVecs = 8;
RowPlan distill_plan(int64_t n, int64_t cols, int per_vec) {
  const int64_t vecs = (cols + per_vec - 1) / per_vec;
  if (vecs > 512 && (vecs <= 4096 ? n < 512 : n >= 128)) return {kLongThreads, kLongVecs, static_cast<int>(cols), 1};
  return log_probs_plan(n, cols, per_vec);
}

int64_t distill_workspace_bytes(int64_t n, int64_t cols) {
  if (n == 0) return 0;
  int64_t most = 0;                            // the element type is not known here
  for (int per_vec : {4, 8}) {
    const RowPlan p = distill_plan(n, cols, per_vec);
    if (p.chunks > 1) most = std::max<int64_t>(most, n * p.chunks);
  }
  return most * static_cast<int64_t>(sizeof(DistillStat));
}

template <typename T>
hipError_t distill_typed(const DistillArgs& a, hipStream_t s) {
  const RowPlan p = distill_plan(a.n, a.cols, Elem<T>::kPerVec);
  DistillStat* stats = static_cast<DistillStat*>(a.workspace);
  const size_t slots = teacher_lds_bytes(a.n_teacher);
  const size_t lds = slots + static_cast<size_t>(p.threads) * p.vecs + 32;      // RowTile::kBitBytes, in words of 16
  const int64_t items = a.n * p.chunks;
  const hipError_t e = in_slices(items, [&](int64_t at, unsigned grid) {
    if (p.chunks > 1) {
      if (p.vecs == 8) distill_tile_kernel<T, 256, 8, false><<<grid, 256, lds, s>>>(a, at, p.chunk, p.chunks, stats);
      else distill_tile_kernel<T, 256, 16, false><<<grid, 256, lds, s>>>(a, at, p.chunk, p.chunks, stats);
    } else if (p.threads == 64) {
      if (p.vecs == 2) distill_tile_kernel<T, 64, 2, true><<<grid, 64, lds, s>>>(a, at, p.chunk, 1, stats);
      else distill_tile_kernel<T, 64, 8, true><<<grid, 64, lds, s>>>(a, at, p.chunk, 1, stats);
    } else if (p.threads == 256) {
      if (p.vecs == 8) distill_tile_kernel<T, 256, 8, true><<<grid, 256, lds, s>>>(a, at, p.chunk, 1, stats);
      else distill_tile_kernel<T, 256, 16, true><<<grid, 256, lds, s>>>(a, at, p.chunk, 1, stats);
    } else {
      distill_long_kernel<T, kLongThreads, kLongVecs><<<grid, kLongThreads, lds, s>>>(a, at);
    }
  });
  if (e != hipSuccess || p.chunks == 1) return e;
  const int per_row = a.grad_out ? p.chunks : 1;
  return in_slices(a.n * per_row, [&](int64_t at, unsigned grid) {
    if (!a.grad_out) distill_join_kernel<T, 64, 2><<<grid, 64, slots, s>>>(a, at, p.chunk, p.chunks, 1, stats);
    else if (p.vecs == 8) distill_join_kernel<T, 256, 8><<<grid, 256, slots, s>>>(a, at, p.chunk, p.chunks, per_row, stats);
    else distill_join_kernel<T, 256, 16><<<grid, 256, slots, s>>>(a, at, p.chunk, p.chunks, per_row, stats);
  });
}

hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
  switch (a.n == 0 ? -1 : a.dtype) {
    case -1: return hipSuccess;
    case kElemF32: return distill_typed<float>(a, s);
    case kElemF16: return distill_typed<_Float16>(a, s);
    default: return distill_typed<__bf16>(a, s);
  }
}

}  // namespace ifvs
