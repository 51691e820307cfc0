// Embedding lookup and the gradient of its table (Section 2, opening
// paragraph: alpha is a sum of rows of a table; the training paragraph sends
// gradients back into the rows).
//
//   lookup:   out[i] = scale * sum over j of table[ids[i][j]]
//   gradient: G[r] = scale * sum over the slots (i, j) that name r of grad[i]
//
// Both move bytes and add: HBM bounds them.  The gradient sorts the slots by
// table row (stable, so equal rows stay in slot order), cuts the sorted slots
// into equal pieces, and sums each piece's runs in order; runs that cross
// pieces leave fp32 partial sums that a last launch adds in order.  So a row
// that half of the slots name costs no more than as many rows, no sum depends
// on scheduling, and each gradient row is read once.  The table is cleared
// beside the sort.
#include <algorithm>
#include <cmath>

#include "rows_device.h"

namespace ifvs {

namespace {

constexpr int kEmbThreads = 256;

// Lanes that share a row: the smallest power of two that holds its vectors,
// at most a workgroup (wider rows go to several workgroups).
int lanes_per_row(int vecs) {
  int l = 1;
  while (l < vecs && l < kEmbThreads) l *= 2;
  return l;
}

// The columns of a lane: vector `vec` of a row of dim elements.  The last
// vector of a row that does not divide ends at the row's end: it overlaps its
// neighbour, and only `own` of its elements (the last ones) are the lane's.
template <typename T>
struct LaneCols {
  static constexpr int kE = Elem<T>::kPerVec;
  int start, own;
  bool narrow;                        // dim < kE: element by element
  __device__ __forceinline__ LaneCols(int vec, int dim) {
    narrow = dim < kE;
    start = narrow ? 0 : min(vec * kE, dim - kE);
    own = min(kE, dim - vec * kE);
  }
  // The lane's vector of a row, packed.
  __device__ __forceinline__ Word4 load_raw(const T* row) const {
    if (!narrow) return *reinterpret_cast<const Word4At2*>(row + start);
    float f[kE];
#pragma unroll
    for (int j = 0; j < kE; ++j) f[j] = j < own ? elem_load(row + j) : 0.0f;
    return Elem<T>::pack(f);
  }
  // Elements of another type O at the same columns.
  template <typename O>
  __device__ __forceinline__ void load_old(const O* row, float* f) const {
    constexpr int kO = Elem<O>::kPerVec;
    if (own == kE) {
#pragma unroll
      for (int j = 0; j < kE; j += kO) {
        const Word4 w = *reinterpret_cast<const Word4At2*>(row + start + j);
        Elem<O>::unpack(w, f + j);
      }
      return;
    }
    const int skip = narrow ? 0 : kE - own;
#pragma unroll
    for (int j = 0; j < kE; ++j) f[j] = j >= skip && (!narrow || j < own) ? elem_load(row + start + j) : 0.0f;
  }
  template <typename O>
  __device__ __forceinline__ void store(O* row, const float* f) const {
    if (own == kE) {
      constexpr int kO = Elem<O>::kPerVec;
#pragma unroll
      for (int j = 0; j < kE; j += kO) store_words(row + start + j, Elem<O>::pack(f + j));
    } else {
      const int skip = narrow ? 0 : kE - own;
#pragma unroll
      for (int j = 0; j < kE; ++j)
        if (j >= skip && (!narrow || j < own)) row[start + j] = elem_round<O>(f[j]);
    }
  }
};

// grid.x: groups of kRows output rows, grid.y: kEmbThreads vectors of a row.
template <typename T, int kRows>
__global__ __launch_bounds__(kEmbThreads) void embed_lookup_kernel(const EmbedArgs a, int lanes, int64_t group0) {
  constexpr int kE = Elem<T>::kPerVec;
  const T* table = static_cast<const T*>(a.table);
  const int lane = threadIdx.x & (lanes - 1);
  const int groups = kEmbThreads / lanes;
  const int64_t i0 = ((group0 + blockIdx.x) * groups + threadIdx.x / lanes) * kRows;
  const int vec = blockIdx.y * kEmbThreads + lane;
  if (vec * kE >= a.dim || i0 >= a.n) return;
  const LaneCols<T> cols(vec, a.dim);
  float sum[kRows][kE];
#pragma unroll
  for (int u = 0; u < kRows; ++u)
#pragma unroll
    for (int e = 0; e < kE; ++e) sum[u][e] = 0.0f;
  for (int j = 0; j < a.bag; ++j) {
    // Absent slots and rows past the end read row 0 and drop it: no load
    // waits for a branch.
    uint32_t id[kRows];
    Word4 w[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) id[u] = static_cast<uint32_t>(a.ids[min(i0 + u, a.n - 1) * a.bag + j]);
#pragma unroll
    for (int u = 0; u < kRows; ++u)
      w[u] = cols.load_raw(table + (id[u] < static_cast<uint32_t>(a.rows) ? static_cast<int64_t>(id[u]) : 0) * a.table_ld);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      float f[kE];
      Elem<T>::unpack(w[u], f);
#pragma unroll
      for (int e = 0; e < kE; ++e) sum[u][e] += id[u] < static_cast<uint32_t>(a.rows) ? f[e] : 0.0f;
    }
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u)
    if (i0 + u < a.n) {
#pragma unroll
      for (int e = 0; e < kE; ++e) sum[u][e] *= a.scale;
      cols.store(static_cast<T*>(a.out) + (i0 + u) * a.out_ld, sum[u]);
    }
}

// ---------------------------------------------------- sorting slots by row
// Stable radix sort, least significant digit first.  A workgroup of 16
// wavefronts takes tiles of 4096 entries: a wavefront ranks 64 entries at a
// time among those of their digit (ballots over the digit's bits), so no
// atomics order anything.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortRounds = 4;
constexpr int kSortTile = kSortThreads * kSortRounds;
constexpr int kSortMaxBits = 10;
constexpr int kSortMaxGroups = 256;
// One launch (sort_owned_kernel) up to this many slots and owners: each owner
// reads all ids, so its time grows with slots x owners, and the owner of
// frequent rows sorts alone; the four launches of the radix sort cost the same
// for any ids.  Whole gradients, one launch / four, us (45000 rows of 64
// columns; ids uniform, Zipf scattered over the table, Zipf in its first rows,
// half of them one row): 16384 slots 26/40, 36/44, 49/44, 60/61 (beyond, an
// owner no longer holds the ids in registers); 20480 35/43, 42/45, 60/46,
// 71/62; 32768 43/48, 57/50, 81/51, 93/71.
// What is cleared beside the sort hides part of that: one slot more for every
// 32 KB cleared, up to twice as many.  131072 rows, clearing 173 MiB (up to
// 21920 slots): 20480 slots 51/65, 51/62, 79/62, 78/71, 24576 55/67, 58/62,
// 90/63, 86/73; 256 MiB (24576): 20480 67/78, 65/72, 83/72, 79/82, 32768 74/85,
// 76/78, 115/78, 112/91; 512 MiB (32768): 32768 139/146, 130/136, 149/132,
// 142/147.  Over three heights of the table, eight sizes of the clear and 16384
// to 32768 slots of those four kinds the choice costs 3.0% over the better of
// the two in the mean and 35% at worst; 28 to 40 KB a slot do the same, a limit
// of 16384 slots for all 4.0%, of 32768 from 128 MiB on 4.5% (79% at worst).
constexpr int64_t kOwnedSlots = 1 << 14;
constexpr int64_t kClearPerSlot = 1 << 15;            // bytes
constexpr int kOwnersFull = 256;
constexpr int64_t kMostOwners = 1 << 9;

struct SortBufs {
  uint32_t* key;       // table row; `rows` for absent slots
  uint32_t* from;      // gradient row
};

struct SortArgs {
  const int32_t* ids;  // the first pass reads these
  int64_t slots;
  uint32_t rows;
  int bag;
  SortBufs in, out;
  int shift, bits;
  int groups;
  int64_t per_group;   // slots of a workgroup, a multiple of kSortTile
  uint32_t* hist;      // [groups][1 << bits]
};

// Where a pass reads its entries: the ids themselves, a buffer, or the LDS.
struct FromIds {
  const int32_t* ids;
  uint32_t rows, bag;
  __device__ __forceinline__ uint2 operator()(int64_t at) const {
    const uint32_t slot = static_cast<uint32_t>(at);
    return {min(static_cast<uint32_t>(ids[at]), rows), bag == 1 ? slot : slot / bag};
  }
};
struct FromBuf {
  SortBufs in;
  __device__ __forceinline__ uint2 operator()(int64_t at) const { return {in.key[at], in.from[at]}; }
};
struct FromLds {
  const uint2* list;
  int64_t start;
  __device__ __forceinline__ uint2 operator()(int64_t at) const { return list[at - start]; }
};

// Exclusive sum over 1024 threads.
__device__ __forceinline__ uint32_t sort_scan(uint32_t v, uint32_t* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = v;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t below = __shfl_up(sum, o, 64);
    if (lane >= o) sum += below;
  }
  if (lane == 63) s_wave[wave] = sum;
  __syncthreads();
  uint32_t base = 0;
  for (int w = 0; w < wave; ++w) base += s_wave[w];
  __syncthreads();
  return base + sum - v;
}

struct SortLds {
  uint16_t count[kSortWaves][1 << kSortMaxBits];     // of a tile: at most 4096
  uint32_t base[1 << kSortMaxBits];                  // where the digit's next entry goes
  uint32_t wave[kSortWaves];
};

// Counts of the digits of [lo, hi) into s.base.
template <typename Src>
__device__ __forceinline__ void sort_count(const SortArgs& a, const Src& src, int64_t lo, int64_t hi, SortLds& s) {
  const uint32_t mask = (1u << a.bits) - 1;
  s.base[threadIdx.x] = 0;
  __syncthreads();
  for (int64_t at = lo + threadIdx.x; at < hi; at += kSortThreads)
    atomicAdd(&s.base[(src(at).x >> a.shift) & mask], 1u);
  __syncthreads();
}

// Moves [lo, hi) to its places; s.base holds each digit's first one.
template <typename Src>
__device__ __forceinline__ void sort_move(const SortArgs& a, const Src& src, int64_t lo, int64_t hi, SortLds& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t mask = (1u << a.bits) - 1;
  const bool digit_thread = tid <= static_cast<int>(mask);
  for (int64_t tile = lo; tile < hi; tile += kSortTile) {
    if (digit_thread)
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) s.count[w][tid] = 0;
    __syncthreads();
    const int64_t mine = tile + wave * kSortRounds * 64;
    uint2 entry[kSortRounds];
    uint32_t rank[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      entry[r] = mine + r * 64 + lane < hi ? src(mine + r * 64 + lane) : uint2{0, 0};
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (mine + r * 64 < hi) {
        const bool live = mine + r * 64 + lane < hi;
        const uint32_t digit = (entry[r].x >> a.shift) & mask;
        uint64_t peers = __ballot(live);
        for (int b = 0; b < a.bits; ++b) {
          const uint64_t set = __ballot((digit >> b) & 1u);
          peers &= (digit >> b) & 1u ? set : ~set;
        }
        const uint32_t before = s.count[wave][digit];
        const int below = __popcll(peers & ((1ull << lane) - 1));
        rank[r] = before + below;
        group_sync<64>();
        if (live && below == 0) s.count[wave][digit] = static_cast<uint16_t>(before + __popcll(peers));
        group_sync<64>();
      }
    __syncthreads();
    // the tile's entries of digit `tid` before each wavefront's
    uint32_t of_digit = 0;
    if (digit_thread) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t n = s.count[w][tid];
        s.count[w][tid] = static_cast<uint16_t>(of_digit);
        of_digit += n;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (mine + r * 64 + lane < hi) {
        const uint32_t digit = (entry[r].x >> a.shift) & mask;
        const uint32_t to = s.base[digit] + s.count[wave][digit] + rank[r];
        a.out.key[to] = entry[r].x;
        a.out.from[to] = entry[r].y;
      }
    __syncthreads();
    if (digit_thread) s.base[tid] += of_digit;
  }
}

// Clears the table beside the sort (whose few workgroups wait for memory most
// of the time): rows that slots name are written again later, which costs less
// than to wait for the sort's answer which those are.
struct ClearArgs {
  char* out;
  int64_t rows, row_bytes, stride, last_bytes;   // rows of row_bytes, the last one of last_bytes
  int threads;                                    // of a row: a workgroup or a wavefront
  int64_t row0, row1, blocks;                     // a launch's share of them and its workgroups
};

// Share `k` of `of` equal ones.
ClearArgs clear_share(ClearArgs c, int64_t k, int64_t of) {
  const int64_t per = kSortThreads / c.threads;
  c.row0 = c.rows * k / of;
  c.row1 = c.rows * (k + 1) / of;
  c.blocks = std::min<int64_t>((c.row1 - c.row0 + per - 1) / per, 1 << 20);
  return c;
}

__device__ __forceinline__ void clear_rows(const ClearArgs& c, int64_t block) {
  const Word4 zero{0, 0, 0, 0};
  const int per = kSortThreads / c.threads, lane = threadIdx.x & (c.threads - 1);
  for (int64_t r = c.row0 + block * per + threadIdx.x / c.threads; r < c.row1; r += c.blocks * per) {
    char* out = c.out + r * c.stride;
    const int64_t bytes = r == c.rows - 1 ? c.last_bytes : c.row_bytes;
    const int64_t vecs = bytes >> 4;
    for (int64_t v = lane; v < vecs; v += c.threads) store_words(out + (v << 4), zero);
    for (int64_t h = (vecs << 3) + lane; h < bytes >> 1; h += c.threads) reinterpret_cast<uint16_t*>(out)[h] = 0;
  }
}

__global__ __launch_bounds__(kSortThreads) void clear_kernel(const ClearArgs c) { clear_rows(c, blockIdx.x); }

// Few slots, in one launch: every workgroup owns 1 << bits table rows, looks
// through all ids for them (the L2 holds the ids), lists its slots in order (in
// LDS, or where they lie in the whole order: it has counted the smaller ids on
// the way), and sorts them by one pass.  The owner of the last rows takes
// the absent slots.
__global__ __launch_bounds__(kSortThreads) void sort_owned_kernel(const SortArgs a, const ClearArgs c) {
  __shared__ SortLds s;
  __shared__ uint2 s_list[kSortTile];
  __shared__ uint32_t s_below[kSortWaves];
  if (static_cast<int>(blockIdx.x) >= a.groups) {
    clear_rows(c, blockIdx.x - a.groups);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t first = blockIdx.x << a.bits, last = first + (1u << a.bits);
  // a wavefront's slots, 64 a round; kHeld rounds stay in registers, so up to
  // 16384 slots are read once and with one wait
  const int64_t per_wave = (a.slots + kSortThreads - 1) / kSortThreads * 64;
  const int64_t lo = wave * per_wave, hi = min(a.slots, lo + per_wave);
  constexpr int kHeld = 16;
  uint32_t key[kHeld];
  bool held = false;
  auto each = [&](auto&& fn) {
    for (int64_t at = lo; at < hi; at += 64 * kHeld) {
      if (!held) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
          key[u] = 0;
          if (at + u * 64 < hi) key[u] = min(static_cast<uint32_t>(a.ids[min(at + u * 64 + lane, a.slots - 1)]), a.rows);
        }
      }
#pragma unroll
      for (int u = 0; u < kHeld; ++u) {
        const int64_t mine = at + u * 64 + lane;
        if (at + u * 64 < hi) fn(mine, mine < hi, key[u]);
      }
    }
    held = per_wave <= 64 * kHeld;
  };
  uint32_t below = 0, own = 0;
  each([&](int64_t, bool live, uint32_t key) {
    below += __popcll(__ballot(live && key < first));
    own += __popcll(__ballot(live && key >= first && key < last));
  });
  if (lane == 0) {
    s_below[wave] = below;
    s.wave[wave] = own;
  }
  __syncthreads();
  uint32_t start = 0, to = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    start += s_below[w];
    if (w < wave) to += s.wave[w];
    total += s.wave[w];
  }
  to += start;
  if (total == 0) return;
  const bool in_lds = total <= kSortTile;
  if (own > 0)
    each([&](int64_t at, bool live, uint32_t key) {
      const bool mine = live && key >= first && key < last;
      const uint64_t hits = __ballot(mine);
      if (mine) {
        const uint32_t p = to + __popcll(hits & ((1ull << lane) - 1));
        const uint32_t from = a.bag == 1 ? static_cast<uint32_t>(at) : static_cast<uint32_t>(at) / static_cast<uint32_t>(a.bag);
        if (in_lds) {
          s_list[p - start] = {key, from};
        } else {
          a.in.key[p] = key;
          a.in.from[p] = from;
        }
      }
      to += __popcll(hits);
    });
  __syncthreads();
  auto sort = [&](auto&& src) {
    sort_count(a, src, start, start + total, s);
    const uint32_t n = s.base[tid];
    __syncthreads();
    const uint32_t base = sort_scan(n, s.wave);
    s.base[tid] = start + base;
    __syncthreads();
    sort_move(a, src, start, start + total, s);
  };
  if (in_lds) sort(FromLds{s_list, start});
  else sort(FromBuf{a.in});
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs a, int first, const ClearArgs c) {
  __shared__ SortLds s;
  if (static_cast<int>(blockIdx.x) >= a.groups) {
    clear_rows(c, blockIdx.x - a.groups);
    return;
  }
  const int64_t lo = blockIdx.x * a.per_group;
  const int64_t hi = min(a.slots, lo + a.per_group);
  if (first) sort_count(a, FromIds{a.ids, a.rows, static_cast<uint32_t>(a.bag)}, lo, hi, s);
  else sort_count(a, FromBuf{a.in}, lo, hi, s);
  if (threadIdx.x < (1u << a.bits)) a.hist[(blockIdx.x << a.bits) + threadIdx.x] = s.base[threadIdx.x];
}

__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(const SortArgs a, int first, const ClearArgs c) {
  __shared__ SortLds s;
  if (static_cast<int>(blockIdx.x) >= a.groups) {
    clear_rows(c, blockIdx.x - a.groups);
    return;
  }
  const int tid = threadIdx.x;
  uint32_t total = 0, before = 0;
  constexpr int kAtOnce = 8;
  if (tid < (1 << a.bits))
    for (int g = 0; g < a.groups; g += kAtOnce) {
      uint32_t n[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) n[u] = g + u < a.groups ? a.hist[((g + u) << a.bits) + tid] : 0;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (g + u < static_cast<int>(blockIdx.x)) before += n[u];
        total += n[u];
      }
    }
  const uint32_t base = sort_scan(total, s.wave);
  s.base[tid] = base + before;
  __syncthreads();
  const int64_t lo = blockIdx.x * a.per_group;
  const int64_t hi = min(a.slots, lo + a.per_group);
  if (first) sort_move(a, FromIds{a.ids, a.rows, static_cast<uint32_t>(a.bag)}, lo, hi, s);
  else sort_move(a, FromBuf{a.in}, lo, hi, s);
}

// ------------------------------------------------------------ summing runs
// Sorted slots of a piece: about kPieces of them fill the GPU, up to kLongPiece
// slots each; kMaxPieces bounds the longest join, so past 262144 slots a piece
// has 1 / 8192 of them (of 2^30 slots 131072, added one after another).
constexpr int64_t kPieces = 1024;
constexpr int64_t kLongPiece = 32;
constexpr int64_t kMaxPieces = 1 << 13;
constexpr int kAhead = 8;                  // gradient rows in flight per lane

struct SumArgs {
  const uint32_t* key;       // sorted
  const uint32_t* from;
  int64_t slots;
  int64_t pieces;
  int piece;
  float* partial;            // [pieces][2][pitch]: sums of runs that come in / go on
  int pitch;
  int lanes, col_blocks;
};

template <typename O, typename T>
__device__ __forceinline__ void put_row(const EmbedArgs& a, const LaneCols<T>& cols, uint32_t row, const float* sum) {
  constexpr int kE = Elem<T>::kPerVec;
  O* out = static_cast<O*>(a.out) + static_cast<int64_t>(row) * a.out_ld;
  float f[kE];
  if (a.accumulate) {
    cols.load_old(out, f);
#pragma unroll
    for (int e = 0; e < kE; ++e) f[e] += sum[e] * a.scale;
  } else {
#pragma unroll
    for (int e = 0; e < kE; ++e) f[e] = sum[e] * a.scale;
  }
  cols.store(out, f);
}

template <typename T, typename O>
__global__ __launch_bounds__(kEmbThreads) void embed_sum_kernel(const EmbedArgs a, const SumArgs s) {
  constexpr int kE = Elem<T>::kPerVec;
  const int64_t block = static_cast<int64_t>(blockIdx.x);
  const int lane = threadIdx.x & (s.lanes - 1);
  const int groups = kEmbThreads / s.lanes;
  const int64_t piece = block / s.col_blocks * groups + threadIdx.x / s.lanes;
  const int vec = static_cast<int>(block % s.col_blocks) * kEmbThreads + lane;
  if (piece >= s.pieces || vec * kE >= a.dim) return;
  const int64_t lo = piece * s.piece, hi = min(s.slots, lo + s.piece);
  const LaneCols<T> cols(vec, a.dim);
  const T* grad = static_cast<const T*>(a.grad);
  float* partial = s.partial + piece * 2 * s.pitch + vec * kE;
  const uint32_t rows = static_cast<uint32_t>(a.rows);
  bool came_in = lo > 0 && s.key[lo - 1] == s.key[lo];
  float sum[kE];
#pragma unroll
  for (int e = 0; e < kE; ++e) sum[e] = 0.0f;
  uint32_t run = s.key[lo];
  auto flush = [&](bool goes_on) {
    if (run >= rows) return;
    if (came_in || goes_on) {
      float* to = partial + (came_in ? 0 : s.pitch);
#pragma unroll
      for (int e = 0; e < kE; e += 4) *reinterpret_cast<float4*>(to + e) = {sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
    } else {
      put_row<O>(a, cols, run, sum);
    }
  };
  // Absent slots' rows are read too (their run is dropped), and past the end
  // the last slot's again: no load waits for a branch.  A step's keys are read
  // during the step before it.
  uint32_t key[kAhead], from[kAhead];
  auto read_keys = [&](int64_t at) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      key[u] = s.key[min(at + u, hi - 1)];
      from[u] = s.from[min(at + u, hi - 1)];
    }
  };
  read_keys(lo);
  for (int64_t at = lo; at < hi; at += kAhead) {
    Word4 w[kAhead];
    uint32_t now[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      w[u] = cols.load_raw(grad + static_cast<int64_t>(from[u]) * a.grad_ld);
      now[u] = key[u];
    }
    read_keys(at + kAhead);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (now[u] != run && at + u < hi) {
        flush(false);
        came_in = false;
        run = now[u];
#pragma unroll
        for (int e = 0; e < kE; ++e) sum[e] = 0.0f;
      }
      if (at + u < hi) {
        float f[kE];
        Elem<T>::unpack(w[u], f);
#pragma unroll
        for (int e = 0; e < kE; ++e) sum[e] += f[e];
      }
    }
  }
  flush(hi < s.slots && s.key[hi] == run);
}

// A run that starts in a piece and goes on over `count` more: one workgroup per
// piece and 64 vectors of columns (a CU reads some 40 GB/s, so a long run's
// columns are spread).  Its four wavefronts each add a quarter of the partial
// sums in order, and the quarters are added in order.
constexpr int kJoinWaves = 4;
constexpr uint32_t kJoinAhead = 8;              // partial sums in flight per lane
template <typename T, typename O>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(const EmbedArgs a, const SumArgs s,
                                                                     int col_blocks) {
  constexpr int kE = Elem<T>::kPerVec;
  __shared__ float s_sum[kJoinWaves - 1][kE][64];
  const int64_t piece = static_cast<int64_t>(blockIdx.x) / col_blocks;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t lo = piece * s.piece, hi = lo + s.piece;
  if (hi >= s.slots) return;
  const uint32_t run = s.key[hi - 1];
  if (run >= static_cast<uint32_t>(a.rows) || s.key[hi] != run) return;
  if (s.key[lo] == run && lo > 0 && s.key[lo - 1] == run) return;      // it started earlier
  int64_t count = 0;
  for (int64_t p = piece + 1;; p += 64 * kJoinWaves) {
    const bool in = p + tid < s.pieces && s.key[(p + tid) * s.piece] == run;
    const int n = __syncthreads_count(in ? 1 : 0);
    count += n;
    if (n < 64 * kJoinWaves) break;
  }
  const int vec = static_cast<int>(blockIdx.x % col_blocks) * 64 + lane;
  const bool live = vec * kE < a.dim;
  float sum[kE];
#pragma unroll
  for (int e = 0; e < kE; ++e) sum[e] = 0.0f;
  if (live) {
    const int64_t p1 = piece + 1 + count * (wave + 1) / kJoinWaves;
    int64_t p0 = piece + 1 + count * wave / kJoinWaves;
    auto from = [&](int64_t p, int side) { return s.partial + (p * 2 + side) * s.pitch + vec * kE; };
    if (wave == 0) {
      const float* first = from(piece, 1);
#pragma unroll
      for (int e = 0; e < kE; ++e) sum[e] = first[e];
    }
    for (; p0 < p1; p0 += kJoinAhead) {
      float4 f[kJoinAhead][kE / 4];
#pragma unroll
      for (uint32_t u = 0; u < kJoinAhead; ++u)
#pragma unroll
        for (int e = 0; e < kE / 4; ++e) f[u][e] = *reinterpret_cast<const float4*>(from(min(p0 + u, p1 - 1), 0) + 4 * e);
#pragma unroll
      for (uint32_t u = 0; u < kJoinAhead; ++u)
        if (p0 + u < p1) {
#pragma unroll
          for (int e = 0; e < kE / 4; ++e) {
            sum[4 * e] += f[u][e].x;
            sum[4 * e + 1] += f[u][e].y;
            sum[4 * e + 2] += f[u][e].z;
            sum[4 * e + 3] += f[u][e].w;
          }
        }
    }
  }
  if (wave > 0)
#pragma unroll
    for (int e = 0; e < kE; ++e) s_sum[wave - 1][e][lane] = sum[e];
  __syncthreads();
  if (wave > 0 || !live) return;
#pragma unroll
  for (int w = 0; w < kJoinWaves - 1; ++w)
#pragma unroll
    for (int e = 0; e < kE; ++e) sum[e] += s_sum[w][e][lane];
  put_row<O>(a, LaneCols<T>(vec, a.dim), run, sum);
}

// Few slots: one workgroup per sorted slot and 64 vectors of columns sums the
// run that starts at the slot (others leave at once), its four wavefronts a
// quarter each, so one launch does without pieces and joins (512 slots of 384
// columns: 14 us against 17; a run of all 1024 slots 44 against 21).
constexpr int64_t kRunSlots = 1024;
template <typename T, typename O>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_run_kernel(const EmbedArgs a, const SumArgs s,
                                                                    int col_blocks) {
  constexpr int kE = Elem<T>::kPerVec;
  __shared__ float s_sum[kJoinWaves - 1][kE][64];
  const int slots = static_cast<int>(s.slots);
  const int e = static_cast<int>(blockIdx.x) / col_blocks;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t run = s.key[e];
  if (run >= static_cast<uint32_t>(a.rows) || (e > 0 && s.key[e - 1] == run)) return;
  int count = 0;
  for (int at = e;; at += 64 * kJoinWaves) {
    const int n = __syncthreads_count(at + tid < slots && s.key[min(at + tid, slots - 1)] == run ? 1 : 0);
    count += n;
    if (n < 64 * kJoinWaves) break;
  }
  const int vec = static_cast<int>(blockIdx.x) % col_blocks * 64 + lane;
  const bool live = vec * kE < a.dim;
  const LaneCols<T> cols(live ? vec : 0, a.dim);
  float sum[kE];
#pragma unroll
  for (int j = 0; j < kE; ++j) sum[j] = 0.0f;
  const int hi = e + count * (wave + 1) / kJoinWaves;
  for (int at = e + count * wave / kJoinWaves; at < hi; at += kAhead) {
    uint32_t from[kAhead];
    Word4 w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) from[u] = s.from[min(at + u, hi - 1)];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      w[u] = cols.load_raw(static_cast<const T*>(a.grad) + static_cast<int64_t>(from[u]) * a.grad_ld);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (at + u < hi) {
        float f[kE];
        Elem<T>::unpack(w[u], f);
#pragma unroll
        for (int j = 0; j < kE; ++j) sum[j] += f[j];
      }
  }
  if (wave > 0)
#pragma unroll
    for (int j = 0; j < kE; ++j) s_sum[wave - 1][j][lane] = sum[j];
  __syncthreads();
  if (wave > 0 || !live) return;
#pragma unroll
  for (int q = 0; q < kJoinWaves - 1; ++q)
#pragma unroll
    for (int j = 0; j < kE; ++j) sum[j] += s_sum[q][j][lane];
  put_row<O>(a, cols, run, sum);
}

// ---------------------------------------------------------------- the plan
struct EmbedPlan {
  int bits, passes, groups;          // passes 0: sort_owned_kernel, groups owners
  int64_t per_group, pieces;
  int piece;
  int64_t off_a, off_b, off_hist, off_partial, bytes;
  int pitch;
};

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// clear_bytes: of the table's gradient (0: needs the most workspace).
EmbedPlan embed_plan(int64_t rows, int dim, int64_t slots, int64_t clear_bytes) {
  EmbedPlan p{};
  if (slots == 0) return p;                           // nothing to sort: the table is cleared at most
  int bits = 1;
  while ((rows >> bits) != 0) ++bits;                 // `rows` itself is a key
  int own = 6;
  while (own < kSortMaxBits && (rows >> own) >= kOwnersFull) ++own;
  if (slots <= kOwnedSlots + std::min(clear_bytes / kClearPerSlot, kOwnedSlots) && (rows >> own) < kMostOwners) {
    p.bits = own;
    p.groups = static_cast<int>((rows >> own) + 1);
  } else {
    p.passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const int64_t tiles = (slots + kSortTile - 1) / kSortTile;
    p.per_group = (tiles + kSortMaxGroups - 1) / kSortMaxGroups * kSortTile;
    p.groups = static_cast<int>((slots + p.per_group - 1) / p.per_group);
  }
  p.piece = static_cast<int>(round_up(
      std::max({std::min((slots + kPieces - 1) / kPieces, kLongPiece), (slots + kMaxPieces - 1) / kMaxPieces, int64_t{1}}),
      kAhead));
  p.pieces = slots <= kRunSlots ? 0 : (slots + p.piece - 1) / p.piece;
  p.pitch = static_cast<int>(round_up(dim, 8));
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t off = at;
    at += round_up(bytes, 256);
    return off;
  };
  p.off_a = take(slots * 8);
  p.off_b = take(slots * 8);
  p.off_hist = take(p.passes > 0 ? static_cast<int64_t>(p.groups) * 4 << p.bits : 0);
  p.off_partial = take(p.pieces * 2 * p.pitch * 4);
  p.bytes = at;
  return p;
}

template <typename T>
hipError_t lookup_typed(const EmbedArgs& a, hipStream_t s) {
  const int vecs = (a.dim + Elem<T>::kPerVec - 1) / Elem<T>::kPerVec;
  const int lanes = lanes_per_row(vecs), groups = kEmbThreads / lanes;
  const int col_blocks = (vecs + kEmbThreads - 1) / kEmbThreads;
  constexpr int kRows = 4;
  // Four rows a lane keep four loads in flight; fewer rows than fill the GPU
  // twice that way get a lane each.
  const bool many = a.n * lanes * col_blocks >= int64_t{2} * 256 * 1024 * kRows;
  const int per = groups * (many ? kRows : 1);
  const int64_t blocks = (a.n + per - 1) / per;
  constexpr int64_t kMost = 1 << 22;
  for (int64_t at = 0; at < blocks; at += kMost) {
    const dim3 grid(static_cast<unsigned>(std::min(blocks - at, kMost)), col_blocks);
    if (many) embed_lookup_kernel<T, kRows><<<grid, kEmbThreads, 0, s>>>(a, lanes, at);
    else embed_lookup_kernel<T, 1><<<grid, kEmbThreads, 0, s>>>(a, lanes, at);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Sorts the slots; its launches clear the table beside it (c.rows 0: nothing).
hipError_t sort_slots(const EmbedArgs& a, const EmbedPlan& p, int64_t slots, char* ws, const ClearArgs& c,
                      hipStream_t s, SumArgs& sum) {
  SortArgs o{};
  o.ids = a.ids;
  o.slots = slots;
  o.rows = static_cast<uint32_t>(a.rows);
  o.bag = a.bag;
  o.bits = p.bits;
  o.groups = p.groups;
  o.per_group = p.per_group;
  o.hist = reinterpret_cast<uint32_t*>(ws + p.off_hist);
  SortBufs buf[2];
  buf[0].key = reinterpret_cast<uint32_t*>(ws + p.off_a);
  buf[1].key = reinterpret_cast<uint32_t*>(ws + p.off_b);
  for (SortBufs& b : buf) b.from = b.key + slots;
  int to = 0;
  if (p.passes == 0) {
    o.in = buf[1];
    o.out = buf[0];
    const ClearArgs all = clear_share(c, 0, 1);
    sort_owned_kernel<<<static_cast<unsigned>(p.groups + all.blocks), kSortThreads, 0, s>>>(o, all);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  } else {
    const int launches = 2 * p.passes;
    for (int pass = 0; pass < p.passes; ++pass) {
      to = pass & 1;
      o.shift = pass * p.bits;
      o.in = buf[to ^ 1];
      o.out = buf[to];
      const ClearArgs one = clear_share(c, 2 * pass, launches), two = clear_share(c, 2 * pass + 1, launches);
      sort_count_kernel<<<static_cast<unsigned>(p.groups + one.blocks), kSortThreads, 0, s>>>(o, pass == 0, one);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      sort_move_kernel<<<static_cast<unsigned>(p.groups + two.blocks), kSortThreads, 0, s>>>(o, pass == 0, two);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
  }
  sum.key = buf[to].key;
  sum.from = buf[to].from;
  return hipSuccess;
}

template <typename T, typename O>
hipError_t gradient_typed(const EmbedArgs& a, hipStream_t s) {
  const int64_t slots = a.n * a.bag;
  const EmbedPlan p = embed_plan(a.rows, a.dim, slots, a.accumulate ? 0 : a.rows * a.dim * static_cast<int64_t>(sizeof(O)));
  char* ws = static_cast<char*>(a.workspace);
  ClearArgs c{};
  c.out = static_cast<char*>(a.out);
  c.rows = a.rows;
  c.row_bytes = c.last_bytes = static_cast<int64_t>(a.dim) * sizeof(O);
  c.stride = a.out_ld * static_cast<int64_t>(sizeof(O));
  c.threads = 64;
  if (c.stride == c.row_bytes) {
    // One run of bytes: 256 KB a workgroup, less where that leaves CUs idle
    // (512 MB and the sums: 142 us; 64 KB 145, 1 MB 156; stores that stay in
    // the caches 179).
    const int64_t all = c.rows * c.row_bytes;
    int64_t each = 262144;
    while (each > 16384 && all / each < 1024) each /= 2;
    c.row_bytes = c.stride = each;
    c.rows = (all + c.stride - 1) / c.stride;
    c.last_bytes = all - (c.rows - 1) * c.stride;
    c.threads = kSortThreads;
  }
  if (a.accumulate) c.rows = 0;
  SumArgs sum{};
  if (slots == 0) {
    const ClearArgs all = clear_share(c, 0, 1);
    clear_kernel<<<static_cast<unsigned>(all.blocks), kSortThreads, 0, s>>>(all);
    return hipGetLastError();
  }
  if (hipError_t e = sort_slots(a, p, slots, ws, c, s, sum); e != hipSuccess) return e;
  const int vecs = (a.dim + Elem<T>::kPerVec - 1) / Elem<T>::kPerVec;
  sum.slots = slots;
  sum.piece = p.piece;
  sum.pieces = p.pieces;
  sum.partial = reinterpret_cast<float*>(ws + p.off_partial);
  sum.pitch = p.pitch;
  sum.lanes = lanes_per_row(vecs);
  sum.col_blocks = (vecs + kEmbThreads - 1) / kEmbThreads;
  if (slots <= kRunSlots) {
    const int col_blocks = (vecs + 63) / 64;
    embed_run_kernel<T, O><<<static_cast<unsigned>(slots * col_blocks), 64 * kJoinWaves, 0, s>>>(a, sum, col_blocks);
    return hipGetLastError();
  }
  const int groups = kEmbThreads / sum.lanes;
  embed_sum_kernel<T, O><<<static_cast<unsigned>((p.pieces + groups - 1) / groups * sum.col_blocks), kEmbThreads, 0,
                           s>>>(a, sum);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || p.pieces <= 1) return e;
  const int col_blocks = (vecs + 63) / 64;
  embed_join_kernel<T, O><<<static_cast<unsigned>((p.pieces - 1) * col_blocks), 64 * kJoinWaves, 0, s>>>(a, sum, col_blocks);
  return hipGetLastError();
}

}  // namespace

int64_t embed_workspace_bytes(int64_t rows, int dim, int64_t slots) { return embed_plan(rows, dim, slots, 0).bytes; }

hipError_t launch_embed_lookup(const EmbedArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  switch (a.dtype) {
    case kElemF32: return lookup_typed<float>(a, s);
    case kElemF16: return lookup_typed<_Float16>(a, s);
    default: return lookup_typed<__bf16>(a, s);
  }
}

hipError_t launch_embed_gradient(const EmbedArgs& a, hipStream_t s) {
  const bool wide = a.out_dtype == kElemF32;
  switch (a.dtype) {
    case kElemF32: return gradient_typed<float, float>(a, s);
    case kElemF16: return wide ? gradient_typed<_Float16, float>(a, s) : gradient_typed<_Float16, _Float16>(a, s);
    default: return wide ? gradient_typed<__bf16, float>(a, s) : gradient_typed<__bf16, __bf16>(a, s);
  }
}

}  // namespace ifvs
