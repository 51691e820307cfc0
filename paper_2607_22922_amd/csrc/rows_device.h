// Element types and row helpers of the row operators (k_embed.hip,
// k_rows.hip): loads and stores of fp32, fp16 and bf16 rows that start at any
// element, a row held in registers, and reductions in a fixed order.
#pragma once

#include "ifvs_internal.h"

namespace ifvs {

// Sixteen bytes at any element's alignment (one global_load_dwordx4: gfx950
// takes them unaligned).
typedef uint32_t Word4 __attribute__((ext_vector_type(4)));
typedef Word4 Word4At2 __attribute__((aligned(2)));

__device__ __forceinline__ Word4 load_words(const void* p) {
  return __builtin_nontemporal_load(static_cast<const Word4At2*>(p));
}
__device__ __forceinline__ Word4 load_words_again(const void* p) { return *static_cast<const Word4At2*>(p); }
__device__ __forceinline__ void store_words(void* p, Word4 w) {
  __builtin_nontemporal_store(w, static_cast<Word4At2*>(p));
}

template <typename T>
__device__ __forceinline__ float elem_load(const T* p) {
  return static_cast<float>(*p);
}

// One rounding, to nearest even (past the range of fp16: infinity).
template <typename T>
__device__ __forceinline__ T elem_round(float v) {
  return static_cast<T>(v);
}

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int kLowBit = 0;          // of an element's fp32 bits: below it all are 0
  static constexpr int kPerVec = 4;
  static constexpr uint32_t kNegInfWord = 0xFF800000u;
  static __device__ __forceinline__ void unpack(const Word4& w, float* f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(w[j]);
  }
  static __device__ __forceinline__ Word4 pack(const float* f) {
    Word4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(f[j]);
    return w;
  }
};
template <>
struct Elem<_Float16> {
  static constexpr int kLowBit = 13;          // of an element's fp32 bits: below it all are 0
  static constexpr int kPerVec = 8;
  static constexpr uint32_t kNegInfWord = 0xFC00FC00u;
  static __device__ __forceinline__ void unpack(const Word4& w, float* f) {
    typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
    const Half8 h = __builtin_bit_cast(Half8, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = static_cast<float>(h[j]);
  }
  static __device__ __forceinline__ Word4 pack(const float* f) {
    typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
    Half8 h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = static_cast<_Float16>(f[j]);
    return __builtin_bit_cast(Word4, h);
  }
};
template <>
struct Elem<__bf16> {
  static constexpr int kLowBit = 16;          // of an element's fp32 bits: below it all are 0
  static constexpr int kPerVec = 8;
  static constexpr uint32_t kNegInfWord = 0xFF80FF80u;
  static __device__ __forceinline__ void unpack(const Word4& w, float* f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[2 * j] = __uint_as_float(w[j] << 16);
      f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ Word4 pack(const float* f) {
    typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
    Bf8 h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = static_cast<__bf16>(f[j]);
    return __builtin_bit_cast(Word4, h);
  }
};

// ---- reductions over a wavefront, the same value in every lane: four steps
// on the vector unit's lane permutations (pairs, quads, eights, sixteens: no
// LDS), then the four sixteens through scalar registers.
template <int kCtrl>
__device__ __forceinline__ float lane_perm(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), kCtrl, 0xF, 0xF, true));
}
template <int kCtrl>
__device__ __forceinline__ double lane_perm(double v) {
  const int lo = __builtin_amdgcn_mov_dpp(__double2loint(v), kCtrl, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_mov_dpp(__double2hiint(v), kCtrl, 0xF, 0xF, true);
  return __hiloint2double(hi, lo);
}
constexpr int kPermXor1 = 0xB1, kPermXor2 = 0x4E, kPermHalfMirror = 0x141, kPermMirror = 0x140;

__device__ __forceinline__ float lane_of(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                          __builtin_amdgcn_readlane(__double2loint(v), lane));
}

__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, lane_perm<kPermXor1>(v));
  return fmaxf(v, lane_perm<kPermXor2>(v));
}
__device__ __forceinline__ float sixteen_max(float v) {
  v = quad_max(v);
  v = fmaxf(v, lane_perm<kPermHalfMirror>(v));
  return fmaxf(v, lane_perm<kPermMirror>(v));
}
__device__ __forceinline__ float wave_max(float v) {
  v = sixteen_max(v);
  return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ double wave_add(double v) {
  v += lane_perm<kPermXor1>(v);
  v += lane_perm<kPermXor2>(v);
  v += lane_perm<kPermHalfMirror>(v);
  v += lane_perm<kPermMirror>(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ double wave_max(double v) {
  v = fmax(v, lane_perm<kPermXor1>(v));
  v = fmax(v, lane_perm<kPermXor2>(v));
  v = fmax(v, lane_perm<kPermHalfMirror>(v));
  v = fmax(v, lane_perm<kPermMirror>(v));
  return fmax(fmax(lane_of(v, 0), lane_of(v, 16)), fmax(lane_of(v, 32), lane_of(v, 48)));
}

// A barrier that a workgroup of one wavefront does not need: its own LDS
// operations stay in order.
template <int kThreads>
__device__ __forceinline__ void group_sync() {
  if constexpr (kThreads > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Elements before the first 16-byte boundary at or after p, at most len.
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int len) {
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
  return min(len, ((16 - off) & 15) / static_cast<int>(sizeof(T)));
}

// Up to kThreads * kVecs aligned vectors of a row, and its edges (less than a
// vector before the first and after the last), in the registers of a
// workgroup: thread t holds vectors t, t + kThreads, ... and edge element t;
// places past the end hold -inf.  (Vectors that straddle cache lines cost a
// fifth: 2048 rows of 50001 fp16 logits 47 us unaligned, of 50048 39.)  Loops
// step over vector rounds that lie wholly past the end.
template <typename T, int kThreads, int kVecs>
struct RowTile {
  static constexpr int kE = Elem<T>::kPerVec;
  static constexpr int kCapacity = kThreads * kVecs * kE;
  Word4 v[kVecs];
  float edge;
  int head, nvec, nedge;       // elements before the first vector, vectors, edge elements

  // The layout of len elements at x, without reading them.
  __device__ __forceinline__ void place(const T* x, int len) {
    head = head_of(x, len);
    nvec = (len - head) / kE;
    nedge = len - nvec * kE;
  }
  // kOnce: nothing reads these bytes again soon (they pass the caches by).
  template <bool kOnce = true>
  __device__ __forceinline__ void load(const T* x, int len) {
    const int tid = threadIdx.x;
    place(x, len);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      // a scalar base and bound per round, one offset per thread
      const char* from = reinterpret_cast<const char*>(x + head) + static_cast<int64_t>(i) * kThreads * 16;
      v[i] = Word4{Elem<T>::kNegInfWord, Elem<T>::kNegInfWord, Elem<T>::kNegInfWord, Elem<T>::kNegInfWord};
      if (tid < nvec - i * kThreads) v[i] = kOnce ? load_words(from + tid * 16u) : load_words_again(from + tid * 16u);
    }
    edge = tid < nedge ? elem_load(x + edge_column()) : -INFINITY;
  }
  __device__ __forceinline__ bool has(int i) const { return i * kThreads < nvec; }
  __device__ __forceinline__ int column(int i, int j) const {
    return head + (i * kThreads + static_cast<int>(threadIdx.x)) * kE + j;
  }
  __device__ __forceinline__ int edge_column() const {
    const int tid = threadIdx.x;
    return tid < head ? tid : nvec * kE + tid;
  }
  // A bit per column: byte and bit of a column; the edges' two bytes follow
  // the vectors'.
  static constexpr int kBitBytes = kThreads * kVecs + 2;
  __device__ __forceinline__ int bit_of(int column) const {
    const int in = column - head;
    if (in >= 0 && in < nvec * kE) return in / kE * 8 + in % kE;
    return kThreads * kVecs * 8 + (in < 0 ? column : column - nvec * kE);
  }

  // The thread's elements one by one: f(x, column).
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (static_cast<int>(threadIdx.x) < nvec - i * kThreads) {
        float y[kE];
        Elem<T>::unpack(v[i], y);
#pragma unroll
        for (int j = 0; j < kE; ++j) f(y[j], column(i, j));
        __builtin_amdgcn_sched_barrier(0);
      }
    if (static_cast<int>(threadIdx.x) < nedge) f(edge, edge_column());
  }

  // The same from memory, for rare paths that must not cost the others
  // registers.
  template <typename F>
  __device__ __forceinline__ void each_from_memory(const T* x, F&& f) const {
#pragma unroll 1
    for (int i = 0; i < kVecs; ++i)
      if (static_cast<int>(threadIdx.x) < nvec - i * kThreads)
#pragma unroll 1
        for (int j = 0; j < kE; ++j) f(elem_load(x + column(i, j)), column(i, j));
    if (static_cast<int>(threadIdx.x) < nedge) f(elem_load(x + edge_column()), edge_column());
  }

  // The same a vector a load, columns ascending (an edge before the vectors, or
  // the one after them), until f returns false.  f sees all of a vector.
  template <typename F>
  __device__ __forceinline__ void each_vector_from_memory(const T* x, F&& f) const {
    const int tid = threadIdx.x;
    if (tid < head && !f(elem_load(x + tid), tid)) return;
#pragma unroll 1
    for (int i = 0; i < kVecs && tid < nvec - i * kThreads; ++i) {
      float y[kE];
      Elem<T>::unpack(load_words_again(x + column(i, 0)), y);
      bool more = true;
#pragma unroll
      for (int j = 0; j < kE; ++j) more = f(y[j], column(i, j)) && more;
      if (!more) return;
    }
    if (tid >= head && tid < nedge) f(elem_load(x + edge_column()), edge_column());
  }

  // Between two passes over the tile: the compiler would keep every unpacked
  // element of the first alive for the second (two to three times the registers).
  __device__ __forceinline__ void forget_unpacked() {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) asm volatile("" : "+v"(v[i]));
  }

  // Maximum of the thread's elements (NaN ones are passed over).
  __device__ __forceinline__ float thread_max() const {
    float m = edge;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (has(i)) {
        float f[kE];
        Elem<T>::unpack(v[i], f);
#pragma unroll
        for (int j = 0; j < kE; j += 2) m = fmaxf(fmaxf(m, f[j]), f[j + 1]);
      }
    return m;
  }
};

}  // namespace ifvs
