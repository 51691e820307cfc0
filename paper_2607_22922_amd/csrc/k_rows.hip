// Row operators over logits: log probabilities of given columns with the
// row's entropy and its best columns, and the distillation loss with its
// gradient (the training paragraph of Section 2 follows labels; these follow
// scores).
//
// Both rest on one row statistic.  With c = log2(e) / tau and a reference b
// near max(x) c, e_v = 2^(x_v c - b): one fused multiply-add whose only
// rounding is that of the small exponent, so rows far from 0 lose nothing.
// Then S = sum e_v, log2 q_v = x_v c - b - log2 S, and the entropy is
// log S - (sum e_v (x_v c - b)) ln 2 / S: every term has one sign.
// Maximum times c can pass the range of fp32 (masks of the lowest value);
// such rows take (x - max) c instead.
#include <cmath>

#include "rows_device.h"

namespace ifvs {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;
constexpr float kExpFloor = -200.0f;          // 2^-200 is 0 in fp32
constexpr double kLn2 = 0.69314718055994530942;

// The exponent of a column relative to the row's reference.
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

__device__ __forceinline__ int64_t row_cols(const int32_t* n_valid, int64_t i, int64_t cols) {
  if (!n_valid) return cols;
  const int64_t v = n_valid[i];
  return v < 0 ? 0 : (v < cols ? v : cols);
}

// One workgroup per row: three passes over it, then one per alternative.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void log_probs_kernel(const LogProbArgs a) {
  __shared__ double s_red[kRowWaves];
  __shared__ float s_val[kRowWaves];
  __shared__ int s_at[kRowWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t i = blockIdx.x;
  const T* x = static_cast<const T*>(a.logits) + i * a.ld;
  const int len = static_cast<int>(row_cols(a.n_valid, i, a.cols));
  float mx = -INFINITY;
  double bad = 0.0;
  for (int v = tid; v < len; v += kRowThreads) {
    const float f = elem_load(x + v);
    if (isnan(f) || f == INFINITY) bad = 1.0;
    mx = fmaxf(mx, f);
  }
  mx = block_max<kRowWaves>(mx, s_red);
  const RowRef ref = row_ref(mx, a.c);
  float sum = 0.0f, wsum = 0.0f;
  for (int v = tid; v < len; v += kRowThreads) {
    const float z = ref.exponent(elem_load(x + v));
    const float e = exp2f(z);
    sum += e;
    wsum += e * fmaxf(z, kExpFloor);
  }
  const double S = block_add<kRowWaves>(sum, s_red);
  const double Z = block_add<kRowWaves>(wsum, s_red);
  const bool nan = block_add<kRowWaves>(bad, s_red) > 0.0;
  const bool empty = mx == -INFINITY;           // no column above -inf: no distribution
  const double log2S = log2(S);
  auto logp = [&](float f) -> float {
    if (nan) return NAN;
    if (empty) return -INFINITY;
    return static_cast<float>((ref.exponent64(f) - log2S) * kLn2);
  };
  if (a.entropy_out && tid == 0)
    a.entropy_out[i] = nan ? NAN : (empty ? 0.0f : static_cast<float>((log2S - Z / S) * kLn2));
  for (int g = tid; g < a.n_given; g += kRowThreads) {
    const int64_t v = a.given[i * a.n_given + g];
    a.given_out[i * a.n_given + g] = v >= 0 && v < len ? logp(elem_load(x + v)) : -INFINITY;
  }
  float last = INFINITY;
  int last_at = -1;
  for (int t = 0; t < a.n_top; ++t) {
    float best = -INFINITY;
    int at = len;
    if (!nan)
      for (int v = tid; v < len; v += kRowThreads) {
        const float f = elem_load(x + v);
        if ((f < last || (f == last && v > last_at)) && f > best) {
          best = f;
          at = v;
        }
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float f = __shfl_xor(best, o, 64);
      const int v = __shfl_xor(at, o, 64);
      if (f > best || (f == best && v < at)) {
        best = f;
        at = v;
      }
    }
    if (lane == 0) {
      s_val[wave] = best;
      s_at[wave] = at;
    }
    __syncthreads();
    best = s_val[0];
    at = s_at[0];
    for (int w = 1; w < kRowWaves; ++w)
      if (s_val[w] > best || (s_val[w] == best && s_at[w] < at)) {
        best = s_val[w];
        at = s_at[w];
      }
    __syncthreads();
    const bool none = best == -INFINITY;
    if (tid == 0) {
      a.top_ids_out[i * a.n_top + t] = none ? -1 : at;
      a.top_out[i * a.n_top + t] = none ? (nan ? NAN : -INFINITY) : logp(best);
    }
    if (!none) {
      last = best;
      last_at = at;
    } else {
      last = -INFINITY;
    }
  }
}

// One workgroup per row.  The teacher's probabilities are held in LDS; a
// column's teacher probability is looked up among the slots.
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
  const int len = static_cast<int>(row_cols(a.n_valid, i, a.cols));
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
  const RowRef ref = row_ref(mx, a.c), ref_rest = row_ref(mx_rest, a.c);
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

int64_t log_probs_workspace_bytes(int64_t, int64_t, int) { return 0; }
int64_t distill_workspace_bytes(int64_t, int64_t) { return 0; }

hipError_t launch_log_probs(const LogProbArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(a.n)), block(kRowThreads);
  switch (a.dtype) {
    case kElemF32: log_probs_kernel<float><<<grid, block, 0, s>>>(a); break;
    case kElemF16: log_probs_kernel<_Float16><<<grid, block, 0, s>>>(a); break;
    default: log_probs_kernel<__bf16><<<grid, block, 0, s>>>(a); break;
  }
  return hipGetLastError();
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
