// Embedding lookup and the gradient of its table (Section 2, opening
// paragraph: alpha is a sum of rows of a table; the training paragraph sends
// gradients back into the rows).
//
//   lookup:   out[i] = scale * sum over j of table[ids[i][j]]
//   gradient: G[r] = scale * sum over the slots (i, j) that name r of grad[i]
#include <cmath>

#include "rows_device.h"

namespace ifvs {

namespace {

constexpr int kEmbThreads = 256;

// One workgroup per output row.
template <typename T>
__global__ __launch_bounds__(kEmbThreads) void embed_lookup_kernel(const EmbedArgs a) {
  const T* table = static_cast<const T*>(a.table);
  T* out = static_cast<T*>(a.out);
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x)
    for (int d = threadIdx.x; d < a.dim; d += kEmbThreads) {
      float sum = 0.0f;
      for (int j = 0; j < a.bag; ++j) {
        const int64_t id = a.ids[i * a.bag + j];
        if (id >= 0 && id < a.rows) sum += elem_load(table + id * a.table_ld + d);
      }
      out[i * a.out_ld + d] = elem_round<T>(sum * a.scale);
    }
}

// One workgroup per table row: it looks through all slots in order.
template <typename T, typename O>
__global__ __launch_bounds__(kEmbThreads) void embed_gradient_kernel(const EmbedArgs a) {
  __shared__ int64_t s_hit[kEmbThreads];
  const T* grad = static_cast<const T*>(a.grad);
  O* out = static_cast<O*>(a.out);
  const int64_t slots = a.n * a.bag;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x)
    for (int d0 = 0; d0 < a.dim; d0 += kEmbThreads) {
      const int d = d0 + threadIdx.x;
      float sum = 0.0f;
      bool any = false;
      for (int64_t s0 = 0; s0 < slots; s0 += kEmbThreads) {
        const int64_t s = s0 + threadIdx.x;
        const bool hit = s < slots && a.ids[s] == r;
        if (!__syncthreads_or(hit ? 1 : 0)) continue;
        s_hit[threadIdx.x] = hit ? s / a.bag : -1;
        __syncthreads();
        for (int e = 0; e < kEmbThreads; ++e)
          if (s_hit[e] >= 0) {
            any = true;
            if (d < a.dim) sum += elem_load(grad + s_hit[e] * a.grad_ld + d);
          }
        __syncthreads();
      }
      if (d < a.dim && (any || !a.accumulate)) {
        const float old = a.accumulate ? elem_load(out + r * a.out_ld + d) : 0.0f;
        out[r * a.out_ld + d] = elem_round<O>(old + sum * a.scale);
      }
    }
}

}  // namespace

int64_t embed_workspace_bytes(int64_t, int, int64_t) { return 0; }

hipError_t launch_embed_lookup(const EmbedArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(a.n < 65536 ? a.n : 65536)), block(kEmbThreads);
  switch (a.dtype) {
    case kElemF32: embed_lookup_kernel<float><<<grid, block, 0, s>>>(a); break;
    case kElemF16: embed_lookup_kernel<_Float16><<<grid, block, 0, s>>>(a); break;
    default: embed_lookup_kernel<__bf16><<<grid, block, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

hipError_t launch_embed_gradient(const EmbedArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.rows < 65536 ? a.rows : 65536)), block(kEmbThreads);
  const bool wide = a.out_dtype == kElemF32;
  switch (a.dtype) {
    case kElemF32: embed_gradient_kernel<float, float><<<grid, block, 0, s>>>(a); break;
    case kElemF16:
      if (wide) embed_gradient_kernel<_Float16, float><<<grid, block, 0, s>>>(a);
      else embed_gradient_kernel<_Float16, _Float16><<<grid, block, 0, s>>>(a);
      break;
    default:
      if (wide) embed_gradient_kernel<__bf16, float><<<grid, block, 0, s>>>(a);
      else embed_gradient_kernel<__bf16, __bf16><<<grid, block, 0, s>>>(a);
      break;
  }
  return hipGetLastError();
}

}  // namespace ifvs
