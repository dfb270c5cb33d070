// Declarations of the kernels around attention: query/key norms and rotation, paged cache.
#pragma once
#include "../../include/distr_attn.h"
#include "da_common.h"

namespace da {

// Norm and rotation of queries ([0]) and keys ([1]; no heads: none). Strides of a batch, a head, a row, in elements: in_stride
// of x (backward: and of its gradient y), out_stride of y (backward: of the gradient g).
struct QkProblem {
  int B, N, d, dtype;
  int heads[2];
  const void* x[2];
  const void* g[2];
  void* y[2];
  int64_t in_stride[2][3], out_stride[2][3];
  const void* weight[2];
  da_rotary rotary;
  const int32_t* positions;
};
hipError_t launch_qk_forward(const QkProblem& p, hipStream_t stream);
size_t qk_backward_scratch_bytes(const QkProblem& p);
// part: qk_backward_scratch_bytes, or null where neither weight gradient is asked for
hipError_t launch_qk_backward(const QkProblem& p, float* const dweight[2], float* part, hipStream_t stream);

hipError_t launch_cache_append(const void* k, const void* v, void* k_pages, void* v_pages, const da_paged& p, hipStream_t stream);

// Attention over the pages. Scratch for the sums of keys that are dealt out: paged_scratch_bytes at most; with less (or none) the
// kernels take fewer workgroups or keep a row's keys together.
size_t paged_scratch_bytes(const da_paged& p);
hipError_t launch_paged(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                        size_t scratch_bytes, hipStream_t stream);
size_t paged_f32_scratch_bytes(const da_paged& p);
hipError_t launch_paged_f32(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                            size_t scratch_bytes, hipStream_t stream);

// The same over a cache of 4-bit codes.
hipError_t launch_cache4_append(const void* k, const void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream);
hipError_t launch_cache4_read(void* k, void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream);
size_t paged4_scratch_bytes(const da_paged& p);
hipError_t launch_paged4(const void* q, void* o, const da_cache4& cache, const da_paged& p, float scale, void* scratch, size_t scratch_bytes,
                         hipStream_t stream);
size_t paged4_f32_scratch_bytes(const da_paged& p);
hipError_t launch_paged4_f32(const void* q, void* o, const da_cache4& cache, const da_paged& p, float scale, void* scratch, size_t scratch_bytes,
                             hipStream_t stream);

}  // namespace da
