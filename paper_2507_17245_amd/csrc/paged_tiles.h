// Pieces of the bf16 kernels over a paged cache: direct loads of a page's rows, values that are no numbers.
#pragma once
#include "attn_bf16_impl.h"

namespace da {

namespace {

// One direct load into LDS: 16 bytes a lane from `offset` and `more` (of all lanes) bytes behind base, zeros where they end behind `bytes`.
// ONCE: what is read is not kept in the caches for longer.
template <bool ONCE = false>
__device__ inline void load_lds(const char* base, unsigned bytes, int offset, int more, char* to) {
  typedef __attribute__((address_space(3))) void lds_void;
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)to, 16, offset, more, 0, ONCE ? 2 : 0);
}

// Whether one of eight values is an infinity or a NaN.
__device__ inline bool has_odd(bf16x8 x) {
  const u32x4 b = __builtin_bit_cast(u32x4, x);
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) odd |= (b[j] & 0x7f80u) == 0x7f80u || (b[j] & 0x7f800000u) == 0x7f800000u;
  return odd;
}
template <int TT, int NMB, typename READ>
__device__ inline bool any_odd(READ operand) {
  bool odd = false;
#pragma unroll
  for (int tt = 0; tt < TT; ++tt) {
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb) odd |= has_odd(operand(tt, mb));
    __builtin_amdgcn_sched_barrier(0);
  }
  return __builtin_amdgcn_ballot_w64(odd) != 0;
}
// P.V of a tile whose keys not every row sees, and whose values hold an infinity or a NaN: the product would bring it to the rows with P = 0, too
// (0 times it). The finite values as they are; then, for either infinity and for NaN, the weight with which a row sees
// one: where that is not 0 it decides the row's result.
template <int TT, int NMB, typename READ>
__device__ inline void odd_values(f32x16 (&oacc)[NMB], const bf16x8 (&pop)[TT], READ operand) {
#pragma unroll
  for (int mb = 0; mb < NMB; ++mb) {
#pragma unroll 1
    for (int kind = 0; kind < 4; ++kind) {   // finite, infinity, minus infinity, NaN
      f32x16 z;
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = kind == 0 ? oacc[mb][i] : 0.0f;
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) {
        const s16x8 x = __builtin_bit_cast(s16x8, operand(tt, mb));
        s16x8 y;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int is = (x[j] & 0x7f80) != 0x7f80 ? 0 : (x[j] & 0x7f) != 0 ? 3 : x[j] < 0 ? 2 : 1;
          y[j] = is != kind ? (short)0 : kind == 0 ? x[j] : (short)0x3f80;
        }
        z = mfma_32x32x16(__builtin_bit_cast(bf16x8, y), pop[tt], z);
        __builtin_amdgcn_sched_barrier(0);   // (one operand's registers at a time)
      }
      const float what = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : __builtin_nanf("");
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[mb][i] = kind == 0 ? z[i] : oacc[mb][i] + (z[i] > 0.0f ? what : 0.0f);
    }
  }
}

}  // namespace

}  // namespace da
