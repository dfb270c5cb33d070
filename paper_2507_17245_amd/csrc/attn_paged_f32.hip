// Attention of new tokens over a paged cache, float tensors in float arithmetic: the reference-precision form of attn_paged.hip. Kernel and
// work split: paged_f32.h.
//
// Bound: the float products, 1/16 of the bf16 rate. A lane's operands are 16-byte loads (V at d = 64: 8).
// Measured, us: three chunks of up to 48 on up to 700, H8 d64 17.7 (latency: 13, and the combine kernel's 4.2); 100 tokens on 2000, H16 Hkv4 d128 51;
// 16 chunks of 40 on up to 2000, H8 d64 63 (27 % of the products' rate: each unit reads the keys again, K one tile ahead); 64 single tokens of up to
// 8192, H32 Hkv8 d64 335 (3.7 TB/s). The kernel as a template for both caches takes 1 % more at d = 64 and the same at d = 128.
#include "paged_f32.h"

namespace da {

namespace {

template <int D>
struct FloatPages {
  static constexpr int NMB = D / 32, HALF = D / 2;
  const char *k, *v;
  int64_t page_bytes, head_bytes, row_bytes;

  typedef PageWindow Window;
  struct Head {
    const char *k, *v;
    int64_t page_bytes, row_bytes;
    int lq, hh;
    __device__ Head(const FloatPages& p, int head, int lq, int hh)
        : k(p.k + head * p.head_bytes), v(p.v + head * p.head_bytes), page_bytes(p.page_bytes), row_bytes(p.row_bytes), lq(lq), hh(hh) {}
    __device__ Window window(const int* __restrict__ table, int key, int n_keys, int page_size, int n_pages) const {
      return page_window(table, key, n_keys, page_size, n_pages, page_bytes, row_bytes);
    }
  };
  // (of an absent key, the cache's first row)
  struct Keys {
    float x[HALF];
    __device__ void load(const Head& h, const Window& w) {
      const char* at = h.k + (w.lo | (uint64_t)w.hi << 32) + h.hh * HALF * 4;
#pragma unroll
      for (int s = 0; s < HALF; s += 4) {
        const f32x4 y = *(const f32x4*)(at + s * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[s + j] = w.there ? y[j] : 0.0f;
      }
    }
    __device__ float value(int s) const { return x[s]; }
  };
  // By the tile's two groups of 16 keys, which lie in a page each: rows that are absent come as zeros.
  struct Values {
    float x[16][NMB];
    __device__ void load(const Head& h, const Window& w, uint32_t there, int left) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const uint64_t off = (uint32_t)__builtin_amdgcn_readlane((int)w.lo, 16 * g) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)w.hi, 16 * g) << 32;
        const int rows = min(left - 16 * g, 16), row = (int)h.row_bytes;
        const unsigned bytes = there >> (16 * g) & 1 ? (unsigned)((rows - 1) * row + D * 4) : 0u;
        const __amdgpu_buffer_rsrc_t rsrc = head_rsrc(h.v + off, bytes);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = 4 * h.hh * row + h.lq * NMB * 4, more = (8 * (j >> 2) + (j & 3)) * row;
          if constexpr (NMB == 4) {
            const f32x4 y = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, more, 0));
#pragma unroll
            for (int mb = 0; mb < 4; ++mb) x[8 * g + j][mb] = y[mb];
          } else {
            const f32x2 y = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, more, 0));
            x[8 * g + j][0] = y[0];
            x[8 * g + j][1] = y[1];
          }
        }
      }
    }
    __device__ void get(float (&to)[16][NMB]) const {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb) to[i][mb] = x[i][mb];
    }
  };
};

template <int D>
hipError_t launch_d(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                    size_t scratch_bytes, hipStream_t stream) {
  const FloatPages<D> pages = {(const char*)k_pages, (const char*)v_pages, p.page_stride * 4, p.head_stride * 4, p.row_stride * 4};
  return launch_paged_f32_as<FloatPages<D>, D>(q, pages, o, p, scale, scratch, paged_f32_launch(p, scratch_bytes), stream);
}

}  // namespace

size_t paged_f32_scratch_bytes(const da_paged& p) { return paged_launch_bytes(paged_f32_resident(p), kRows, p.d); }

hipError_t launch_paged_f32(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                            size_t scratch_bytes, hipStream_t stream) {
  return p.d == 64 ? launch_d<64>(q, k_pages, v_pages, o, p, scale, scratch, scratch_bytes, stream)
                   : launch_d<128>(q, k_pages, v_pages, o, p, scale, scratch, scratch_bytes, stream);
}

}  // namespace da
