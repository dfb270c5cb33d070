// Attention of new tokens over a paged cache of 4-bit codes (fp4.h), float tensors in float arithmetic. Kernel and work split: paged_f32.h.
//
// Bound: the float products. Keys are converted behind their products' other operands; a lane's channels of V (two at d = 64, four at 128) are a
// byte or two of a row, asked for key by key.
#include "fp4.h"
#include "paged_f32.h"

namespace da {

namespace {

// Where a key lies: offsets of its row's codes and scales in a kv head's pages.
struct Window4 {
  uint64_t code, scale;
  int there;
};

template <int D>
struct CodePages {
  static constexpr int NMB = D / 32, HALF = D / 2;
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  int64_t code_page, code_head, code_row, scale_page, scale_head, scale_row;   // bytes

  typedef Window4 Window;
  struct Head {
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    int64_t code_page, code_row, scale_page, scale_row;
    int lq, hh;
    __device__ Head(const CodePages& p, int head, int lq, int hh)
        : k_codes(p.k_codes + head * p.code_head), k_scales(p.k_scales + head * p.scale_head), v_codes(p.v_codes + head * p.code_head),
          v_scales(p.v_scales + head * p.scale_head), code_page(p.code_page), code_row(p.code_row), scale_page(p.scale_page), scale_row(p.scale_row),
          lq(lq), hh(hh) {}
    __device__ Window window(const int* __restrict__ table, int key, int n_keys, int page_size, int n_pages) const {
      Window w = {0, 0, 0};
      if (key < n_keys) {
        const unsigned page = (unsigned)key / (unsigned)page_size;
        const int id = table[page], row = (int)((unsigned)key - page * (unsigned)page_size);
        if (id >= 0 && id < n_pages) w = Window{(uint64_t)(id * code_page + row * code_row), (uint64_t)(id * scale_page + row * scale_row), 1};
      }
      return w;
    }
  };
  struct Keys {
    uint32_t codes[HALF / 8];
    int scale[HALF / 32];
    // (of an absent key the cache's first row is read, and taken as zeros)
    __device__ void load(const Head& h, const Window& w) {
      const u32x4* from = (const u32x4*)(h.k_codes + w.code + h.hh * (HALF / 2));
#pragma unroll
      for (int s = 0; s < HALF / 32; ++s) {
        const u32x4 x = from[s];
#pragma unroll
        for (int j = 0; j < 4; ++j) codes[4 * s + j] = w.there ? x[j] : 0u;
        const int e = h.k_scales[w.scale + h.hh * (HALF / 32) + s];
        scale[s] = w.there ? e : 0;
      }
    }
    __device__ float value(int s) const {
      const uint32_t c = codes[s / 8];
      const float by = scale_value(scale[s / 32]);
      f32x2 y;
      switch (s / 2 % 4) {
        case 0: y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, by, 0); break;
        case 1: y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, by, 1); break;
        case 2: y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, by, 2); break;
        default: y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, by, 3);
      }
      return y[s & 1];
    }
  };
  struct Values {
    uint32_t codes[16], scale[16];
    __device__ void load(const Head& h, const Window& w, uint32_t there, int left) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        auto lane_of = [&](uint64_t x) {
          return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, 16 * g) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), 16 * g) << 32;
        };
        const int rows = min(left - 16 * g, 16), code_row = (int)h.code_row, scale_row = (int)h.scale_row;
        const bool is = there >> (16 * g) & 1;
        const __amdgpu_buffer_rsrc_t code_rsrc = head_rsrc(h.v_codes + lane_of(w.code), is ? (unsigned)((rows - 1) * code_row + D / 2) : 0u);
        const __amdgpu_buffer_rsrc_t scale_rsrc = head_rsrc(h.v_scales + lane_of(w.scale), is ? (unsigned)((rows - 1) * scale_row + D / 32) : 0u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int more = 8 * (j >> 2) + (j & 3);
          if constexpr (NMB == 4) codes[8 * g + j] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(code_rsrc, 4 * h.hh * code_row + h.lq * 2, more * code_row, 0);
          else codes[8 * g + j] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(code_rsrc, 4 * h.hh * code_row + h.lq, more * code_row, 0);
          scale[8 * g + j] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(scale_rsrc, 4 * h.hh * scale_row + h.lq * NMB / 32, more * scale_row, 0);
        }
      }
    }
    __device__ void get(float (&to)[16][NMB]) const {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], scale_value(scale[i]), 0);
        to[i][0] = lo[0];
        to[i][1] = lo[1];
        if constexpr (NMB == 4) {
          const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], scale_value(scale[i]), 1);
          to[i][2] = hi[0];
          to[i][3] = hi[1];
        }
      }
    }
  };
};

template <int D>
hipError_t launch_d(const void* q, void* o, const da_cache4& c, const da_paged& p, float scale, void* scratch, size_t scratch_bytes, hipStream_t stream) {
  const CodePages<D> pages = {(const uint8_t*)c.k_codes, (const uint8_t*)c.k_scales, (const uint8_t*)c.v_codes, (const uint8_t*)c.v_scales,
                              c.code_stride[0], c.code_stride[1], c.code_stride[2], c.scale_stride[0], c.scale_stride[1], c.scale_stride[2]};
  return launch_paged_f32_as<CodePages<D>, D>(q, pages, o, p, scale, scratch, paged_f32_launch(p, scratch_bytes), stream);
}

}  // namespace

size_t paged4_f32_scratch_bytes(const da_paged& p) { return paged_launch_bytes(paged_f32_resident(p), kRows, p.d); }

hipError_t launch_paged4_f32(const void* q, void* o, const da_cache4& cache, const da_paged& p, float scale, void* scratch, size_t scratch_bytes,
                             hipStream_t stream) {
  return p.d == 64 ? launch_d<64>(q, o, cache, p, scale, scratch, scratch_bytes, stream) : launch_d<128>(q, o, cache, p, scale, scratch, scratch_bytes, stream);
}

}  // namespace da
