// New keys and values into a paged cache of 4-bit codes, and out of it again (fp4.h has the form).
//
// Bound: k and v and their codes, each moved once. A workgroup takes successive rows, heads fastest; one wave finds where their tokens lie.
// Append: lanes as in cache_append.hip, two pieces of eight channels each; the scale of 32 channels is the largest of its four pieces' (which lanes
// of one row hold, wherever the rotation puts them), exchanged through LDS.
// The codes are those of the exact row: with norm or rotation the row is taken in 32 bits with a bound on its error, and where a code or a scale
// differs between the two ends of that bound (one wave of a hundred), the wave takes its rows again in 64 bits.
// Read: a lane converts eight channels, 4 bytes to 16 or 32.
#include "fp4.h"
#include "token_rows.h"

namespace da {

namespace {

constexpr int kThreads4 = 256, kMostTokens4 = 64;

struct Cache4 {   // strides in bytes
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  int64_t code_page, code_head, code_row, scale_page, scale_head, scale_row;
};
struct Batch4 {
  const int* __restrict__ page_table;
  const int* __restrict__ kv_len;
  const int* __restrict__ q_start;
  int Hkv, n_seq, n_tokens, n_pages, page_size, max_pages;
};
struct Tokens4 {     // of a workgroup that reads
  int tokens;
  uint32_t by_heads; // 2^31 / Hkv, rounded up: 2 x * by_heads >> 32 is x / Hkv for x < 2^16 (several tokens to a workgroup, so Hkv < 2^15)
};

// Where the workgroup's tokens lie.
struct Places4 {
  int at[kMostTokens4];   // place in the sequence; -1: none in the cache
  int64_t code[kMostTokens4], scale[kMostTokens4];
  __device__ void find(const Cache4& cache, const Batch4& b, int first) {   // of the tokens from `first` on
    if (threadIdx.x < 64) {
      const int token = min(first + (int)threadIdx.x, b.n_tokens - 1);
      const bool real = first + (int)threadIdx.x < b.n_tokens;
      const TokenPlace place(token, real, b.q_start, b.kv_len, b.page_table, b.n_seq, b.page_size, b.max_pages);
      const bool is = real && place.page >= 0 && place.page < b.n_pages;
      const int row = is ? place.at % (unsigned)b.page_size : 0, page = is ? place.page : 0;
      at[threadIdx.x] = is ? place.at : -1;
      code[threadIdx.x] = page * cache.code_page + row * cache.code_row;
      scale[threadIdx.x] = page * cache.scale_page + row * cache.scale_row;
    }
    __syncthreads();
  }
};
// Row `pair` of the workgroup's: its token there and its head.
__device__ inline void row_of(const Tokens4& w, int Hkv, unsigned pair, int& token, int& head) {
  token = w.tokens == 1 ? 0 : (int)__umulhi(2 * pair, w.by_heads);
  head = (int)pair - token * Hkv;
}

template <int LPR>
__device__ inline double row_sum(double x) {
#pragma unroll
  for (int i = 1; i < LPR; i *= 2) x += __shfl_xor(x, i, LPR);
  return x;
}

// A lane's sixteen channels of a row in 64 bits; weights and angles are loaded again.
template <typename E, int D, int ROPE>
__device__ inline void exact_row(double (&y)[16], const Eight<E> (&row)[2], const void* weight, const Rotary& r, int head, const LanePlace<ROPE>& at, int pos) {
  constexpr int LPR = D / 16;
  float x[16];
  row[0].values(x);
  row[1].values(x + 8);
#pragma unroll
  for (int j = 0; j < 16; ++j) y[j] = (double)x[j];
  if (r.norm) {
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < 16; ++j) s += y[j] * y[j];
    const double rms = 1.0 / __builtin_sqrt(row_sum<LPR>(s) * (1.0 / (16 * LPR)) + (double)r.eps);
    load_weight<D>(x, weight, r, head, at);
#pragma unroll
    for (int j = 0; j < 16; ++j) y[j] = y[j] * rms * (double)x[j];
  }
  if (at.turn) {
    Angles t;
    t.load(r, pos, at.pair, true);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int ia = ROPE == 1 ? j : 2 * j, ib = ROPE == 1 ? 8 + j : 2 * j + 1;
      const double a = y[ia], b = y[ib], c = t.c[j], s = t.s[j];
      y[ia] = a * c - b * s;
      y[ib] = a * s + b * c;
    }
  }
}

// Largest of eight magnitudes; NaN stays.
template <typename T>
__device__ inline T most_of(const T* x) {
  T m = __builtin_elementwise_abs(x[0]);
#pragma unroll
  for (int j = 1; j < 8; ++j) m = __builtin_elementwise_maximum(m, __builtin_elementwise_abs(x[j]));
  return m;
}

// Eight channels as they come, to codes.
template <typename E>
struct Plain8;
template <>
struct Plain8<float> {
  static __device__ float most(const Eight<float>& x) {
    float y[8];
    x.values(y);
    return most_of(y);
  }
  static __device__ uint32_t codes(const Eight<float>& x, int e) {
    float y[8];
    x.values(y);
    return codes_of(y, e);
  }
};
template <>
struct Plain8<bf16> {
  static __device__ float most(const Eight<bf16>& x) {   // (by the bits: a NaN is above the infinity)
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x.raw[j] & 0x7fff7fffu));
    return __builtin_bit_cast(float, (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16);
  }
  static __device__ uint32_t codes(const Eight<bf16>& x, int e) {
    const float s = scale_value(e);
    const uint32_t w[4] = {x.raw[0], x.raw[1], x.raw[2], x.raw[3]};
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), s, 3);
  }
};

template <typename E, int D, int ROPE, bool ONCE>
__global__ __launch_bounds__(kThreads4) void cache4_append_kernel(const E* __restrict__ k, const E* __restrict__ v, const Cache4 cache, const Batch4 b,
                                                                 const int* __restrict__ positions, const void* __restrict__ weight, const Rotary r,
                                                                 int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head) {
  constexpr int LPR = D / 16, PIECES = D / 8, STEP = kThreads4 / LPR;
  __shared__ Places4 places;
  __shared__ __attribute__((aligned(16))) int k_most[STEP][PIECES], v_most[STEP][PIECES];   // scale bytes of the pieces of 8 channels
  const LanePlace<ROPE> at(threadIdx.x % LPR, r.rot_dim);
  // (rows of the whole call stay below 2^31; a workgroup's are those of 64 tokens at most)
  const unsigned rows = (unsigned)b.n_tokens * (unsigned)b.Hkv, row = threadIdx.x / LPR, from = blockIdx.x * STEP, pair = min(from + row, rows - 1);
  const int first = (int)(from / (unsigned)b.Hkv), token = (int)(pair / (unsigned)b.Hkv), head = (int)(pair - (unsigned)token * (unsigned)b.Hkv);
  Eight<E> kp[2], vp[2];
  const E* k_row = k + token * k_token + head * k_head;
  const E* v_row = v + token * v_token + head * v_head;
  kp[0].template load<ONCE>(k_row + at.lo);
  kp[1].template load<ONCE>(k_row + at.hi);
  vp[0].template load<ONCE>(v_row + at.lo);
  vp[1].template load<ONCE>(v_row + at.hi);
  places.find(cache, b, first);
  const int place = places.at[token - first];
  const bool stored = from + row < rows && place >= 0;
  const bool exact = r.norm == 0 && r.rope == 0;   // keys go as they come
  Angles angles;
  bool there = true;
  if (at.turn) {
    const int pos = positions ? positions[token] : place;
    there = pos >= 0 && pos < r.n_pos;
    angles.load(r, there ? pos : 0, at.pair, true);
  }
  int* const k_mine = k_most[row];
  int* const v_mine = v_most[row];
  constexpr float part = 0x1p-19f;
  bool doubt = false;
  int k_scale[2], v_scale[2];
  uint32_t code[2], v_code[2];
  float y[16], off[16];
  if (exact) {
#pragma unroll
    for (int h = 0; h < 2; ++h) k_mine[(h ? at.hi : at.lo) / 8] = scale_of(Plain8<E>::most(kp[h]));
  } else {
    kp[0].values(y);
    kp[1].values(y + 8);
    if (r.norm) {
      float w[16];
      load_weight<D>(w, weight, r, head, at);
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < 16; ++j) s = __builtin_fmaf(y[j], y[j], s);
      s = __builtin_fmaf(row_sum<LPR>(s), 1.0f / (16 * LPR), r.eps);
      doubt = !(s > 0x1p-90f && s < 0x1p120f);   // (squares that leave a float's range)
      // (a channel that is no full float before its weight, 2^-150 off, counts for less than `part` of the scale by a weight of up to 2^24 only)
      doubt |= !(most_of(w) <= 0x1p24f && most_of(w + 8) <= 0x1p24f);
      const float rms = 1.0f / __builtin_sqrtf(s);
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] = y[j] * rms * w[j];
    }
    // What y may be off by. A channel without rotation: 15 roundings of 2^-24 (the squares' sum, of 20, counts half). A rotated one, a c - b s: those and two
    // more, of |a c| + |b s| <= sqrt((a^2 + b^2) (c^2 + s^2)), the length of the pair that comes out, and no more than |y_a| + |y_b|. `part` is 32 of them,
    // not 17, for what is itself rounded here.
    if (at.turn) {
      rotate<ROPE, 1>(y, angles);
      if (!there) {
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = __builtin_nanf("");
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int ia = ROPE == 1 ? j : 2 * j, ib = ROPE == 1 ? 8 + j : 2 * j + 1;
        off[ia] = off[ib] = __builtin_fabsf(y[ia]) + __builtin_fabsf(y[ib]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) off[j] = __builtin_fabsf(y[j]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float most = most_of(y + 8 * h), by = most_of(off + 8 * h) * part, hi = most + by;
      const int e = scale_of(hi);
      // (what is no number in 32 bits, or near the least of them, is for 64 to say)
      doubt |= e != scale_of(most - by) || !(hi < INFINITY) || (hi < 0x1p-100f && hi > 0.0f);
      k_mine[(h ? at.hi : at.lo) / 8] = e;
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) v_mine[(h ? at.hi : at.lo) / 8] = scale_of(Plain8<E>::most(vp[h]));
  wave_order();
  typedef __attribute__((ext_vector_type(4))) int i32x4;
  auto of_group = [&](const int* mine, int h) {
    const i32x4 s = *(const i32x4*)&mine[(h ? at.hi : at.lo) / 32 * 4];
    return max(max(s[0], s[1]), max(s[2], s[3]));
  };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    k_scale[h] = of_group(k_mine, h);
    v_scale[h] = of_group(v_mine, h);
    v_code[h] = v_scale[h] == kScaleNaN ? 0u : Plain8<E>::codes(vp[h], v_scale[h]);
    if (exact) {
      code[h] = Plain8<E>::codes(kp[h], k_scale[h]);
    } else {
      auto end = [&](float part) {   // codes at an end of the error
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(off[8 * h + j], part, y[8 * h + j]);
        return codes_of(x, k_scale[h]);
      };
      code[h] = end(part);
      doubt |= code[h] != end(-part);
    }
  }
  if (!exact && __builtin_amdgcn_ballot_w64(doubt && stored) != 0) {
    double z[16];
    exact_row<E, D, ROPE>(z, kp, weight, r, head, at, at.turn ? positions ? positions[token] : place : 0);
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h) k_mine[(h ? at.hi : at.lo) / 8] = scale_of(most_of(z + 8 * h));
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      k_scale[h] = of_group(k_mine, h);
      code[h] = codes_of(z + 8 * h, k_scale[h]);
    }
  }
  if (!stored) return;
  const int64_t codes = places.code[token - first] + head * cache.code_head, scale = places.scale[token - first] + head * cache.scale_head;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = h ? at.hi : at.lo;
    *(uint32_t*)(cache.k_codes + codes + c / 2) = k_scale[h] == kScaleNaN ? 0u : code[h];
    *(uint32_t*)(cache.v_codes + codes + c / 2) = v_code[h];
    if (c % 32 == 0) {
      cache.k_scales[scale + c / 32] = (uint8_t)k_scale[h];
      cache.v_scales[scale + c / 32] = (uint8_t)v_scale[h];
    }
  }
}

template <typename E, int D, bool ONCE>
__global__ __launch_bounds__(kThreads4) void cache4_read_kernel(E* __restrict__ k, E* __restrict__ v, const Cache4 cache, const Batch4 b, const Tokens4 w,
                                                               int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head) {
  typedef Values16<E> Values;   // 16 bytes
  constexpr int CH = Values::CHANNELS, LPR = D / CH, STEP = kThreads4 / LPR, FLIGHT = 4;   // rows of a lane on their way at once
  __shared__ Places4 places;
  const int c = threadIdx.x % LPR * CH, row = threadIdx.x / LPR, first = blockIdx.x * w.tokens;
  const unsigned rows = (unsigned)min(w.tokens, b.n_tokens - first) * (unsigned)b.Hkv;
  places.find(cache, b, first);
  for (unsigned base = row; base < rows; base += FLIGHT * STEP) {
    typename Values::Codes kc[FLIGHT], vc[FLIGHT];
    int ks[FLIGHT], vs[FLIGHT], t[FLIGHT], head[FLIGHT];
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) {
      row_of(w, b.Hkv, min(base + i * STEP, rows - 1), t[i], head[i]);
      const int64_t codes = places.code[t[i]] + head[i] * cache.code_head + c / 2, scale = places.scale[t[i]] + head[i] * cache.scale_head + c / 32;
      kc[i] = *(const typename Values::Codes*)(cache.k_codes + codes);
      vc[i] = *(const typename Values::Codes*)(cache.v_codes + codes);
      ks[i] = cache.k_scales[scale];
      vs[i] = cache.v_scales[scale];
    }
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) {
      if (base + i * STEP >= rows || places.at[t[i]] < 0) continue;
      Values(kc[i], scale_value(ks[i])).template store<ONCE>(k + (first + t[i]) * k_token + head[i] * k_head + c);
      Values(vc[i], scale_value(vs[i])).template store<ONCE>(v + (first + t[i]) * v_token + head[i] * v_head + c);
    }
  }
}

Cache4 cache_of(const da_cache4& c) {
  return Cache4{(uint8_t*)c.k_codes, (uint8_t*)c.k_scales, (uint8_t*)c.v_codes, (uint8_t*)c.v_scales,
                c.code_stride[0], c.code_stride[1], c.code_stride[2], c.scale_stride[0], c.scale_stride[1], c.scale_stride[2]};
}
Batch4 batch_of(const da_paged& p) {
  return Batch4{p.page_table, p.kv_len, p.q_start, p.Hkv, p.n_seq, p.n_tokens, p.n_pages, p.page_size, p.max_pages};
}
// lanes: of a row. Workgroups of eight rounds over their rows where there are tokens for more than fill the chip, and at least a token each.
Tokens4 tokens_of(const da_paged& p, int lanes) {
  const long long rows = (long long)p.n_tokens * p.Hkv, round = kThreads4 / lanes;
  const long long want = std::max(1LL, std::min(8 * round, rows / (4 * kComputeUnits)));   // rows of a workgroup
  const int tokens = (int)std::max(1LL, std::min({want / p.Hkv, (long long)kMostTokens4, 65535LL / p.Hkv}));
  return Tokens4{tokens, (uint32_t)(((1u << 31) + (unsigned)p.Hkv - 1) / (unsigned)p.Hkv)};
}

template <typename E, int D, int ROPE>
void append(const void* k, const void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream) {
  const Rotary r = {p.rotary.norm, p.rotary.eps, p.rotary.weight_dtype, p.rotary.weight_heads, p.rotary.rope,
                    p.rotary.rope ? p.rotary.rot_dim : 0, p.rotary.n_pos, p.rotary.cos_table, p.rotary.sin_table};
  const unsigned step = kThreads4 / (D / 16), grid = (unsigned)(((long long)p.n_tokens * p.Hkv + step - 1) / step);
  // What is read is not needed again. us, kept in the caches | past them: 28 MB of k and v 23.3 | 24.4, 74 MB 52 | 46 (with their reads); floats: no difference.
  constexpr bool kCan = sizeof(E) == 2;
  const bool once = kCan && (long long)p.n_tokens * p.Hkv * D * 2 * (long long)sizeof(E) > kPastCaches / 2;
  hipLaunchKernelGGL((once ? cache4_append_kernel<E, D, ROPE, kCan> : cache4_append_kernel<E, D, ROPE, false>), dim3(grid), dim3(kThreads4), 0, stream, (const E*)k, (const E*)v, cache_of(cache), batch_of(p),
                     p.positions, p.rotary.k_weight, r, p.k_stride[0], p.k_stride[1], p.v_stride[0], p.v_stride[1]);
}
template <typename E, int D>
void read(void* k, void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream) {
  const Tokens4 w = tokens_of(p, D / Values16<E>::CHANNELS);
  // us, kept in the caches | past them: 40 MB of k and v 16.7 | 16.0, 268 MB 69 | 43.5, floats, 127 MB 39 | 25.6 (the smaller ones may be found there by who reads them next)
  const bool once = (long long)p.n_tokens * p.Hkv * D * 2 * (long long)sizeof(E) > kPastCaches / 2;
  hipLaunchKernelGGL((once ? cache4_read_kernel<E, D, true> : cache4_read_kernel<E, D, false>), dim3((unsigned)((p.n_tokens + w.tokens - 1) / w.tokens)), dim3(kThreads4), 0, stream, (E*)k, (E*)v,
                     cache_of(cache), batch_of(p), w, p.k_stride[0], p.k_stride[1], p.v_stride[0], p.v_stride[1]);
}

}  // namespace

hipError_t launch_cache4_append(const void* k, const void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream) {
#define DA_APPEND(E, D) (p.rotary.rope == 1 ? append<E, D, 1>(k, v, cache, p, stream) : append<E, D, 2>(k, v, cache, p, stream))
  if (p.dtype == DA_BF16) p.d == 64 ? DA_APPEND(bf16, 64) : DA_APPEND(bf16, 128);
  else p.d == 64 ? DA_APPEND(float, 64) : DA_APPEND(float, 128);
#undef DA_APPEND
  return hipGetLastError();
}

hipError_t launch_cache4_read(void* k, void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream) {
  if (p.dtype == DA_BF16) p.d == 64 ? read<bf16, 64>(k, v, cache, p, stream) : read<bf16, 128>(k, v, cache, p, stream);
  else p.d == 64 ? read<float, 64>(k, v, cache, p, stream) : read<float, 128>(k, v, cache, p, stream);
  return hipGetLastError();
}

}  // namespace da
