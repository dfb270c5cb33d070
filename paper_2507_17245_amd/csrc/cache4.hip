// New keys and values into a paged cache of 4-bit codes, and out of it again (fp4.h has the form).
//
// Bound: k and v and their codes, each moved once. Append: lanes as in cache_append.hip, two pieces of eight channels each; the scale of 32 channels is the
// largest of its four pieces' (which lanes of one row hold, wherever the rotation puts them), exchanged through LDS.
// The codes are those of the exact row: with norm or rotation the row is taken in 32 bits with a bound on its error, and where a code or a scale
// differs between the two ends of that bound (one wave of a hundred), the wave takes its rows again in 64 bits.
// Read: a lane converts eight channels, 4 bytes to 16 or 32.
#include "fp4.h"
#include "token_rows.h"

namespace da {

namespace {

constexpr int kThreads4 = 256;

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

template <int LPR>
__device__ inline double row_sum(double x) {
#pragma unroll
  for (int i = 1; i < LPR; i *= 2) x += __shfl_xor(x, i, LPR);
  return x;
}

// The row in 64 bits: x as loaded, w its weights (norm), t its angles (turn).
template <int LPR, int ROPE>
__device__ inline void exact_row(double (&y)[16], const float (&x)[16], const float (&w)[16], const Angles& t, bool norm, float eps, bool turn) {
  double rms = 1.0;
  if (norm) {
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < 16; ++j) s += (double)x[j] * (double)x[j];
    rms = 1.0 / __builtin_sqrt(row_sum<LPR>(s) * (1.0 / (16 * LPR)) + (double)eps);
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) y[j] = norm ? (double)x[j] * rms * (double)w[j] : (double)x[j];
  if (turn) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int ia = ROPE == 1 ? j : 2 * j, ib = ROPE == 1 ? 8 + j : 2 * j + 1;
      const double a = y[ia], b = y[ib], c = t.c[j], s = t.s[j];
      y[ia] = a * c - b * s;
      y[ib] = a * s + b * c;
    }
  }
}
template <typename T>
__device__ inline T most_of(const T* x) {   // of eight magnitudes; NaN stays
  T m = __builtin_elementwise_abs(x[0]);
#pragma unroll
  for (int j = 1; j < 8; ++j) m = __builtin_elementwise_maximum(m, __builtin_elementwise_abs(x[j]));
  return m;
}

template <typename E, int D, int ROPE>
__global__ __launch_bounds__(kThreads4) void cache4_append_kernel(const E* __restrict__ k, const E* __restrict__ v, const Cache4 cache, const Batch4 b,
                                                                 const int* __restrict__ positions, const void* __restrict__ weight, const Rotary r,
                                                                 int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head) {
  constexpr int LPR = D / 16, PIECES = D / 8;
  // Scale bytes of the pieces of 8 channels: K at the upper and at the lower end of its error, V.
  __shared__ __attribute__((aligned(16))) uint32_t scales[kThreads4 / LPR][PIECES];
  const long long pair = ((long long)blockIdx.x * kThreads4 + threadIdx.x) / LPR;
  const LanePlace<ROPE> at(threadIdx.x % LPR, r.rot_dim);
  const int token = (int)min(pair / b.Hkv, (long long)b.n_tokens - 1), head = (int)(pair % b.Hkv);
  Eight<E> kl, kh, vl, vh;
  const E* kp = k + token * k_token + head * k_head;
  const E* vp = v + token * v_token + head * v_head;
  kl.load(kp + at.lo);
  kh.load(kp + at.hi);
  vl.load(vp + at.lo);
  vh.load(vp + at.hi);
  const TokenPlace place(token, pair / b.Hkv < b.n_tokens, b.q_start, b.kv_len, b.page_table, b.n_seq, b.page_size, b.max_pages);
  const bool stored = place.page >= 0 && place.page < b.n_pages;

  float x[16], y[16], w[16], u[16];
  kl.values(x);
  kh.values(x + 8);
  vl.values(u);
  vh.values(u + 8);
  Angles angles;
  if (at.turn) angles.load(r, positions ? positions[token] : place.at, at.pair, true);
  bool doubt = false;
#pragma unroll
  for (int j = 0; j < 16; ++j) y[j] = x[j];
  if (r.norm) {
    load_weight<D>(w, weight, r, head, at);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 16; ++j) s = __builtin_fmaf(x[j], x[j], s);
    s = __builtin_fmaf(row_sum<LPR>(s), 1.0f / (16 * LPR), r.eps);
    doubt = !(s > 0x1p-90f && s < 0x1p120f);   // (squares that leave a float's range)
    const float rms = 1.0f / __builtin_sqrtf(s);
#pragma unroll
    for (int j = 0; j < 16; ++j) y[j] = x[j] * rms * w[j];
  }
  // What y may be off by: 19 roundings of 2^-24 at most in what a channel is the sum of (the squares' sum counts half), with room.
  float off[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) off[j] = __builtin_fabsf(y[j]);
  if (at.turn) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int ia = ROPE == 1 ? j : 2 * j, ib = ROPE == 1 ? 8 + j : 2 * j + 1;
      const float a = off[ia], c = off[ib], tc = __builtin_fabsf(angles.c[j]), ts = __builtin_fabsf(angles.s[j]);
      off[ia] = __builtin_fmaf(a, tc, c * ts);
      off[ib] = __builtin_fmaf(a, ts, c * tc);
    }
    rotate<ROPE, 1>(y, angles);
  }
  const float part = r.norm || r.rope ? 0x1p-19f : 0.0f;
  float up[16], down[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    up[j] = part != 0.0f ? __builtin_fmaf(off[j], part, y[j]) : y[j];   // (-0 stays)
    down[j] = part != 0.0f ? __builtin_fmaf(off[j], -part, y[j]) : y[j];
  }
  // (the ends' magnitudes may be either's: both bounds of the largest one)
  uint32_t* mine = scales[threadIdx.x / LPR];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float pu = most_of(up + 8 * h), pd = most_of(down + 8 * h);
    float hi = __builtin_elementwise_maximum(pu, pd), lo = 0.0f;
#pragma unroll
    for (int j = 8 * h; j < 8 * h + 8; ++j) lo = fmaxf(lo, fminf(__builtin_fabsf(up[j]), __builtin_fabsf(down[j])));
    // (what is no number in 32 bits, or near the least of them, is for 64 to say)
    if (part != 0.0f) doubt |= !(hi < INFINITY) || (hi < 0x1p-100f && hi > 0.0f);
    mine[(h ? at.hi : at.lo) / 8] = (uint32_t)scale_of(hi) | (uint32_t)scale_of(lo) << 8 | (uint32_t)scale_of(most_of(u + 8 * h)) << 16;
  }
  wave_order();
  int k_scale[2], v_scale[2];
  uint32_t code[2], v_code[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const u32x4 s = *(const u32x4*)&mine[(h ? at.hi : at.lo) / 32 * 4];
    auto most = [&](int shift) { return (int)max(max(s[0] >> shift & 255, s[1] >> shift & 255), max(s[2] >> shift & 255, s[3] >> shift & 255)); };
    k_scale[h] = most(0);
    if (part != 0.0f) doubt |= k_scale[h] != most(8);
    code[h] = codes_of(up + 8 * h, k_scale[h]);
    if (part != 0.0f) doubt |= code[h] != codes_of(down + 8 * h, k_scale[h]);
    v_scale[h] = most(16);
    v_code[h] = v_scale[h] == kScaleNaN ? 0u : codes_of(u + 8 * h, v_scale[h]);
  }
  if (__builtin_amdgcn_ballot_w64(doubt && stored) != 0) {
    double z[16];
    exact_row<LPR, ROPE>(z, x, w, angles, r.norm, r.eps, at.turn);
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h) mine[(h ? at.hi : at.lo) / 8] = (uint32_t)scale_of(most_of(z + 8 * h));
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 s = *(const u32x4*)&mine[(h ? at.hi : at.lo) / 32 * 4];
      k_scale[h] = (int)max(max(s[0], s[1]), max(s[2], s[3]));
      code[h] = codes_of(z + 8 * h, k_scale[h]);
    }
  }
  if (!stored) return;
  const int64_t codes = place.page * cache.code_page + head * cache.code_head + place.at % b.page_size * cache.code_row;
  const int64_t scale = place.page * cache.scale_page + head * cache.scale_head + place.at % b.page_size * cache.scale_row;
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

template <typename E, int D>
__global__ __launch_bounds__(kThreads4) void cache4_read_kernel(E* __restrict__ k, E* __restrict__ v, const Cache4 cache, const Batch4 b, int64_t k_token,
                                                               int64_t k_head, int64_t v_token, int64_t v_head) {
  constexpr int LPR = D / 8;
  const long long pair = ((long long)blockIdx.x * kThreads4 + threadIdx.x) / LPR;
  const int c = threadIdx.x % LPR * 8;
  const int token = (int)min(pair / b.Hkv, (long long)b.n_tokens - 1), head = (int)(pair % b.Hkv);
  const TokenPlace place(token, pair / b.Hkv < b.n_tokens, b.q_start, b.kv_len, b.page_table, b.n_seq, b.page_size, b.max_pages);
  if (place.page < 0 || place.page >= b.n_pages) return;
  const int64_t codes = place.page * cache.code_page + head * cache.code_head + place.at % b.page_size * cache.code_row + c / 2;
  const int64_t scale = place.page * cache.scale_page + head * cache.scale_head + place.at % b.page_size * cache.scale_row + c / 32;
  const uint32_t kc = *(const uint32_t*)(cache.k_codes + codes), vc = *(const uint32_t*)(cache.v_codes + codes);
  const float ks = scale_value(cache.k_scales[scale]), vs = scale_value(cache.v_scales[scale]);
  typedef Values8<E> Values;
  *(Values*)(k + token * k_token + head * k_head + c) = Values(kc, ks);
  *(Values*)(v + token * v_token + head * v_head + c) = Values(vc, vs);
}

Cache4 cache_of(const da_cache4& c) {
  return Cache4{(uint8_t*)c.k_codes, (uint8_t*)c.k_scales, (uint8_t*)c.v_codes, (uint8_t*)c.v_scales,
                c.code_stride[0], c.code_stride[1], c.code_stride[2], c.scale_stride[0], c.scale_stride[1], c.scale_stride[2]};
}
Batch4 batch_of(const da_paged& p) {
  return Batch4{p.page_table, p.kv_len, p.q_start, p.Hkv, p.n_seq, p.n_tokens, p.n_pages, p.page_size, p.max_pages};
}
unsigned grid_of(const da_paged& p, int lanes) {
  return (unsigned)(((long long)p.n_tokens * p.Hkv * lanes + kThreads4 - 1) / kThreads4);
}

template <typename E, int D, int ROPE>
void append(const void* k, const void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream) {
  const Rotary r = {p.rotary.norm, p.rotary.eps, p.rotary.weight_dtype, p.rotary.weight_heads, p.rotary.rope,
                    p.rotary.rope ? p.rotary.rot_dim : 0, p.rotary.n_pos, p.rotary.cos_table, p.rotary.sin_table};
  hipLaunchKernelGGL((cache4_append_kernel<E, D, ROPE>), dim3(grid_of(p, D / 16)), dim3(kThreads4), 0, stream, (const E*)k, (const E*)v, cache_of(cache),
                     batch_of(p), p.positions, p.rotary.k_weight, r, p.k_stride[0], p.k_stride[1], p.v_stride[0], p.v_stride[1]);
}
template <typename E, int D>
void read(void* k, void* v, const da_cache4& cache, const da_paged& p, hipStream_t stream) {
  hipLaunchKernelGGL((cache4_read_kernel<E, D>), dim3(grid_of(p, D / 8)), dim3(kThreads4), 0, stream, (E*)k, (E*)v, cache_of(cache), batch_of(p),
                     p.k_stride[0], p.k_stride[1], p.v_stride[0], p.v_stride[1]);
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
