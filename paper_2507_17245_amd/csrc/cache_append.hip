// New keys and values into a paged cache, the keys normed and rotated on the way.
//
// Bound: reading k and v and writing their places once. Lanes are dealt to (token, head) pairs, heads fastest: a wave's
// reads are one run of k and of v, and lanes of one token load the same angles. A token finds its sequence by counting the starts up
// to its wave's first token, 64 at a time, then its place, its page and the row in it.
// Measured, us: five prompts of up to 4096, Hkv16 d128 bf16 27.7 (5.4 TB/s), float 62 (4.7 TB/s); 64 single tokens, a kernel of 4.2 (that chain of loads).
#include "paged.h"
#include "token_rows.h"

namespace da {

namespace {

constexpr int kAppendThreads = 256;

template <typename E, int D, int ROPE, bool ONCE>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(
    const E* __restrict__ k, const E* __restrict__ v, E* __restrict__ k_pages, E* __restrict__ v_pages, const int* __restrict__ page_table,
    const int* __restrict__ kv_len, const int* __restrict__ q_start, const int* __restrict__ positions, const void* __restrict__ weight,
    const Rotary r, int Hkv, int n_seq, int n_tokens, int n_pages, int page_size, int max_pages, int64_t page_stride, int64_t head_stride,
    int64_t row_stride, int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head) {
  constexpr int LPR = D / 16;
  const long long pair = ((long long)blockIdx.x * kAppendThreads + threadIdx.x) / LPR;
  const LanePlace<ROPE> at(threadIdx.x % LPR, r.rot_dim);
  const int token = (int)min(pair / Hkv, (long long)n_tokens - 1), head = (int)(pair % Hkv);
  const bool real = pair / Hkv < n_tokens;
  Eight<E> kl, kh, vl, vh;
  const E* kp = k + token * k_token + head * k_head;
  const E* vp = v + token * v_token + head * v_head;
  kl.template load<ONCE>(kp + at.lo);
  kh.template load<ONCE>(kp + at.hi);
  vl.template load<ONCE>(vp + at.lo);
  vh.template load<ONCE>(vp + at.hi);

  const TokenPlace place(token, real, q_start, kv_len, page_table, n_seq, page_size, max_pages);
  const int page = place.page;
  float x[16];
  kl.values(x);
  kh.values(x + 8);
  if (r.norm) {
    float w[16];
    load_weight<D>(w, weight, r, head, at);
    const float rms = inverse_rms<LPR>(x, r.eps);
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = x[j] * rms * w[j];
  }
  if (page < 0 || page >= n_pages) return;
  if (at.turn) {
    Angles angles;
    angles.load(r, positions ? positions[token] : place.at, at.pair, true);
    rotate<ROPE, 1>(x, angles);
  }
  const int64_t to = page * page_stride + head * head_stride + place.at % page_size * row_stride;
  Eight<E>::template store<ONCE>(k_pages + to + at.lo, x);
  Eight<E>::template store<ONCE>(k_pages + to + at.hi, x + 8);
  vl.template put<ONCE>(v_pages + to + at.lo);
  vh.template put<ONCE>(v_pages + to + at.hi);
}

template <typename E, int D, int ROPE>
void append(const void* k, const void* v, void* k_pages, void* v_pages, const da_paged& p, hipStream_t stream) {
  const Rotary r = {p.rotary.norm, p.rotary.eps, p.rotary.weight_dtype, p.rotary.weight_heads, p.rotary.rope,
                    p.rotary.rope ? p.rotary.rot_dim : 0, p.rotary.n_pos, p.rotary.cos_table, p.rotary.sin_table};
  const long long lanes = (long long)p.n_tokens * p.Hkv * (D / 16);
  constexpr bool kCan = sizeof(E) == 2;
  const bool once = kCan && lanes * 16 * 2 * 4 > kPastCaches;
  hipLaunchKernelGGL((once ? cache_append_kernel<E, D, ROPE, kCan> : cache_append_kernel<E, D, ROPE, false>), dim3((unsigned)((lanes + kAppendThreads - 1) / kAppendThreads)), dim3(kAppendThreads),
                     0, stream, (const E*)k, (const E*)v, (E*)k_pages, (E*)v_pages, p.page_table, p.kv_len, p.q_start, p.positions,
                     p.rotary.k_weight, r, p.Hkv, p.n_seq, p.n_tokens, p.n_pages, p.page_size, p.max_pages, p.page_stride, p.head_stride,
                     p.row_stride, p.k_stride[0], p.k_stride[1], p.v_stride[0], p.v_stride[1]);
}

}  // namespace

hipError_t launch_cache_append(const void* k, const void* v, void* k_pages, void* v_pages, const da_paged& p, hipStream_t stream) {
#define DA_APPEND(E, D) \
  (p.rotary.rope == 1 ? append<E, D, 1>(k, v, k_pages, v_pages, p, stream) : append<E, D, 2>(k, v, k_pages, v_pages, p, stream))
  if (p.dtype == DA_BF16) p.d == 64 ? DA_APPEND(bf16, 64) : DA_APPEND(bf16, 128);
  else p.d == 64 ? DA_APPEND(float, 64) : DA_APPEND(float, 128);
#undef DA_APPEND
  return hipGetLastError();
}

}  // namespace da
