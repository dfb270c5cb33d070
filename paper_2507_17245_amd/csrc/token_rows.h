// Norm and rotation of rows of d channels, a few lanes to a row: what the kernels that make queries and keys share.
//
//   n = x / sqrt(mean(x^2) + eps) * w;   (a, b) -> (a cos - b sin, a sin + b cos) for the pairs of the first rot_dim channels
//
// d / 16 lanes take a row, each two pieces of eight channels (16-byte loads of bf16): in the rotated part the pieces are the
// two halves of eight pairs, so that a rotation needs no exchange between lanes, and only the mean does (two or three DPP
// steps). Everything in 32 bits; the result is rounded once, where it is stored.
#pragma once
#include "da_common.h"

namespace da {

namespace {

// Position rotation and norm as the kernels take them (da_rotary; weights of the tensor at hand).
struct Rotary {
  int norm;
  float eps;
  int weight_dtype, weight_heads;
  int rope, rot_dim, n_pos;
  const float* cos_table;
  const float* sin_table;
};

// Calls that read and write more than 128 MB leave the caches (256 MB) alone: what they hold would be gone before it is read again. us, in the
// caches | past them: rows of B4 H16 Hkv16 N8192 d128, forward and gradient (537 and 805 MB) 278 | 252, appends of 149 MB 33.5 | 27.8; but
// appends of 71 MB 14.1 | 15.5, rows of 43 MB 11.5 | 16.0, forward and gradient of 43 and 64 MB 30 | 40, of 84 and 126 MB 52 | 57. Not
// floats, whose eight channels are two accesses that share a line (forward and gradient of 270 and 405 MB 151 | 161).
constexpr long long kPastCaches = 128LL << 20;
template <bool ONCE, typename V>
__device__ inline V read16(const V* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE, typename V>
__device__ inline void write16(V* p, V x) {
  if constexpr (ONCE) __builtin_nontemporal_store(x, p);
  else *p = x;
}

template <typename E>
struct Eight;   // eight consecutive channels, as loaded
template <>
struct Eight<bf16> {
  u32x4 raw;
  template <bool ONCE = false>
  __device__ void load(const bf16* p) { raw = read16<ONCE>((const u32x4*)p); }
  template <bool ONCE>
  __device__ void put(bf16* p) const { write16<ONCE>((u32x4*)p, raw); }
  __device__ void values(float* x) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __builtin_bit_cast(float, raw[j] << 16);
      x[2 * j + 1] = __builtin_bit_cast(float, raw[j] & 0xffff0000u);
    }
  }
  template <bool ONCE>
  static __device__ void store(bf16* p, const float* x) {
    bf16x8 y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = (bf16)x[j];
    write16<ONCE>((bf16x8*)p, y);
  }
};
template <>
struct Eight<float> {
  f32x4 raw[2];
  template <bool ONCE = false>
  __device__ void load(const float* p) {
    raw[0] = *(const f32x4*)p;
    raw[1] = *(const f32x4*)(p + 4);
  }
  template <bool ONCE>
  __device__ void put(float* p) const {
    *(f32x4*)p = raw[0];
    *(f32x4*)(p + 4) = raw[1];
  }
  __device__ void values(float* x) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = raw[j >> 2][j & 3];
  }
  template <bool ONCE>
  static __device__ void store(float* p, const float* x) {
    *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
};

// The lane's place in a row: channels lo .. lo + 7 and hi .. hi + 7; `turn`: they are rotated, as pairs 8 l .. 8 l + 7.
template <int ROPE>
struct LanePlace {
  int lo, hi, pair;
  bool turn;
  __device__ LanePlace(int l, int rot_dim) {
    turn = 16 * l < rot_dim;
    pair = 8 * l;
    lo = 16 * l;
    hi = lo + 8;
    if (ROPE == 1 && turn) {
      lo = 8 * l;
      hi = lo + rot_dim / 2;
    }
  }
};

struct Angles {
  float c[8], s[8];
  // position `pos` of the tables; a position outside of them gives NaN
  __device__ void load(const Rotary& r, int pos, int pair, bool turn) {
    if (!turn) return;
    const bool there = pos >= 0 && pos < r.n_pos;
    const size_t at = (size_t)(there ? pos : 0) * (r.rot_dim / 2) + pair;
    const f32x4 c0 = *(const f32x4*)(r.cos_table + at), c1 = *(const f32x4*)(r.cos_table + at + 4);
    const f32x4 s0 = *(const f32x4*)(r.sin_table + at), s1 = *(const f32x4*)(r.sin_table + at + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      c[j] = there ? (j < 4 ? c0[j & 3] : c1[j & 3]) : __builtin_nanf("");
      s[j] = there ? (j < 4 ? s0[j & 3] : s1[j & 3]) : __builtin_nanf("");
    }
  }
};

// x: the lane's sixteen channels, lo then hi. SIGN 1: forward, -1: by the negative angle (the transposed map, for gradients).
template <int ROPE, int SIGN>
__device__ inline void rotate(float (&x)[16], const Angles& t) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int ia = ROPE == 1 ? j : 2 * j, ib = ROPE == 1 ? 8 + j : 2 * j + 1;
    const float a = x[ia], b = x[ib], s = SIGN > 0 ? t.s[j] : -t.s[j];
    x[ia] = a * t.c[j] - b * s;
    x[ib] = a * s + b * t.c[j];
  }
}

template <int CTRL>
__device__ inline float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// Sum over the LPR (4 or 8) lanes of a row, in every one of them.
template <int LPR>
__device__ inline float row_sum(float x) {
  x += dpp<0xb1>(x);    // quad_perm 1 0 3 2
  x += dpp<0x4e>(x);    // quad_perm 2 3 0 1
  if constexpr (LPR == 8) x += dpp<0x141>(x);   // row_half_mirror
  return x;
}

template <int LPR>
__device__ inline float inverse_rms(const float (&x)[16], float eps) {
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < 16; ++j) s = __builtin_fmaf(x[j], x[j], s);
  return 1.0f / __builtin_sqrtf(__builtin_fmaf(row_sum<LPR>(s), 1.0f / (16 * LPR), eps));
}

// The lane's weights (ones where there are none)
template <int D, int ROPE>
__device__ inline void load_weight(float (&w)[16], const void* weight, const Rotary& r, int head, const LanePlace<ROPE>& at) {
  if (weight == nullptr) {
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = 1.0f;
    return;
  }
  const size_t base = r.weight_heads ? (size_t)head * D : 0;
  if (r.weight_dtype == 0) {
    Eight<bf16> a, b;
    a.load((const bf16*)weight + base + at.lo);
    b.load((const bf16*)weight + base + at.hi);
    a.values(w);
    b.values(w + 8);
  } else {
    Eight<float> a, b;
    a.load((const float*)weight + base + at.lo);
    b.load((const float*)weight + base + at.hi);
    a.values(w);
    b.values(w + 8);
  }
}

// Where a lane's token (of the batch's rows, ascending over the wave) lies in its sequence, and the page of the table there (-1: none).
struct TokenPlace {
  int at = -1, page = -1;
  __device__ TokenPlace(int token, bool real, const int* __restrict__ q_start, const int* __restrict__ kv_len, const int* __restrict__ page_table, int n_seq,
                        int page_size, int max_pages) {
    // sequences that begin at or before the wave's first token
    const int first = __builtin_amdgcn_readfirstlane(token), lane = threadIdx.x & 63;
    int seq = -1;
    for (int s = 0; s <= n_seq; s += 64) {
      const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(s + lane <= n_seq && q_start[min(s + lane, n_seq)] <= first));
      seq += n;
      if (n < 64) break;
    }
    // the lane's own token: one sequence on for every token in between where each has one, else step by step
    const int guess = seq + token - first;
    if (guess > seq && guess < n_seq && seq >= 0 && q_start[guess] == token && q_start[guess + 1] > token) {
      seq = guess;
    } else {
      while (seq < n_seq && q_start[seq + 1] <= token) ++seq;
    }
    if (real && seq >= 0 && seq < n_seq) {
      at = kv_len[seq] - (q_start[seq + 1] - token);
      if (at >= 0 && at / page_size < max_pages) page = page_table[(size_t)seq * max_pages + at / page_size];
    }
  }
};

}  // namespace

}  // namespace da
