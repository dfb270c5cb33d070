// Pieces of the bf16 kernels over a paged cache of 4-bit codes: where keys lie, and the walk of a unit with up to 16 rows.
#pragma once
#include <cfloat>

#include "attn_bf16_impl.h"
#include "fp4.h"
#include "paged.h"
#include "paged_units.h"

namespace da {

namespace {

constexpr float kLift = 8.0f;   // the reference follows when a score is 2^8 times it (weights and sums have room, and rounding is relative)

struct Codes {   // strides in bytes
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  int64_t code_page, code_head, scale_page, scale_head;
  int code_row, scale_row;
};

// Where 16 successive keys lie, a lane for each such group of a wave's next 64: offsets of the first one's codes and scales, or, in a cache of more than
// 2 GB, its page and row (far). The 16 lie in one page, so all of their rows are the cache's, whatever the sequence's length is; in the place of
// keys that are in none of its pages stands its first row.
struct CodeWindow {
  uint32_t code, scale;
  uint64_t there;   // groups that lie in the cache
  template <bool FAR>
  __device__ void place(int page, int row, int n_pages, const Codes& c) {
    const bool is = page >= 0 && page < n_pages;
    page = is ? page : 0;
    row = is ? row : 0;
    code = FAR ? (uint32_t)page : (uint32_t)page * (uint32_t)c.code_page + (uint32_t)row * (uint32_t)c.code_row;
    scale = FAR ? (uint32_t)row : (uint32_t)page * (uint32_t)c.scale_page + (uint32_t)row * (uint32_t)c.scale_row;
    there = __builtin_amdgcn_ballot_w64(is);
  }
};
__device__ inline __amdgpu_buffer_rsrc_t rows_rsrc(const uint8_t* base) { return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0xffffffffu, 0x00020000); }

// Nothing is known of x from here on: what is computed of it stays where it is used.
__device__ inline int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ inline f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// Largest and sum over the four lanes of a row (16 apart).
__device__ inline float quarter_max(float x) {
  x = half_swap_max(x);
  return fmaxf(x, __shfl_xor(x, 16));
}
__device__ inline float quarter_sum(float x) {
  x = half_swap_sum(x);
  return x + __shfl_xor(x, 16);
}

struct Paged4Call {
  const bf16* __restrict__ q;
  Codes cache;
  bf16* __restrict__ o;
  const int* __restrict__ page_table;
  const int* __restrict__ q_start;
  const int* __restrict__ kv_len;
  float* __restrict__ lse;
  int H, Hkv, n_seq, n_tokens, n_pages, page_size, max_pages;
  int64_t q_token, q_head;
  int causal;
  float scale_log2e;
  int ranges, least;
  int near;   // successive heads' rows of codes lie next to each other
  unsigned most;
  float* __restrict__ part_o;
  f32x4* __restrict__ part_stat;
  PagedCut* __restrict__ cuts;
};

// Rows m0 .. of unit u (16 at most) against the tiles t0 .. t1 - 1 of BC keys, by all waves of the workgroup. Every wave has all rows and every WAVES-th
// tile of its own (4352 bytes of keys and values: 64 keys at d = 64, 32 at 128), with a softmax state of its own and no barrier until the states
// meet. Bound: reading the codes, and beside it the conversions and exponentials.
//   S^T = K Q^T   by v_mfma_f32_16x16x32_bf16. A lane loads of a key what it is the operand for (8 or 16 bytes: the contraction is dealt out so), converts it with
//                 its scale (every value of a code is a bf16 number) and multiplies; no LDS.
//   O^T = V^T P^T P is where it is needed. V is converted with its scales, written to LDS a wave's tile at a time and read transposed.
// K of the next tile is asked for when this one's is converted, V likewise (one | two tiles ahead, us: 1000 sequences of up to 300 H16 d64 107 | 171, 64 of up to
// 8192 45.5 | 48.7, one of 100003 H16 d128 74 | 77: registers that other waves need). buffer(wave): 8 KB of a wave's own. slot: place of the rows' sums in
// scratch, where not the whole of a unit's tiles is walked. ONCE: what is read is not kept in the caches.
template <int D, bool STATS, int WAVES, bool FAR, bool ONCE, typename BUFFER>
__device__ inline void few_rows(const Paged4Call& p, const PagedUnit& u, int head, int m0, int t0, int t1, bool whole, size_t slot, int wave,
                                BUFFER buffer, f32x4 (*stat_lds)[16]) {
  constexpr int ROWS = 16, BC = 64, FT = D == 64 ? 64 : 32, GROUPS = FT / 16, KSTEPS = D / 32, NCT = D / 16, WORDS = D / 32;
  constexpr int WINDOW = 64 / GROUPS, ROWB = D * 2;
  static_assert(FT * ROWB >= ROWS * D * 4, "a wave's sums take the place of its tile");
  const int tid = here(threadIdx.x), lane = tid & 63, m = lane & 15, g = lane >> 4, group = p.H / p.Hkv;
  const int n_keys = min(u.len, p.max_pages * p.page_size);
  const int* table = p.page_table + (int64_t)u.seq * p.max_pages;
  const int m1 = min(m0 + ROWS, u.rows), mr = min(m0 + m, u.rows - 1);   // this lane's row (surplus rows: a valid one, never stored)
  const int token = u.q0 + mr / group, q_of = head * group + mr % group;
  const int lim = min(p.causal ? u.len - u.nq + mr / group : n_keys - 1, n_keys - 1);   // last key this row sees
  const int n_seen = p.causal ? min(n_keys, max(u.len - u.nq + (m1 - 1) / group + 1, 0)) : n_keys;   // no row sees more
  const int all_see = p.causal ? min(max(u.len - u.nq + m0 / group + 1, 0), n_keys) : n_keys;   // keys below this every row sees

  // Operands of Q: the channels of a lane's pieces of K.
  bf16x8 qop[KSTEPS];
  {
    const bf16* q_row = p.q + token * p.q_token + q_of * p.q_head + g * (D / 4);
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) qop[s] = *(const bf16x8*)(q_row + 8 * s);
  }
  const uint8_t* k_codes = p.cache.k_codes + head * p.cache.code_head;
  const uint8_t* v_codes = p.cache.v_codes + head * p.cache.code_head;
  const uint8_t* k_scales = p.cache.k_scales + head * p.cache.scale_head;
  const uint8_t* v_scales = p.cache.v_scales + head * p.cache.scale_head;
  const int k_at = m * p.cache.code_row + g * (D / 8), ks_at = m * p.cache.scale_row + g * (D / 4) / 32;
  const int vr = lane >> 2, vp = lane & 3;   // row of 16 and quarter of it that the lane brings of V
  const int v_at = vr * p.cache.code_row + vp * (D / 8), vs_at = vr * p.cache.scale_row + vp * (D / 4) / 32;
  // LDS: the 16-byte pieces of a row are exchanged so that neither a write (of eight lanes at a time: a piece of every quarter of two rows) nor a transposing read
  // (two pieces of eight rows) meets a bank twice
  auto piece_at = [](int row, int piece) {
    return D == 64 ? piece ^ ((row >> 1 & 3) << 1 | ((row ^ row >> 1) & 1)) : piece ^ (piece >> 3) ^ (row & 7) << 1;
  };
  char* const vb = buffer(wave);
  const int r_row = 4 * g + (m >> 2);
  const int r_at = r_row * ROWB + (piece_at(r_row, (m & 3) >> 1) << 4) + 8 * (m & 1);

  int tile = t0 * (BC / FT) + wave;
  const int t_end = min(t1 * (BC / FT), (n_seen + FT - 1) / FT);
  // the window's lane for this wave's tile tile + WAVES i is that of i * GROUPS, and of the groups of 16 keys behind it
  auto key_of = [&](int first) { return (first + (lane / GROUPS) * WAVES) * FT + lane % GROUPS * 16; };
  auto page_of = [&](int key) { return key < n_seen ? table[(unsigned)key / (unsigned)p.page_size] : -1; };
  CodeWindow now;
  now.template place<FAR>(page_of(key_of(tile)), key_of(tile) % (unsigned)p.page_size, p.n_pages, p.cache);
  int page_next = page_of(key_of(tile + WINDOW * WAVES));
  int at = 0;   // place in the window of the tile that is asked for
  uint32_t kc[GROUPS][WORDS], vc[GROUPS][WORDS];
  int ks[GROUPS], vs[GROUPS];
  // Loads in this order and nowhere else: the waits for a tile's keys leave its values, and the next one's keys, on their way.
  auto ask = [&](const uint8_t* codes, const uint8_t* scales, int code_at, int scale_at, uint32_t (&c)[GROUPS][WORDS], int (&e)[GROUPS]) {
    constexpr int kKeep = ONCE ? 2 : 0;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int a = __builtin_amdgcn_readlane((int)now.code, at * GROUPS + i), b = __builtin_amdgcn_readlane((int)now.scale, at * GROUPS + i);
      const __amdgpu_buffer_rsrc_t code_rsrc = rows_rsrc(FAR ? codes + (a * p.cache.code_page + (int64_t)b * p.cache.code_row) : codes);
      const __amdgpu_buffer_rsrc_t scale_rsrc = rows_rsrc(FAR ? scales + (a * p.cache.scale_page + (int64_t)b * p.cache.scale_row) : scales);
      e[i] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(scale_rsrc, scale_at, FAR ? 0 : b, 0);
      if constexpr (WORDS == 2) {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(code_rsrc, code_at, FAR ? 0 : a, kKeep));
        c[i][0] = x[0];
        c[i][1] = x[1];
      } else {
        const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(code_rsrc, code_at, FAR ? 0 : a, kKeep));
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = x[j];
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto there_of = [&]() { return (int)(now.there >> (at * GROUPS) & ((1 << GROUPS) - 1)); };
  // (also behind the last tile: the waits then know how many loads are on their way)
  int there = there_of();
  ask(k_codes, k_scales, k_at, ks_at, kc, ks);
  ask(v_codes, v_scales, v_at, vs_at, vc, vs);
  f32x4 oacc[NCT], lacc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) oacc[ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (bf16)1.0f;
  // The reference is a score, unscaled (a scaled one is rounded, which shows on large scores); sum before rounding, over this lane's keys.
  float ref = -FLT_MAX, e_run = 0.0f;
  for (; tile < t_end; tile += WAVES) {
    const int seen = there;
    f32x4 sc[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      sc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) sc[i] = mfma_16x16x32(values_of(kc[i][s], scale_value(ks[i])), qop[s], sc[i]);
    }
    if (++at == WINDOW) {
      const int first = key_of(tile + WAVES);
      at = 0;
      now.template place<FAR>(page_next, first % (unsigned)p.page_size, p.n_pages, p.cache);
      page_next = page_of(first + WINDOW * WAVES * FT);
    }
    there = there_of();
    ask(k_codes, k_scales, k_at, ks_at, kc, ks);
    const int n0 = tile * FT;
    const bool some = n0 + FT > all_see || seen != (1 << GROUPS) - 1;
    if (some) {
      const int past = here(lim - n0 - 4 * g);   // keys of the lane's that the row sees
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (16 * i + j > past || !(seen >> i & 1)) sc[i][j] = -INFINITY;
    }
    float mx = sc[0][0];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sc[i][j]);
    if (__builtin_amdgcn_ballot_w64((mx - ref) * p.scale_log2e > kLift) != 0) {
      const float ref_new = fmaxf(ref, quarter_max(mx));
      const float alpha = __builtin_amdgcn_exp2f((ref - ref_new) * p.scale_log2e);
      lacc *= alpha;
      if constexpr (STATS) e_run *= alpha;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) oacc[ct] *= alpha;
      ref = ref_new;
    }
    // P rounded to bf16 as the operands of P.V; the row sum is taken over the rounded values (on the matrix pipe), so that the rounding of a
    // row's largest weights cancels
    bf16x8 pop[FT / 32];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = __builtin_amdgcn_exp2f((sc[i][j] - ref) * p.scale_log2e);
        if constexpr (STATS) e_run += x;
        pop[i / 2][i % 2 * 4 + j] = (bf16)x;
      }
    // V. Rows that none of the unit's sees are taken as zeros.
    bool odd = false;   // a value may be an infinity or a NaN
    if (some) {
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        if (n0 + 16 * i + vr >= n_seen || !(seen >> i & 1)) vs[i] = 0;
        odd |= vs[i] > kScaleMost;
      }
      odd = __builtin_amdgcn_ballot_w64(odd) != 0;
    }
    wave_order();   // the reads of the previous tile come first
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int s = 0; s < WORDS; ++s)
        *(bf16x8*)(vb + (i * 16 + vr) * ROWB + (piece_at(vr, vp * WORDS + s) << 4)) = values_of(vc[i][s], scale_value(vs[i]));
    wave_order();
    if (odd) {
      // Keys that not every row sees, and an infinity or a NaN among their values: the product would bring it to the rows with P = 0, too. Those
      // that a row sees are added to its sums, key by key; the product goes without.
      const int last = here(lim - n0);
#pragma unroll 1
      for (int key = 0; key < FT; ++key) {
        const bool sees = key <= last && (seen >> (key >> 4) & 1);
        const char* row = vb + key * ROWB + 8 * (g & 1);
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
          const bf16x4 x = *(const bf16x4*)(row + (piece_at(key & 15, 2 * ct + (g >> 1)) << 4));
#pragma unroll
          for (int j = 0; j < 4; ++j) oacc[ct][j] += sees && !(__builtin_fabsf((float)x[j]) < INFINITY) ? (float)x[j] : 0.0f;
        }
      }
      wave_order();
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
#pragma unroll
        for (int s = 0; s < WORDS; ++s) {
          bf16x8* at = (bf16x8*)(vb + (i * 16 + vr) * ROWB + (piece_at(vr, vp * WORDS + s) << 4));
          bf16x8 x = *at;
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = __builtin_fabsf((float)x[j]) < INFINITY ? x[j] : (bf16)0.0f;
          *at = x;
        }
      wave_order();
    }
    auto operand = [&](int tt, int ct) {
      const char* p0 = vb + (r_at ^ (piece_at(0, 2 * ct) << 4)) + 32 * tt * ROWB;
      return lds_read_tr_pair<bf16x8>(p0, p0 + 16 * ROWB);
    };
    ask(v_codes, v_scales, v_at, vs_at, vc, vs);
#pragma unroll
    for (int tt = 0; tt < FT / 32; ++tt) lacc = mfma_16x16x32(ones, pop[tt], lacc);
#pragma unroll
    for (int tt = 0; tt < FT / 32; ++tt)
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) oacc[ct] = mfma_16x16x32(operand(tt, ct), pop[tt], oacc[ct]);
    // (behind a branch the compiler does not wait long enough for the products on every path)
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 7");
  }
  // the waves' states meet
  const float l_tot = lacc[0], e_tot = STATS ? quarter_sum(e_run) : 0.0f;
  if (g == 0) stat_lds[wave][m] = f32x4{ref, l_tot, e_tot, 0.0f};
  __syncthreads();
  float ref_all = stat_lds[0][m][0], l_all = 0.0f, e_all = 0.0f;
#pragma unroll
  for (int j = 1; j < WAVES; ++j) ref_all = fmaxf(ref_all, stat_lds[j][m][0]);
#pragma unroll
  for (int j = 0; j < WAVES; ++j) {
    const f32x4 st = stat_lds[j][m];
    const float x = __builtin_amdgcn_exp2f((st[0] - ref_all) * p.scale_log2e);
    l_all += st[1] * x;
    e_all += st[2] * x;
  }
  // (a row that sees nothing has sum 0 and is 0)
  const float weight = __builtin_amdgcn_exp2f((ref - ref_all) * p.scale_log2e) * (!whole ? 1.0f : l_all == 0.0f ? 0.0f : 1.0f / l_all);
  // a wave's sums: 16 rows of D floats in its buffer, the 16-byte pieces exchanged by the row
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) *(f32x4*)(vb + m * (D * 4) + (((4 * ct + g) ^ m) << 4)) = oacc[ct] * weight;
  __syncthreads();
  for (int i = tid; i < (m1 - m0) * (D / 4); i += WAVES * 64) {
    const int row = i / (D / 4), piece = i % (D / 4), r = m0 + row;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < WAVES; ++j) x += *(const f32x4*)(buffer(j) + row * (D * 4) + ((piece ^ row) << 4));
    if (whole) {
      const bf16x4 y = {(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
      *(bf16x4*)(p.o + ((int64_t)(u.q0 + r / group) * p.H + head * group + r % group) * D + piece * 4) = y;
    } else {
      *(f32x4*)(p.part_o + (slot + row) * D + piece * 4) = x;
    }
  }
  if (wave == 0 && g == 0 && m0 + m < m1) {
    if (!whole) p.part_stat[slot + m] = f32x4{ref_all * p.scale_log2e, l_all, e_all, 0.0f};
    else if (STATS) p.lse[(int64_t)token * p.H + q_of] = row_statistic(ref_all * p.scale_log2e, e_all);
  }
}

}  // namespace

}  // namespace da
