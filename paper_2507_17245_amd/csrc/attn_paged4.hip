// Attention of new tokens over a paged cache of 4-bit codes (fp4.h), bf16. Work split: paged_units.h.
//
//   O = softmax(scale Q K^T) V over the keys that a row sees, one pass: running reference and sum of every row.
//
// A unit is up to 16 query rows of a sequence and a kv head (all query heads of the kv head, token after token). Every wave of a workgroup has all rows
// and every WAVES-th tile of its own (4352 bytes of keys and values: 64 keys at d = 64, 32 at 128), with a softmax state of its own and no
// barrier until the states meet. Bound: reading the codes, and beside it the conversions and exponentials.
//   S^T = K Q^T   by v_mfma_f32_16x16x32_bf16. A lane loads of a key what it is the operand for (8 or 16 bytes: the contraction is dealt out so), converts it with
//                 its scale (every value of a code is a bf16 number) and multiplies; no LDS.
//   O^T = V^T P^T P is where it is needed. V is converted with its scales, written to LDS a wave's tile at a time and read transposed.
// K of the next tile is asked for when this one's is converted, V likewise.
#include <cfloat>

#include "attn_bf16_impl.h"
#include "fp4.h"
#include "paged.h"
#include "paged_units.h"

namespace da {

namespace {

constexpr int kRows4 = 16, kKeys4 = 64;   // rows of a unit, keys of the line's tiles
constexpr int paged4_pad(int waves) { return waves == 8 ? 6 : 3; }
constexpr float kLift = 8.0f;   // the reference follows when a score is 2^8 times it (weights and sums have room, and rounding is relative)

struct Codes {   // strides in bytes
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  int64_t code_page, code_head, scale_page, scale_head;
  int code_row, scale_row;
};

// Where 16 successive keys lie: the page (-1: in none of the cache's) and the row in it. A lane for each such group of a wave's next 64.
struct CodeWindow {
  int page, row;
};
__device__ inline CodeWindow code_window(const int* __restrict__ table, int key, int n_keys, int page_size, int n_pages) {
  CodeWindow w = {-1, 0};
  if (key < n_keys) {
    const unsigned at = (unsigned)key / (unsigned)page_size;
    const int id = table[at];
    if (id >= 0 && id < n_pages) w = CodeWindow{id, (int)((unsigned)key - at * (unsigned)page_size)};
  }
  return w;
}

__device__ inline f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline __amdgpu_buffer_rsrc_t rows_rsrc(const uint8_t* base, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00020000);
}
// Largest and sum over the four lanes of a row (16 apart).
__device__ inline float quarter_max(float x) {
  x = half_swap_max(x);
  return fmaxf(x, __shfl_xor(x, 16));
}
__device__ inline float quarter_sum(float x) {
  x = half_swap_sum(x);
  return x + __shfl_xor(x, 16);
}

template <int D, bool STATS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void paged4_kernel(
    const bf16* __restrict__ q, const Codes cache, bf16* __restrict__ o, const int* __restrict__ page_table, const int* __restrict__ q_start,
    const int* __restrict__ kv_len, float* __restrict__ lse, int H, int Hkv, int n_seq, int n_tokens, int n_pages, int page_size, int max_pages,
    int64_t q_token, int64_t q_head, int causal, float scale_log2e, int ranges, int least, unsigned most, float* __restrict__ part_o,
    f32x4* __restrict__ part_stat, PagedCut* __restrict__ cuts) {
  constexpr int ROWS = kRows4, BC = kKeys4, FT = D == 64 ? 64 : 32, GROUPS = FT / 16, KSTEPS = D / 32, NCT = D / 16, WORDS = D / 32;
  constexpr int WINDOW = 64 / GROUPS;
  constexpr int TILEB = FT * D * 2, ROWB = D * 2;
  static_assert(TILEB >= ROWS * D * 4, "a wave's sums take the place of its tile");
  __shared__ __attribute__((aligned(1024))) char v_lds[WAVES][TILEB];
  __shared__ f32x4 stat_lds[WAVES][ROWS];
  __shared__ PagedLds line_lds;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int group = H / Hkv;
  const PagedBatch batch = {q_start, kv_len, n_seq, n_tokens, group, max_pages * page_size, most};
  const PagedLine<ROWS, BC, paged4_pad(WAVES)> line(batch, &line_lds, wave, WAVES);
  unsigned pos = 0, end = 1;
  int wg = blockIdx.x;
  if (ranges) {
    // Ranges that follow each other on one XCD: their units read the same keys.
    if ((gridDim.x & 7) == 0) wg = (wg & 7) * (gridDim.x >> 3) + (wg >> 3);
    const unsigned total = line.total * (unsigned)Hkv, length = paged_range(total, gridDim.x, least);
    pos = paged_cut(line, wg, length, total);
    end = paged_cut(line, wg + 1, length, total);
    const PagedCut cut = paged_mark<ROWS>(line, pos, end, length, total);
    if (tid == 0) cuts[wg] = cut;
  }
  while (pos < end) {
    PagedUnit u;
    int head, t0, t1;
    if (ranges) {
      head = (int)(pos / line.total);
      const unsigned at = pos - (unsigned)head * line.total;
      if (!line.template find<false>(at, &u)) return;
      t0 = (int)(at - u.first);
      t1 = min(u.places, t0 + (int)(end - pos));
    } else {
      // (a kv head's units on one XCD where there are eight of them; those of a sequence that see the most keys first)
      head = wg % Hkv;
      if (!line.template find<true>(wg / Hkv, &u)) return;
      u.m0 = (u.rows - 1) / ROWS * ROWS - u.m0;
      t0 = 0;
      t1 = u.places;
    }
    const bool whole = t0 == 0 && t1 == u.places;
    pos += (unsigned)(t1 - t0);

    const int n_keys = min(u.len, batch.max_keys);
    const int* table = page_table + (int64_t)u.seq * max_pages;
    const int m1 = min(u.m0 + ROWS, u.rows), mr = min(u.m0 + m, u.rows - 1);   // this lane's row (surplus rows: a valid one, never stored)
    const int token = u.q0 + mr / group, q_of = head * group + mr % group;
    const int lim = min(causal ? u.len - u.nq + mr / group : n_keys - 1, n_keys - 1);   // last key this row sees
    const int n_seen = causal ? min(n_keys, max(u.len - u.nq + (m1 - 1) / group + 1, 0)) : n_keys;   // no row sees more
    const int all_see = causal ? min(max(u.len - u.nq + u.m0 / group + 1, 0), n_keys) : n_keys;   // keys below this every row sees

    // Operands of Q: the channels of a lane's pieces of K.
    bf16x8 qop[KSTEPS];
    {
      const bf16* q_row = q + token * q_token + q_of * q_head + g * (D / 4);
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) qop[s] = *(const bf16x8*)(q_row + 8 * s);
    }
    const uint8_t* k_codes = cache.k_codes + head * cache.code_head;
    const uint8_t* v_codes = cache.v_codes + head * cache.code_head;
    const uint8_t* k_scales = cache.k_scales + head * cache.scale_head;
    const uint8_t* v_scales = cache.v_scales + head * cache.scale_head;
    const int k_at = m * cache.code_row + g * (D / 8), ks_at = m * cache.scale_row + g * (D / 4) / 32;
    const int vr = lane >> 2, vp = lane & 3;   // row of 16 and quarter of it that the lane brings of V
    const int v_at = vr * cache.code_row + vp * (D / 8), vs_at = vr * cache.scale_row + vp * (D / 4) / 32;
    // LDS: 16-byte pieces exchanged so that neither the writes (a piece of 4 rows' quarters at a time) nor the transposing reads (two pieces of 8 rows) meet in a bank
    auto swizzle = [](int row) { return D == 64 ? (row >> 1 & 3) << 1 | (row >> 1 & 1) : (row & 7) | (row & 1) << 3; };
    char* const vb = v_lds[wave];
    const int w_at = vr * ROWB, w_swz = swizzle(vr);
    const int r_row = 4 * g + (m >> 2);
    const int r_at = r_row * ROWB + ((((m & 3) >> 1) ^ swizzle(r_row)) << 4) + 8 * (m & 1);

    int tile = t0 * (BC / FT) + wave;
    const int t_end = min(t1 * (BC / FT), (n_seen + FT - 1) / FT);
    // the window's lane for this wave's tile tile + WAVES i is that of i * GROUPS, and of the groups of 16 keys behind it
    auto window_of = [&](int first) {
      const int t = first + (lane / GROUPS) * WAVES;
      return code_window(table, t * FT + lane % GROUPS * 16, n_seen, page_size, n_pages);
    };
    CodeWindow now = window_of(tile), next = window_of(tile + WINDOW / 2 * WAVES);
    int at = 0;   // place in the window of the tile that is asked for
    uint32_t kc[GROUPS][WORDS], vc[GROUPS][WORDS];
    int ks[GROUPS], vs[GROUPS];
    auto ask = [&](int t, const uint8_t* codes, const uint8_t* scales, int code_at, int scale_at, uint32_t (&c)[GROUPS][WORDS], int (&e)[GROUPS]) -> int {
      int there = 0;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        const int page = __builtin_amdgcn_readlane(now.page, at * GROUPS + i), row = __builtin_amdgcn_readlane(now.row, at * GROUPS + i);
        const int rows = min(n_seen - (t * FT + 16 * i), 16), id = max(page, 0);
        there |= (page >= 0 ? 1 : 0) << i;
        const __amdgpu_buffer_rsrc_t code_rsrc = rows_rsrc(codes + (id * cache.code_page + (int64_t)row * cache.code_row), page >= 0 ? (unsigned)((rows - 1) * cache.code_row + D / 2) : 0u);
        const __amdgpu_buffer_rsrc_t scale_rsrc = rows_rsrc(scales + (id * cache.scale_page + (int64_t)row * cache.scale_row), page >= 0 ? (unsigned)((rows - 1) * cache.scale_row + D / 32) : 0u);
        if constexpr (WORDS == 2) {
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(code_rsrc, code_at, 0, 0));
          c[i][0] = x[0];
          c[i][1] = x[1];
        } else {
          const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(code_rsrc, code_at, 0, 0));
#pragma unroll
          for (int j = 0; j < 4; ++j) c[i][j] = x[j];
        }
        e[i] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(scale_rsrc, scale_at, 0, 0);
      }
      return there;
    };
    int there = 0;
    if (tile < t_end) {
      there = ask(tile, k_codes, k_scales, k_at, ks_at, kc, ks);
      ask(tile, v_codes, v_scales, v_at, vs_at, vc, vs);
    }
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
        for (int s = 0; s < KSTEPS; ++s) sc[i] = mfma_16x16x32(Values8<bf16>(kc[i][s], scale_value(ks[i])).x, qop[s], sc[i]);
      }
      const bool more = tile + WAVES < t_end;
      if (more) {
        ++at;
        there = ask(tile + WAVES, k_codes, k_scales, k_at, ks_at, kc, ks);
      }
      const int n0 = tile * FT;
      const bool some = n0 + FT > all_see || seen != (1 << GROUPS) - 1;
      if (some) {
#pragma unroll
        for (int i = 0; i < GROUPS; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (n0 + 16 * i + 4 * g + j > lim || !(seen >> i & 1)) sc[i][j] = -INFINITY;
      }
      float mx = sc[0][0];
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sc[i][j]);
      if (__builtin_amdgcn_ballot_w64((mx - ref) * scale_log2e > kLift) != 0) {
        const float ref_new = fmaxf(ref, quarter_max(mx));
        const float alpha = __builtin_amdgcn_exp2f((ref - ref_new) * scale_log2e);
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
          const float x = __builtin_amdgcn_exp2f((sc[i][j] - ref) * scale_log2e);
          if constexpr (STATS) e_run += x;
          pop[i / 2][i % 2 * 4 + j] = (bf16)x;
        }
      // V: values, and where rows do not all see a tile's keys and 32 channels are NaN, first without those, then they alone
      bool odd = false;
      if (some) {
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) odd |= vs[i] == kScaleNaN;
        odd = __builtin_amdgcn_ballot_w64(odd) != 0;
      }
      auto convert = [&](auto value) {   // value(i, s): eight channels
        wave_order();   // the reads of the previous tile come first
#pragma unroll
        for (int i = 0; i < GROUPS; ++i)
#pragma unroll
          for (int s = 0; s < WORDS; ++s) *(bf16x8*)(vb + i * 16 * ROWB + w_at + (((vp * WORDS + s) ^ w_swz) << 4)) = value(i, s);
        wave_order();
      };
      auto operand = [&](int tt, int ct) {
        const char* p0 = vb + (r_at ^ (ct * 32)) + 32 * tt * ROWB;
        return lds_read_tr_pair<bf16x8>(p0, p0 + 16 * ROWB);
      };
      if (odd) {
        bf16 one = (bf16)1.0f;
        bf16x8 zeros, all;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          zeros[j] = (bf16)0.0f;
          all[j] = one;
        }
        convert([&](int i, int) { return vs[i] == kScaleNaN ? all : zeros; });
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
          f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int tt = 0; tt < FT / 32; ++tt) {
            bf16x8 sees;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int i = 2 * tt + j / 4;
              sees[j] = (bf16)(n0 + 16 * i + 4 * g + j % 4 > lim || !(seen >> i & 1) ? 0.0f : 1.0f);
            }
            z = mfma_16x16x32(operand(tt, ct), sees, z);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (z[j] > 0.0f) oacc[ct][j] = __builtin_nanf("");
        }
        convert([&](int i, int s) { return vs[i] == kScaleNaN ? zeros : Values8<bf16>(vc[i][s], scale_value(vs[i])).x; });
      } else {
        convert([&](int i, int s) { return Values8<bf16>(vc[i][s], scale_value(vs[i])).x; });
      }
      if (more) ask(tile + WAVES, v_codes, v_scales, v_at, vs_at, vc, vs);
#pragma unroll
      for (int tt = 0; tt < FT / 32; ++tt) {
        lacc = mfma_16x16x32(ones, pop[tt], lacc);
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) oacc[ct] = mfma_16x16x32(operand(tt, ct), pop[tt], oacc[ct]);
      }
      if (at == WINDOW / 2) {   // (the next to be asked for is behind it)
        at = 0;
        now = next;
        next = window_of(tile + (1 + WINDOW / 2) * WAVES);
      }
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
      const float x = __builtin_amdgcn_exp2f((st[0] - ref_all) * scale_log2e);
      l_all += st[1] * x;
      e_all += st[2] * x;
    }
    // (a row that sees nothing has sum 0 and is 0)
    const float weight = __builtin_amdgcn_exp2f((ref - ref_all) * scale_log2e) * (!whole ? 1.0f : l_all == 0.0f ? 0.0f : 1.0f / l_all);
    // a wave's sums: 16 rows of D floats in its buffer, the 16-byte pieces exchanged by the row
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) *(f32x4*)(vb + m * (D * 4) + (((4 * ct + g) ^ m) << 4)) = oacc[ct] * weight;
    __syncthreads();
    const size_t slot = (2 * (size_t)wg + (t0 == 0 ? 2 : 1)) * ROWS;
    for (int i = tid; i < (m1 - u.m0) * (D / 4); i += WAVES * 64) {
      const int row = i / (D / 4), piece = i % (D / 4), r = u.m0 + row;
      f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < WAVES; ++j) x += *(const f32x4*)(v_lds[j] + row * (D * 4) + ((piece ^ row) << 4));
      if (whole) {
        const bf16x4 y = {(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
        *(bf16x4*)(o + ((int64_t)(u.q0 + r / group) * H + head * group + r % group) * D + piece * 4) = y;
      } else {
        *(f32x4*)(part_o + (slot + row) * D + piece * 4) = x;
      }
    }
    if (wave == 0 && g == 0 && u.m0 + m < m1) {
      if (!whole) part_stat[slot + m] = f32x4{ref_all * scale_log2e, l_all, e_all, 0.0f};
      else if (STATS) lse[(int64_t)token * H + q_of] = row_statistic(ref_all * scale_log2e, e_all);
    }
    __syncthreads();   // (the next tiles take the place of the sums)
  }
}

template <int D, int WAVES>
hipError_t launch_as(const void* q, void* o, const Codes& cache, const da_paged& p, float scale, void* scratch, const PagedLaunch& l, hipStream_t stream) {
  const float scale_log2e = scale * 1.4426950408889634f;
  const PagedScratch at(scratch, l.workgroups, kRows4, D);
  hipLaunchKernelGGL((p.lse_out ? paged4_kernel<D, true, WAVES> : paged4_kernel<D, false, WAVES>), dim3((unsigned)l.workgroups), dim3(WAVES * 64), 0, stream,
                     (const bf16*)q, cache, (bf16*)o, p.page_table, p.q_start, p.kv_len, p.lse_out, p.H, p.Hkv, p.n_seq, p.n_tokens, p.n_pages, p.page_size,
                     p.max_pages, p.q_stride[0], p.q_stride[1], p.causal, scale_log2e, l.ranges, l.least, l.most, at.sums, at.stats, at.cuts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !l.ranges) return e;
  hipLaunchKernelGGL((paged_combine_kernel<bf16, D, kRows4>), dim3((unsigned)(l.workgroups * (kRows4 * D / 1024))), dim3(256), 0, stream, at.sums, at.stats,
                     at.cuts, (bf16*)o, p.lse_out, p.H, p.Hkv);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const void* q, void* o, const Codes& cache, const da_paged& p, float scale, void* scratch, size_t scratch_bytes, hipStream_t stream) {
  const long long units = (long long)p.n_seq * p.Hkv;   // that there are about
  auto launch = [&](int waves) { return paged_launch(p, kRows4, kKeys4, paged4_pad(waves), 8 * kComputeUnits / waves, 20, scratch_bytes); };
  if (units <= kComputeUnits) return launch_as<D, 8>(q, o, cache, p, scale, scratch, launch(8), stream);
  return launch_as<D, 4>(q, o, cache, p, scale, scratch, launch(4), stream);
}

}  // namespace

size_t paged4_scratch_bytes(const da_paged& p) {
  return p.dtype == DA_F32 ? paged4_f32_scratch_bytes(p) : paged_launch_bytes(2 * kComputeUnits, kRows4, p.d);
}

hipError_t launch_paged4(const void* q, void* o, const da_cache4& c, const da_paged& p, float scale, void* scratch, size_t scratch_bytes, hipStream_t stream) {
  if (p.dtype == DA_F32) return launch_paged4_f32(q, o, c, p, scale, scratch, scratch_bytes, stream);
  const Codes cache = {(const uint8_t*)c.k_codes, (const uint8_t*)c.k_scales, (const uint8_t*)c.v_codes, (const uint8_t*)c.v_scales, c.code_stride[0],
                       c.code_stride[1], c.scale_stride[0], c.scale_stride[1], (int)c.code_stride[2], (int)c.scale_stride[2]};
  return p.d == 64 ? launch_d<64>(q, o, cache, p, scale, scratch, scratch_bytes, stream) : launch_d<128>(q, o, cache, p, scale, scratch, scratch_bytes, stream);
}

}  // namespace da
