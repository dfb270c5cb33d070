// Attention of new tokens over a paged cache, bf16: single tokens and short chunks. Work split: paged_units.h.
//
//   O = softmax(scale Q K^T) V over the keys that a row sees, one pass: running maximum and sum of every row.
//
// Bound: reading the keys and values once. A unit is 32 query rows of a kv head (all of its query heads share every tile); the
// four waves of a workgroup deal its key tiles out among themselves, each with a softmax state of its own: no barrier on the walk. A wave's
// tile is 8 KB of K and of V, brought into LDS by direct loads one tile ahead, 16 keys at a time: 16 rows lie in one page, so
// that a scalar base and limit place them, and rows behind the sequence's end or on a page that is none of the cache's come as zeros and are never
// read. The page table's entries are loaded for 64 such groups at once, a lane for each.
// Operand layouts as in attn_bf16_few.hip.
#include <cfloat>

#include "attn_bf16_impl.h"
#include "paged.h"
#include "paged_tiles.h"
#include "paged_units.h"

namespace da {

namespace {

constexpr int kFewRows = 32, kFewWaves = 4, kFewThreads = kFewWaves * 64;
constexpr int kFewTileBytes = 8192;   // of K, and of V, per wave and buffer
template <int D>
constexpr int kFewKeys = kFewTileBytes / (2 * D);

// STATS: row statistics are asked for. They take a sum of their own, of the weights before they are rounded (the sum over the rounded ones is
// off by their rounding, 1e-4 of a statistic).
template <int D, bool STATS>
__global__ __launch_bounds__(kFewThreads, 1) void paged_few_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k_pages, const bf16* __restrict__ v_pages, bf16* __restrict__ o,
    const int* __restrict__ page_table, const int* __restrict__ q_start, const int* __restrict__ kv_len, float* __restrict__ lse, int H, int Hkv,
    int n_seq, int n_tokens, int n_pages, int page_size, int max_pages, int64_t page_bytes, int64_t head_bytes, int row_bytes, int64_t q_token,
    int64_t q_head, int causal, float scale_log2e, int ranges, int least, float* __restrict__ part_o, f32x4* __restrict__ part_stat) {
  constexpr int ROWB = D * 2, CH = D / 8, KT = kFewKeys<D>;
  constexpr int MB = KT / 32, TT = KT / 16, KS = D / 16, NMB = D / 32;
  constexpr int GROUPS = KT / 16, LPG = 16 * ROWB / 1024;   // groups of 16 keys in a tile, direct loads of one
  constexpr int CPT = GROUPS * LPG;
  constexpr int WINDOW = 64 / GROUPS;                       // a wave's tiles in a page window
  __shared__ __attribute__((aligned(1024))) char k_lds0[kFewWaves][kFewTileBytes];
  __shared__ __attribute__((aligned(1024))) char k_lds1[kFewWaves][kFewTileBytes];
  __shared__ __attribute__((aligned(1024))) char v_lds0[kFewWaves][kFewTileBytes];
  __shared__ __attribute__((aligned(1024))) char v_lds1[kFewWaves][kFewTileBytes];
  __shared__ f32x4 stat_lds[kFewWaves][kFewRows];   // reference, sum, sum before rounding

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, hh = lane >> 5;
  const int group = H / Hkv;
  const PagedBatch batch = {q_start, kv_len, n_seq, n_tokens, Hkv, group, (int)min((long long)max_pages * page_size, 0x7fffffffLL), causal};

  // lanes' places in a group's loads
  int dma_k[LPG], dma_v[LPG];
#pragma unroll
  for (int j = 0; j < LPG; ++j) {
    const int slot = j * 64 + lane, row = slot / CH, pc = slot % CH;
    dma_k[j] = row * row_bytes + (pc ^ (D == 128 ? (row & 15) : ((row >> 1) & 7))) * 16;
    dma_v[j] = row * row_bytes + ((((pc >> 1) ^ v_swizzle<ROWB>(row)) << 1) | (pc & 1)) * 16;
  }
  // and in the operands
  int ka_off[KS], va_off[NMB];
#pragma unroll
  for (int s = 0; s < KS; ++s) ka_off[s] = lq * ROWB + ((2 * s + hh) ^ (D == 128 ? (lq & 15) : ((lq >> 1) & 7))) * 16;
  {
    const int row_l = 4 * hh + ((lane & 15) >> 2);
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb)
      va_off[mb] = row_l * ROWB + ((2 * mb + ((lane >> 4) & 1)) ^ v_swizzle<ROWB>(row_l)) * 32 + 8 * (lane & 3);
  }

  // this workgroup's range of the line
  const PagedLine<kFewRows, KT> line(batch);
  long long pos = 0, end = 1, per_head = 1, length = 1;
  if (ranges) {
    per_head = line.total;
    length = paged_range(per_head * Hkv, gridDim.x, least);
    pos = paged_cut(line, blockIdx.x, length, per_head * Hkv, per_head);
    end = paged_cut(line, blockIdx.x + 1LL, length, per_head * Hkv, per_head);
  }
  while (pos < end) {
    PagedUnit u;
    int head, t0, t1;
    if (ranges) {
      head = (int)(pos / per_head);
      const unsigned at = (unsigned)(pos - head * per_head);
      if (!line.template find<false>(at, &u)) return;
      t0 = (int)(at - u.first);
      t1 = (int)min((long long)u.tiles, t0 + (end - pos));
    } else {
      head = blockIdx.x % Hkv;
      if (!line.template find<true>(blockIdx.x / Hkv, &u)) return;
      t0 = 0;
      t1 = u.tiles;
    }
    const bool whole = t0 == 0 && t1 == u.tiles;
    pos += t1 - t0;

    const int m = u.m0 + lq, m_ld = min(m, u.rows - 1);   // this lane's row (surplus rows: a valid one, never stored)
    const int token = u.q0 + m_ld / group;
    const int n_keys = min(u.len, batch.max_keys);
    const int lim = min(causal ? u.len - u.nq + m_ld / group : n_keys - 1, n_keys - 1);   // last key this row sees
    // no row of the unit sees more
    const int n_seen = causal ? min(n_keys, max(u.len - u.nq + (min(u.m0 + kFewRows, u.rows) - 1) / group + 1, 0)) : n_keys;
    const int all_see = causal ? min(max(u.len - u.nq + u.m0 / group + 1, 0), n_keys) : n_keys;   // keys below this every row sees
    const int t_end = min(t1, (n_seen + KT - 1) / KT);
    const bf16* q_row = q + token * q_token + (head * group + m_ld % group) * q_head;
    bf16x8 qop[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) qop[s] = *(const bf16x8*)(q_row + 16 * s + 8 * hh);

    const int* table = page_table + (int64_t)u.seq * max_pages;
    const char* k_base = (const char*)k_pages + head * head_bytes;
    const char* v_base = (const char*)v_pages + head * head_bytes;
    int tile = t0 + wave;
    // the window's lane for this wave's tile tile + 4 i is that of i * GROUPS, and of the groups of 16 keys behind it
    auto window_of = [&](int first) {
      const int t = first + (lane / GROUPS) * kFewWaves;
      return page_window(table, t * KT + lane % GROUPS * 16, n_seen, page_size, n_pages, page_bytes, row_bytes);
    };
    PageWindow window = window_of(tile), window_next = window_of(tile + WINDOW * kFewWaves);
    int in_window = 0;
    // The next tile in turn; returns a bit for each group of it that lies in the cache.
    auto load_tile = [&](auto par_c, int t) -> int {
      if (in_window == WINDOW) {
        in_window = 0;
        window = window_next;
        window_next = window_of(t + WINDOW * kFewWaves);
      }
      char* kd = decltype(par_c)::value ? k_lds1[wave] : k_lds0[wave];
      char* vd = decltype(par_c)::value ? v_lds1[wave] : v_lds0[wave];
      int there = 0;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int from = in_window * GROUPS + g;
        const uint64_t off = (uint32_t)__builtin_amdgcn_readlane((int)window.lo, from) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)window.hi, from) << 32;
        const int is = __builtin_amdgcn_readlane(window.there, from);
        const int rows = min(n_seen - (t * KT + 16 * g), 16);   // (`is` says that there is one)
        const unsigned bytes = is ? (unsigned)((rows - 1) * row_bytes + ROWB) : 0u;
        there |= is << g;
#pragma unroll
        for (int j = 0; j < LPG; ++j) {
          load_lds(k_base + off, bytes, dma_k[j], 0, kd + (g * LPG + j) * 1024);
          load_lds(v_base + off, bytes, dma_v[j], 0, vd + (g * LPG + j) * 1024);
        }
      }
      ++in_window;
      return there;
    };
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qop[s]));   // (here before the tiles are asked for)
    int there = tile < t_end ? load_tile(even, tile) : 0;

    f32x16 oacc[NMB];
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[mb][i] = 0.0f;
    // The reference is the largest score so far, unscaled (a scaled one is rounded, which shows on large scores).
    float ref = -FLT_MAX, l_run = 0.0f, e_run = 0.0f;   // the sums are over this lane's half of the keys

    auto step = [&](auto par_c, int t) {
      constexpr int par = decltype(par_c)::value;
      const char* kb = par ? k_lds1[wave] : k_lds0[wave];
      const char* vb = par ? v_lds1[wave] : v_lds0[wave];
      const int seen = there;
      // the next tile into the other buffer, whose reads are done; then this tile has to be there
      if (t + kFewWaves < t_end) {
        there = load_tile(std::integral_constant<int, par ^ 1>(), t + kFewWaves);
        asm volatile("s_waitcnt vmcnt(%0)" ::"i"(2 * CPT) : "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      f32x16 sc[MB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[mb][i] = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s) sc[mb] = mfma_32x32x16(*(const bf16x8*)(kb + ka_off[s] + mb * 32 * ROWB), qop[s], sc[mb]);
      }
      const int n0 = t * KT;
      auto v_operand = [&](int tt, int mb) {
        const char* p0 = vb + va_off[mb] + 16 * tt * ROWB;
        return lds_read_tr_pair<bf16x8>(p0, p0 + 8 * ROWB);
      };
      bool odd = false;
      if (n0 + KT > all_see || seen != (1 << GROUPS) - 1) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (n0 + 32 * mb + 8 * (i >> 2) + 4 * hh + (i & 3) > lim || !(seen >> (2 * mb + (i >> 3)) & 1)) sc[mb][i] = -INFINITY;
        odd = any_odd<TT, NMB>(v_operand);
      }
      float mx = sc[0][0];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[mb][i]);
      const float ref_new = fmaxf(ref, half_swap_max(mx));
      if (__builtin_amdgcn_ballot_w64(ref_new > ref) != 0) {
        const float alpha = __builtin_amdgcn_exp2f((ref - ref_new) * scale_log2e);
        l_run *= alpha;
        if constexpr (STATS) e_run *= alpha;
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[mb][i] *= alpha;
        ref = ref_new;
      }
      // P rounded to bf16 as the operands of P.V; the row sum is taken over the rounded values, so that the rounding of a row's
      // largest weights cancels
      bf16x8 pop[TT];
      const bf16x2 ones = {(bf16)1.0f, (bf16)1.0f};
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float x0 = __builtin_amdgcn_exp2f((sc[mb][i] - ref) * scale_log2e), x1 = __builtin_amdgcn_exp2f((sc[mb][i + 1] - ref) * scale_log2e);
          const bf16x2 pr = {(bf16)x0, (bf16)x1};
          if constexpr (STATS) e_run += x0 + x1;
          pop[mb * 2 + (i >> 3)][i & 7] = pr[0];
          pop[mb * 2 + (i >> 3)][(i & 7) + 1] = pr[1];
          l_run = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_run, false);
        }
      if (odd) {
        odd_values<TT, NMB>(oacc, pop, v_operand);
        return;
      }
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb) oacc[mb] = mfma_32x32x16(v_operand(tt, mb), pop[tt], oacc[mb]);
    };
    while (tile < t_end) {
      step(even, tile);
      tile += kFewWaves;
      if (tile >= t_end) break;
      step(odd, tile);
      // (the wait behind these products as in attn_bf16_few.hip)
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 1");
      tile += kFewWaves;
    }

    // ---- the waves' states meet ----------------------------------------------------------------------
    const float l_tot = half_swap_sum(l_run), e_tot = STATS ? half_swap_sum(e_run) : 0.0f;
    if (hh == 0) stat_lds[wave][lq] = f32x4{ref, l_tot, e_tot, 0.0f};
    __syncthreads();   // also: nobody reads tiles any more
    float ref_all = stat_lds[0][lq][0], l_all = 0.0f, e_all = 0.0f;
#pragma unroll
    for (int j = 1; j < kFewWaves; ++j) ref_all = fmaxf(ref_all, stat_lds[j][lq][0]);
#pragma unroll
    for (int j = 0; j < kFewWaves; ++j) {
      const f32x4 st = stat_lds[j][lq];
      const float x = __builtin_amdgcn_exp2f((st[0] - ref_all) * scale_log2e);
      l_all += st[1] * x;
      e_all += st[2] * x;
    }
    // (a row that sees nothing has sum 0 and is 0)
    const float weight = __builtin_amdgcn_exp2f((ref - ref_all) * scale_log2e) * (!whole ? 1.0f : l_all == 0.0f ? 0.0f : 1.0f / l_all);
    // wave w's sums: 32 rows of D floats, the 16-byte pieces exchanged by the row (its own buffers: K at
    // d = 64, K and V at d = 128)
    float* half0 = (float*)k_lds0[wave];
    float* half1 = (float*)(D == 128 ? v_lds0[wave] : k_lds0[wave]);
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int piece = 8 * mb + 2 * i4 + hh;   // channels 4*piece ..
        float* dst = mb < 2 ? half0 : half1;
        const f32x4 x = {oacc[mb][4 * i4] * weight, oacc[mb][4 * i4 + 1] * weight, oacc[mb][4 * i4 + 2] * weight, oacc[mb][4 * i4 + 3] * weight};
        *(f32x4*)&dst[lq * 64 + (((piece & 15) ^ (lq & 15)) << 2)] = x;
      }
    __syncthreads();
    const size_t slot = 2 * (size_t)blockIdx.x + (t0 == 0 ? 2 : 1);   // (the part in front of the next one's cut)
    auto finish = [&](const char (*sums)[kFewTileBytes], int c0) {   // 64 channels from c0 on
#pragma unroll
      for (int i = tid; i < kFewRows * 16; i += kFewThreads) {
        const int row = i / 16, piece = i % 16, mr = u.m0 + row;
        if (mr >= u.rows) continue;
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kFewWaves; ++j) x += *(const f32x4*)((const float*)sums[j] + row * 64 + ((piece ^ (row & 15)) << 2));
        if (whole) {
          const bf16x4 y = {(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
          *(bf16x4*)(o + ((int64_t)(u.q0 + mr / group) * H + head * group + mr % group) * D + c0 + piece * 4) = y;
        } else {
          *(f32x4*)(part_o + (slot * kFewRows + row) * D + c0 + piece * 4) = x;
        }
      }
    };
    finish(k_lds0, 0);
    if constexpr (D == 128) finish(v_lds0, 64);
    if (wave == 0 && hh == 0 && m < u.rows) {
      if (!whole) part_stat[slot * kFewRows + lq] = f32x4{ref_all * scale_log2e, l_all, e_all, 0.0f};
      else if (STATS) lse[(int64_t)token * H + head * group + m % group] = row_statistic(ref_all * scale_log2e, e_all);
    }
    __syncthreads();   // (the next unit's tiles take the place of the sums)
  }
}

template <int D>
hipError_t launch_few(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                      const PagedLaunch& l, hipStream_t stream) {
  const float scale_log2e = scale * 1.4426950408889634f;
  float* part_o = (float*)scratch;
  f32x4* part_stat = (f32x4*)((char*)scratch + paged_sum_bytes(l.workgroups, kFewRows, D));
  hipLaunchKernelGGL((p.lse_out ? paged_few_kernel<D, true> : paged_few_kernel<D, false>), dim3((unsigned)l.workgroups), dim3(kFewThreads), 0, stream, (const bf16*)q, (const bf16*)k_pages,
                     (const bf16*)v_pages, (bf16*)o, p.page_table, p.q_start, p.kv_len, p.lse_out, p.H, p.Hkv, p.n_seq, p.n_tokens, p.n_pages,
                     p.page_size, p.max_pages, p.page_stride * 2, p.head_stride * 2, (int)(p.row_stride * 2), p.q_stride[0], p.q_stride[1],
                     p.causal, scale_log2e, l.ranges, l.least, part_o, part_stat);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !l.ranges) return e;
  hipLaunchKernelGGL((paged_combine_kernel<bf16, D, kFewRows, kFewKeys<D>>), dim3(paged_combine_grid(p, kFewRows)), dim3(256), 0,
                     stream, part_o, part_stat, (bf16*)o, p.q_start, p.kv_len, p.lse_out, p.H, p.Hkv, p.n_seq, p.n_tokens,
                     p.max_pages * p.page_size, l.workgroups, l.least);
  return hipGetLastError();
}

// One workgroup per compute unit (its tiles take the LDS).
PagedLaunch few_launch(const da_paged& p, size_t scratch_bytes) {
  return paged_launch(p, kFewRows, p.d == 64 ? kFewKeys<64> : kFewKeys<128>, kComputeUnits, scratch_bytes);
}

}  // namespace

// Whether the call has sequences with enough rows for the kernel of units of 128. The host knows the rows of all of them alone.
static bool paged_many_rows(const da_paged& p) {
  return true;
}

size_t paged_scratch_bytes(const da_paged& p) {
  if (p.dtype == DA_BF16 && paged_many_rows(p)) return paged_chunk_scratch_bytes(p);
  return paged_launch_bytes(p.dtype == DA_F32 ? 2 * kComputeUnits : kComputeUnits, kFewRows, p.d);
}

hipError_t launch_paged(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                        size_t scratch_bytes, hipStream_t stream) {
  if (p.dtype == DA_F32) return launch_paged_f32(q, k_pages, v_pages, o, p, scale, scratch, scratch_bytes, stream);
  if (paged_many_rows(p)) return launch_paged_chunk(q, k_pages, v_pages, o, p, scale, scratch, scratch_bytes, stream);
  const PagedLaunch l = few_launch(p, scratch_bytes);
  return p.d == 64 ? launch_few<64>(q, k_pages, v_pages, o, p, scale, scratch, l, stream)
                   : launch_few<128>(q, k_pages, v_pages, o, p, scale, scratch, l, stream);
}

}  // namespace da
