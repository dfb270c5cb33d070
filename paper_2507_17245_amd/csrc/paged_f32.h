// Attention of new tokens over a paged cache in float arithmetic: the kernel, for caches of floats (attn_paged_f32.hip) and of 4-bit
// codes (attn_paged4_f32.hip), which bring the loads of keys and values.
//
// Units of 32 rows and ranges of tiles (paged_units.h); four waves deal 32-key tiles out among themselves. Products by
// v_mfma_f32_32x32x2_f32, S^T = K Q^T and O^T = V^T P^T, with the contraction dealt out so that a lane's operands are what it can
// load itself: channels s and s + d / 2 in step s of the first (a lane walks half a row of K), keys
// acc_row(i, 0 / 1) in step i of the second, where P already is, with channels r * d / 32 + mb as row r of block mb (a lane takes consecutive
// ones of a row of V). V of a tile is asked for before its scores are taken and K of the next one behind them. Operands do not pass through LDS.
//
// PAGES: what the kernel is given of the cache; Head: the lane's places in a kv head's; Window: where the lane's key of a tile lies (`there`:
// whether it does); Keys: half a row of K, load() and the channels' values; Values: load() and the operands of the second product. Absent
// keys' values are zeros.
#pragma once
#include <cfloat>

#include "f32_tiles.h"
#include "paged.h"
#include "paged_units.h"

namespace da {

namespace {

constexpr int kPad = 3, kWaves = 4, kThreads = kWaves * 64, kRows = 32;

template <typename PAGES, int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 2 : 1) void paged_f32_kernel(
    const float* __restrict__ q, const PAGES pages, float* __restrict__ o,
    const int* __restrict__ page_table, const int* __restrict__ q_start, const int* __restrict__ kv_len, float* __restrict__ lse, int H, int Hkv,
    int n_seq, int n_tokens, int n_pages, int page_size, int max_pages, int64_t q_token,
    int64_t q_head, int causal, float scale_log2e, int ranges, int least, unsigned most, float* __restrict__ part_o, f32x4* __restrict__ part_stat, PagedCut* __restrict__ cuts) {
  constexpr int NMB = D / 32, HALF = D / 2;
  __shared__ __attribute__((aligned(16))) float sums[kWaves][kRows][D + 4];
  __shared__ f32x2 stat_lds[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, hh = lane >> 5;
  const int group = H / Hkv;
  const PagedBatch batch = {q_start, kv_len, n_seq, n_tokens, group, max_pages * page_size, most};

  __shared__ PagedLds line_lds;
  const PagedLine<kRows, kTile, kPad> line(batch, &line_lds, wave, kWaves);
  unsigned pos = 0, end = 1;
  if (ranges) {
    const unsigned total = line.total * (unsigned)Hkv, length = paged_range(total, gridDim.x, least);
    pos = paged_cut(line, blockIdx.x, length, total);
    end = paged_cut(line, blockIdx.x + 1, length, total);
    const PagedCut cut = paged_mark<kRows>(line, pos, end, length, total);
    if (tid == 0) cuts[blockIdx.x] = cut;
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
      head = blockIdx.x % Hkv;
      if (!line.template find<true>(blockIdx.x / Hkv, &u)) return;
      t0 = 0;
      t1 = u.places;
    }
    const bool whole = t0 == 0 && t1 == u.places;
    pos += (unsigned)(t1 - t0);

    const int m = u.m0 + lq, m_ld = min(m, u.rows - 1);
    const int token = u.q0 + m_ld / group;
    const int n_keys = min(u.len, batch.max_keys);
    const int lim = min(causal ? u.len - u.nq + m_ld / group : n_keys - 1, n_keys - 1);
    const int n_seen = causal ? min(n_keys, max(u.len - u.nq + (min(u.m0 + kRows, u.rows) - 1) / group + 1, 0)) : n_keys;
    const int all_see = causal ? min(max(u.len - u.nq + u.m0 / group + 1, 0), n_keys) : n_keys;   // keys below this every row sees
    const int t_end = min(t1, (n_seen + kTile - 1) / kTile);
    const float* q_row = q + token * q_token + (head * group + m_ld % group) * q_head + hh * HALF;
    float qv[HALF];
#pragma unroll
    for (int s = 0; s < HALF; s += 4) {
      const f32x4 x = *(const f32x4*)(q_row + s);
#pragma unroll
      for (int j = 0; j < 4; ++j) qv[s + j] = x[j];
    }
    const int* table = page_table + (int64_t)u.seq * max_pages;
    const typename PAGES::Head at(pages, head, lq, hh);

    f32x16 oacc[NMB];
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb) zero(oacc[mb]);
    float ref = -FLT_MAX, l_run = 0.0f;
    // Lane lq of either half: where key tile * 32 + lq lies.
    auto window_of = [&](int t) { return at.window(table, t * kTile + lq, n_seen, page_size, n_pages); };
    typename PAGES::Keys keys;
    int t = t0 + wave;
    typename PAGES::Window now = window_of(t), next = window_of(t + kWaves);
    if (t < t_end) keys.load(at, now);
    for (; t < t_end; t += kWaves) {
      const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(now.there != 0);
      typename PAGES::Values values;
      values.load(at, now, there, n_seen - t * kTile);
      ChannelSum<HALF> chain;
#pragma unroll
      for (int s = 0; s < HALF; ++s) chain.step(s, keys.value(s), qv[s]);
      f32x16 sc = chain.sum();
      now = next;
      next = window_of(t + 2 * kWaves);
      if (t + kWaves < t_end) keys.load(at, now);
      const bool some = t * kTile + kTile > all_see;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (t * kTile + acc_row(i, hh) > lim || !(there >> acc_row(i, hh) & 1)) sc[i] = -INFINITY;
      float mx = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
      const float ref_new = fmaxf(ref, half_swap_max(mx));
      if (__builtin_amdgcn_ballot_w64(ref_new > ref) != 0) {
        const float alpha = __builtin_amdgcn_exp2f((ref - ref_new) * scale_log2e);
        l_run *= alpha;
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[mb][i] *= alpha;
        ref = ref_new;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sc[i] = __builtin_amdgcn_exp2f((sc[i] - ref) * scale_log2e);
        l_run += sc[i];
      }
      float vv[16][NMB];   // V[key acc_row(i, hh)][channel lq * NMB + mb]
      values.get(vv);
      bool odd = false;
      if (some) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int mb = 0; mb < NMB; ++mb) odd |= !(__builtin_fabsf(vv[i][mb]) < INFINITY);
      }
      if (__builtin_amdgcn_ballot_w64(odd) == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int mb = 0; mb < NMB; ++mb) oacc[mb] = mfma(vv[i][mb], sc[i], oacc[mb]);
        continue;
      }
      // An infinity or a NaN among values that not every row sees: it must not reach the rows with P = 0 (0 times it). The finite
      // values, then the weight with which a row sees either infinity or a NaN.
#pragma unroll 1
      for (int kind = 0; kind < 4; ++kind) {
        const float what = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : __builtin_nanf("");
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb) {
          f32x16 z;
#pragma unroll
          for (int i = 0; i < 16; ++i) z[i] = kind == 0 ? oacc[mb][i] : 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float x = vv[i][mb];
            const int is = __builtin_fabsf(x) < INFINITY ? 0 : x != x ? 3 : x < 0.0f ? 2 : 1;
            z = mfma(is != kind ? 0.0f : kind == 0 ? x : 1.0f, sc[i], z);
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (a few operands' registers at a time)
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[mb][i] = kind == 0 ? z[i] : oacc[mb][i] + (z[i] > 0.0f ? what : 0.0f);
        }
      }
    }

    const float l_tot = half_swap_sum(l_run);
    if (hh == 0) stat_lds[wave][lq] = f32x2{ref, l_tot};
    __syncthreads();
    float ref_all = stat_lds[0][lq][0], l_all = 0.0f;
#pragma unroll
    for (int j = 1; j < kWaves; ++j) ref_all = fmaxf(ref_all, stat_lds[j][lq][0]);
#pragma unroll
    for (int j = 0; j < kWaves; ++j) l_all += stat_lds[j][lq][1] * __builtin_amdgcn_exp2f((stat_lds[j][lq][0] - ref_all) * scale_log2e);
    const float weight = __builtin_amdgcn_exp2f((ref - ref_all) * scale_log2e) * (!whole ? 1.0f : l_all == 0.0f ? 0.0f : 1.0f / l_all);
#pragma unroll
    for (int i = 0; i < 16; ++i) {   // channels acc_row(i, hh) * NMB ..
      float* to = &sums[wave][lq][acc_row(i, hh) * NMB];
      if constexpr (NMB == 4) *(f32x4*)to = f32x4{oacc[0][i] * weight, oacc[1][i] * weight, oacc[2][i] * weight, oacc[3][i] * weight};
      else *(f32x2*)to = f32x2{oacc[0][i] * weight, oacc[1][i] * weight};
    }
    __syncthreads();
    const size_t slot = 2 * (size_t)blockIdx.x + (t0 == 0 ? 2 : 1);   // (the part in front of the next one's cut)
    for (int i = tid; i < kRows * (D / 4); i += kThreads) {
      const int row = i / (D / 4), c = i % (D / 4) * 4, mr = u.m0 + row;
      if (mr >= u.rows) continue;
      f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kWaves; ++j) x += *(const f32x4*)&sums[j][row][c];
      if (whole) *(f32x4*)(o + ((int64_t)(u.q0 + mr / group) * H + head * group + mr % group) * D + c) = x;
      else *(f32x4*)(part_o + (slot * kRows + row) * D + c) = x;
    }
    if (wave == 0 && hh == 0 && m < u.rows) {
      if (!whole) part_stat[slot * kRows + lq] = f32x4{ref_all * scale_log2e, l_all, l_all, 0.0f};
      else if (lse) lse[(int64_t)token * H + head * group + m % group] = row_statistic(ref_all * scale_log2e, l_all);
    }
    __syncthreads();
  }
}

template <typename PAGES, int D>
hipError_t launch_paged_f32_as(const void* q, const PAGES& pages, void* o, const da_paged& p, float scale, void* scratch, const PagedLaunch& l,
                               hipStream_t stream) {
  const float scale_log2e = scale * 1.4426950408889634f;
  const PagedScratch at(scratch, l.workgroups, kRows, D);
  hipLaunchKernelGGL((paged_f32_kernel<PAGES, D>), dim3((unsigned)l.workgroups), dim3(kThreads), 0, stream, (const float*)q, pages,
                     (float*)o, p.page_table, p.q_start, p.kv_len, p.lse_out, p.H, p.Hkv, p.n_seq, p.n_tokens, p.n_pages,
                     p.page_size, p.max_pages, p.q_stride[0], p.q_stride[1], p.causal,
                     scale_log2e, l.ranges, l.least, l.most, at.sums, at.stats, at.cuts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !l.ranges) return e;
  hipLaunchKernelGGL((paged_combine_kernel<float, D, kRows>), dim3((unsigned)(l.workgroups * (kRows * D / 1024))), dim3(256), 0, stream, at.sums, at.stats,
                     at.cuts, (float*)o, p.lse_out, p.H, p.Hkv);
  return hipGetLastError();
}

// Workgroups at a time (registers).
inline int paged_f32_resident(const da_paged& p) { return (p.d == 64 ? 2 : 1) * kComputeUnits; }

// Ranges where the table has room for more tiles than a workgroup takes in two rounds (one at d = 128), and the more the better units fill the chip by
// themselves (units whole | ranges, us): H8 Hkv8 d64 one of 300 17.0 | 14.7, 600 24.4 | 14.8, 40 tokens each of 16 of up to 400 22.8 | 31.1, 620 28.6 |
// 36.5; d128 one of 150 21.5 | 18.5, of 600 44.6 | 19.7.
inline PagedLaunch paged_f32_launch(const da_paged& p, size_t scratch_bytes) {
  const int from = (p.d == 64 ? 8 : 5) + (int)std::min(paged_units(p, kRows) * p.Hkv, (long long)kComputeUnits) / 16;
  return paged_launch(p, kRows, kTile, kPad, paged_f32_resident(p), from, scratch_bytes);
}

}  // namespace

}  // namespace da
