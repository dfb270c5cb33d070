// Attention of new tokens over a paged cache, bf16: single tokens to chunks of a prompt. Work split: paged_units.h.
//
//   O = softmax(scale Q K^T) V over the keys that a row sees, one pass: running maximum and sum of every row.
//
// A unit is up to 128 query rows of a sequence and a kv head, all of its query heads together, so that grouped heads share every tile; of calls
// with single tokens up to 32 rows, by a kernel with the second walk alone. Eight waves a compute unit (their tiles take the LDS), two to a
// SIMD, one exponentiating while the other multiplies, in one workgroup or several (paged_form).
//   more than 32 rows: waves own 32 rows each, and of eight waves each of a pair with the same rows walks half of the unit's tiles (64 keys)
//     in buffers of its half's own. Bound: the matrix products (at d = 64 the exponentials beside them). Loop, layouts, online softmax and
//     the exchange of the halves are those of attn_bf16_impl.h.
//   up to 32 rows (decoding): every wave has all rows and tiles of 8 KB in turn. Bound: reading the keys and values.
// Tiles come 16 keys at a time, which lie in one page, by a scalar base and limit: rows behind the sequence's end, and keys on
// pages that are none of the cache's, are never read. The page table's entries are held for the tiles ahead, a lane for each, with a bit for
// those that lie in the cache.
// Measured, us: 64 sequences of up to 8192 tokens, H32 Hkv8 d64 107 (5.9 TB/s); one of 100003, H16 d128 137 (6.0 TB/s); 2048 tokens on 16384,
// H32 Hkv8, d64 289 (890 TFLOP/s), d128 488 (1055); two chunks of 250 beside 14 single tokens, of up to 4096, d128 66; one token on 777 10.8.
#include <cfloat>

#include "attn_bf16_impl.h"
#include "paged.h"
#include "paged_tiles.h"
#include "paged_units.h"

namespace da {

namespace {

constexpr int kUnitRows = 128, kFewRows = 32, kTileKeys = 64, kRW = 4;   // rows and keys of the line's units and tiles, waves over the rows

// Places of the line for what beginning and ending a unit takes, in tiles (paged_units.h).
constexpr int paged_pad(int rows, int waves) { return rows != kFewRows ? 8 : waves == 8 ? 6 : 3; }

// Nothing is known of x from here on: what is computed of it stays where it is used, instead of in registers that the walk has not got.
__device__ inline int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
// A lane's places: in the loads of 16 keys, and in the operands. Swizzles as in attn_bf16_impl.h; they are exclusive ors, so that
// load j and operands s and mb differ from the first by one, too.
template <int D>
struct Places {
  static constexpr int ROWB = D * 2, CH = D / 8, LPG = 16 * ROWB / 1024, RPL = 16 / LPG;   // loads of 16 keys, rows of one
  int lq, hh;
  int row, kc, v, ka, va;
  __device__ Places(int lane, int row_bytes) {
    lq = lane & 31;
    hh = lane >> 5;
    const int pc = lane % CH;
    row = lane / CH * row_bytes;
    kc = (pc ^ (lane >> 4)) * 16;
    v = row + ((((pc >> 1) ^ v_swizzle<ROWB>(lane / CH)) << 1) | (pc & 1)) * 16;
    ka = lq * ROWB + (hh ^ (D == 128 ? (lq & 15) : ((lq >> 1) & 7))) * 16;
    const int row_l = 4 * hh + ((lane & 15) >> 2);
    va = row_l * ROWB + (((lane >> 4) & 1) ^ v_swizzle<ROWB>(row_l)) * 32 + 8 * (lane & 3);
  }
  // 16 rows of K or V, `bytes` of them from `from` on
  template <bool ONCE = false>
  __device__ void load_k(const char* from, unsigned bytes, int row_bytes, char* to) const {
    const int c = here(kc);
#pragma unroll
    for (int j = 0; j < LPG; ++j) load_lds<ONCE>(from, bytes, row + (c ^ (j * 64)), j * RPL * row_bytes, to + j * 1024);
  }
  template <bool ONCE = false>
  __device__ void load_v(const char* from, unsigned bytes, int row_bytes, char* to) const {
#pragma unroll
    for (int j = 0; j < LPG; ++j) load_lds<ONCE>(from, bytes, v, j * RPL * row_bytes, to + j * 1024);
  }
  // operands of the products: rows 32 mb + lq of K, channels 16 s + 8 hh ..; rows 16 tt .. of V, channels 32 mb ..
  __device__ static bf16x8 k_operand(const char* tile, int ka, int mb, int s) { return *(const bf16x8*)(tile + (ka ^ (s * 32)) + mb * 32 * ROWB); }
  __device__ static bf16x8 v_operand(const char* tile, int va, int tt, int mb) {
    const char* p0 = tile + (va ^ (mb * 64)) + 16 * tt * ROWB;
    return lds_read_tr_pair<bf16x8>(p0, p0 + 8 * ROWB);
  }
};

// ROWS: 128, or 32 for single tokens: without the loop for more rows, whose code and registers are in the way of a short call. WAVES: 8, one
// workgroup a compute unit; 4 (and 2 with 32 rows): two (four), one beginning or ending its units beside the others' walks.
// CUT: whether there may be ranges (without, prompts of H16 d128 with row statistics 114 -> 109 us: fewer registers in memory).
template <int D, bool STATS, int ROWS, int WAVES, bool CUT>
__global__ __launch_bounds__(WAVES * 64, 2) void paged_kernel(
    const bf16* __restrict__ q, const bf16* __restrict__ k_pages, const bf16* __restrict__ v_pages, bf16* __restrict__ o,
    const int* __restrict__ page_table, const int* __restrict__ q_start, const int* __restrict__ kv_len, float* __restrict__ lse, int H, int Hkv,
    int n_seq, int n_tokens, int n_pages, int page_size, int max_pages, int64_t page_bytes, int64_t head_bytes, int row_bytes, int64_t q_token,
    int64_t q_head, int causal, float scale_log2e, int ranges, int least, unsigned most, float* __restrict__ part_o, f32x4* __restrict__ part_stat, PagedCut* __restrict__ cuts) {
  constexpr int BC = kTileKeys, ROWB = D * 2, TILEB = BC * ROWB;
  constexpr int MB = BC / 32, TT = BC / 16, KSTEPS = D / 16, NMB = D / 32;
  constexpr int LPG = 16 * ROWB / 1024;   // direct loads of 16 keys
  constexpr float kSumTrigger = (BC / 2) * 256.0f;   // (as in attn_bf16_impl.h)
  // Two tiles of K and V for each half; or, with few rows, one of 8 KB for each wave.
  constexpr int kThreads = WAVES * 64, HALVES = WAVES == 2 * kRW ? 2 : 1;
  constexpr int FEWB = 8192, FT = FEWB / ROWB, BUFB = WAVES / 2 * FEWB;
  static_assert(ROWS == kFewRows || HALVES * TILEB <= BUFB, "a buffer holds the halves' tiles");
  __shared__ __attribute__((aligned(1024))) char k_lds0[BUFB];
  __shared__ __attribute__((aligned(1024))) char k_lds1[BUFB];
  __shared__ __attribute__((aligned(1024))) char v_lds0[BUFB];
  __shared__ __attribute__((aligned(1024))) char v_lds1[BUFB];
  __shared__ f32x4 few_stat[WAVES][32];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % kRW, half = HALVES == 1 ? 0 : wave / kRW;
  const int group = H / Hkv;
  const PagedBatch batch = {q_start, kv_len, n_seq, n_tokens, group, max_pages * page_size, most};
  auto k_buf = [&](int par) -> char* { return (par ? k_lds1 : k_lds0) + half * TILEB; };
  auto v_buf = [&](int par) -> char* { return (par ? v_lds1 : v_lds0) + half * TILEB; };

  __shared__ PagedLds line_lds;
  const PagedLine<ROWS, BC, paged_pad(ROWS, WAVES)> line(batch, &line_lds, wave, WAVES);
  unsigned pos = 0, end = 1;
  int wg = blockIdx.x;
  if (CUT && ranges) {
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
    if (CUT && ranges) {
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
    const bool whole = !CUT || (t0 == 0 && t1 == u.places);
    pos += (unsigned)(t1 - t0);

    const int n_keys = min(u.len, batch.max_keys);
    const int* table = page_table + (int64_t)u.seq * max_pages;
    const char* k_base = (const char*)k_pages + head * head_bytes;
    const char* v_base = (const char*)v_pages + head * head_bytes;
    // The unit's rows: up to 128 at once, or 32 from m0 on.
    bool few = ROWS == kFewRows || u.rows - u.m0 <= 32;
    for (int m0 = u.m0;;) {
      const int m1 = min(m0 + (few ? 32 : ROWS), u.rows);
      const int n_seen = causal ? min(n_keys, max(u.len - u.nq + (m1 - 1) / group + 1, 0)) : n_keys;   // no row sees more
      const int all_see = causal ? min(max(u.len - u.nq + m0 / group + 1, 0), n_keys) : n_keys;   // keys below this every row sees
      if (few) {
        // ---- few rows: a wave has all of them, and every eighth (fourth, second) tile of 8 KB. Bound: reading the keys and values. ----
        // Each wave has a softmax state of its own and no barrier; K of its next tile is asked for when the scores are
        // taken, V when it is multiplied, so that 128 KB a compute unit are on their way most of the time.
        constexpr int GROUPS = FT / 16, FMB = FT / 32, FTT = FT / 16, CPT = FEWB / 1024, WINDOW = 64 / GROUPS;
        const int lane = here(tid) & 63;
        const Places<D> at_lane(lane, row_bytes);
        const int lq = at_lane.lq, hh = at_lane.hh;
        const int m = m0 + lq, m_ld = min(m, u.rows - 1);
        const int token = u.q0 + m_ld / group, q_of = head * group + m_ld % group;
        const int lim = min(causal ? u.len - u.nq + m_ld / group : n_keys - 1, n_keys - 1);
        bf16x8 qop[KSTEPS];
        const bf16* q_row = q + token * q_token + q_of * q_head;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) qop[s] = *(const bf16x8*)(q_row + 16 * s + 8 * hh);
        int tile = t0 * (BC / FT) + wave;
        const int t_end = min(t1 * (BC / FT), (n_seen + FT - 1) / FT);
        // the window's lane for this wave's tile tile + 8 i is that of i * GROUPS, and of the groups of 16 keys behind it
        auto window_of = [&](int first) {
          const int t = first + (lane / GROUPS) * WAVES;
          return page_window(table, t * FT + lane % GROUPS * 16, n_seen, page_size, n_pages, page_bytes, row_bytes);
        };
        // Every key is read once. Calls that read more than the caches hold (256 MB) leave them alone: B1 H16 100003 keys d128 171 -> 159 us, 64
        // sequences of 5 on 4096 159 -> 144; smaller ones may find in them what a program read a step ago (14 sequences of 1100-3900 39, 41 so).
        const bool once = (long long)line.tiles * Hkv * (2 * TILEB) > 256LL << 20;
        // Two windows, the second from the middle of the first on; it takes the first's place when that half is asked for.
        PageWindow now = window_of(tile), next = window_of(tile + WINDOW / 2 * WAVES);
        int at = 0;   // place in the window of the tile that is asked for
        auto ask = [&](auto of_k, const char* from, int t, char* to) -> int {
          int there = 0;
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) {
            const int l = at * GROUPS + g;
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)now.lo, l), hi = (uint32_t)__builtin_amdgcn_readlane((int)now.hi, l);
            const int is = __builtin_amdgcn_readlane(now.there, l);
            const int rows = min(n_seen - (t * FT + 16 * g), 16);
            const unsigned bytes = is ? (unsigned)((rows - 1) * row_bytes + ROWB) : 0u;
            there |= is << g;
            const char* rows_at = from + (lo | (uint64_t)hi << 32);
            char* rows_to = to + g * LPG * 1024;
            if constexpr (decltype(of_k)::value) {
              if (once) at_lane.template load_k<true>(rows_at, bytes, row_bytes, rows_to);
              else at_lane.load_k(rows_at, bytes, row_bytes, rows_to);
            } else {
              if (once) at_lane.template load_v<true>(rows_at, bytes, row_bytes, rows_to);
              else at_lane.load_v(rows_at, bytes, row_bytes, rows_to);
            }
          }
          return there;
        };
        const std::true_type of_k;
        const std::false_type of_v;
        char* kb = (wave < WAVES / 2 ? k_lds0 : k_lds1) + wave % (WAVES / 2) * FEWB;
        char* vb = (wave < WAVES / 2 ? v_lds0 : v_lds1) + wave % (WAVES / 2) * FEWB;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) asm volatile("" : "+v"(qop[s]));   // (here before the tiles are asked for)
        int there = 0;
        if (tile < t_end) {
          there = ask(of_k, k_base, tile, kb);
          ask(of_v, v_base, tile, vb);
        }
        f32x16 oacc[NMB];
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[mb][i] = 0.0f;
        // The reference is the largest score so far, unscaled (a scaled one is rounded, which shows on large scores).
        float ref = -FLT_MAX, l_run = 0.0f, e_run = 0.0f;
        for (; tile < t_end; tile += WAVES) {
          const int seen = there;
          asm volatile("s_waitcnt vmcnt(%0)" ::"i"(CPT) : "memory");   // K is there
          const int ka = here(at_lane.ka), va = here(at_lane.va);
          f32x16 sc[FMB];
#pragma unroll
          for (int mb = 0; mb < FMB; ++mb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[mb][i] = 0.0f;
#pragma unroll
            for (int s = 0; s < KSTEPS; ++s) sc[mb] = mfma_32x32x16(at_lane.k_operand(kb, ka, mb, s), qop[s], sc[mb]);
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // and read
          const bool more = tile + WAVES < t_end;
          if (more) {
            ++at;
            there = ask(of_k, k_base, tile + WAVES, kb);
          }
          const int n0 = tile * FT;
          const bool some = n0 + FT > all_see || seen != (1 << GROUPS) - 1;
          if (some) {
#pragma unroll
            for (int mb = 0; mb < FMB; ++mb)
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (n0 + 32 * mb + 8 * (i >> 2) + 4 * hh + (i & 3) > lim || !(seen >> (2 * mb + (i >> 3)) & 1)) sc[mb][i] = -INFINITY;
          }
          float mx = sc[0][0];
#pragma unroll
          for (int mb = 0; mb < FMB; ++mb)
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
          bf16x8 pop[FTT];
          const bf16x2 ones = {(bf16)1.0f, (bf16)1.0f};
#pragma unroll
          for (int mb = 0; mb < FMB; ++mb)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const float x0 = __builtin_amdgcn_exp2f((sc[mb][i] - ref) * scale_log2e), x1 = __builtin_amdgcn_exp2f((sc[mb][i + 1] - ref) * scale_log2e);
              const bf16x2 pr = {(bf16)x0, (bf16)x1};
              if constexpr (STATS) e_run += x0 + x1;
              pop[mb * 2 + (i >> 3)][i & 7] = pr[0];
              pop[mb * 2 + (i >> 3)][(i & 7) + 1] = pr[1];
              l_run = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_run, false);
            }
          if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"i"(CPT) : "memory");   // V is there
          else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          auto v_operand = [&](int tt, int mb) { return at_lane.v_operand(vb, va, tt, mb); };
          bool odd = false;
          if (some) odd = any_odd<FTT, NMB>(v_operand);
          if (odd) {
            odd_values<FTT, NMB>(oacc, pop, v_operand);
          } else {
#pragma unroll
            for (int tt = 0; tt < FTT; ++tt)
#pragma unroll
              for (int mb = 0; mb < NMB; ++mb) oacc[mb] = mfma_32x32x16(v_operand(tt, mb), pop[tt], oacc[mb]);
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          if (more) ask(of_v, v_base, tile + WAVES, vb);
          if (at == WINDOW / 2) {   // (the next to be asked for is behind it)
            at = 0;
            now = next;
            next = window_of(tile + (1 + WINDOW / 2) * WAVES);
          }
          // (the wait behind these products as in attn_bf16_few.hip)
          __builtin_amdgcn_sched_barrier(0);
          asm volatile("s_nop 1");
        }
        // the waves' states meet
        const float l_tot = half_swap_sum(l_run), e_tot = STATS ? half_swap_sum(e_run) : 0.0f;
        if (hh == 0) few_stat[wave][lq] = f32x4{ref, l_tot, e_tot, 0.0f};
        __syncthreads();
        float ref_all = few_stat[0][lq][0], l_all = 0.0f, e_all = 0.0f;
#pragma unroll
        for (int j = 1; j < WAVES; ++j) ref_all = fmaxf(ref_all, few_stat[j][lq][0]);
#pragma unroll
        for (int j = 0; j < WAVES; ++j) {
          const f32x4 st = few_stat[j][lq];
          const float x = __builtin_amdgcn_exp2f((st[0] - ref_all) * scale_log2e);
          l_all += st[1] * x;
          e_all += st[2] * x;
        }
        // (a row that sees nothing has sum 0 and is 0)
        const float weight = __builtin_amdgcn_exp2f((ref - ref_all) * scale_log2e) * (!whole ? 1.0f : l_all == 0.0f ? 0.0f : 1.0f / l_all);
        // wave w's sums: 32 rows of D floats in its own buffers (K at d = 64, K and V at d = 128), the 16-byte pieces exchanged by the row
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const int piece = 8 * mb + 2 * i4 + hh;   // channels 4*piece ..
            float* dst = (float*)(mb < 2 ? kb : vb);
            const f32x4 x = {oacc[mb][4 * i4] * weight, oacc[mb][4 * i4 + 1] * weight, oacc[mb][4 * i4 + 2] * weight, oacc[mb][4 * i4 + 3] * weight};
            *(f32x4*)&dst[lq * 64 + (((piece & 15) ^ (lq & 15)) << 2)] = x;
          }
        __syncthreads();
        const size_t slot = (2 * (size_t)wg + (t0 == 0 ? 2 : 1)) * ROWS + (m0 - u.m0);
        for (int i = tid; i < (m1 - m0) * (D / 4); i += kThreads) {
          const int row = i / (D / 4), piece = i % (D / 4), mr = m0 + row;
          const int at = row * 256 + (((piece & 15) ^ (row & 15)) << 4);
          f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int j = 0; j < WAVES; ++j) {
            const char* of = piece < 16 ? (j < WAVES / 2 ? k_lds0 : k_lds1) : (j < WAVES / 2 ? v_lds0 : v_lds1);
            x += *(const f32x4*)(of + j % (WAVES / 2) * FEWB + at);
          }
          if (whole) {
            const bf16x4 y = {(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
            *(bf16x4*)(o + ((int64_t)(u.q0 + mr / group) * H + head * group + mr % group) * D + piece * 4) = y;
          } else {
            *(f32x4*)(part_o + (slot + row) * D + piece * 4) = x;
          }
        }
        if (wave == 0 && hh == 0 && m < m1) {
          if (!whole) part_stat[slot + lq] = f32x4{ref_all * scale_log2e, l_all, e_all, 0.0f};
          else if (STATS) lse[(int64_t)token * H + q_of] = row_statistic(ref_all * scale_log2e, e_all);
        }
        __syncthreads();   // (the next tiles take the place of the sums)
        m0 += 32;
        if (m0 >= min(u.m0 + ROWS, u.rows)) break;
        continue;
      }
      const int lane = here(tid) & 63;
      const Places<D> at_lane(lane, row_bytes);
      const int lq = at_lane.lq, hh = at_lane.hh;
      const int m = u.m0 + rw * 32 + lq, m_ld = min(m, u.rows - 1);   // this lane's row (surplus rows: a valid one, never stored)
      const int token = u.q0 + m_ld / group, q_of = head * group + m_ld % group;
      const int lim = min(causal ? u.len - u.nq + m_ld / group : n_keys - 1, n_keys - 1);   // last key this row sees
      const int seen_tiles = (n_seen + BC - 1) / BC;
      // the halves' tiles; a half without any walks one behind the last key: zeros, masked out
      const int n_all = max(min(t1, seen_tiles) - t0, 0), n_most = max((n_all + HALVES - 1) / HALVES, 1);
      const int n_tiles = half ? max(n_all - n_most, 1) : n_most;
      const int tile0 = half ? (n_all > 1 ? t0 + n_most : seen_tiles) : (n_all > 0 ? t0 : seen_tiles);
      const bool idle = u.m0 + rw * 32 >= u.rows;   // a wave without rows brings its part of the tiles in

      bf16x8 qop[KSTEPS];
      {
        const bf16* q_row = q + token * q_token + q_of * q_head;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) qop[s] = *(const bf16x8*)(q_row + 16 * s + 8 * hh);
      }
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) asm volatile("" : "+v"(qop[s]));   // (here before the tiles are asked for)

      // Lane i: where the wave's 16 keys of tile (first + i) of the half lie, and which of the tile's groups lie in the cache.
      struct Window {
        uint32_t lo, hi;
        int there;
      };
      auto window_of = [&](int first) {
        Window w = {0, 0, 0};
        const int key = (tile0 + first + lane) * BC;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const PageWindow p = page_window(table, key + 16 * g, n_seen, page_size, n_pages, page_bytes, row_bytes);
          w.there |= p.there << g;
          if (g == rw) {
            w.lo = p.lo;
            w.hi = p.hi;
          }
        }
        return w;
      };
      // Two windows, the second from the middle of the first on; it takes the first's place when that half is done with.
      int base;
      Window now, next;
      auto advance = [&](int it) {   // tiles before `it` are done with: those up to it + 31 lie in the window from here on
        if (it < base + 32) return;
        base += 32;
        now = next;
        next = window_of(base + 32);
      };
      auto there_of = [&](int it) { return __builtin_amdgcn_readlane(now.there, it - base); };
      const std::true_type yes;
      const std::false_type no;
      // The wave's 16 keys of a tile: where they lie, and how many bytes from there on. A tile's are taken when K is asked for and used for V, too.
      struct Group {
        uint32_t lo, hi;
        unsigned bytes;
      };
      auto group_of = [&](int it) {
        const int l = it - base, is = there_of(it) >> rw & 1, rows = min(n_seen - ((tile0 + it) * BC + 16 * rw), 16);
        return Group{(uint32_t)__builtin_amdgcn_readlane((int)now.lo, l), (uint32_t)__builtin_amdgcn_readlane((int)now.hi, l),
                     is ? (unsigned)((rows - 1) * row_bytes + ROWB) : 0u};
      };
      auto load_k = [&](const Group& g, int par) { at_lane.load_k(k_base + (g.lo | (uint64_t)g.hi << 32), g.bytes, row_bytes, k_buf(par) + rw * LPG * 1024); };
      auto load_v = [&](const Group& g, int par) { at_lane.load_v(v_base + (g.lo | (uint64_t)g.hi << 32), g.bytes, row_bytes, v_buf(par) + rw * LPG * 1024); };
      Group ahead1, ahead2;   // of tiles it + 1 and it + 2
      // What tile `it` brings in: K(it + 2) where K(it) was, V(it + 1) where V(it - 1) was.
      auto feed = [&](int it, int par) {
        if (it + 2 < n_tiles) load_k(ahead2, par);
        load_v(ahead1, par ^ 1);
      };
      auto fed = [&](int it) {
        ahead1 = ahead2;
        ahead2 = group_of(it + 3);
      };
      auto dma_wait = [&]() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
      auto masked = [&](int it) { return (tile0 + it) * BC + BC > all_see || there_of(it) != 15; };

      f32x16 oacc[NMB];
      float nref, l_run, e_run;   // negated reference (exp2 domain), sums over this lane's half of the keys
      float trigger;              // below zero until the row has met a score above -infinity: its first one becomes the reference
      bool far = false;           // a row of the wave has left a reference beyond kFar

      auto qk = [&](int par, f32x16 (&sacc)[MB]) {
        const char* at = k_buf(par);
        const int ka = at_lane.ka;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
          for (int i = 0; i < 16; ++i) sacc[mb][i] = 0.0f;
#pragma unroll
          for (int s = 0; s < KSTEPS; ++s) sacc[mb] = mfma_32x32x16(at_lane.k_operand(at, ka, mb, s), qop[s], sacc[mb]);
        }
      };
      auto apply_mask = [&](int it, f32x16 (&sc)[MB]) {
        const int there = there_of(it);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if ((tile0 + it) * BC + 32 * mb + 8 * (i >> 2) + 4 * hh + (i & 3) > lim || !(there >> (2 * mb + (i >> 3)) & 1)) sc[mb][i] = -INFINITY;
      };
      auto tile_max = [&](const f32x16 (&sc)[MB]) -> float {
        float mt = sc[0][0];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) mt = fmaxf(mt, sc[mb][i]);
        return __builtin_fmaf(half_swap_max(mt), scale_log2e, nref);
      };
      auto exp_tile = [&](const f32x16 (&sc)[MB], bf16x8 (&pop)[TT]) -> float {   // -> sum before rounding, with STATS
        float sum = 0.0f;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mb][i], scale_log2e, nref));
            const float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mb][i + 1], scale_log2e, nref));
            const bf16x2 pr = {(bf16)x0, (bf16)x1};
            pop[mb * 2 + (i >> 3)][i & 7] = pr[0];
            pop[mb * 2 + (i >> 3)][(i & 7) + 1] = pr[1];
            if constexpr (STATS) sum += x0 + x1;
          }
        return sum;
      };
      const RowSum row_sum(lane);
      auto shift_reference = [&](float delta) {
        nref -= delta;
        const float alpha = __builtin_amdgcn_exp2f(fminf(-delta, 0.0f));   // (a first reference has no sums)
        l_run *= alpha;
        if constexpr (STATS) e_run *= alpha;
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[mb][i] *= alpha;
      };
      // One tile, as in attn_bf16_impl.h. clean_c: neither it nor the next needs the mask.
      auto body = [&](auto clean_c, auto next_c, int it, int par, f32x16 (&sc)[MB], f32x16 (&sn)[MB]) {
        constexpr bool CLEAN = decltype(clean_c)::value, HAS_NEXT = decltype(next_c)::value;
        if constexpr (HAS_NEXT) {
          feed(it, par);
          qk(par ^ 1, sn);
          fed(it);
        }
        bf16x8 pop[TT];
        float es = exp_tile(sc, pop);
        float rs = row_sum(pop);
        // (d = 64: out of the loop's way, 2048 tokens on 16384 285 | 281 us with the look at the reference below; d = 128 472.5 | 474)
        const bool lift = __builtin_amdgcn_ballot_w64(!(rs <= trigger)) != 0;
        if (D == 64 ? __builtin_expect(lift, 0) : lift) {
          far |= __builtin_amdgcn_ballot_w64(!(__builtin_fabsf(nref) <= kFar)) != 0;
          const float mt = tile_max(sc);
          const bool first = trigger < 0.0f && mt > -INFINITY;
          if (first) trigger = kSumTrigger;
          shift_reference(mt > kTau || first ? mt : 0.0f);
          es = exp_tile(sc, pop);
          rs = RowSum::by_lanes(pop);
        }
        l_run += rs;
        if constexpr (STATS) e_run += es;
        const char* vb = v_buf(par);
        const int va = at_lane.va;
        auto v_operand = [&](int tt, int mb) { return at_lane.v_operand(vb, va, tt, mb); };
        {
          constexpr int PF = (4 / NMB < TT) ? 4 / NMB : TT - 1;
          bf16x8 va[PF + 1][NMB];
#pragma unroll
          for (int s = 0; s < PF; ++s)
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) va[s][mb] = v_operand(s, mb);
#pragma unroll
          for (int tt = 0; tt < TT; ++tt) {
            if (tt + PF < TT) {
#pragma unroll
              for (int mb = 0; mb < NMB; ++mb) va[(tt + PF) % (PF + 1)][mb] = v_operand(tt + PF, mb);
            }
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) oacc[mb] = mfma_32x32x16(va[tt % (PF + 1)][mb], pop[tt], oacc[mb]);
          }
          __builtin_amdgcn_sched_group_barrier(0x100, 2 * NMB * PF, 0);
#pragma unroll
          for (int i = 0; i < (TT - PF) * NMB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x008, PF * NMB, 0);
        }
        if constexpr (!CLEAN) {   // (the wait behind these products as in attn_bf16_few.hip)
          __builtin_amdgcn_sched_barrier(0);
          asm volatile("s_nop 3");
        }
        if constexpr (HAS_NEXT) {
          if constexpr (!CLEAN) {
            if (masked(it + 1)) apply_mask(it + 1, sn);
          }
          dma_wait();
        }
        __syncthreads();
      };

#pragma unroll
      for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[mb][i] = 0.0f;
      nref = l_run = e_run = 0.0f;
      trigger = kSumTrigger;
      base = 0;
      now = window_of(0);
      next = window_of(32);
      ahead2 = group_of(0);
      load_v(ahead2, 0);
      load_k(ahead2, 0);
      ahead1 = group_of(1);
      if (n_tiles > 1) load_k(ahead1, 1);
      ahead2 = group_of(2);
      dma_wait();
      __syncthreads();
      if (idle) {
        __syncthreads();
        for (int it = 0; it < n_tiles - 1; ++it) {
          advance(it);
          feed(it, it & 1);
          fed(it);
          dma_wait();
          __syncthreads();
        }
        __syncthreads();
      } else {
        f32x16 s0[MB], s1[MB];
        qk(0, s0);
        if (masked(0)) apply_mask(0, s0);
        const float first_max = tile_max(s0);
        if (first_max > -INFINITY) nref -= first_max;
        else trigger = -1.0f;
        __syncthreads();
        const int n_full = min(max(all_see / BC - tile0, 0), n_tiles);   // tiles that need no mask for their place
        int it = 0;
        while (it < n_tiles - 1) {
          advance(it);
          if ((it & 1) == 0) {
            // clean tiles of the window from `it` on
            const uint64_t bad = __builtin_amdgcn_ballot_w64(now.there != 15) >> (it - base);
            const int clean = min(min(n_full, it + (bad ? __builtin_ctzll(bad) : 64)), base + 61);   // (four tiles ahead are looked up)
            if (it + 2 < clean) {
              do {
                body(yes, yes, it, 0, s0, s1);
                body(yes, yes, it + 1, 1, s1, s0);
                __builtin_amdgcn_sched_barrier(0);   // (as above, for the way out of this loop)
                asm volatile("s_nop 3");
                it += 2;
              } while (it + 2 < clean);
              continue;
            }
          }
          body(no, yes, it, it & 1, s0, s1);
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) s0[mb] = s1[mb];
          ++it;
        }
        advance(it);
        body(no, no, it, it & 1, s0, s1);
      }
      if (HALVES == 2 && n_tiles < n_most) __syncthreads();   // (the other half's last tile)
      // Taken again as few rows, 32 at a time: a unit with sums that are no numbers where some rows do not see all keys of a tile (an infinity or a NaN among
      // its values reaches their sums, 0 times it; few rows look at the values), and one that has had a reference beyond kFar, its last or an earlier one.
      {
        float odd = !far && __builtin_fabsf(nref) <= kFar ? 0.0f : 1.0f;
        if (n_seen > all_see) {
#pragma unroll
          for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd = __builtin_fmaf(oacc[mb][i], 0.0f, odd);
        }
        if (__syncthreads_or(odd != 0.0f)) {   // (NaN is)
          few = true;
          continue;
        }
      }

      // ---- the halves meet: each hands the other one half of the channels and finishes the rest ----------------
      constexpr int OB = NMB / HALVES;
      const int c0 = HALVES == 2 ? half * (D / 2) : 0;
      float l_tot = half_swap_sum(l_run), e_tot = STATS ? half_swap_sum(e_run) : 0.0f;
      float ref = -nref;
      f32x16 out[OB];
      if constexpr (HALVES == 2) {
        static_assert(ROWS == kFewRows || (kRW * OB * 4096 <= BUFB && WAVES * 512 <= BUFB), "the exchange fits the tile buffers");
        f32x4* stat = (f32x4*)k_lds0;
        f32x4* give = (f32x4*)(half ? v_lds1 : v_lds0) + rw * (OB * 256) + lane;
        const f32x4* take = (const f32x4*)(half ? v_lds0 : v_lds1) + rw * (OB * 256) + lane;
        if (hh == 0) stat[wave * 32 + lq] = f32x4{-nref, l_tot, e_tot, 0.0f};
#pragma unroll
        for (int mb = 0; mb < OB; ++mb) {
          f32x16 theirs;
          if (half) {
            theirs = oacc[mb];
            out[mb] = oacc[mb + OB];
          } else {
            theirs = oacc[mb + OB];
            out[mb] = oacc[mb];
          }
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) give[(mb * 4 + i4) * 64] = f32x4{theirs[4 * i4], theirs[4 * i4 + 1], theirs[4 * i4 + 2], theirs[4 * i4 + 3]};
        }
        __syncthreads();
        // (a half that saw nothing of a row has sum 0 and no reference; a NaN sum makes the row NaN)
        const f32x4 st = stat[(wave ^ kRW) * 32 + lq];
        const float mine_ref = l_tot == 0.0f ? -FLT_MAX : -nref, other_ref = st[1] == 0.0f ? -FLT_MAX : st[0];
        ref = fmaxf(mine_ref, other_ref);
        const float wm = __builtin_amdgcn_exp2f(mine_ref - ref), wo = __builtin_amdgcn_exp2f(other_ref - ref);
        l_tot = __builtin_fmaf(wm, l_tot, wo * st[1]);
        e_tot = __builtin_fmaf(wm, e_tot, wo * st[2]);
#pragma unroll
        for (int mb = 0; mb < OB; ++mb)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const f32x4 x = take[(mb * 4 + i4) * 64];
#pragma unroll
            for (int j = 0; j < 4; ++j) out[mb][4 * i4 + j] = __builtin_fmaf(wm, out[mb][4 * i4 + j], wo * x[j]);
          }
      } else {
        if (l_tot == 0.0f) ref = -FLT_MAX;   // (as above, for the unit's other parts: a row that saw nothing has no reference)
#pragma unroll
        for (int mb = 0; mb < OB; ++mb) out[mb] = oacc[mb];
      }
      const float inv = !whole ? 1.0f : l_tot == 0.0f ? 0.0f : 1.0f / l_tot;
      if (m < u.rows) {
        const int64_t row = (int64_t)token * H + q_of;
        const size_t slot = (2 * (size_t)wg + (t0 == 0 ? 2 : 1)) * ROWS + rw * 32 + lq;
        if (hh == 0 && half == 0) {
          if (!whole) part_stat[slot] = f32x4{ref, l_tot, e_tot, 0.0f};
          else if (STATS) lse[row] = row_statistic(ref, e_tot);
        }
#pragma unroll
        for (int mb = 0; mb < OB; ++mb)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const int c = c0 + 32 * mb + 8 * i4 + 4 * hh;
            const f32x4 x = f32x4{out[mb][4 * i4], out[mb][4 * i4 + 1], out[mb][4 * i4 + 2], out[mb][4 * i4 + 3]} * inv;
            if (whole) *(bf16x4*)(o + row * D + c) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
            else *(f32x4*)(part_o + slot * D + c) = x;
          }
      }
      __syncthreads();   // (the next unit's tiles take the place of the sums)
      break;
    }
  }
}

template <int D, int ROWS, int WAVES, bool CUT>
hipError_t launch_as(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                     const PagedLaunch& l, hipStream_t stream) {
  const float scale_log2e = scale * 1.4426950408889634f;
  const PagedScratch at(scratch, l.workgroups, ROWS, D);
  hipLaunchKernelGGL((p.lse_out ? paged_kernel<D, true, ROWS, WAVES, CUT> : paged_kernel<D, false, ROWS, WAVES, CUT>), dim3((unsigned)l.workgroups), dim3(WAVES * 64),
                     0, stream, (const bf16*)q, (const bf16*)k_pages, (const bf16*)v_pages, (bf16*)o, p.page_table, p.q_start, p.kv_len, p.lse_out, p.H,
                     p.Hkv, p.n_seq, p.n_tokens, p.n_pages, p.page_size, p.max_pages, p.page_stride * 2, p.head_stride * 2, (int)(p.row_stride * 2),
                     p.q_stride[0], p.q_stride[1], p.causal, scale_log2e, l.ranges, l.least, l.most, at.sums, at.stats, at.cuts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !l.ranges) return e;
  hipLaunchKernelGGL((paged_combine_kernel<bf16, D, ROWS>), dim3((unsigned)(l.workgroups * (ROWS * D / 1024))), dim3(256), 0, stream, at.sums, at.stats,
                     at.cuts, (bf16*)o, p.lse_out, p.H, p.Hkv);
  return hipGetLastError();
}

// How a call is launched. us:
//   units of 32 rows for no more new tokens than sequences (units of 128 | of 32, both with eight waves): H32 Hkv8 one of 777 d64 12.8 | 11.5, 32 of up
//     to 8000 d128 123 | 112. Tokens that are all one sequence's take longer: 250 on 2000 among 256 places 25 | 30, 500 on 4000 among 512 d128 61 | 101.
//   workgroups of eight, four, two waves by the units that there are at least, so that as many begin at once as compute units hold (eight | four |
//     two waves; H32 Hkv8 d64): 16 of 8000 42 | 44 | 44, one of 100003 49 | 54 | 61; 48 of up to 1000 23 | 19 | 25; 128 of up to 300 34 | 23 | 18.
//     With 128 rows eight | four: 1024 on 4096 49 | 59; 64 of 8 new tokens H16 71 | 65.
//   whole units where the full ones alone are more than compute units (ranges | whole): a prompt of 1400, H32 Hkv8 d64 42 | 26, 1900 on 6000 122 | 105; of
//     fewer it is not known whether they fill the chip: 1000 on 16000 165 | 200. And where the table has no room for more tiles of a sequence than beginning,
//     ending and joining units take, the more the better the units fill the chip by themselves: single tokens H32 Hkv8 d64 of one sequence of 1200
//     13.6 | 12.1, 2000 13.0 | 16.2, of 16 of up to 2000 20.1 | 17.4, 4000 25.1 | 25.9; d128 of one of 1000 14.3 | 15.6, 1300 14.3 | 17.2, of 16 of up to
//     1300 23.0 | 19.9; 60 new of two of 16 of up to 1300 d64 25.0 | 21.0, 3200 31.2 | 34.6.
struct PagedForm {
  int rows, waves;   // of a unit, of a workgroup
  PagedLaunch launch;
};
PagedForm paged_form(const da_paged& p, size_t scratch_bytes) {
  const int group = p.H / p.Hkv;
  const long long heads = (long long)p.n_seq * p.Hkv, full = (long long)p.n_tokens * group / kUnitRows * p.Hkv;
  const int units = (int)std::min(std::max(heads, full), (long long)kComputeUnits);   // that there are at least
  auto form = [&](int rows, int waves) {
    const int from = rows == kUnitRows ? 16 + units / 6 : p.d == 64 ? 20 + std::min(units, kComputeUnits / 2) / 4 : 12 + std::min(units, kComputeUnits / 2) / 6;
    return PagedForm{rows, waves, paged_launch(p, rows, kTileKeys, paged_pad(rows, waves), kComputeUnits * 8 / waves, from, scratch_bytes)};
  };
  if (p.n_tokens <= p.n_seq && group <= kFewRows) return form(kFewRows, heads <= kComputeUnits ? 8 : heads <= 2 * kComputeUnits ? 4 : 2);
  if (full > kComputeUnits) return PagedForm{kUnitRows, 4, PagedLaunch{(int)(paged_units(p, kUnitRows) * p.Hkv), 0, 0, 0}};
  if (heads > kComputeUnits) {
    const PagedForm f = form(kUnitRows, 4);
    if (!f.launch.ranges || f.launch.workgroups > kComputeUnits) return f;   // (a smaller scratch: one workgroup a compute unit)
  }
  return form(kUnitRows, 8);
}

template <int D>
hipError_t launch_d(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                    size_t scratch_bytes, hipStream_t stream) {
  const PagedForm f = paged_form(p, scratch_bytes);
  const auto launch = f.rows == kFewRows ? (f.waves == 2 ? launch_as<D, kFewRows, 2, true> : f.waves == 4 ? launch_as<D, kFewRows, 4, true> : launch_as<D, kFewRows, 8, true>)
                      : f.waves == 8     ? launch_as<D, kUnitRows, 8, true>
                      : f.launch.ranges  ? launch_as<D, kUnitRows, 4, true>
                                         : launch_as<D, kUnitRows, 4, false>;
  return launch(q, k_pages, v_pages, o, p, scale, scratch, f.launch, stream);
}

}  // namespace

size_t paged_scratch_bytes(const da_paged& p) {
  return p.dtype == DA_F32 ? paged_f32_scratch_bytes(p) : paged_launch_bytes(2 * kComputeUnits, kUnitRows, p.d);
}

hipError_t launch_paged(const void* q, const void* k_pages, const void* v_pages, void* o, const da_paged& p, float scale, void* scratch,
                        size_t scratch_bytes, hipStream_t stream) {
  if (p.dtype == DA_F32) return launch_paged_f32(q, k_pages, v_pages, o, p, scale, scratch, scratch_bytes, stream);
  return p.d == 64 ? launch_d<64>(q, k_pages, v_pages, o, p, scale, scratch, scratch_bytes, stream)
                   : launch_d<128>(q, k_pages, v_pages, o, p, scale, scratch, scratch_bytes, stream);
}

}  // namespace da
