// Attention of new tokens over a paged cache of 4-bit codes (fp4.h), bf16: single tokens to chunks of a prompt. Work split: paged_units.h.
//
//   O = softmax(scale Q K^T) V over the keys that a row sees, one pass: running reference and sum of every row.
//
// A unit is up to 128 query rows of a sequence and a kv head (all query heads of the kv head, token after token); of calls with single tokens up to
// 16 rows, by a kernel with the walk of few rows alone (paged4_few.h).
//   more than 32 rows: as in attn_paged.hip: waves own 32 rows each, and of eight waves each of a pair with the same rows walks half of the unit's
//     tiles of 64 keys in buffers of its half's own. The four waves that share a tile load 16 keys of it each, convert them and write them to LDS
//     as bf16, keys two tiles ahead of the products, values one; codes are asked for a tile before. Bound: the matrix products (at d = 64 the
//     exponentials beside them); the conversions are 16 (d = 64) or 32 instructions a wave and tile.
//   up to 32 rows: 16 at a time as few rows.
#include "paged4_few.h"
#include "paged4_split.h"

namespace da {

namespace {

constexpr int kRW = 4;   // waves over the 128 rows of a unit

// Where the 16-byte pieces of a row of 64 keys lie in LDS: neither the writes (eight lanes at a time: a piece of every quarter of two rows) nor the reads of K (the
// same piece of eight rows) and the transposing ones of V (two pairs of pieces of four rows) meet in a bank. (Counted at d = 128: none. At d = 64 conflicts take 9 % of a
// compute unit's cycles; exchanged by row >> 1 for sixteen lanes at a time, 2048 tokens on 16384 take the same, 298 us.)
template <int D>
__device__ inline int k_piece(int row, int piece) {
  return D == 64 ? piece ^ (row & 7) : piece ^ (piece >> 3) ^ (row & 7) << 1 ^ (row >> 3 & 1);
}
template <int D>
__device__ inline int v_piece(int row, int piece) {
  return D == 64 ? piece ^ ((row >> 1 & 1) << 2 | (row & 1)) : piece ^ (piece >> 3) ^ ((row & 3) << 2 | (row & 1) << 1);
}

// Codes of 16 keys or values, on their way or here: a lane has a quarter of a row.
template <int D>
struct Quarter {
  static constexpr int WORDS = D / 32;
  uint32_t codes[WORDS];
  int scale;
  __device__ void load(const uint8_t* from, const uint8_t* scales, uint64_t code, uint64_t at_scale, int code_at, int scale_at) {
    scale = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rows_rsrc(scales + at_scale), scale_at, 0, 0);
    if constexpr (WORDS == 2) {
      const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows_rsrc(from + code), code_at, 0, 0));
      codes[0] = x[0];
      codes[1] = x[1];
    } else {
      const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows_rsrc(from + code), code_at, 0, 0));
#pragma unroll
      for (int j = 0; j < 4; ++j) codes[j] = x[j];
    }
  }
  template <typename AT>
  __device__ void store(AT at, bool zero) const {   // at(piece of the quarter): where it lies
    const float s = scale_value(zero ? 0 : scale);
#pragma unroll
    for (int j = 0; j < WORDS; ++j) *(bf16x8*)at(j) = values_of(codes[j], s);
  }
};

// Single tokens: units of 16 rows.
template <int D, bool STATS, int WAVES, bool FAR>
__global__ __launch_bounds__(WAVES * 64, kSimdWaves) void paged4_few_kernel(const Paged4Call p) {
  __shared__ __attribute__((aligned(1024))) char v_lds[WAVES][8192];
  __shared__ f32x4 stat_lds[WAVES][16];
  __shared__ PagedLds line_lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const PagedBatch batch = {p.q_start, p.kv_len, p.n_seq, p.n_tokens, p.H / p.Hkv, p.max_pages * p.page_size, p.most};
  typedef PagedLine<kFewRows, kTileKeys, paged4_pad(kFewRows, WAVES)> Line;
  const Line line(batch, &line_lds, wave, WAVES);
  Share<Paged4Call, Line, kFewRows> share(p, line);
  // Every key is read once. Calls of more than 64 MB leave the caches alone where a head's rows lie together (else heads share lines): 64 sequences of up to 8192 d64
  // 47.1 -> 44.4 us, one of 100003 Hkv8 d128 34.4 -> 30.5, 200 of up to 2500 79 -> 74.5; but 16 of up to 2000 d64 14.8 -> 15.6, and tokens outside, H16 d128 73.7 -> 76.8.
  const bool once = (long long)line.tiles * p.Hkv * (kTileKeys * 2 * (D / 2 + D / 32)) > 64LL << 20 && p.cache.code_row == D / 2;
  PagedUnit u;
  int t0, t1;
  while (share.next(p, line, u, t0, t1)) {
    const size_t slot = (2 * (size_t)share.wg + (t0 == 0 ? 2 : 1)) * kFewRows;
    const bool whole = t0 == 0 && t1 == u.places;
    auto buffer = [&](int w) { return v_lds[w]; };
    if (!FAR && once) few_rows<D, STATS, WAVES, FAR, !FAR>(p, u, share.head, u.m0, t0, t1, whole, slot, wave, buffer, stat_lds);
    else few_rows<D, STATS, WAVES, FAR, false>(p, u, share.head, u.m0, t0, t1, whole, slot, wave, buffer, stat_lds);
    __syncthreads();   // (the next tiles take the place of the sums)
  }
}

// Chunks and mixed batches: units of 128 rows. WAVES: 8, one workgroup a compute unit; 4: two, one beginning or ending its units beside the others' walks.
template <int D, bool STATS, int WAVES, bool FAR>
__global__ __launch_bounds__(WAVES * 64, 2) void paged4_rows_kernel(const Paged4Call p) {
  constexpr int ROWS = kUnitRows, BC = kTileKeys, ROWB = D * 2, TILEB = BC * ROWB;
  constexpr int MB = BC / 32, TT = BC / 16, KSTEPS = D / 16, NMB = D / 32, WORDS = D / 32;
  constexpr float kSumTrigger = (BC / 2) * 256.0f;   // (as in attn_bf16_impl.h)
  constexpr int HALVES = WAVES == 2 * kRW ? 2 : 1, BUFB = HALVES * TILEB;
  static_assert(BUFB >= WAVES / 4 * 8192, "room for the waves' tiles with few rows");
  __shared__ __attribute__((aligned(1024))) char k_lds0[BUFB];
  __shared__ __attribute__((aligned(1024))) char k_lds1[BUFB];
  __shared__ __attribute__((aligned(1024))) char v_lds0[BUFB];
  __shared__ __attribute__((aligned(1024))) char v_lds1[BUFB];
  __shared__ f32x4 stat_lds[WAVES][16];
  __shared__ PagedLds line_lds;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % kRW, half = HALVES == 1 ? 0 : wave / kRW;
  const int group = p.H / p.Hkv;
  const PagedBatch batch = {p.q_start, p.kv_len, p.n_seq, p.n_tokens, group, p.max_pages * p.page_size, p.most};
  auto k_buf = [&](int par) -> char* { return (par ? k_lds1 : k_lds0) + half * TILEB; };
  auto v_buf = [&](int par) -> char* { return (par ? v_lds1 : v_lds0) + half * TILEB; };
  auto few_buf = [&](int w) -> char* {   // 8 KB of a wave's own
    constexpr int EACH = WAVES / 4;
    char* const from = w / EACH == 0 ? k_lds0 : w / EACH == 1 ? k_lds1 : w / EACH == 2 ? v_lds0 : v_lds1;
    return from + w % EACH * 8192;
  };
  typedef PagedLine<ROWS, BC, paged4_pad(ROWS, WAVES), 2 * kFewRows> Line;
  const Line line(batch, &line_lds, wave, WAVES);
  Share<Paged4Call, Line, ROWS> share(p, line);
  PagedUnit u;
  int t0, t1;
  while (share.next(p, line, u, t0, t1)) {
    const int head = share.head;
    const bool whole = t0 == 0 && t1 == u.places;
    const size_t slot0 = (2 * (size_t)share.wg + (t0 == 0 ? 2 : 1)) * ROWS;
    const int unit_end = min(u.m0 + ROWS, u.rows);
    const int few_tiles = u.rows <= 2 * kFewRows ? kFewTiles : 1;   // of a place
    bool few = u.rows - u.m0 <= 2 * kFewRows;
    if (!few) {
      const int lane = here(tid) & 63, lq = lane & 31, hh = lane >> 5;
      const int n_keys = min(u.len, batch.max_keys);
      const int* table = p.page_table + (int64_t)u.seq * p.max_pages;
      const int n_seen = p.causal ? min(n_keys, max(u.len - u.nq + (unit_end - 1) / group + 1, 0)) : n_keys;   // no row sees more
      const int all_see = p.causal ? min(max(u.len - u.nq + u.m0 / group + 1, 0), n_keys) : n_keys;   // keys below this every row sees
      const int m = u.m0 + rw * 32 + lq, m_ld = min(m, u.rows - 1);   // this lane's row (surplus rows: a valid one, never stored)
      const int token = u.q0 + m_ld / group, q_of = head * group + m_ld % group;
      const int lim = min(p.causal ? u.len - u.nq + m_ld / group : n_keys - 1, n_keys - 1);   // last key this row sees
      const int seen_tiles = (n_seen + BC - 1) / BC;
      // the halves' tiles; a half without any walks one behind the last key: zeros, masked out
      const int n_all = max(min(t1, seen_tiles) - t0, 0), n_most = max((n_all + HALVES - 1) / HALVES, 1);
      const int n_tiles = half ? max(n_all - n_most, 1) : n_most;
      const int tile0 = half ? (n_all > 1 ? t0 + n_most : seen_tiles) : (n_all > 0 ? t0 : seen_tiles);
      const bool idle = u.m0 + rw * 32 >= u.rows;   // a wave without rows brings its part of the tiles in

      bf16x8 qop[KSTEPS];
      {
        const bf16* q_row = p.q + token * p.q_token + q_of * p.q_head;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) qop[s] = *(const bf16x8*)(q_row + 16 * s + 8 * hh);
      }

      // Lane i: where the wave's 16 keys of tile (first + i) of the half lie, and which of the tile's groups lie in the cache.
      struct Window {
        uint32_t code, scale;
        int there;
      };
      auto window_of = [&](int first) {
        Window w = {0, 0, 0};
        const int key = (tile0 + first + lane) * BC;
        int pages[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) pages[i] = table[(unsigned)max(min(key + 16 * i, n_seen - 1), 0) / (unsigned)p.page_size];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = key + 16 * i, page = at < n_seen ? pages[i] : -1;
          CodeWindow c;
          c.template place<FAR>(page, at % (unsigned)p.page_size, p.n_pages, p.cache);
          w.there |= (page >= 0 && page < p.n_pages ? 1 : 0) << i;
          if (i == rw) {
            w.code = c.code;
            w.scale = c.scale;
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

      const int vr = lane >> 2, vp = lane & 3;   // row of the wave's 16 and quarter of it that the lane brings
      const int code_at = vr * p.cache.code_row + vp * (D / 8), scale_at = vr * p.cache.scale_row + vp * (D / 4) / 32;
      const uint8_t* k_codes = p.cache.k_codes + head * p.cache.code_head;
      const uint8_t* v_codes = p.cache.v_codes + head * p.cache.code_head;
      const uint8_t* k_scales = p.cache.k_scales + head * p.cache.scale_head;
      const uint8_t* v_scales = p.cache.v_scales + head * p.cache.scale_head;
      Quarter<D> k_ahead, v_ahead;   // of the tiles whose turn is next
      auto ask = [&](Quarter<D>& to, const uint8_t* codes, const uint8_t* scales, int it) {
        const int a = __builtin_amdgcn_readlane((int)now.code, it - base), b = __builtin_amdgcn_readlane((int)now.scale, it - base);
        to.load(codes, scales, FAR ? (uint64_t)(a * p.cache.code_page + (int64_t)b * p.cache.code_row) : (uint64_t)(uint32_t)a,
                FAR ? (uint64_t)(a * p.cache.scale_page + (int64_t)b * p.cache.scale_row) : (uint64_t)(uint32_t)b, code_at, scale_at);
      };
      auto ask_k = [&](int it) { ask(k_ahead, k_codes, k_scales, it); };
      auto ask_v = [&](int it) { ask(v_ahead, v_codes, v_scales, it); };
      auto put_k = [&](const Quarter<D>& from, int par) {
        char* const to = k_buf(par) + (16 * rw + vr) * ROWB;
        from.store([&](int j) { return to + (k_piece<D>(vr, vp * WORDS + j) << 4); }, false);
      };
      auto put_v = [&](int it, int par) {   // rows that none of the unit's sees: zeros
        char* const to = v_buf(par) + (16 * rw + vr) * ROWB;
        const bool hidden = (tile0 + it) * BC + 16 * rw + vr >= n_seen || !(there_of(it) >> rw & 1);
        v_ahead.store([&](int j) { return to + (v_piece<D>(vr, vp * WORDS + j) << 4); }, hidden);
      };
      // What tile `it` brings in: K(it + 2) where K(it) was, V(it + 1) where V(it - 1) was; and the codes of the next ones.
      auto feed = [&](int it, int par) {
        put_k(k_ahead, par);
        put_v(it + 1, par ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        ask_k(it + 3);
        ask_v(it + 2);
        __builtin_amdgcn_sched_barrier(0);
      };
      auto masked = [&](int it) { return (tile0 + it) * BC + BC > all_see || there_of(it) != 15; };

      f32x16 oacc[NMB];
      float nref, l_run, e_run;   // negated reference (exp2 domain), sums over this lane's half of the keys
      float trigger;              // below zero until the row has met a score above -infinity: its first one becomes the reference
      bool far = false;           // a row of the wave has left a reference beyond kFar
      const int ka = lq * ROWB + (k_piece<D>(lq, hh) << 4);
      const int row_l = 4 * hh + ((lane & 15) >> 2);
      const int va = row_l * ROWB + (v_piece<D>(row_l, (lane >> 4 & 1) << 1 | (lane & 3) >> 1) << 4) + 8 * (lane & 1);
      auto v_operand = [&](const char* tile, int tt, int mb) {
        const char* p0 = tile + (va ^ (v_piece<D>(0, 4 * mb) << 4)) + 16 * tt * ROWB;
        return lds_read_tr_pair<bf16x8>(p0, p0 + 8 * ROWB);
      };

      auto qk = [&](int par, f32x16 (&sacc)[MB]) {
        const char* at = k_buf(par);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
          for (int i = 0; i < 16; ++i) sacc[mb][i] = 0.0f;
#pragma unroll
          for (int s = 0; s < KSTEPS; ++s)
            sacc[mb] = mfma_32x32x16(*(const bf16x8*)(at + (ka ^ (k_piece<D>(0, 2 * s) << 4)) + mb * 32 * ROWB), qop[s], sacc[mb]);
        }
      };
      auto apply_mask = [&](int it, f32x16 (&sc)[MB]) {
        const int there = there_of(it), past = here(lim - (tile0 + it) * BC - 4 * hh);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * mb + 8 * (i >> 2) + (i & 3) > past || !(there >> (2 * mb + (i >> 3)) & 1)) sc[mb][i] = -INFINITY;
      };
      auto tile_max = [&](const f32x16 (&sc)[MB]) -> float {
        float mt = sc[0][0];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) mt = fmaxf(mt, sc[mb][i]);
        return __builtin_fmaf(half_swap_max(mt), p.scale_log2e, nref);
      };
      auto exp_tile = [&](const f32x16 (&sc)[MB], bf16x8 (&pop)[TT]) -> float {   // -> sum before rounding, with STATS
        float sum = 0.0f;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mb][i], p.scale_log2e, nref));
            const float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mb][i + 1], p.scale_log2e, nref));
            const bf16x2 pr = {(bf16)x0, (bf16)x1};
            pop[mb * 2 + (i >> 3)][i & 7] = pr[0];
            pop[mb * 2 + (i >> 3)][(i & 7) + 1] = pr[1];
            if constexpr (STATS) {
              sum += x0 + x1;
              asm volatile("" : "+v"(sum));   // (at once: pairs that wait for their turn do not fit the registers, d = 128 with row statistics 570 -> 505 us)
            }
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
        }
        bf16x8 pop[TT];
        float es = exp_tile(sc, pop);
        float rs = row_sum(pop);
        if (__builtin_amdgcn_ballot_w64(!(rs <= trigger)) != 0) {
          far |= __builtin_amdgcn_ballot_w64(!(__builtin_fabsf(nref) <= kFar)) != 0;
          const float mt = tile_max(sc);
          const bool first = trigger < 0.0f && mt > -INFINITY;
          if (first) trigger = kSumTrigger;
          shift_reference(mt > kLift || first ? mt : 0.0f);
          es = exp_tile(sc, pop);
          rs = RowSum::by_lanes(pop);
        }
        l_run += rs;
        if constexpr (STATS) e_run += es;
        const char* vb = v_buf(par);
        {
          constexpr int PF = (4 / NMB < TT) ? 4 / NMB : TT - 1;
          bf16x8 va[PF + 1][NMB];
#pragma unroll
          for (int s = 0; s < PF; ++s)
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) va[s][mb] = v_operand(vb, s, mb);
#pragma unroll
          for (int tt = 0; tt < TT; ++tt) {
            if (tt + PF < TT) {
#pragma unroll
              for (int mb = 0; mb < NMB; ++mb) va[(tt + PF) % (PF + 1)][mb] = v_operand(vb, tt + PF, mb);
            }
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) oacc[mb] = mfma_32x32x16(va[tt % (PF + 1)][mb], pop[tt], oacc[mb]);
          }
        }
        if constexpr (!CLEAN) {   // (the wait behind these products as in attn_bf16_few.hip)
          __builtin_amdgcn_sched_barrier(0);
          asm volatile("s_nop 3");
        }
        if constexpr (HAS_NEXT && !CLEAN) {
          if (masked(it + 1)) apply_mask(it + 1, sn);
        }
        lds_barrier();
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
      {
        Quarter<D> first;
        ask(first, k_codes, k_scales, 0);
        ask_v(0);
        ask_k(1);
        put_k(first, 0);
        put_v(0, 0);
        put_k(k_ahead, 1);
      }
      ask_k(2);
      ask_v(1);
      __syncthreads();
      if (idle) {
        lds_barrier();
        for (int it = 0; it < n_tiles - 1; ++it) {
          advance(it);
          feed(it, it & 1);
          lds_barrier();
        }
        lds_barrier();
      } else {
        f32x16 s0[MB], s1[MB];
        qk(0, s0);
        if (masked(0)) apply_mask(0, s0);
        const float first_max = tile_max(s0);
        if (first_max > -INFINITY) nref -= first_max;
        else trigger = -1.0f;
        lds_barrier();
        const int n_full = min(max(all_see / BC - tile0, 0), n_tiles);   // tiles that need no mask for their place
        int it = 0;
        while (it < n_tiles - 1) {
          advance(it);
          if ((it & 1) == 0) {
            // clean tiles of the window from `it` on
            const uint64_t bad = __builtin_amdgcn_ballot_w64(now.there != 15) >> (it - base);
            const int clean = min(min(n_full, it + (bad ? __builtin_ctzll(bad) : 64)), base + 60);   // (four tiles ahead are looked up)
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
      if (HALVES == 2 && n_tiles < n_most) lds_barrier();   // (the other half's last tile)
      // Taken again as few rows: a unit with sums that are no numbers where some rows do not see all keys of a tile (an infinity or a NaN among its values
      // reaches their sums, 0 times it; few rows look at the values), and one that has had a reference beyond kFar, its last or an earlier one.
      {
        float odd = !far && __builtin_fabsf(nref) <= kFar ? 0.0f : 1.0f;
        if (n_seen > all_see) {
#pragma unroll
          for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd = __builtin_fmaf(oacc[mb][i], 0.0f, odd);
        }
        few = __syncthreads_or(odd != 0.0f);   // (NaN is)
      }
      if (!few) {
        // ---- the halves meet: each hands the other one half of the channels and finishes the rest ----------------
        constexpr int OB = NMB / HALVES;
        const int c0 = HALVES == 2 ? half * (D / 2) : 0;
        float l_tot = half_swap_sum(l_run), e_tot = STATS ? half_swap_sum(e_run) : 0.0f;
        float ref = -nref;
        f32x16 out[OB];
        if constexpr (HALVES == 2) {
          static_assert(kRW * OB * 4096 <= BUFB && WAVES * 512 <= BUFB, "the exchange fits the tile buffers");
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
          const int64_t row = (int64_t)token * p.H + q_of;
          const size_t slot = slot0 + rw * 32 + lq;
          if (hh == 0 && half == 0) {
            if (!whole) p.part_stat[slot] = f32x4{ref, l_tot, e_tot, 0.0f};
            else if (STATS) p.lse[row] = row_statistic(ref, e_tot);
          }
#pragma unroll
          for (int mb = 0; mb < OB; ++mb)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
              const int c = c0 + 32 * mb + 8 * i4 + 4 * hh;
              const f32x4 x = f32x4{out[mb][4 * i4], out[mb][4 * i4 + 1], out[mb][4 * i4 + 2], out[mb][4 * i4 + 3]} * inv;
              if (whole) *(bf16x4*)(p.o + row * D + c) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
              else *(f32x4*)(p.part_o + slot * D + c) = x;
            }
        }
      }
      __syncthreads();   // (the next unit's tiles take the place of the sums)
    }
    if (few) {
      for (int m0 = u.m0; m0 < unit_end; m0 += kFewRows) {
        few_rows<D, STATS, WAVES, FAR, false>(p, u, head, m0, t0 * few_tiles, t1 * few_tiles, whole, slot0 + (m0 - u.m0), wave, few_buf, stat_lds);
        __syncthreads();
      }
    }
  }
}

template <int D, int ROWS, int WAVES, bool FAR>
hipError_t launch_as(Paged4Call call, void* scratch, const PagedLaunch& l, hipStream_t stream) {
  const PagedScratch at(scratch, l.workgroups, ROWS, D);
  call.ranges = l.ranges;
  call.least = l.least;
  call.most = l.most;
  call.part_o = at.sums;
  call.part_stat = at.stats;
  call.cuts = at.cuts;
  const dim3 grid((unsigned)l.workgroups), block(WAVES * 64);
  if constexpr (ROWS == kFewRows) {
    if (call.lse) hipLaunchKernelGGL((paged4_few_kernel<D, true, WAVES, FAR>), grid, block, 0, stream, call);
    else hipLaunchKernelGGL((paged4_few_kernel<D, false, WAVES, FAR>), grid, block, 0, stream, call);
  } else {
    if (call.lse) hipLaunchKernelGGL((paged4_rows_kernel<D, true, WAVES, FAR>), grid, block, 0, stream, call);
    else hipLaunchKernelGGL((paged4_rows_kernel<D, false, WAVES, FAR>), grid, block, 0, stream, call);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !l.ranges) return e;
  hipLaunchKernelGGL((paged_combine_kernel<bf16, D, ROWS>), dim3((unsigned)(l.workgroups * (ROWS * D / 1024))), dim3(256), 0, stream, at.sums, at.stats,
                     at.cuts, call.o, call.lse, call.H, call.Hkv);
  return hipGetLastError();
}

template <int D, int WAVES>
auto few_launch(bool far) {
  return far ? launch_as<D, kFewRows, WAVES, true> : launch_as<D, kFewRows, WAVES, false>;
}
template <int D, int WAVES>
auto rows_launch(bool far) {
  return far ? launch_as<D, kUnitRows, WAVES, true> : launch_as<D, kUnitRows, WAVES, false>;
}
template <int D>
hipError_t launch_d(const Paged4Call& call, bool far, const da_paged& p, void* scratch, size_t scratch_bytes, hipStream_t stream) {
  const Paged4Form f = paged4_form(p, scratch_bytes);
  const auto launch = f.rows == kUnitRows ? (f.waves == 8 ? rows_launch<D, 8>(far) : rows_launch<D, 4>(far))
                      : f.waves == 8      ? few_launch<D, 8>(far)
                      : f.waves == 4      ? few_launch<D, 4>(far)
                                          : few_launch<D, 2>(far);
  return launch(call, scratch, f.launch, stream);
}

}  // namespace

size_t paged4_scratch_bytes(const da_paged& p) {
  return p.dtype == DA_F32 ? paged4_f32_scratch_bytes(p) : paged_launch_bytes(kSimdWaves * kComputeUnits, kUnitRows, p.d);
}

hipError_t launch_paged4(const void* q, void* o, const da_cache4& c, const da_paged& p, float scale, void* scratch, size_t scratch_bytes, hipStream_t stream) {
  if (p.dtype == DA_F32) return launch_paged4_f32(q, o, c, p, scale, scratch, scratch_bytes, stream);
  const Codes cache = {(const uint8_t*)c.k_codes, (const uint8_t*)c.k_scales, (const uint8_t*)c.v_codes, (const uint8_t*)c.v_scales, c.code_stride[0],
                       c.code_stride[1], c.scale_stride[0], c.scale_stride[1], (int)c.code_stride[2], (int)c.scale_stride[2]};
  // whether a kv head's pages reach farther than offsets of 31 bits
  auto reaches = [&](const int64_t* stride) { return (p.n_pages - 1) * (double)stride[0] + (p.page_size - 1) * (double)stride[2] + p.d > 2e9; };
  const bool far = reaches(c.code_stride) || reaches(c.scale_stride);
  Paged4Call call = {};
  call.q = (const bf16*)q;
  call.cache = cache;
  call.o = (bf16*)o;
  call.page_table = p.page_table;
  call.q_start = p.q_start;
  call.kv_len = p.kv_len;
  call.lse = p.lse_out;
  call.H = p.H;
  call.Hkv = p.Hkv;
  call.n_seq = p.n_seq;
  call.n_tokens = p.n_tokens;
  call.n_pages = p.n_pages;
  call.page_size = p.page_size;
  call.max_pages = p.max_pages;
  call.q_token = p.q_stride[0];
  call.q_head = p.q_stride[1];
  call.causal = p.causal;
  call.near = c.code_stride[1] == p.d / 2 && c.code_stride[2] > p.d / 2;
  call.scale_log2e = scale * 1.4426950408889634f;
  return p.d == 64 ? launch_d<64>(call, far, p, scratch, scratch_bytes, stream) : launch_d<128>(call, far, p, scratch, scratch_bytes, stream);
}

}  // namespace da
