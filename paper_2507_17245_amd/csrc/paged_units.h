// How the attention over a paged cache is dealt out to workgroups.
//
// A unit is a run of `rows` query rows of one sequence and kv head (all query heads of the kv head, token after token) against the
// keys that they see, in tiles. The lengths lie on the device, so every workgroup finds its own work: it sums the
// units and tiles of the sequences, 64 at a time, a lane for each.
//   whole units   workgroup w takes unit w / Hkv of kv head w % Hkv.
//   ranges        all tiles, unit after unit and kv head after kv head, are one line, which is cut into equal ranges, one a workgroup:
//                 each has the same walk whatever the lengths are. Beginning and ending a unit costs as much as several
//                 tiles: behind its tiles a unit has PAD places without one, and a cut on them or less than `snap` tiles from
//                 either end of the tiles moves to the end. A unit that cuts fall into is put together by the
//                 combine kernel from the sums of its parts: those of the part in front of its first cut, which workgroup w begins
//                 at, at 2 w, those of a part that begins with workgroup w's cut at 2 w + 1.
//                 PAD 0 | as it is (ranges, us): three chunks of up to 48 on 700, float H8 d64 24.0 | 18.2; decoding H32 Hkv8 d64, 16 sequences of up
//                 to 2000 25.5 | 19.9, one of 8000 18.6 | 15.6; 60 and one new token each of four of up to 4000, d128 40.7 | 35.7. (One
//                 prompt of 512 on 4096, whose units half a range fits without, 34.6 | 36.3.) Places spread over the tiles, more snap: 5-20 % more.
#pragma once
#include <cfloat>

#include "da_common.h"
#include "paged.h"

namespace da {

namespace {

struct PagedBatch {
  const int* __restrict__ q_start;
  const int* __restrict__ kv_len;
  int n_seq, n_tokens;
  int group;       // query heads of a kv head
  int max_keys;    // that a row of the page table has room for
  unsigned most;   // places of a kv head's line that starts in ascending order may make
};

struct PagedUnit {
  int seq, q0, nq;     // sequence, its first new token and their number
  int len;             // its keys (as told, not cut to the table's room)
  int m0, rows;        // first query row of the unit (token * group + head), rows of the sequence
  int places;          // the line's for it: a tile each for the sequence's keys and PAD behind them
  unsigned first;      // the unit's first place among a kv head's
};

template <int CTRL, int ROWS>
__device__ inline unsigned dpp_add(unsigned x) {
  return x + (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
__device__ inline unsigned wave_scan(unsigned x) {   // sums over the lanes up to one's own
  x = dpp_add<0x111, 0xf>(x);   // row_shr 1, 2, 4, 8: sums within rows of 16 lanes
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);   // row_bcast 15: a row's last lane to the next row
  return dpp_add<0x143, 0xc>(x);   // row_bcast 31: the second row's last lane to the upper two
}

// The sum of all lanes' x, given wave_scan(x); the largest number where it is beyond 32 bits.
__device__ inline unsigned wave_total(unsigned x, unsigned scan) {
  return __builtin_amdgcn_ballot_w64(scan < x) == 0 ? (unsigned)__builtin_amdgcn_readlane((int)scan, 63) : ~0u;
}

struct PagedLds {   // of a workgroup
  int seq[7][64];                     // the first 64 sequences
  unsigned places[64], units[64];     // of each 64 sequences, up to 4096 of them
};

template <int ROWS, int KEYS, int PAD>
struct PagedSequence {   // what a lane knows of its sequence
  int q0, nq, len, units, places;   // (places of a unit)
  unsigned sum, unit_sum;   // places and units of the sequences up to it, in its 64
  __device__ PagedSequence(const PagedBatch& b, int s) {
    q0 = nq = len = units = places = 0;
    if (s < b.n_seq) {
      const int at = b.q_start[s], to = b.q_start[s + 1], keys = b.kv_len[s];
      q0 = min(max(at, 0), b.n_tokens);
      nq = max(min(max(to, 0), b.n_tokens) - q0, 0);
      len = max(keys, 0);
      units = (int)(((unsigned)nq * (unsigned)b.group + (ROWS - 1)) / ROWS);
      places = max((min(len, b.max_keys) + KEYS - 1) / KEYS, 1) + PAD;
    }
    sum = wave_scan((unsigned)units * (unsigned)places);
    unit_sum = wave_scan((unsigned)units);
  }
  __device__ PagedSequence(const PagedLds* lds, int lane)
      : q0(lds->seq[0][lane]), nq(lds->seq[1][lane]), len(lds->seq[2][lane]), units(lds->seq[3][lane]), places(lds->seq[4][lane]),
        sum((unsigned)lds->seq[5][lane]), unit_sum((unsigned)lds->seq[6][lane]) {}
  __device__ void store(PagedLds* lds, int lane) const {
    const int x[7] = {q0, nq, len, units, places, (int)sum, (int)unit_sum};
#pragma unroll
    for (int i = 0; i < 7; ++i) lds->seq[i][lane] = x[i];
  }
  __device__ unsigned all_places() const { return wave_total((unsigned)units * (unsigned)places, sum); }
  __device__ unsigned all_units() const { return (unsigned)__builtin_amdgcn_readlane((int)unit_sum, 63); }
};

// The line of a kv head. The first 64 sequences stay in LDS. Of more, up to 4096, LDS has the sums of each 64, which the waves
// take a share of, and the 64 that are asked for are loaded again; beyond, the sums are taken again, too.
// Starts out of order may count the same tokens many times, more than 32 bits hold and than the parts of units have scratch for: sums stay at the
// largest number then, and a line of more places than ascending starts can make is taken as empty (no range has work).
template <int ROWS, int KEYS, int PAD>
struct PagedLine {
  typedef PagedSequence<ROWS, KEYS, PAD> Sequence;
  static constexpr unsigned kPad = PAD;
  const PagedBatch b;
  PagedLds* const lds;
  unsigned total, tiles;   // its places, those of them that are tiles
  // (called by all threads of the workgroup)
  __device__ PagedLine(const PagedBatch& batch, PagedLds* to, int wave, int waves) : b(batch), lds(to) {
    const int lane = threadIdx.x & 63, n = (b.n_seq + 63) / 64;
    const Sequence head(b, lane);
    if (wave == 0) head.store(lds, lane);
    total = head.all_places();
    unsigned units = head.all_units();
    if (n > 64) {
      for (int c = 1; c < n; ++c) {
        const Sequence q(b, c * 64 + lane);
        const unsigned more = q.all_places();
        total = total + more < more ? ~0u : total + more;
        units += q.all_units();
      }
    } else if (n > 1) {
      for (int c = wave; c < n; c += waves) {
        const Sequence q(b, c * 64 + lane);
        const unsigned all = q.all_places();
        if (lane == 63) {
          lds->places[c] = all;
          lds->units[c] = q.unit_sum;
        }
      }
    }
    __syncthreads();
    if (n > 1 && n <= 64) {
      const unsigned all = lane < n ? lds->places[lane] : 0u;
      total = wave_total(all, wave_scan(all));
      units = (unsigned)__builtin_amdgcn_readlane((int)wave_scan(lane < n ? lds->units[lane] : 0u), 63);
    }
    tiles = total - units * (unsigned)PAD;
    if (total > b.most) total = 0;
  }
  // The unit that holds place `x` (BY_UNIT: the x-th unit); false behind the last one.
  template <bool BY_UNIT>
  __device__ bool find(unsigned x, PagedUnit* out) const {
    const int lane = threadIdx.x & 63, n = (b.n_seq + 63) / 64;
    if (n == 1) return in<BY_UNIT>(Sequence(lds, lane), 0, x, 0, out);
    if (n <= 64) {
      const unsigned t = lane < n ? lds->places[lane] : 0u, u = lane < n ? lds->units[lane] : 0u, ts = wave_scan(t), us = wave_scan(u);
      const uint64_t past = __builtin_amdgcn_ballot_w64((BY_UNIT ? us : ts) > x);
      if (past == 0) return false;
      const int c = __builtin_ctzll(past);
      const unsigned places = (unsigned)__builtin_amdgcn_readlane((int)(ts - t), c), units = (unsigned)__builtin_amdgcn_readlane((int)(us - u), c);
      return in<BY_UNIT>(Sequence(b, c * 64 + lane), c * 64, x - (BY_UNIT ? units : places), places, out);
    }
    unsigned places = 0, units = 0;
    for (int c = 0; c < n; ++c) {
      const Sequence q(b, c * 64 + lane);
      if (in<BY_UNIT>(q, c * 64, x - (BY_UNIT ? units : places), places, out)) return true;
      places += q.all_places();
      units += q.all_units();
    }
    return false;
  }

 private:
  // among 64 sequences from s0 on, with `before` places in front of them
  template <bool BY_UNIT>
  __device__ bool in(const Sequence& q, int s0, unsigned x, unsigned before, PagedUnit* out) const {
    const uint64_t past = __builtin_amdgcn_ballot_w64((BY_UNIT ? q.unit_sum : q.sum) > x);
    if (past == 0) return false;
    const int i = __builtin_ctzll(past);
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, i); };
    const unsigned first = (unsigned)of((int)(q.sum - (unsigned)q.units * (unsigned)q.places));
    const int places = of(q.places);
    const int unit = BY_UNIT ? (int)(x - (unsigned)of((int)(q.unit_sum - (unsigned)q.units))) : (int)((x - first) / (unsigned)places);
    out->seq = s0 + i;
    out->q0 = of(q.q0);
    out->nq = of(q.nq);
    out->len = of(q.len);
    out->m0 = unit * ROWS;
    out->rows = out->nq * b.group;
    out->places = places;
    out->first = before + first + (unsigned)unit * (unsigned)places;
    return true;
  }
};

// (All kv heads' places stay below 2^32, by the call's checks: 2e9 tiles and 2.5e8 units of up to 8 places more.)
// Length of a range: equal ones for `workgroups` of them, none shorter than `least` tiles.
__device__ inline unsigned paged_range(unsigned total, int workgroups, int least) {
  return max((total + (unsigned)workgroups - 1) / (unsigned)workgroups, (unsigned)least);
}
__device__ inline unsigned paged_snap(unsigned length) { return min(max(length / 8, 1u), 6u); }
// Where range w begins.
template <typename LINE>
__device__ inline unsigned paged_cut(const LINE& line, unsigned w, unsigned length, unsigned total) {
  const unsigned at = w * length;
  if (at >= total) return total;
  PagedUnit u;
  const unsigned head = at / line.total;
  if (!line.template find<false>(at - head * line.total, &u)) return total;
  const unsigned in = at - head * line.total - u.first, snap = paged_snap(length);
  return in < snap ? at - in : (unsigned)u.places - in < snap + LINE::kPad ? at - in + (unsigned)u.places : at;
}

// Where the keys of 16 successive places lie: a lane for each such group of a wave's next 64. The group's first row of
// the page, in bytes, and whether the page is one of the cache's.
struct PageWindow {
  uint32_t lo, hi;
  int there;
};
__device__ inline PageWindow page_window(const int* __restrict__ table, int key, int n_keys, int page_size, int n_pages,
                                         int64_t page_bytes, int64_t row_bytes) {
  PageWindow w = {0, 0, 0};
  if (key < n_keys) {
    const unsigned at = (unsigned)key / (unsigned)page_size;
    const int id = table[at];
    if (id >= 0 && id < n_pages) {
      const uint64_t off = (uint64_t)(id * page_bytes + (int64_t)((unsigned)key - at * (unsigned)page_size) * row_bytes);
      w = PageWindow{(uint32_t)off, (uint32_t)(off >> 32), 1};
    }
  }
  return w;
}

// log-sum-exp of a row from its reference (log2 units) and the sum relative to it
__device__ inline float row_statistic(float ref, float sum) { return sum == 0.0f ? -INFINITY : 0.6931471805599453f * (ref + __builtin_log2f(sum)); }

// What the combine kernel knows of a unit that cuts fall into, left by the workgroup of its first part (rows 0: there is none).
struct PagedCut {
  int rows, q0, m0, head;   // of the unit
  int last;                 // its last cut; the first is the next workgroup's
  int unused[3];
};
// The range from `begin` to `end`: whether a unit that begins in it is cut at its end.
template <int ROWS, typename LINE>
__device__ inline PagedCut paged_mark(const LINE& line, unsigned begin, unsigned end, unsigned length, unsigned total) {
  PagedCut cut = {0, 0, 0, 0, 0, {0, 0, 0}};
  PagedUnit u;
  if (end >= total) return cut;
  const unsigned head = end / line.total;
  if (!line.template find<false>(end - head * line.total, &u)) return cut;
  const unsigned first = head * line.total + u.first;
  if (first == end || first < begin) return cut;
  const unsigned last = (first + (unsigned)u.places - LINE::kPad - paged_snap(length)) / length;   // (in front of the line's end, which the last range has)
  return PagedCut{min(ROWS, u.rows - u.m0), u.q0, u.m0, (int)head, (int)last, {0, 0, 0}};
}

// Units that cuts fall into, from the sums of their parts: a workgroup for every 1024 / D rows that a unit may have, behind every cut. Where
// there are fewer rows, lanes share a row's parts. E: type of o.
template <typename E, int D, int ROWS>
__global__ __launch_bounds__(256) void paged_combine_kernel(
    const float* __restrict__ part_o, const f32x4* __restrict__ part_stat, const PagedCut* __restrict__ cuts, E* __restrict__ o,
    float* __restrict__ lse, int H, int Hkv) {
  constexpr int TAKE = 1024 / D, C4 = D / 4;
  __shared__ f32x4 x_lds[256], stat_lds[256];
  constexpr int PIECES = ROWS / TAKE;
  // (pieces shifted by the cut: neither one cut's pieces nor the first pieces of all cuts end up on one XCD)
  const int group = H / Hkv, wg = blockIdx.x / PIECES, piece = (blockIdx.x + wg) % PIECES;
  const PagedCut u = cuts[wg];
  const int rows = min(u.rows - piece * TAKE, TAKE);
  if (rows <= 0) return;
  int side = 1;   // lanes' rows side by side, a power of two
  while (side < rows) side *= 2;
  const int c = threadIdx.x % C4 * 4, at_row = threadIdx.x / C4 % side, share = threadIdx.x / (C4 * side), shares = TAKE / side;
  const int row = piece * TAKE + min(at_row, rows - 1), first = wg + 1, parts = u.last - first + 2;
  auto slot_of = [&](int i) { return (i == 0 ? 2 * (size_t)first : 2 * (size_t)(first + i - 1) + 1) * ROWS + row; };
  f32x4 all = {-FLT_MAX, 0.0f, 0.0f, 0.0f}, x = {0.0f, 0.0f, 0.0f, 0.0f};   // reference, sum, sum before rounding
  auto add = [&](f32x4 st, f32x4 y) {
    const float ref = fmaxf(all[0], st[0]);
    const float a = __builtin_amdgcn_exp2f(all[0] - ref), b = __builtin_amdgcn_exp2f(st[0] - ref);
    all = f32x4{ref, __builtin_fmaf(b, st[1], a * all[1]), __builtin_fmaf(b, st[2], a * all[2]), 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf(b, y[i], a * x[i]);
  };
  for (int i = share; i < parts; i += 4 * shares) {   // four parts in flight
    f32x4 st[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const size_t slot = slot_of(min(i + j * shares, parts - 1));
      st[j] = part_stat[slot];
      y[j] = *(const f32x4*)(part_o + slot * D + c);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j * shares < parts) add(st[j], y[j]);
  }
  if (shares > 1) {
    x_lds[threadIdx.x] = x;
    stat_lds[threadIdx.x] = all;
    __syncthreads();
    if (share == 0)
      for (int j = 1; j < shares; ++j) add(stat_lds[threadIdx.x + j * C4 * side], x_lds[threadIdx.x + j * C4 * side]);
  }
  if (share != 0 || at_row >= rows) return;
  const int mr = u.m0 + row;
  const int64_t at = (int64_t)(u.q0 + mr / group) * H + u.head * group + mr % group;
  x *= all[1] == 0.0f ? 0.0f : 1.0f / all[1];
  typedef __attribute__((ext_vector_type(4))) E Four;
  *(Four*)(o + at * D + c) = Four{(E)x[0], (E)x[1], (E)x[2], (E)x[3]};
  if (lse && c == 0) lse[at] = row_statistic(all[0], all[2]);
}

// How a call is launched: units dealt out whole, or ranges with sums of their parts in scratch.
struct PagedLaunch {
  int workgroups, ranges, least;
  unsigned most;   // places of a kv head's line
};
// (no more units than this, whatever the sequences' shares of the tokens are)
inline long long paged_units(const da_paged& p, int rows) { return (long long)p.n_tokens * (p.H / p.Hkv) / rows + std::min(p.n_seq, p.n_tokens); }
// Scratch: sums [2 * workgroups][rows][d], their statistics [2 * workgroups][rows][4], cuts [workgroups].
inline size_t paged_launch_bytes(int workgroups, int rows, int d) { return (size_t)workgroups * (2 * (size_t)rows * (d + 4) * 4 + sizeof(PagedCut)); }
struct PagedScratch {
  float* sums;
  f32x4* stats;
  PagedCut* cuts;
  PagedScratch(void* at, int workgroups, int rows, int d) {
    sums = (float*)at;
    stats = (f32x4*)(sums + (size_t)2 * workgroups * rows * d);
    cuts = (PagedCut*)(stats + (size_t)2 * workgroups * rows);
  }
};
// `most` workgroups are resident at a time. Ranges of `least` places or more, as many as there are places in all and the scratch has room for, where
// the table has room for `from` tiles of a sequence.
inline PagedLaunch paged_launch(const da_paged& p, int rows, int keys, int pad, int most, int from, size_t scratch_bytes) {
  constexpr int least = 4;
  const long long room = ((long long)p.max_pages * p.page_size + keys - 1) / keys, line = (room + pad) * paged_units(p, rows), places = line * p.Hkv;
  const int n = (int)std::min({(long long)most, (places + least - 1) / least, (long long)(scratch_bytes / paged_launch_bytes(1, rows, p.d))});
  if (n >= 2 && room >= from) return PagedLaunch{n, 1, least, (unsigned)line};
  return PagedLaunch{(int)(paged_units(p, rows) * p.Hkv), 0, least, (unsigned)line};
}

}  // namespace

}  // namespace da
