// How the attention over a paged cache is dealt out to workgroups.
//
// A unit is a run of `rows` query rows of one sequence and kv head (all query heads of the kv head, token after token) against the
// keys that they see, in tiles. The lengths lie on the device, so every workgroup finds its own work: it sums the
// units and tiles of the sequences, 64 at a time, a lane for each.
//   whole units   workgroup w takes unit w / Hkv of kv head w % Hkv.
//   ranges        all tiles, unit after unit and kv head after kv head, are one line, which is cut into equal ranges: every
//                 workgroup has the same walk whatever the lengths are. A unit that ranges cut is put together by the combine kernel from the
//                 sums that they leave: workgroup w those of the unit that its range begins in at 2 w, of the one that it ends in, if that
//                 is another, at 2 w + 1. The ones in between are whole.
#pragma once
#include <cfloat>

#include "da_common.h"
#include "paged.h"

namespace da {

namespace {

struct PagedBatch {
  const int* __restrict__ q_start;
  const int* __restrict__ kv_len;
  int n_seq, n_tokens, n_heads_kv;
  int group;       // query heads of a kv head
  int max_keys;    // that a row of the page table has room for
  int causal;
};

struct PagedUnit {
  int seq, q0, nq;     // sequence, its first new token and their number
  int len;             // its keys (as told, not cut to the table's room)
  int m0, rows;        // first query row of the unit (token * group + head), rows of the sequence
  int tiles;           // of the sequence's keys: those that the line counts for the unit
  unsigned first;      // place of the unit's first tile among a kv head's
};

__device__ inline unsigned wave_scan(unsigned x) {   // sums over the lanes up to one's own
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned y = (unsigned)__builtin_amdgcn_ds_bpermute((((threadIdx.x & 63) - d) & 63) << 2, (int)x);
    if ((int)(threadIdx.x & 63) >= d) x += y;
  }
  return x;
}

template <int ROWS, int KEYS>
struct PagedSequence {   // what a lane knows of its sequence
  int q0, nq, len, units, tiles;
  __device__ PagedSequence(const PagedBatch& b, int s) {
    q0 = nq = len = units = tiles = 0;
    if (s >= b.n_seq) return;
    q0 = min(max(b.q_start[s], 0), b.n_tokens);
    nq = max(min(max(b.q_start[s + 1], 0), b.n_tokens) - q0, 0);
    len = max(b.kv_len[s], 0);
    units = (int)(((long long)nq * b.group + ROWS - 1) / ROWS);
    tiles = max((min(len, b.max_keys) + KEYS - 1) / KEYS, 1);
  }
};

// All tiles of a kv head.
template <int ROWS, int KEYS>
__device__ inline unsigned paged_total(const PagedBatch& b) {
  unsigned total = 0;
  for (int s0 = 0; s0 < b.n_seq; s0 += 64) {
    const PagedSequence<ROWS, KEYS> q(b, s0 + (threadIdx.x & 63));
    total += (unsigned)__builtin_amdgcn_readlane((int)wave_scan((unsigned)q.units * (unsigned)q.tiles), 63);
  }
  return total;
}

// The unit that holds place `x` of a kv head's line (BY_UNIT: its x-th unit); false behind the last one.
template <int ROWS, int KEYS, bool BY_UNIT>
__device__ inline bool paged_find(const PagedBatch& b, unsigned x, PagedUnit* out) {
  unsigned before = 0, tiles_before = 0;
  for (int s0 = 0; s0 < b.n_seq; s0 += 64) {
    const PagedSequence<ROWS, KEYS> q(b, s0 + (threadIdx.x & 63));
    const unsigned w = (unsigned)q.units * (unsigned)q.tiles, sum = wave_scan(w);
    const unsigned at = BY_UNIT ? wave_scan((unsigned)q.units) : sum;
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + at > x);
    if (past != 0) {
      const int i = __builtin_ctzll(past);
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, i); };
      const unsigned in = x - before - (unsigned)of((int)(at - (BY_UNIT ? (unsigned)q.units : w)));
      const int tiles = of(q.tiles);
      const int unit = BY_UNIT ? (int)in : (int)(in / (unsigned)tiles);
      out->seq = s0 + i;
      out->q0 = of(q.q0);
      out->nq = of(q.nq);
      out->len = of(q.len);
      out->m0 = unit * ROWS;
      out->rows = out->nq * b.group;
      out->tiles = tiles;
      out->first = tiles_before + (unsigned)of((int)(sum - w)) + (unsigned)unit * (unsigned)tiles;
      return true;
    }
    before += (unsigned)__builtin_amdgcn_readlane((int)at, 63);
    tiles_before += (unsigned)__builtin_amdgcn_readlane((int)sum, 63);
  }
  return false;
}

// Length of a range: equal ones for `workgroups` of them, none shorter than `least` tiles.
__device__ inline long long paged_range(long long total, int workgroups, int least) {
  return max((total + workgroups - 1) / workgroups, (long long)least);
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

// Units that ranges have cut, from the sums of their parts. E: type of o.
template <typename E, int D, int ROWS, int KEYS>
__global__ __launch_bounds__(256) void paged_combine_kernel(
    const float* __restrict__ part_o, const f32x4* __restrict__ part_stat, E* __restrict__ o, const int* __restrict__ q_start,
    const int* __restrict__ kv_len, float* __restrict__ lse, int H, int Hkv, int n_seq, int n_tokens, int max_keys, int workgroups, int least) {
  const int group = H / Hkv, head = blockIdx.x % Hkv;
  const PagedBatch batch = {q_start, kv_len, n_seq, n_tokens, Hkv, group, max_keys, 0};
  PagedUnit u;
  if (!paged_find<ROWS, KEYS, true>(batch, blockIdx.x / Hkv, &u)) return;
  const long long per_head = paged_total<ROWS, KEYS>(batch);
  const long long length = paged_range(per_head * Hkv, workgroups, least);
  const long long first = head * per_head + u.first, last = first + u.tiles - 1;
  const int w0 = (int)(first / length), w1 = (int)(last / length);
  if (w0 == w1) return;
  const int rows = min(ROWS, u.rows - u.m0);
  for (int i = threadIdx.x; i < rows * (D / 4); i += 256) {
    const int row = i / (D / 4), c = i % (D / 4) * 4;
    // (all but the first part begin with their range)
    const size_t slot0 = (2 * (size_t)w0 + (w0 * length >= first ? 0 : 1)) * ROWS + row;
    auto slot_of = [&](int w) { return w == w0 ? slot0 : 2 * (size_t)w * ROWS + row; };
    float ref = -FLT_MAX;
#pragma unroll 4
    for (int w = w0; w <= w1; ++w) ref = fmaxf(ref, part_stat[slot_of(w)][0]);
    float l = 0.0f, e = 0.0f;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int w = w0; w <= w1; ++w) {
      const size_t slot = slot_of(w);
      const f32x4 st = part_stat[slot];
      const float weight = __builtin_amdgcn_exp2f(st[0] - ref);
      l = __builtin_fmaf(weight, st[1], l);
      e = __builtin_fmaf(weight, st[2], e);
      const f32x4 y = *(const f32x4*)(part_o + slot * D + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(weight, y[j], x[j]);
    }
    const int mr = u.m0 + row;
    const int64_t at = (int64_t)(u.q0 + mr / group) * H + head * group + mr % group;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[at * D + c + j] = (E)(x[j] * inv);
    if (lse && c == 0) lse[at] = row_statistic(ref, e);
  }
}

// How a call is launched: units dealt out whole, or ranges with sums of their parts in scratch.
struct PagedLaunch {
  int workgroups, ranges, least;
};
// (no more units than this, whatever the sequences' shares of the tokens are)
inline long long paged_units(const da_paged& p, int rows) { return (long long)p.n_tokens * (p.H / p.Hkv) / rows + std::min(p.n_seq, p.n_tokens); }
inline size_t paged_sum_bytes(int workgroups, int rows, int d) { return (size_t)2 * workgroups * rows * d * 4; }
inline size_t paged_launch_bytes(int workgroups, int rows, int d) { return (size_t)2 * workgroups * rows * (d + 4) * 4; }
// `most` workgroups are resident at a time. Ranges, unless no sequence is long enough for two of them, with what fits the scratch.
inline PagedLaunch paged_launch(const da_paged& p, int rows, int keys, int most, size_t scratch_bytes) {
  const long long room = ((long long)p.max_pages * p.page_size + keys - 1) / keys;
  const int least = 4;
  const int n = (int)std::min((long long)most, (long long)(scratch_bytes / paged_launch_bytes(1, rows, p.d)));
  if (n >= 2 && room >= 20) return PagedLaunch{n, 1, least};
  return PagedLaunch{(int)(paged_units(p, rows) * p.Hkv), 0, least};
}

}  // namespace

}  // namespace da
