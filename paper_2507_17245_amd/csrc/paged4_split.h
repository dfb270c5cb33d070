// How the bf16 attention over a paged cache of 4-bit codes is dealt out (paged_units.h): forms of a call, a workgroup's share. Here every kv head has a
// line of its own, cut into the same number of ranges.
#pragma once
#include <numeric>

#include "paged_units.h"

namespace da {

namespace {

// Places of the line: a tile of a unit of 128 rows takes 2600 cycles where its keys come from memory, one of few rows 410: four of them are one place.
constexpr int kUnitRows = 128, kFewRows = 16, kTileKeys = 64;   // rows and keys of the line's units and tiles
constexpr int paged4_pad(int rows, int waves) { return rows != kFewRows ? 8 : waves == 8 ? 10 : 6; }
constexpr int kSimdWaves = 2;   // (2 | 3, us: 64 sequences of up to 8192 d64 47.4 | 48.3, 200 of up to 2500 d128 79.6 | 86: registers, and more parts to join)

// The workgroup's work: pos .. end of a line (ranges), or one unit.
template <typename CALL, typename LINE, int ROWS>
struct Share {
  unsigned pos = 0, end = 1;
  int wg = blockIdx.x, head = 0;
  __device__ Share(const CALL& p, const LINE& line) {
    if (!p.ranges) return;
    // Every kv head's line is cut into the same `ranges` ones. What follows each other here lies on one XCD: with few rows those of one place in the lines, as
    // several heads' scales (and, tokens outside, codes) lie in one line of 128 bytes; with units of 128 rows those of one head, which read the same keys.
    if ((gridDim.x & 7) == 0) wg = (wg & 7) * (gridDim.x >> 3) + (wg >> 3);
    const int part = ROWS == kFewRows ? wg / p.Hkv : wg % p.ranges;
    head = ROWS == kFewRows ? wg % p.Hkv : wg / p.ranges;
    wg = head * p.ranges + part;
    const unsigned length = paged_range(line.total, p.ranges, p.least);
    pos = paged_cut(line, part, length, line.total);
    end = paged_cut(line, part + 1, length, line.total);
    PagedCut cut = paged_mark<ROWS>(line, pos, end, length, line.total);
    cut.head = head;
    cut.last += head * p.ranges;
    if (threadIdx.x == 0) p.cuts[wg] = cut;
  }
  // The next unit and its tiles; false: none.
  __device__ bool next(const CALL& p, const LINE& line, PagedUnit& u, int& t0, int& t1) {
    if (pos >= end) return false;
    if (p.ranges) {
      if (!line.template find<false>(pos, &u)) return false;
      t0 = (int)(pos - u.first);
      t1 = min(u.places, t0 + (int)(end - pos));
    } else {
      // A kv head's units on one XCD where there are eight of them; those of a sequence that see the most keys first. Few rows of heads whose rows of codes lie next
      // to each other and share lines of 128 bytes: every eighth unit's heads on one XCD (else | so, us, H32 Hkv8: 200 sequences of up to 2500 d64 109 | 72, d128 129 |
      // 100, 64 of up to 1000 20.3 | 14.6; heads outside tokens d128, which share none, 67 | 69).
      int unit = wg / p.Hkv;
      head = wg % p.Hkv;
      if (ROWS == kFewRows && p.near && wg < (int)(gridDim.x / (8u * (unsigned)p.Hkv)) * 8 * p.Hkv) {
        unit = (wg >> 3) / p.Hkv * 8 + (wg & 7);
        head = (wg >> 3) % p.Hkv;
      }
      if (!line.template find<true>(unit, &u)) return false;
      u.m0 = (u.rows - 1) / ROWS * ROWS - u.m0;
      t0 = 0;
      t1 = u.places;
    }
    pos += (unsigned)(t1 - t0);
    return true;
  }
};

// How a call is launched. us, H32 Hkv8, sequences of random lengths from a quarter of the given one on:
//   units of 16 rows for no more new tokens than sequences. Workgroups of eight waves up to 256 units, else of four, of two for more than 512 where the table has
//     room for 1280 keys (four | two waves: 256 sequences of up to 100 d64 17.1 | 11.1, 600 24.2 | 19.8, 1000 32.3 | 28.6; 1000 of up to 300 79.5 | 58.8, d128 104 | 79; but
//     200 of up to 2500 d64 48.2 | 51.4, d128 72.4 | 77).
//   their units stay whole (ranges | whole: 64 sequences of up to 1000 d64 18.7 | 12.2, d128 20 | 14.9; 256 of up to 1500 51 | 41.6; 200 of up to 2500 d128 77.6 | 73) unless the table
//     has room for so many keys that the longest one holds up the others: d64 one sequence of 2500 11.2 | 12.4, 16 of up to 6000 19.5 | 21.3, 64 of up to 8192
//     45.6 | 48, 32 of up to 16000, which fill the chip once, 46 | 49; d128 one of 1500 11.4 | 12.0, 16 of up to 4000 19.1 | 21.5, 64 of up to 6000 54.5 | 57.4.
//   units of 128 rows otherwise: as in attn_paged.hip.
struct Paged4Form {
  int rows, waves;   // of a unit, of a workgroup
  PagedLaunch launch;
};
inline Paged4Form paged4_form(const da_paged& p, size_t scratch_bytes) {
  const int group = p.H / p.Hkv;
  const long long heads = (long long)p.n_seq * p.Hkv, full = (long long)p.n_tokens * group / kUnitRows * p.Hkv, room = (long long)p.max_pages * p.page_size;
  const int units = (int)std::min(std::max(heads, full), (long long)kComputeUnits);   // that there are at least
  auto form = [&](int rows, int waves, int from) {
    PagedLaunch l = paged_launch(p, rows, kTileKeys, paged4_pad(rows, waves), 4 * kSimdWaves * kComputeUnits / waves, from, scratch_bytes);
    if (l.ranges) {
      l.ranges = l.workgroups / p.Hkv;
      const int whole = 8 / std::gcd(8, p.Hkv);   // of a number of workgroups that the XCDs share evenly
      if (l.ranges > 16 * whole) l.ranges -= l.ranges % whole;
      if (l.ranges < 2) l.ranges = 0;
      l.workgroups = l.ranges ? l.ranges * p.Hkv : (int)(paged_units(p, rows) * p.Hkv);
    }
    return Paged4Form{rows, waves, l};
  };
  if (p.n_tokens <= p.n_seq && group <= 2 * kFewRows) {
    const int few = (int)std::min(heads, (long long)kComputeUnits);
    const int from = heads > kComputeUnits ? (p.d == 64 ? 96 : 64) : p.d == 64 ? 24 + few / 2 : 18 + few / 4;
    return form(kFewRows, heads <= kComputeUnits ? 8 : heads > 2 * kComputeUnits && room <= 20 * kTileKeys ? 2 : 4, from);
  }
  if (full > kComputeUnits) return Paged4Form{kUnitRows, 4, PagedLaunch{(int)(paged_units(p, kUnitRows) * p.Hkv), 0, 0, 0}};
  return form(kUnitRows, heads > kComputeUnits ? 4 : 8, 16 + units / 6);
}

}  // namespace

}  // namespace da
