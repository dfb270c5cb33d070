// The work split of the attention over a paged cache of 4-bit codes (csrc/paged4_split.h) on the CPU, by the lanes of paged_split_driver.cpp: every
// tile of every unit once, parts in places of their own within the scratch, for every form that a call is launched in.
#define main paged_split_main
#include "paged_split_driver.cpp"
#undef main

#include "paged4_split.h"

namespace da {
namespace {

struct Call4 {
  int ranges, Hkv, least, near;
  PagedCut* cuts;
};

template <int ROWS, int WAVES>
void check4(const char* name, const Batch& b, const PagedLaunch& l, size_t scratch) {
  typedef PagedLine<ROWS, kTileKeys, paged4_pad(ROWS, WAVES), ROWS == kUnitRows ? 2 * kFewRows : 0> Line;
  typedef Share<Call4, Line, ROWS> Work;
  const da_paged& p = b.p;
  const int group = p.H / p.Hkv, max_keys = p.max_pages * p.page_size;
  CHECK(l.workgroups >= 1);
  CHECK(!l.ranges || (l.workgroups == l.ranges * p.Hkv && l.ranges >= 2 && paged_launch_bytes(l.workgroups, ROWS, p.d) <= scratch));
  CHECK(l.ranges || l.workgroups >= 1);
  const PagedBatch batch = {b.start.data(), b.len.data(), p.n_seq, p.n_tokens, group, max_keys, l.most};
  std::vector<Part> parts;
  std::vector<PagedCut> cuts(l.workgroups, PagedCut{-1, 0, 0, 0, 0, {0, 0, 0}});
  static int turn = 0;   // (heads' rows next to each other or not)
  const Call4 call = {l.ranges, p.Hkv, l.least, ++turn / 2 % 2, cuts.data()};
  PagedLds lds;
  unsigned line_total = 0;
  gridDim.x = (unsigned)l.workgroups;
  for (int wg = 0; wg < l.workgroups && g_failed == 0; ++wg) {
    std::vector<Part> mine;
    blockIdx.x = (unsigned)wg;
    wave::run([&] {
      const bool tell = wave::current == 0;
      const Line line(batch, &lds, 0, 1);
      Work share(call, line);
      if (tell) line_total = line.total;
      Part x;
      for (int n = 0; share.next(call, line, x.u, x.t0, x.t1); ++n) {
        if (n > 4000) {   // (far more than any of these batches has)
          if (tell) CHECK(!"a range ends");
          return;
        }
        x.wg = share.wg;
        x.head = share.head;
        if (tell) mine.push_back(x);
      }
    });
    parts.insert(parts.end(), mine.begin(), mine.end());
  }
  std::set<size_t> slots;
  std::map<std::vector<int>, std::vector<size_t>> parts_of;   // (head, sequence, first row) -> slots
  for (const Part& x : parts) {
    const PagedUnit& u = x.u;
    CHECK(x.wg >= 0 && x.wg < l.workgroups && x.head >= 0 && x.head < p.Hkv && u.seq >= 0 && u.seq < p.n_seq);
    CHECK(u.q0 >= 0 && u.nq > 0 && u.q0 + u.nq <= p.n_tokens && u.rows == u.nq * group);
    CHECK(u.m0 >= 0 && u.m0 % ROWS == 0 && u.m0 < u.rows);
    CHECK(x.t0 >= 0 && x.t0 < x.t1 && x.t1 <= u.places && u.places <= (max_keys + kTileKeys - 1) / kTileKeys + (int)Line::kPad);
    if (x.t0 == 0 && x.t1 == u.places) continue;
    const size_t slot = 2 * (size_t)x.wg + (x.t0 == 0 ? 2 : 1);
    CHECK(slot < 2 * (size_t)l.workgroups);
    CHECK(slots.insert(slot).second);
    parts_of[{x.head, u.seq, u.m0}].push_back(slot);
  }
  for (int wg = 0; l.ranges && wg < l.workgroups; ++wg) {
    const PagedCut& c = cuts[wg];
    CHECK(c.rows >= 0);   // (every workgroup leaves one)
    if (c.rows <= 0) continue;
    CHECK(c.last > wg && c.last < l.workgroups);
    CHECK(c.rows <= ROWS && c.head >= 0 && c.head < p.Hkv && c.q0 >= 0 && c.m0 >= 0);
    CHECK((long long)c.q0 * group + c.m0 + c.rows <= (long long)p.n_tokens * group);
  }
  if (!b.ascending()) return;
  std::map<std::vector<int>, std::vector<std::pair<int, int>>> walked;
  for (const Part& x : parts) walked[{x.head, x.u.seq, x.u.m0}].push_back({x.t0, x.t1});
  size_t units = 0;
  unsigned long long all_places = 0;
  for (int s = 0; s < p.n_seq; ++s) {
    const int n = (b.start[s + 1] - b.start[s]) * group, keys = std::min(std::max(b.len[s], 0), max_keys);
    const int keys_of = ROWS == kUnitRows && n <= 2 * kFewRows ? kTileKeys * kFewTiles : kTileKeys;
    const int places = std::max((keys + keys_of - 1) / keys_of, 1) + (int)Line::kPad;
    for (int m0 = 0; m0 < n; m0 += ROWS) {
      all_places += places;
      for (int h = 0; h < p.Hkv; ++h, ++units) {
        auto& w = walked[{h, s, m0}];
        std::sort(w.begin(), w.end());
        int at = 0;
        for (const auto& t : w) {
          CHECK(t.first == at);
          at = t.second;
        }
        CHECK(at == places);
      }
    }
  }
  CHECK(walked.size() == units);
  CHECK(!l.ranges || line_total == all_places);
  std::map<std::vector<int>, std::vector<size_t>> joined;
  for (int wg = 0; l.ranges && wg < l.workgroups; ++wg) {
    const PagedCut& c = cuts[wg];
    if (c.rows <= 0) continue;
    int s = 0;
    while (!(b.start[s] == c.q0 && b.start[s + 1] > c.q0)) ++s;
    CHECK(c.rows == std::min(ROWS, (b.start[s + 1] - b.start[s]) * group - c.m0));
    auto& to = joined[{c.head, s, c.m0}];
    CHECK(to.empty());
    for (int i = 0; i < c.last - (wg + 1) + 2; ++i) to.push_back(i == 0 ? 2 * (size_t)(wg + 1) : 2 * (size_t)(wg + i) + 1);
  }
  for (auto& x : parts_of) std::sort(x.second.begin(), x.second.end());
  for (auto& x : joined) std::sort(x.second.begin(), x.second.end());
  CHECK(joined == parts_of);
}

std::set<std::vector<int>> g_forms;   // rows, waves, ranges or not

void all_forms4(const char* name, const Batch& b) {
  static int turn = 0;   // (all of it every other time: the forms of calls with a workspace)
  const size_t sizes[] = {(size_t)1 << 20, (size_t)32 << 20, 300000, 0};
  for (size_t scratch : {turn % 2 ? (size_t)128 << 20 : sizes[turn / 2 % 4]}) {
    ++turn;
    const Paged4Form f = paged4_form(b.p, scratch);
    g_forms.insert({f.rows, f.waves, f.launch.ranges > 0});
    if (f.rows == kFewRows) {
      if (f.waves == 8) check4<kFewRows, 8>(name, b, f.launch, scratch);
      else if (f.waves == 4) check4<kFewRows, 4>(name, b, f.launch, scratch);
      else check4<kFewRows, 2>(name, b, f.launch, scratch);
    } else {
      if (f.waves == 8) check4<kUnitRows, 8>(name, b, f.launch, scratch);
      else check4<kUnitRows, 4>(name, b, f.launch, scratch);
    }
  }
}

int run4() {
  std::mt19937 rng(2);
  auto in = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  for (int group : {1, 4, 34})
    for (int Hkv : {1, 3, 8})
      for (int n_seq : {1, 5, 64, 180}) {
        if (n_seq * Hkv > 600) continue;
        for (int kind = 0; kind < 3; ++kind) {   // one token or none each; a few; a chunk among single ones
          std::vector<int> fresh;
          int T = 0;
          for (int s = 0; s < n_seq; ++s) {
            fresh.push_back(kind == 0 ? in(0, 8) > 0 : kind == 1 ? in(0, 3) : s == n_seq / 2 ? in(2, 500) / std::min(group, 8) + 1 : 1);
            T += fresh.back();
          }
          Batch b = make(Hkv * group, Hkv, in(0, 1) ? 64 : 128, n_seq, T + (kind > 0 ? 3 : 0), 16, in(0, 2) == 0 ? 12 : in(0, 1) ? 150 : 600);
          if (b.p.n_tokens == 0) continue;
          b.start[0] = kind > 0 ? 1 : 0;
          for (int s = 0; s < n_seq; ++s) {
            b.start[s + 1] = b.start[s] + fresh[s];
            b.len[s] = in(0, 6) == 0 ? 0 : in(0, 2) == 0 ? b.p.max_pages * 16 + in(-3, 3) : in(1, b.p.max_pages * 16 / 3);
          }
          all_forms4("in order", b);
        }
      }
  // more sequences than a wave's lanes have sums of in LDS, many heads
  for (int n_seq : {700, 4200}) {
    Batch b = make(8, 2, 64, n_seq, n_seq, 16, 20);
    for (int s = 0; s <= n_seq; ++s) b.start[s] = s;
    for (int s = 0; s < n_seq; ++s) b.len[s] = in(0, 320);
    const Paged4Form f = paged4_form(b.p, (size_t)128 << 20);
    const char* name = "many";
    g_forms.insert({f.rows, f.waves, f.launch.ranges > 0});
    CHECK(f.rows == kFewRows && f.waves == 2 && !f.launch.ranges);
    for (int i = 0; i < 3 && n_seq == 700; ++i) check4<kFewRows, 2>("many", b, f.launch, 0);
    check4<kFewRows, 8>("many, ranges", b, PagedLaunch{24, 12, 4, (unsigned)((20 * 16 / 64 + 10) * paged_units(b.p, kFewRows))}, (size_t)128 << 20);
  }
  // starts in no order, lengths of any kind
  for (int kind = 0; kind < 4; ++kind)
    for (int n_seq : {3, 64, 150, 400}) {
      Batch b = make(8, 4, 64, n_seq, 180, 32, 100);
      for (int s = 0; s <= n_seq; ++s)
        b.start[s] = kind == 0 ? (s % 2 ? 180 : 0) : kind == 1 ? 180 - 180 * s / n_seq : kind == 2 ? in(-200, 400) : s % 3 == 0 ? -2147483647 - 1 : 2147483647;
      for (int s = 0; s < n_seq; ++s) b.len[s] = kind == 2 ? in(-2147483647, 2147483647) : b.len[s];
      all_forms4("any order", b);
    }
  // back and forth with more places than 32 bits hold
  struct {
    int H, Hkv, n_seq, T, page, max_pages, len;
  } const far[] = {{32, 8, 4096, 4096, 64, 512, 32768}, {8, 8, 8300, 2048, 64, 1024, 65536}, {8, 1, 64, 250000, 1024, 512, 524288}, {64, 1, 65, 65536, 1024, 256, 262144}};
  for (const auto& f : far) {
    Batch b = make(f.H, f.Hkv, 64, f.n_seq, f.T, f.page, f.max_pages);
    for (int s = 0; s <= f.n_seq; ++s) b.start[s] = s % 2 ? f.T : 0;
    b.len.assign(f.n_seq, f.len);
    const long long tiles = f.max_pages * (long long)f.page / 64;
    check4<kFewRows, 8>("far", b, PagedLaunch{2 * f.Hkv, 2, 4, (unsigned)((tiles + 10) * paged_units(b.p, kFewRows))}, (size_t)128 << 20);
    check4<kUnitRows, 8>("far", b, PagedLaunch{2 * f.Hkv, 2, 4, (unsigned)((tiles + 8) * paged_units(b.p, kUnitRows))}, (size_t)512 << 20);
  }
  for (const std::vector<int>& f : {std::vector<int>{16, 8, 0}, {16, 8, 1}, {16, 4, 0}, {16, 4, 1}, {16, 2, 0}, {128, 8, 0}, {128, 8, 1}, {128, 4, 0}, {128, 4, 1}})
    if (!g_forms.count(f)) {
      printf("not met: %d rows, %d waves, ranges %d\n", f[0], f[1], f[2]);
      ++g_failed;
    }
  return g_failed;
}

}  // namespace
}  // namespace da

int main() {
  if (da::run4() == 0) printf("ok\n");
  return da::g_failed != 0;
}
