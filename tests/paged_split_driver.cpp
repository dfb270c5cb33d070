// The work split of the attention over a paged cache (csrc/paged_units.h) on the CPU: a wave of 64 lanes that run in turn up to each exchange
// between them. The header's own code is what runs; the loop over a workgroup's range is the kernels'.
#include <setjmp.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <functional>
#include <map>
#include <random>
#include <set>
#include <vector>

#include "paged_units.h"

namespace wave {

constexpr int kLanes = 64;
constexpr size_t kStack = 1 << 16;
jmp_buf lanes[kLanes], home;
ucontext_t first[kLanes], back;
std::vector<char> stacks(kLanes* kStack);
bool started[kLanes];
int current, turn[kLanes], values[2][kLanes];
std::function<void()> body;

void go_on(int lane) {   // from whichever lane runs
  current = lane;
  threadIdx.x = (unsigned)lane;
  if (started[lane]) _longjmp(lanes[lane], 1);
  started[lane] = true;
  setcontext(&first[lane]);
}
void yield() {
  const int me = current;
  if (_setjmp(lanes[me]) == 0) go_on((me + 1) % kLanes);
}
void enter() {
  body();
  // (lanes take the same path: they end one after the other)
  if (current + 1 < kLanes) go_on(current + 1);
  _longjmp(home, 1);
}
void run(const std::function<void()>& f) {
  body = f;
  for (int i = 0; i < kLanes; ++i) {
    started[i] = false;
    turn[i] = 0;
    getcontext(&first[i]);
    first[i].uc_stack.ss_sp = stacks.data() + i * kStack;
    first[i].uc_stack.ss_size = kStack;
    first[i].uc_link = nullptr;
    makecontext(&first[i], enter, 0);
  }
  if (_setjmp(home) == 0) go_on(0);
}
// every lane's x, in two buffers in turn: a lane is at most one exchange ahead
const int* all(int x) {
  int* to = values[turn[current]++ & 1];
  to[current] = x;
  yield();
  return to;
}

}  // namespace wave

int __builtin_amdgcn_readlane(int x, int lane) { return wave::all(x)[lane]; }
uint64_t __builtin_amdgcn_ballot_w64(bool x) {
  const int* v = wave::all(x);
  uint64_t m = 0;
  for (int i = 0; i < 64; ++i) m |= (uint64_t)(v[i] != 0) << i;
  return m;
}
int __builtin_amdgcn_update_dpp(int old, int x, int ctrl, int rows, int banks, bool zero) {
  const int* v = wave::all(x);
  const int lane = wave::current, row = lane / 16;
  if (banks != 15 || zero) abort();
  int from = -1;
  if (ctrl > 0x110 && ctrl < 0x120) from = lane % 16 >= ctrl - 0x110 ? lane - (ctrl - 0x110) : -1;   // row_shr
  else if (ctrl == 0x142) from = row > 0 ? 16 * row - 1 : -1;                                       // row_bcast 15
  else if (ctrl == 0x143) from = row > 1 ? 31 : -1;                                                 // row_bcast 31
  else abort();
  return (rows >> row & 1) && from >= 0 ? v[from] : old;
}
float __builtin_amdgcn_exp2f(float x) { return exp2f(x); }
void __syncthreads() { wave::yield(); }

namespace da {
namespace {

int g_failed = 0;
#define CHECK(c)                                                                           \
  do {                                                                                      \
    if (!(c) && g_failed++ < 20) printf("%s:%d: %s\n", name, __LINE__, #c);                 \
  } while (0)

struct Batch {
  da_paged p = {};
  std::vector<int> start, len;
  bool ascending() const {
    for (size_t i = 0; i + 1 < start.size(); ++i)
      if (start[i] > start[i + 1]) return false;
    return start[0] >= 0 && start.back() <= p.n_tokens;
  }
};

struct Part {
  int wg, head, t0, t1;
  PagedUnit u;
};

template <int ROWS, int KEYS, int PAD>
void check(const char* name, const Batch& b, int most_workgroups, size_t scratch, bool must_range) {
  typedef PagedLine<ROWS, KEYS, PAD> Line;
  const da_paged& p = b.p;
  const PagedLaunch l = paged_launch(p, ROWS, KEYS, PAD, most_workgroups, 0, scratch);
  CHECK(!must_range || l.ranges);
  CHECK(l.workgroups >= 1 && (!l.ranges || paged_launch_bytes(l.workgroups, ROWS, p.d) <= scratch));
  const int group = p.H / p.Hkv, max_keys = p.max_pages * p.page_size;
  const PagedBatch batch = {b.start.data(), b.len.data(), p.n_seq, p.n_tokens, group, max_keys, l.most};
  std::vector<Part> parts;
  std::vector<PagedCut> cuts(l.workgroups);
  PagedLds lds;
  unsigned line_total = 0;
  for (int wg = 0; wg < l.workgroups && g_failed == 0; ++wg) {
    std::vector<Part> mine;
    wave::run([&] {
      const bool tell = wave::current == 0;
      const Line line(batch, &lds, 0, 1);
      unsigned pos = 0, end = 1;
      if (l.ranges) {
        const unsigned total = line.total * (unsigned)p.Hkv, length = paged_range(total, l.workgroups, l.least);
        pos = paged_cut(line, wg, length, total);
        end = paged_cut(line, wg + 1, length, total);
        const PagedCut cut = paged_mark<ROWS>(line, pos, end, length, total);
        if (tell) {
          cuts[wg] = cut;
          line_total = line.total;
        }
      }
      for (int n = 0; pos < end; ++n) {
        if (n > 4000) {   // (far more than any of these batches has)
          if (tell) CHECK(!"a range ends");
          return;
        }
        Part x;
        x.wg = wg;
        if (l.ranges) {
          x.head = (int)(pos / line.total);
          const unsigned at = pos - (unsigned)x.head * line.total;
          if (!line.template find<false>(at, &x.u)) return;
          x.t0 = (int)(at - x.u.first);
          x.t1 = min(x.u.places, x.t0 + (int)(end - pos));
        } else {
          x.head = wg % p.Hkv;
          if (!line.template find<true>(wg / p.Hkv, &x.u)) return;
          x.t0 = 0;
          x.t1 = x.u.places;
        }
        pos += (unsigned)(x.t1 - x.t0);
        if (tell) mine.push_back(x);
      }
    });
    parts.insert(parts.end(), mine.begin(), mine.end());
  }
  // whatever the arrays hold: units are runs of a sequence's rows, and parts lie in the scratch, each in a place of its own
  std::set<size_t> slots;
  std::map<std::vector<int>, std::vector<size_t>> parts_of;   // (head, sequence, first row) -> slots
  for (const Part& x : parts) {
    const PagedUnit& u = x.u;
    CHECK(x.head >= 0 && x.head < p.Hkv && u.seq >= 0 && u.seq < p.n_seq);
    CHECK(u.q0 >= 0 && u.nq > 0 && u.q0 + u.nq <= p.n_tokens && u.rows == u.nq * group);
    CHECK(u.m0 >= 0 && u.m0 % ROWS == 0 && u.m0 < u.rows);
    CHECK(x.t0 >= 0 && x.t0 < x.t1 && x.t1 <= u.places && u.places <= (max_keys + KEYS - 1) / KEYS + PAD);
    if (x.t0 == 0 && x.t1 == u.places) continue;
    const size_t slot = 2 * (size_t)x.wg + (x.t0 == 0 ? 2 : 1);
    CHECK(slot < 2 * (size_t)l.workgroups);
    CHECK(slots.insert(slot).second);
    parts_of[{x.head, u.seq, u.m0}].push_back(slot);
  }
  for (int wg = 0; l.ranges && wg < l.workgroups; ++wg) {
    const PagedCut& c = cuts[wg];
    if (c.rows == 0) continue;
    CHECK(c.last > wg && c.last < l.workgroups);
    CHECK(c.rows > 0 && c.rows <= ROWS && c.head >= 0 && c.head < p.Hkv && c.q0 >= 0 && c.m0 >= 0);
    CHECK((long long)c.q0 * group + c.m0 + c.rows <= (long long)p.n_tokens * group);
  }
  if (!b.ascending()) return;
  // starts in order: every place of every unit once, and each unit that is cut is joined from its own parts
  std::map<std::vector<int>, std::vector<std::pair<int, int>>> walked;
  for (const Part& x : parts) walked[{x.head, x.u.seq, x.u.m0}].push_back({x.t0, x.t1});
  size_t units = 0;
  unsigned long long all_places = 0;
  for (int s = 0; s < p.n_seq; ++s) {
    const int n = (b.start[s + 1] - b.start[s]) * group, keys = std::min(std::max(b.len[s], 0), max_keys);
    const int places = std::max((keys + KEYS - 1) / KEYS, 1) + PAD;
    for (int m0 = 0; m0 < n; m0 += ROWS) {
      all_places += places;
      for (int h = 0; h < p.Hkv; ++h, ++units) {
        const auto& w = walked[{h, s, m0}];
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
    if (c.rows == 0) continue;
    int s = 0;
    while (!(b.start[s] == c.q0 && b.start[s + 1] > c.q0)) ++s;
    CHECK(c.rows == std::min(ROWS, (b.start[s + 1] - b.start[s]) * group - c.m0));
    auto& to = joined[{c.head, s, c.m0}];
    CHECK(to.empty());
    for (int i = 0; i < c.last - (wg + 1) + 2; ++i) to.push_back(i == 0 ? 2 * (size_t)(wg + 1) : 2 * (size_t)(wg + i) + 1);
  }
  CHECK(joined == parts_of);
}

Batch make(int H, int Hkv, int d, int n_seq, int n_tokens, int page, int max_pages) {
  Batch b;
  b.p.H = H;
  b.p.Hkv = Hkv;
  b.p.d = d;
  b.p.n_seq = n_seq;
  b.p.n_tokens = n_tokens;
  b.p.page_size = page;
  b.p.max_pages = max_pages;
  b.start.resize(n_seq + 1);
  b.len.assign(n_seq, max_pages * page);
  return b;
}

void all_forms(const char* name, const Batch& b, bool must_range) {
  const size_t full = (size_t)128 << 20;
  check<128, 64, 8>(name, b, 512, full, must_range);
  check<128, 64, 8>(name, b, 256, (size_t)3 << 20, false);
  check<32, 64, 6>(name, b, 256, full, must_range);
  check<32, 64, 3>(name, b, 1024, full, must_range);
  check<32, 32, 3>(name, b, 512, full, must_range);
  check<128, 64, 8>(name, b, 512, 0, false);   // whole units
}

int run() {
  std::mt19937 rng(1);
  auto in = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  // batches in order: few and many sequences (a wave's lanes of them, their sums in LDS, beyond), some without new tokens or keys
  for (int n_seq : {1, 2, 5, 63, 64, 65, 200, 4200}) {
    const int most_new = n_seq > 1000 ? 2 : n_seq > 60 ? 30 : 300;
    std::vector<int> fresh;
    int T = 0;
    for (int s = 0; s < n_seq; ++s) {
      fresh.push_back(n_seq > 1000 && in(0, 20) ? 0 : in(0, 3) == 0 ? in(0, most_new) : 1);
      T += fresh.back();
    }
    Batch b = make(8, 2, 64, n_seq, T + 3, 16, n_seq > 1000 ? 40 : 300);
    b.start[0] = 1;
    for (int s = 0; s < n_seq; ++s) {
      b.start[s + 1] = b.start[s] + fresh[s];
      b.len[s] = in(0, 5) == 0 ? 0 : in(0, 2) == 0 ? b.p.max_pages * 16 + in(-3, 3) : in(1, b.p.max_pages * 16 / 3);
    }
    if (n_seq <= 200) all_forms("in order", b, n_seq > 2);
    else check<32, 64, 3>("very many", b, 6, (size_t)128 << 20, true);
  }
  // as many places as there can be: full tables, one token each, and all tokens one sequence's
  for (int kind = 0; kind < 2; ++kind) {
    Batch b = make(4, 4, 128, 70, 70, 16, 64);
    for (int s = 0; s <= 70; ++s) b.start[s] = kind ? (s > 3 ? 70 : 0) : s;
    all_forms("full", b, true);
  }
  // starts in no order, lengths of any kind
  for (int kind = 0; kind < 4; ++kind)
    for (int n_seq : {3, 64, 150}) {
      Batch b = make(8, 4, 64, n_seq, 180, 32, 100);
      for (int s = 0; s <= n_seq; ++s)
        b.start[s] = kind == 0 ? (s % 2 ? 180 : 0) : kind == 1 ? 180 - 180 * s / n_seq : kind == 2 ? in(-200, 400) : s % 3 == 0 ? -2147483647 - 1 : 2147483647;
      for (int s = 0; s < n_seq; ++s) b.len[s] = kind == 2 ? in(-2147483647, 2147483647) : b.len[s];
      all_forms("any order", b, false);
    }
  // back and forth with more places than 32 bits hold, in the sums of a wave's lanes, of all sequences, of all kv heads
  struct {
    int H, Hkv, n_seq, T, page, max_pages, len;
  } const far[] = {{32, 8, 4096, 4096, 64, 512, 32768}, {32, 8, 4096, 4096, 64, 512, 30001}, {8, 8, 8300, 2048, 64, 1024, 65536},
                   {8, 1, 64, 250000, 1024, 512, 524288}, {64, 1, 65, 65536, 1024, 256, 262144}};
  for (const auto& f : far) {
    Batch b = make(f.H, f.Hkv, 64, f.n_seq, f.T, f.page, f.max_pages);
    for (int s = 0; s <= f.n_seq; ++s) b.start[s] = s % 2 ? f.T : 0;
    b.len.assign(f.n_seq, f.len);
    check<32, 64, 3>("far", b, 16, (size_t)128 << 20, true);
    check<32, 32, 3>("far", b, 7, (size_t)1 << 20, true);
    check<128, 64, 8>("far", b, 16, (size_t)128 << 20, true);
  }
  return g_failed;
}

}  // namespace
}  // namespace da

int main() {
  if (da::run() == 0) printf("ok\n");
  return da::g_failed != 0;
}
