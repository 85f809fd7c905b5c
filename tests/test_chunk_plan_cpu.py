"""The chunk attention's plan, replayed for all CTAs of a call: every step of every item is taken once, in parts whose number and first
CTA are those that the parts are told."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2403_18647_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <map>
#include <tuple>
#include <vector>
#include "chunk_plan.h"
using namespace sdsat;

struct Part { int kb0, kb1, cta, head, parts; };

// stdin: tiles, grid, G, Hk, table columns, b, then b of (rows, length); prints "items cut parts", or what is wrong
int main() {
  int tiles, grid, G, Hk, ld, b;
  while (std::scanf("%d %d %d %d %d %d", &tiles, &grid, &G, &Hk, &ld, &b) == 6) {
    const int pt1 = CH_ROWS / G, pt = tiles * pt1, cap = ld * CH_STEP;
    std::vector<long long> before(b + 1);
    std::vector<ChSeq> seq(b);
    long long total = 0;
    int first = 0, n_items = 0;
    for (int s = 0; s < b; ++s) {
      int n, len;
      if (std::scanf("%d %d", &n, &len) != 2) return 1;
      seq[s] = ch_sequence(first, first + n, len, pt1, tiles, cap);
      before[s] = total;
      total += ch_cost(seq[s], pt, cap) * Hk;
      n_items += ch_items(seq[s], pt, Hk);
      first += n;
    }
    before[b] = total;
    const ChPlan plan = {before.data(), seq.data(), b, Hk, pt, cap, ch_ctas(grid, n_items, total), total};
    auto with_rows = [&](int s) {
      while (s < b && seq[s].n == 0) ++s;
      return s;
    };
    std::map<std::tuple<int, int, int>, std::vector<Part>> got;
    std::map<int, int> at_head;   // items that are counted at a CTA's place
    const char* wrong = nullptr;
    for (int c = 0; c < plan.ctas; ++c) {
      ChPlace a = plan.border(c);
      const ChPlace z = plan.border(c + 1);
      while (a.s < b && !(a.s == z.s && a.hk == z.hk && a.t == z.t && a.kb >= z.kb)) {
        const ChSeq q = seq[a.s];
        const int steps = ch_steps(q, pt, cap, a.t);
        const bool stop = a.s == z.s && a.hk == z.hk && a.t == z.t;
        Part x = {a.kb, stop ? z.kb : steps, c, c, 1};
        if (x.kb0 > 0 || x.kb1 < steps) plan.parts(a, q, x.head, x.parts);
        got[{a.s, a.hk, a.t}].push_back(x);
        if (stop) break;
        a = plan.after(a, q, with_rows);
      }
    }
    long long items = 0, cut = 0, parts = 0;
    for (int s = 0; s < b; ++s)
      for (int hk = 0; hk < Hk; ++hk)
        for (int t = 0; t < ch_count(seq[s], pt); ++t) {
          const auto& x = got[{s, hk, t}];
          ++items;
          if (x.empty()) { wrong = "an item that no CTA takes"; continue; }
          int kb = 0;
          for (size_t i = 0; i < x.size(); ++i) {
            if (x[i].kb0 != kb || x[i].kb1 <= kb) wrong = "steps taken twice or never";
            kb = x[i].kb1;
            if (x[i].parts != (int)x.size() || x[i].head != x[0].cta || x[i].cta != x[0].cta + (int)i) wrong = "parts other than those that run";
          }
          if (kb != ch_steps(seq[s], pt, cap, t)) wrong = "steps missing";
          if (x.size() > 1) {
            ++cut;
            parts += x.size();
            if (at_head[x[0].cta]++) wrong = "two items counted in one place";
          }
        }
    if (wrong) std::printf("%s\n", wrong);
    else std::printf("%lld %lld %lld\n", items, cut, parts);
  }
}
"""


@pytest.fixture(scope="module")
def replay(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "main.cpp").write_text(PROGRAM)
    exe = str(at / "main")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, str(at / "main.cpp"), "-o", exe], check=True)

    def run(calls):
        text = "\n".join(" ".join(map(str, [tiles, grid, G, Hk, ld, len(seqs)] + [x for s in seqs for x in s])) for tiles, grid, G, Hk, ld, seqs in calls)
        lines = subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
        assert len(lines) == len(calls)
        wrong = [(line, call) for line, call in zip(lines, calls) if not line[0].isdigit()]
        assert not wrong, (len(wrong), wrong[:3])
        return [tuple(map(int, line.split())) for line in lines]
    return run


def test_more_rows_than_the_table_holds(replay):
    """(With costs of all of a sequence's rows, a step of these cost more than a stretch.)"""
    for grid in (148, 152):
        got = replay([(2, grid, 1, 1, 8, [(3840, 0)]), (1, grid, 1, 1, 8, [(3785, 0)]), (2, grid, 1, 2, 8, [(3175, 0)])])
        assert all(cut for _, cut, _ in got)


def test_any_batch(replay):
    r = random.Random(1)
    calls = []
    for i in range(4000):
        b = r.choice([1, 1, 2, 3, 9, 40])
        ld = r.choice([1, 2, 7, 8, 12, 30, 100, 300])
        most = r.choice([40, 600, 6000])
        seqs = [(r.choice([0, 1, 1, r.randrange(1, most)]), r.choice([0, r.randrange(0, 64 * ld + 1), r.randrange(0, 64 * ld + 1), 1 << 30])) for _ in range(b)]
        if not any(n for n, _ in seqs):
            continue
        if i % 2:                                       # within the table
            seqs = [(n, max(0, min(m, 64 * ld - n))) for n, m in seqs]
        calls.append((r.choice([1, 2]), r.choice([1, 7, 132, 148, 152]), r.choice([1, 2, 3, 4, 7, 8, 16, 100, 128]), r.choice([1, 2, 3, 8, 40]), ld, seqs))
    got = replay(calls)
    assert sum(cut for _, cut, _ in got) > 5000 and max(parts for _, _, parts in got) > 100


def test_long_sequences(replay):
    replay([(2, 152, 4, 8, 1 << 18, [(1, 1 << 24)]), (1, 152, 1, 40, 1 << 12, [(1 << 17, 0)]), (2, 152, 128, 1, 1 << 16, [(1 << 16, 1 << 21), (1, 5)]),
            (2, 152, 1, 8, 100, [(1, 6000)] * 1024)])
