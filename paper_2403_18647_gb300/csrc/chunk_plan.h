// The plan of the chunk attention: which steps of which items a CTA takes (plain C++, for the host and the device).
//
// Items stand in a line, by sequence, cache head and rows, weighed by what they cost; the line is cut into equal stretches,
// one for a CTA, at the steps nearest to their borders.  What a part of an item needs to know of the others (the CTA of the
// first, their number) follows from the item's place in the line alone.  That only holds if no step costs more than a
// stretch, or else two borders meet in one step and a CTA between them has no part: costs count the keys that an item's
// steps hold, at most the table's.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define CH_HD __host__ __device__ __forceinline__
#define CH_PAST static __host__ __device__ __noinline__
#else
#define CH_HD inline
#define CH_PAST inline
#endif

namespace sdsat {

constexpr int CH_ROWS = 128;          // rows of a tile
constexpr int CH_STEP = 64;           // keys of a step: a page
constexpr int CH_PART = 4;            // steps that a part of an item has at least
// What work costs, in quarters of a key's with one tile: a key with two tiles, an item's start, and that for which a CTA
// is worth its while.  One tile's steps are bound by memory, two tiles' by the products and the softmax: 48 sequences of up to
// 8200 slots, two of them with 100 new rows, take 156 us with these, 189 with equal keys, 179 with a start of 128 keys.
constexpr int CH_TWO = 5, CH_START = 4 * 512, CH_LEAST = 4 * 512;
// A stretch costs half of what the cheapest item does at least (of two CTAs for each item), a step of an item that is cut the
// start's share and its keys.
static_assert(CH_LEAST >= CH_START / 2 && CH_START / 2 > CH_TWO * CH_STEP + CH_START / (2 * CH_PART), "borders lie more than a step apart");

struct ChSeq {
  int first, n, len, w;               // first row, new positions, slots before them; what a key costs
};
struct ChPlace {
  int s, hk, t, kb;                   // sequence (b: behind the last item), cache head, item of the head, step
  long long cost;                     // before the item
};

template <typename T>
CH_HD T ch_min(T a, T z) { return a < z ? a : z; }
template <typename T>
CH_HD T ch_max(T a, T z) { return a > z ? a : z; }

// a sequence of rows first .. last - 1 after len slots; pt1: positions of a tile; cap: slots of the table
CH_HD ChSeq ch_sequence(int first, int last, int len, int pt1, int tiles, int cap) {
  return ChSeq{first, last - first, ch_min(ch_max(len, 0), cap), tiles == 2 && last - first > pt1 ? CH_TWO : 4};
}
// keys of item t, of pt positions
CH_HD int ch_keys(const ChSeq& q, int pt, int cap, int t) {
  return (int)ch_min((long long)cap, q.len + ch_min((long long)q.n, (long long)(t + 1) * pt));
}
CH_HD int ch_steps(const ChSeq& q, int pt, int cap, int t) { return (ch_keys(q, pt, cap, t) + CH_STEP - 1) / CH_STEP; }
// keys that the items before t, those behind the table's end among them, would hold beyond the table (seldom: out of line)
CH_PAST long long ch_past(ChSeq q, int pt, int cap, int t) {
  const int u = (cap - q.len) / pt;   // items within the table
  return (long long)(t - u) * (q.len - cap) + pt * (((long long)t * (t + 1) - (long long)u * (u + 1)) / 2);
}
// cost of item t, and of a head's items before it
CH_HD long long ch_item(const ChSeq& q, int pt, int cap, int t) { return (long long)q.w * ch_keys(q, pt, cap, t) + CH_START; }
CH_HD long long ch_before(const ChSeq& q, int pt, int cap, int t) {
  long long cost = (long long)t * ((long long)q.w * q.len + CH_START) + (long long)q.w * pt * ((long long)t * (t + 1) / 2);
  if (q.len + (long long)t * pt > cap) cost -= q.w * ch_past(q, pt, cap, t);
  return cost;
}
CH_HD int ch_count(const ChSeq& q, int pt) { return q.n > 0 ? (int)((uint32_t)(q.n - 1) / (uint32_t)pt) + 1 : 0; }   // a head's items
CH_HD long long ch_cost(const ChSeq& q, int pt, int cap) {   // of a head's items
  const int t = ch_count(q, pt);
  return t ? ch_before(q, pt, cap, t - 1) + ch_item(q, pt, cap, t - 1) : 0;
}
// items of a sequence, as far as they matter for the number of CTAs
CH_HD int ch_items(const ChSeq& q, int pt, int Hk) { return (int)ch_min(1ll << 15, (long long)ch_count(q, pt) * Hk); }
// how many of the CTAs take part (of two for each item none takes two of them)
CH_HD int ch_ctas(int grid, int n_items, long long total) {
  return (int)ch_max(1ll, ch_min((long long)grid, ch_max(2ll * n_items, total / CH_LEAST)));
}

struct ChPlan {
  const long long* before;   // [b + 1] cost before each sequence
  const ChSeq* seq;          // [b]
  int b, Hk, pt, cap, ctas;
  long long total;

  // the last sequence whose cost before it is at most x
  CH_HD int at_cost(long long x) const {
    int lo = 0, hi = b;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (before[mid] <= x) lo = mid;
      else hi = mid;
    }
    return lo;
  }
  // where CTA c's stretch begins
  CH_HD ChPlace border(int c) const {
    ChPlace a = {b, 0, 0, 0, 0};
    if (c >= ctas || total == 0) return a;
    const long long x = total / ctas * c + total % ctas * c / ctas;
    a.s = at_cost(x);
    const ChSeq q = seq[a.s];
    const long long of_head = ch_cost(q, pt, cap);
    long long rem = x - before[a.s];
    a.hk = (int)(rem / of_head);
    rem -= a.hk * of_head;
    int lo = 0, hi = ch_count(q, pt);
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (ch_before(q, pt, cap, mid) <= rem) lo = mid;
      else hi = mid;
    }
    a.t = lo;
    rem -= ch_before(q, pt, cap, lo);
    a.cost = x - rem;
    // the nearest step, an item's start spread over all of them; an end where that is less than CH_PART steps away
    const int steps = ch_steps(q, pt, cap, a.t);
    const long long cost = ch_item(q, pt, cap, a.t);
    a.kb = (int)((2 * rem * steps + cost) / (2 * cost));
    if (a.kb < CH_PART) {
      a.kb = 0;
    } else if (a.kb > steps - CH_PART) {   // the item that follows
      a.kb = 0;
      a.cost += cost;
      if (++a.t * pt >= q.n) {
        a.t = 0;
        if (++a.hk == Hk) a.hk = 0, a.s = a.cost < total ? at_cost(a.cost) : b;
      }
    }
    return a;
  }
  // the last CTA whose stretch begins less than y behind the item that begins at `cost`
  CH_HD int cta_at(long long cost, long long y) const { return (int)ch_min((long long)ctas - 1, ((cost + y) * ctas - 1) / total); }
  // the CTA of a cut item's first part, and how many parts it has: the CTAs whose first border lies in the item as border() sees it
  CH_HD void parts(const ChPlace& a, const ChSeq& q, int& head, int& n) const {
    const long long steps = ch_steps(q, pt, cap, a.t), cost = ch_item(q, pt, cap, a.t);
    head = cta_at(a.cost, ((2 * CH_PART - 1) * cost + 2 * steps - 1) / (2 * steps));
    n = cta_at(a.cost, ((2 * (steps - CH_PART) + 1) * cost + 2 * steps - 1) / (2 * steps)) - head + 1;
  }
  // the item that follows; with_rows(s): the first sequence from s on that has rows (b: none)
  template <typename F>
  CH_HD ChPlace after(ChPlace a, const ChSeq& q, F&& with_rows) const {
    a.kb = 0;
    a.cost += ch_item(q, pt, cap, a.t);
    if (++a.t * pt >= q.n) {
      a.t = 0;
      if (++a.hk == Hk) a.hk = 0, a.s = with_rows(a.s + 1);
    }
    return a;
  }
};

}  // namespace sdsat
