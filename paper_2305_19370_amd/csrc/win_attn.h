// Attention with a sliding window and sinks: what its kernels share. Query i of a sequence of nq
// queries and nk keys stands at position p = nk - nq + i and sees key k iff k < nk, (not causal
// or k <= p) and (no window, or |p - k| < window, or k < sinks). The visible keys of one query are
// an interval [lo, hi] and the first `se` keys; those of neighbouring queries move by one.
#pragma once

#include "attn_common.h"

namespace bpt {

// lengths of sequence b: queries, keys, and the position of query 0
struct Seq {
  int nq, nk, off;
};
BPT_DEV Seq seq_of(const WinArgs& a, int b) {
  Seq s;
  s.nq = a.q_lens ? min(max(a.q_lens[b], 0), a.Sq) : a.Sq;
  s.nk = a.kv_lens ? min(max(a.kv_lens[b], 0), a.Skv) : a.Skv;
  s.off = s.nk - s.nq;
  return s;
}

// Keys that a query (or a run of queries) sees: lo .. hi, and those below se. None: hi < lo and se = 0.
struct Vis {
  int lo, hi, se;
  BPT_DEV bool sees(int k) const { return (k >= lo && k <= hi) || k < se; }
  BPT_DEV bool any() const { return hi >= lo || se > 0; }
  // a key that is seen, in place of one that is not: what a tile holds beyond the visible keys is
  // never read, whatever it contains
  BPT_DEV int clamp(int k) const {
    const int in = min(max(k, lo), hi);
    return k < se ? k : in;
  }
};
// Keys of the queries at positions p0 .. p1. Where nothing but sinks is left, lo = hi = se - 1.
BPT_DEV Vis vis_of(const WinArgs& a, const Seq& s, int p0, int p1) {
  Vis v;
  v.lo = a.window ? max(p0 - a.window + 1, 0) : 0;
  v.hi = min(a.causal ? p1 : a.window ? p1 + a.window - 1 : s.nk - 1, s.nk - 1);
  v.se = a.window ? max(min(min(a.sinks, s.nk), a.causal ? p1 + 1 : s.nk), 0) : 0;
  return v;
}
// the same for a run: an interval of which each key is seen by some query
BPT_DEV Vis vis_run(const WinArgs& a, const Seq& s, int p0, int p1) {
  Vis v = vis_of(a, s, p0, p1);
  if (v.hi < v.lo) v.lo = v.hi = v.se - 1;       // -1, -1, 0: nothing
  if (v.se == 0 && v.hi < 0) v.lo = 0;           // hi < lo again: any() is false
  return v;
}

// Queries that see a key (or a run of keys k0 .. k1): an interval of i. Sinks see all; `near` leaves out
// what a sink sees beyond the window.
struct QVis {
  int lo, hi;
};
BPT_DEV QVis qvis_of(const WinArgs& a, const Seq& s, int k0, int k1, bool near) {
  const bool wide = !a.window || (!near && k0 < a.sinks);
  QVis v;
  v.lo = max(a.causal ? k0 - s.off : a.window && !wide ? k0 - a.window + 1 - s.off : 0, 0);
  v.hi = min(wide ? s.nq - 1 : k1 + a.window - 1 - s.off, s.nq - 1);
  return v;
}

// Keys (the first ones) whose dK and dV are left in slots, [slot, B Hkv, keys, dK and dV, dh] fp32, dK without its scale
BPT_DEV int win_slot_keys(const WinArgs& a) { return a.chunks > 1 ? a.Skv : a.far > 0 ? min(a.sinks, a.Skv) : 0; }

// Key tiles of T keys that a run of queries visits, in ascending order: those of the sinks, then
// those of the interval.
template <int T>
struct Tiles {
  int ns, first, n;              // sink tiles, first tile of the interval behind them, tiles in all
  BPT_DEV explicit Tiles(const Vis& v) {
    ns = (v.se + T - 1) / T;
    first = max(v.lo / T, ns);
    n = !v.any() ? 0 : ns + max(v.hi / T + 1 - first, 0);
  }
  BPT_DEV int key0(int j) const { return T * (j < ns ? j : j - ns + first); }
};

}  // namespace bpt
