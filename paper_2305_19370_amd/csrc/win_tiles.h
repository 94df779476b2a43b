// What the bf16 kernels of attention with a window and sinks share: the rows of a wave, copies of
// tiles whose invisible rows are not read, the LDS ring's loop and the store of a transposed result.
#pragma once

#include "win_attn.h"

namespace bpt {

// Workgroups of 256 rows (8 waves, one on a CU) or of 128 (4, two on a CU, one at its start or end while the other works): large
// ones for long runs of tiles that fill the chip. Full attention, 32768 tokens, 32 heads of 128, forward / dQ: 9.1 / 11.0 ms
// (small: 9.5 / 11.3). Window of 1024, 8192 tokens, 16 heads: small 94 / 126 us (large: 120 / 146); of 4096, 16384 tokens: 510 / 677
// (573 / 697).
inline bool win_wide(int64_t len, const WinArgs& a) { return !a.window && (len * a.G + 255) / 256 * a.Hkv * a.B > 256; }

BPT_DEV void wait_lgkm() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Products accumulated into x are formed before what follows: the compiler would sink them behind a branch and
// hold their fragments in registers meanwhile.
BPT_DEV void pin(f32x16& x) { asm volatile("" : "+v"(x)); }

// NW waves of 32 rows share tiles of 64 rows of two tensors in a ring of NS stages
template <int DH, int NWAVES, int NSTAGES>
struct WinCfg {
  static constexpr int KSTEPS = DH / 16, DT = DH / 32;
  static constexpr int NW = NWAVES, ROWS = 32 * NW;
  static constexpr int TB = RmTile<DH>::BYTES, STAGE = 2 * TB;
  static constexpr int NS = NSTAGES;
  static constexpr int LDS = NS * STAGE;
  static constexpr int DPS = Ring2<DH, NW>::DPW;    // copies per wave per stage
};

// Adds the sums of wave g + G to those of wave g, g < G, through LDS that is done with. True: a wave that has given its own.
template <int G, int N>
BPT_DEV bool add_halves(char* smem, f32x16 (&x)[N], int wave, int lane) {
  float* red = (float*)smem + (wave % G) * N * 1024 + lane;   // [register][lane]
  __syncthreads();
  if (wave >= G) {
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) red[(16 * t + r) * 64] = x[t][r];
  }
  __syncthreads();
  if (wave >= G) return true;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[t][r] += red[(16 * t + r) * 64];
  return false;
}

// Row r0 + w0 + lane % 32 of a kv head's list r = token * G + head, what it sees, and what its wave and its
// workgroup of n rows (from r0) see. Rows behind the sequence's last stand for its last: they need no masks of their own, and
// their results are left out in the end.
struct Rows {
  int i, head;                 // token, query head in its group
  bool exists;
  Vis mine, first, last, run;  // the row; the wave's first and last row; the workgroup
  BPT_DEV Rows(const WinArgs& a, const Seq& s, int r0, int w0, int n, int lane) {
    const int r = r0 + w0 + (lane & 31);
    i = r / a.G;
    head = r - i * a.G;
    const int end = s.nq - 1;
    exists = i <= end;
    const int i0 = r0 / a.G, i1 = (r0 + n - 1) / a.G;
    mine = first = last = run = Vis{0, -1, 0};
    if (i0 > end) return;      // the workgroup has no row
    auto at = [&](int t) { const int p = s.off + min(t, end); return vis_of(a, s, p, p); };
    mine = at(i);
    first = at((r0 + w0) / a.G);
    last = at((r0 + w0 + 31) / a.G);
    run = vis_run(a, s, s.off + i0, s.off + min(i1, end));
  }
  // the token whose row is read
  BPT_DEV int safe(const Seq& s) const { return min(i, s.nq - 1); }
  // whether all the wave's rows see all of keys k0 .. k0 + 63, or none sees any
  BPT_DEV bool all(int k0) const { return (k0 >= last.lo && k0 + 63 <= first.hi) || k0 + 63 < first.se; }
  BPT_DEV bool none(int k0) const { return !(k0 <= last.hi && k0 + 63 >= first.lo) && k0 >= last.se; }
  // `out` in place of the scores t[mt][r] of keys k0 + 32 mt + acc_row(r, lane) that the row does not see. One comparison per
  // score where the tile lies across one end of the window only.
  template <int N>
  BPT_DEV void mask(f32x16 (&t)[N], int k0, int lane, float out) const {
    const int base = k0 + 4 * (lane >> 5);
    const int lo = mine.lo - base, hi = mine.hi - base, se = mine.se - base;
    auto where = [&](auto seen) {
#pragma unroll
      for (int mt = 0; mt < N; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) t[mt][r] = seen(32 * mt + 8 * (r >> 2) + (r & 3)) ? t[mt][r] : out;
    };
    if (k0 < last.se) {
      where([&](int k) { return (k >= lo && k <= hi) || k < se; });
    } else {
      if (k0 + 32 * N - 1 > first.hi) where([&](int k) { return k <= hi; });
      if (k0 < last.lo) where([&](int k) { return k >= lo; });
    }
  }
};

// ring_issue for rows row0 .. row0 + 63 of two tensors where only rows that `pick` returns may be
// read: pick(row) is a row of the tile itself.
template <int DH, int NW, class Pick>
BPT_DEV void issue_picked(char* stage, const bf16* src0, int ld0, const bf16* src1, int ld1, int row0, int wave, int lane,
                          const Pick& pick) {
  using T = RmTile<DH>;
  const bf16* org0 = src0 + (int64_t)row0 * ld0;
  const bf16* org1 = src1 + (int64_t)row0 * ld1;
  asm volatile("" : "+v"(lane));                    // recomputed at every call, as in ring_issue
#pragma unroll
  for (int i = 0; i < Ring2<DH, NW>::DPW; ++i) {
    const int b = ring_block<DH, NW>(wave, i), t = b >= T::BLOCKS, blk = b - t * T::BLOCKS;
    const int slot = blk * 64 + lane, col = slot % T::SLOTS, row = pick(row0 + slot / T::SLOTS) - row0;
    const uint32_t off = 2u * (uint32_t)(row * (t ? ld1 : ld0) + (col < DH / 8 ? col : 0) * 8);
    dma16s(scalar_ptr(t ? org1 : org0), off, stage + t * T::BYTES + blk * 1024);
  }
}

// What of v lies in a tile of n keys from k0, of which v sees some: clamp() of it stays in the tile.
BPT_DEV Vis seen_in(const Vis& v, int k0, int n) {
  Vis t{max(v.lo, k0), min(v.hi, k0 + n - 1), min(v.se, k0 + n)};
  if (t.lo > t.hi) t.lo = t.hi = t.se - 1;            // sinks alone
  return t;
}

// K and V of keys k0 .. k0 + 63, a tile that holds a key which v's run of rows sees; a key that none of
// them sees is replaced by one of the tile that is.
template <int DH, int NW>
BPT_DEV void issue_keys(char* stage, const bf16* K, int ldk, const bf16* V, int ldv, int k0, const Vis& v,
                        const RingOff<DH, NW>& roff, int wave, int lane) {
  if ((k0 >= v.lo && k0 + 63 <= v.hi) || k0 + 63 < v.se) {
    ring_issue_full<DH, NW>(stage, K, ldk, k0, V, ldv, k0, roff, wave);
    return;
  }
  const Vis t = seen_in(v, k0, 64);
  issue_picked<DH, NW>(stage, K, ldk, V, ldv, k0, wave, lane, [&](int k) { return t.clamp(k); });
}

// The online softmax of the row on a lane (shared with lane ^ 32): reference in base 2 (-inf until the row has seen a key) and
// the lane's part of the sum of weights. The reference moves to a tile's maximum only where that lies more than GROWTH
// above it: weights stay <= 2^GROWTH, the reference left a weight of at least 1 so that no sum vanishes, and the
// numerator is rescaled in few tiles (any of a wave's 32 rows has a new maximum in most).
template <int DT>
struct OnlineRows {
  static constexpr float GROWTH = 8.0f;
  float c;                                           // scale log2(e)
  float ref = NEG_INF, sum = 0.0f;
  // products t become weights against m; the lane's sum
  template <int N>
  BPT_DEV float raw(f32x16 (&t)[N], float m) const {
    float rs = 0.0f;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        t[x][r] = fast_exp2(fmaf(t[x][r], c, -m));
        rs += t[x][r];
      }
    return rs;
  }
  // products t (-inf where unseen) become weights; acc is rescaled where the reference moves
  template <int N>
  BPT_DEV void weights(f32x16 (&t)[N], f32x16 (&acc)[DT]) {
    float mx = NEG_INF;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, t[x][r]);
    mx = max_halves(mx) * c;
    const bool move = mx > ref + GROWTH;             // also from -inf
    if (__ballot(move)) {
      const float corr = move ? fast_exp2(ref - mx) : 1.0f;   // 0 for a row that starts
      sum *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= corr;
      ref = move ? mx : ref;
    }
    sum += raw(t, ref == NEG_INF ? 0.0f : ref);
  }
};

// Makes stage j of n visible to the workgroup and fills the slot of stage j - 1 (C::NS slots; DPS copies per wave and
// stage): stage j has landed once at most the stages issued after it are pending. Every wave calls it.
template <class C, int DPS, class Issue>
BPT_DEV void ring_step(int j, int n, const Issue& issue) {
  if (C::NS == 4 && j + 2 < n) wait_vmcnt<2 * DPS>();
  else if (C::NS == 4 && j + 1 < n) wait_vmcnt<DPS>();
  else wait_vmcnt<0>();
  __syncthreads();                                  // every wave is done with stage j - 1
  if (j + C::NS - 1 < n) issue(j + C::NS - 1);
}
template <class C, class Issue>
BPT_DEV void ring_start(int n, const Issue& issue) {
#pragma unroll
  for (int st = 0; st < C::NS - 1; ++st)
    if (st < n) issue(st);
}
// Walks n stages of a ring that has been started: body(j) runs with stage j in LDS
template <class C, int DPS, class Issue, class Body>
BPT_DEV void ring_loop(int n, const Issue& issue, const Body& body) {
  for (int j = 0; j < n; ++j) {
    ring_step<C, DPS>(j, n, issue);
    body(j);
  }
}

// A transposed result (features x 32 rows) times f: 4 consecutive features per store at p, the lane's row
template <int DH>
BPT_DEV void store_rows(bf16* p, const f32x16 (&acc)[DH / 32], float f, int lane) {
#pragma unroll
  for (int t = 0; t < DH / 32; ++t)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16)(acc[t][4 * rg + e] * f);
      *(bf16x4*)(p + 32 * t + 8 * rg + 4 * (lane >> 5)) = v;
    }
}

}  // namespace bpt
