// What the bf16 kernels of attention with a window and sinks share: the rows of a wave, copies of
// tiles whose invisible rows are not read, the LDS ring's loop and the store of a transposed result.
#pragma once

#include "win_attn.h"

namespace bpt {

// Waves of workgroups of 256 rows (8 waves, one workgroup on a CU) or 128 (4, two): the small ones where the large would
// leave CUs idle.
inline bool win_wide(int64_t len, const WinArgs& a) { return (len * a.G + 255) / 256 * a.Hkv * a.B > 256; }

template <int N = 0> BPT_DEV void wait_lgkm() { asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N) : "memory"); }

// Products accumulated into x are formed before what follows: the compiler would sink them behind a branch and
// hold their fragments in registers meanwhile.
BPT_DEV void pin(f32x16& x) { asm volatile("" : "+v"(x)); }

// NW waves of 32 rows (keys, in the dK dV kernel) share tiles of 64 rows of two tensors in a ring
template <int DH, int NWAVES>
struct WinCfg {
  static constexpr int KSTEPS = DH / 16, DT = DH / 32;
  static constexpr int NW = NWAVES, ROWS = 32 * NW;
  static constexpr int TB = RmTile<DH>::BYTES, STAGE = 2 * TB;
  static constexpr int NS = NW == 8 || DH == 64 ? 4 : 2;   // stages in the ring
  static constexpr int LDS = NS * STAGE;
  static constexpr int DPS = Ring2<DH, NW>::DPW;    // copies per wave per stage
};

// Row r0 + w0 + lane % 32 of a kv head's list r = token * G + head, what it sees, and what its wave and its
// workgroup of n rows (from r0) see.
struct Rows {
  int i, head;                 // token, query head in its group
  bool full;                   // all the wave's rows exist
  Vis mine, first, last, run;  // the row; the wave's first and last row that exist; the workgroup
  BPT_DEV Rows(const WinArgs& a, const Seq& s, int r0, int w0, int n, int lane) {
    const int r = r0 + w0 + (lane & 31);
    i = r / a.G;
    head = r - i * a.G;
    const int last_i = s.nq - 1;
    mine = first = last = run = Vis{0, -1, 0};
    if (i <= last_i) mine = vis_of(a, s, s.off + i, s.off + i);
    const int i0 = r0 / a.G, i1 = min((r0 + n - 1) / a.G, last_i);
    if (i0 <= i1) run = vis_run(a, s, s.off + i0, s.off + i1);
    const int wi0 = (r0 + w0) / a.G, wi1 = (r0 + w0 + 31) / a.G;
    full = wi1 <= last_i;
    if (wi0 <= last_i) {
      first = vis_of(a, s, s.off + wi0, s.off + wi0);
      const int e = s.off + min(wi1, last_i);
      last = vis_of(a, s, e, e);
    }
  }
  // a row that exists, for rows that do not
  BPT_DEV int safe(const Seq& s) const { return min(i, s.nq - 1); }
  // whether all the wave's rows see all of keys k0 .. k0 + 63, or none sees any
  BPT_DEV bool all(int k0) const { return full && ((k0 >= last.lo && k0 + 63 <= first.hi) || k0 + 63 < first.se); }
  BPT_DEV bool none(int k0) const { return !(k0 <= last.hi && k0 + 63 >= first.lo) && k0 >= last.se; }
  // scores t[mt][r] of keys k0 + 32 mt + acc_row(r, lane)
  template <int N>
  BPT_DEV void mask(f32x16 (&t)[N], int k0, int lane, float out) const {
    const int base = k0 + 4 * (lane >> 5);
    const int lo = mine.lo - base, hi = mine.hi - base, se = mine.se - base;
#pragma unroll
    for (int mt = 0; mt < N; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int k = 32 * mt + 8 * (r >> 2) + (r & 3);
        t[mt][r] = (k >= lo && k <= hi) || k < se ? t[mt][r] : out;
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

// K and V of keys k0 .. k0 + 63, a tile that holds a key which v's run of rows sees; a key that none of
// them sees is replaced by one of the tile that is.
template <int DH, int NW>
BPT_DEV void issue_keys(char* stage, const bf16* K, int ldk, const bf16* V, int ldv, int k0, const Vis& v,
                        const RingOff<DH, NW>& roff, int wave, int lane) {
  if ((k0 >= v.lo && k0 + 63 <= v.hi) || k0 + 63 < v.se) {
    ring_issue_full<DH, NW>(stage, K, ldk, k0, V, ldv, k0, roff, wave);
    return;
  }
  const int lo = max(v.lo, k0), hi = min(v.hi, k0 + 63);
  const int se = min(v.se, k0 + 64);
  issue_picked<DH, NW>(stage, K, ldk, V, ldv, k0, wave, lane,
                       [&](int k) { return k < se ? k : lo <= hi ? min(max(k, lo), hi) : se - 1; });
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
    const float use = ref == NEG_INF ? 0.0f : ref;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        t[x][r] = fast_exp2(fmaf(t[x][r], c, -use));
        sum += t[x][r];
      }
  }
};

// Walks n stages of the ring (C::NS slots, DPS copies per wave and stage): body(j) runs with stage j in
// LDS. Every wave of the workgroup reaches every barrier.
template <class C, int DPS, class Issue, class Body>
BPT_DEV void ring_loop(int n, const Issue& issue, const Body& body) {
#pragma unroll
  for (int st = 0; st < C::NS - 1; ++st)
    if (st < n) issue(st);
  for (int j = 0; j < n; ++j) {
    // stage j has landed once at most the stages issued after it are pending
    if (C::NS == 4 && j + 2 < n) wait_vmcnt<2 * DPS>();
    else if (C::NS == 4 && j + 1 < n) wait_vmcnt<DPS>();
    else wait_vmcnt<0>();
    __syncthreads();                                // stage j visible; every wave is done with stage j - 1
    if (j + C::NS - 1 < n) issue(j + C::NS - 1);    // into the slot of stage j - 1
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
