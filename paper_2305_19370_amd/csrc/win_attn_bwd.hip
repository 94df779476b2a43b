// Attention with a sliding window and sinks, bf16 backward: dQ (rows outside, key tiles inside) and dK, dV
// (keys outside, query tiles of all the kv head's query heads inside): 3 and 4 products a visible pair, 2 of them the same,
// so that neither needs atomics. Full attention of 32768 tokens, 32 heads of 128: 27.0 ms, 1140 TFLOP/s; 8192 tokens, 16 heads,
// 4 key heads, window 1024: 274 us, 820. Bound by issue and LDS: each product reads an LDS fragment for every MFMA, and the
// registers of a wave (the sums, its rows' fragments) leave room for one workgroup's latency to be hidden by one other.
// P and dS are formed in fp32 and rounded to bf16 once, where they become operands of the second products (gradients 2.0-2.7e-3 off); Delta
// is a sum of products of the bf16 O that the caller holds, but for rows of few keys (win_delta_kernel).
#include <algorithm>

#include "win_tiles.h"

namespace bpt {

// S^T = K Q^T, dP^T = V dO^T, dS^T = P^T (dP^T - Delta), dQ^T += K^T dS^T; P from the saved
// log-sum-exp. Rows and ring as in the forward.
template <int DH, int NW>
using WinDqCfg = WinCfg<DH, NW, NW == 8 ? 4 : 2>;

template <int DH, int NW>
BPT_DEV void dq_rows(const WinArgs& a, char* smem, int id) {
  using C = WinDqCfg<DH, NW>;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nblk = (a.Sq * a.G + C::ROWS - 1) / C::ROWS;
  int hh, blk;
  xcd_map(id, a.Hkv * a.B, hh, blk);
  const int kvh = hh % a.Hkv, b = hh / a.Hkv;
  const Seq sq = seq_of(a, b);
  const Rows w(a, sq, (nblk - 1 - blk) * C::ROWS, 32 * wave, C::ROWS, lane);   // most keys first
  const int h = kvh * a.G + w.head;
  const float c = a.scale * LOG2E;
  const bf16* Kb = (const bf16*)a.k + (int64_t)b * a.k_sb + (int64_t)kvh * a.k_sh;
  const bf16* Vb = (const bf16*)a.v + (int64_t)b * a.v_sb + (int64_t)kvh * a.v_sh;
  const Tiles<64> tiles(w.run);

  f32x16 acc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t) acc[t] = f32x16{};
  if (tiles.n > 0) {
    const RingOff<DH, NW> roff = ring_offsets<DH, NW>(a.k_st, a.v_st, wave, lane);
    auto issue = [&](int j) {
      issue_keys<DH, NW>(smem + (j % C::NS) * C::STAGE, Kb, a.k_st, Vb, a.v_st, tiles.key0(j), w.run, roff, wave, lane);
    };
    ring_start<C>(tiles.n, issue);                     // on their way before anything is waited for
    bf16x8 qf[C::KSTEPS], dof[C::KSTEPS];
    const int64_t i = w.safe(sq);
    {
      const bf16* q = (const bf16*)a.q + (int64_t)b * a.q_sb + i * a.q_st + (int64_t)h * a.q_sh;
      const bf16* d = (const bf16*)a.dout + (int64_t)b * a.o_sb + i * a.o_st + (int64_t)h * a.o_sh;
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk) {
        qf[kk] = __builtin_bit_cast(bf16x8, ld16(q + 16 * kk + 8 * (lane >> 5)));
        dof[kk] = __builtin_bit_cast(bf16x8, ld16(d + 16 * kk + 8 * (lane >> 5)));
        settle(qf[kk]);
        settle(dof[kk]);
      }
    }
    const int64_t sidx = ((int64_t)b * a.Hq + h) * a.Sqp + i;
    const float nl = a.nlse[sidx], ndl = a.ndelta[sidx];
    settle(nl);
    settle(ndl);
    auto tile = [&](int j, int k0, bool all) {
      const char* kt = smem + (j % C::NS) * C::STAGE;
      const char* vt = kt + C::TB;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        f32x16 s[1], dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[0][r] = nl;                                // the MFMAs leave (score - lse) / scale
          dp[r] = ndl;                                 // and dP^T - Delta
        }
#pragma unroll
        for (int kk = 0; kk < C::KSTEPS; ++kk) {
          s[0] = mfma32x32x16(frag_rows<DH>(kt, 32 * mt, 2 * kk, lane), qf[kk], s[0]);
          dp = mfma32x32x16(frag_rows<DH>(vt, 32 * mt, 2 * kk, lane), dof[kk], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[0][r] = fast_exp2(s[0][r] * c) * dp[r];
        if (!all) {
          pin(s[0]);
          w.mask(s, k0 + 32 * mt, lane, 0.0f);
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const bf16x8 sb = acc_to_b(s[0], hf);
#pragma unroll
          for (int t = 0; t < C::DT; ++t)
            acc[t] = mfma32x32x16(frag_tr<DH>(kt, 32 * mt + 16 * hf, 32 * t, lane), sb, acc[t]);
        }
      }
    };
    ring_loop<C, C::DPS>(tiles.n, issue, [&](int j) {
      const int k0 = tiles.key0(j);
      if (!w.none(k0)) tile(j, k0, w.all(k0));
    });
  }
  if (!w.exists || !w.mine.any()) {                  // nothing seen: 0, beside rows that see a NaN too
#pragma unroll
    for (int t = 0; t < C::DT; ++t) acc[t] = f32x16{};
  }
  if (w.i < a.Sq)
    store_rows<DH>((bf16*)a.dq + (int64_t)b * a.q_sb + (int64_t)w.i * a.q_st + (int64_t)h * a.q_sh, acc, a.dq_scale, lane);
}

// Ring of the dK dV kernel: tiles of 64 queries (Q, dO) and their -lse / scale and -Delta
template <int DH, int KG, int QH>
struct WinKvCfg {
  static constexpr int KSTEPS = DH / 16, DT = DH / 32;
  static constexpr int NW = KG * QH, KEYS = 32 * KG;   // waves: KG groups of 32 keys x QH parts of a tile's queries
  static constexpr int TB = RmTile<DH>::BYTES, STAGE = 2 * TB + 2 * 64 * 4;
  static constexpr int NS = NW == 8 ? 4 : 2;
  static constexpr int LDS = NS * STAGE;
  static constexpr int DPS = Ring2<DH, NW>::DPW + 2;
};

// KG groups of 32 keys of one kv head; QH = 2: two waves for each, with half the queries of a tile, their sums added at the
// end. S = Q K^T and dP = dO V^T have the key on the lane axis, so P and dS feed dV^T += dO^T P
// and dK^T += Q^T dS directly. The tiles of the kv head's query heads follow one another.
//
// Sinks are seen by every query, a key inside by a window of them: one block of keys would take as long as
// all others together. Where that matters (a.far), the blocks keep to the window, and what sinks see
// beyond it is cut into a.far chunks of (query head, tile of 64 queries) for workgroups of their own (FAR: 32 sinks,
// two waves, each half the queries of a tile). All leave the sinks' sums in fp32 slots, which win_sinks adds in order.
// Few blocks of keys with many tiles (grouped heads, small batches) are cut into a.chunks of those in the same way, for all keys.
template <int DH, int KG, int QH, bool FAR>
BPT_DEV void dkdv_keys(const WinArgs& a, char* smem, int id) {
  using C = WinKvCfg<DH, KG, QH>;
  constexpr int NW = C::NW;
  static_assert(!FAR || (KG == 1 && QH == 2), "two waves for the far part");
  static_assert(FAR || QH == 1 || KG * 2 * C::DT * 4096 <= C::LDS, "the second halves fit the ring");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int hh, blk;
  xcd_map(id, a.Hkv * a.B, hh, blk);
  const int kvh = hh % a.Hkv, b = hh / a.Hkv;
  const Seq sq = seq_of(a, b);
  const int chunks = FAR ? a.far : a.chunks, chunk = blk % chunks;
  const int k0 = blk / chunks * C::KEYS, part = wave / KG, kw = k0 + 32 * (wave % KG), key = kw + (lane & 31);
  const float c = a.scale * LOG2E;
  const bool near = FAR || a.far > 0;               // the window alone, or beyond it

  f32x16 adv[C::DT], adk[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t) adv[t] = adk[t] = f32x16{};
  QVis run{0, -1};
  const int kend = FAR ? min(sq.nk, a.sinks) : sq.nk;   // keys from here on are none of this workgroup's
  if (k0 < kend) {
    run = qvis_of(a, sq, k0, min(k0 + C::KEYS, kend) - 1, near);
    if (FAR) run = QVis{a.causal ? max(k0 + a.window - sq.off, 0) : 0, sq.nq - 1};
  }
  const int t0 = run.lo / 64, nt = run.hi >= run.lo ? run.hi / 64 + 1 - t0 : 0;   // tiles of a query head
  const int per = (nt * a.G + chunks - 1) / chunks;
  const int j0 = chunk * per, n = min(per, nt * a.G - j0);
  QVis mine{0, -1};
  if (n > 0) {
    // keys behind the sequence's last stand for it; their results are left out in the end
    mine = qvis_of(a, sq, min(key, sq.nk - 1), min(key, sq.nk - 1), near);
    QVis first{0, -1}, last{0, -1};
    const int kl = min(kw + 31, kend - 1);
    if (kw < sq.nk) {
      first = qvis_of(a, sq, kw, kw, near);
      last = qvis_of(a, sq, kl, kl, near);
    }
    // the queries that all of the wave's keys see: the first key behind the sinks has the lowest end
    const int ks = !near && kw < a.sinks && a.sinks <= kl ? a.sinks : kw;
    const int all_lo = max(first.lo, last.lo), all_hi = min(qvis_of(a, sq, ks, ks, near).hi, last.hi);
    // stages are requested, and worked on, in order: each keeps its own place (query head, tile) of the list
    RingOff<DH, NW> roff;                             // two waves have 19 copies each: too many registers
    if constexpr (!FAR) roff = ring_offsets<DH, NW>(a.q_st, a.o_st, wave, lane);
    int ih = kvh * a.G + j0 / nt, it = j0 % nt, at = it;
    auto issue = [&](int j) {
      const int q0 = 64 * (t0 + it);
      char* st = smem + (j % C::NS) * C::STAGE;
      const bf16* q = (const bf16*)a.q + (int64_t)b * a.q_sb + (int64_t)ih * a.q_sh;
      const bf16* o = (const bf16*)a.dout + (int64_t)b * a.o_sb + (int64_t)ih * a.o_sh;
      if (!FAR && q0 >= run.lo && q0 + 63 <= run.hi) ring_issue_full<DH, NW>(st, q, a.q_st, q0, o, a.o_st, q0, roff, wave);
      else issue_picked<DH, NW>(st, q, a.q_st, o, a.o_st, q0, wave, lane, [&](int r) { return min(max(r, run.lo), run.hi); });
      const int64_t sidx = ((int64_t)b * a.Hq + ih) * a.Sqp + q0;      // Sqp % 64 == 0: in bounds
      dma4s(scalar_ptr(a.nlse + sidx), 4u * lane, st + 2 * C::TB);
      dma4s(scalar_ptr(a.ndelta + sidx), 4u * lane, st + 2 * C::TB + 256);
      if (++it == nt) {
        it = 0;
        ++ih;
      }
    };
    ring_start<C>(n, issue);
    bf16x8 kf[C::KSTEPS], vf[C::KSTEPS];
    {
      const int64_t kr = min(key, kend - 1);
      const bf16* k = (const bf16*)a.k + (int64_t)b * a.k_sb + kr * a.k_st + (int64_t)kvh * a.k_sh;
      const bf16* v = (const bf16*)a.v + (int64_t)b * a.v_sb + kr * a.v_st + (int64_t)kvh * a.v_sh;
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk) {
        kf[kk] = __builtin_bit_cast(bf16x8, ld16(k + 16 * kk + 8 * (lane >> 5)));
        vf[kk] = __builtin_bit_cast(bf16x8, ld16(v + 16 * kk + 8 * (lane >> 5)));
        settle(kf[kk]);
        settle(vf[kk]);
      }
    }
    auto half = [&](int j, int q0, int mt, bool all) {
      const char* qs = smem + (j % C::NS) * C::STAGE;
      const char* ds = qs + C::TB;
      const float* ls = (const float*)(qs + 2 * C::TB);
      f32x16 s, dp;
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const int qi = 32 * mt + 8 * rg + 4 * (lane >> 5);
        const f32x4 l4 = *(const f32x4*)(ls + qi);
        const f32x4 d4 = *(const f32x4*)(ls + 64 + qi);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[4 * rg + e] = l4[e];                     // the MFMAs leave (score - lse) / scale
          dp[4 * rg + e] = d4[e];                    // and dP - Delta
        }
      }
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk) {
        s = mfma32x32x16(frag_rows<DH>(qs, 32 * mt, 2 * kk, lane), kf[kk], s);
        dp = mfma32x32x16(frag_rows<DH>(ds, 32 * mt, 2 * kk, lane), vf[kk], dp);
        if constexpr (DH == 128) __builtin_amdgcn_sched_barrier(0);   // bound the fragments read ahead
      }
      pin(dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fast_exp2(s[r] * c);
      if (!all) {
        const int base = q0 + 32 * mt + 4 * (lane >> 5);
        const int lo = mine.lo - base, hi = mine.hi - base, end = run.hi - base;
        auto where = [&](auto seen) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = seen(8 * (r >> 2) + (r & 3)) ? s[r] : 0.0f;
        };
        if constexpr (FAR) {
          where([&](int q) { return q <= end && (q > hi || (!a.causal && q < lo)); });
        } else {                                     // one comparison per score across one end of the window
          if (q0 + 63 > all_hi) where([&](int q) { return q <= hi; });
          if (q0 < all_lo) where([&](int q) { return q >= lo; });
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] = s[r] * dp[r];                // dS
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const bf16x8 pb = acc_to_b(s, hf), sb = acc_to_b(dp, hf);
#pragma unroll
        for (int t = 0; t < C::DT; ++t) {
          adv[t] = mfma32x32x16(frag_tr<DH>(ds, 32 * mt + 16 * hf, 32 * t, lane), pb, adv[t]);
          adk[t] = mfma32x32x16(frag_tr<DH>(qs, 32 * mt + 16 * hf, 32 * t, lane), sb, adk[t]);
          if constexpr (DH == 128) __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    ring_loop<C, C::DPS>(n, issue, [&](int j) {
      const int q0 = 64 * (t0 + at);
      at = at + 1 == nt ? 0 : at + 1;
      if constexpr (FAR) {
        // columns of keys that are no sinks are never stored and need no mask
        half(j, q0, part, a.causal && q0 > last.hi && q0 + 63 <= run.hi);
      } else if (q0 <= max(first.hi, last.hi) && q0 + 63 >= min(first.lo, last.lo) && kw < sq.nk) {
        const bool all = q0 >= all_lo && q0 + 63 <= all_hi;
        if constexpr (QH == 2) {
          half(j, q0, part, all);
        } else {
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) half(j, q0, mt, all);
        }
      }
    });
  }
  if constexpr (!FAR && QH == 2) {
    f32x16 both[2 * C::DT];
#pragma unroll
    for (int t = 0; t < C::DT; ++t) {
      both[t] = adk[t];
      both[C::DT + t] = adv[t];
    }
    if (add_halves<KG, 2 * C::DT>(smem, both, wave, lane)) return;
#pragma unroll
    for (int t = 0; t < C::DT; ++t) {
      adk[t] = both[t];
      adv[t] = both[C::DT + t];
    }
  }
  // a key that no query sees, behind the sequence's last or in front of the first query's window: whatever it holds is in its own
  // column alone (0 times its dP)
  if (key >= sq.nk || (!FAR && mine.hi < mine.lo)) {
#pragma unroll
    for (int t = 0; t < C::DT; ++t) adv[t] = adk[t] = f32x16{};
  }
  const int ns = win_slot_keys(a);
  if (key < ns) {
    // chunks: one slot for each; far: slot 0 the window's part, then two for each of its chunks
    const int64_t slot = FAR ? 1 + 2 * chunk + part : chunk;
    float* p = a.part_s + ((slot * a.B * a.Hkv + (int64_t)b * a.Hkv + kvh) * ns + key) * 2 * DH;
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const int d = 32 * t + 8 * rg + 4 * (lane >> 5);
        *(f32x4*)(p + d) = f32x4{adk[t][4 * rg], adk[t][4 * rg + 1], adk[t][4 * rg + 2], adk[t][4 * rg + 3]};
        *(f32x4*)(p + DH + d) = f32x4{adv[t][4 * rg], adv[t][4 * rg + 1], adv[t][4 * rg + 2], adv[t][4 * rg + 3]};
      }
  } else if (!FAR && key < a.Skv) {
    store_rows<DH>((bf16*)a.dk + (int64_t)b * a.k_sb + (int64_t)key * a.k_st + (int64_t)kvh * a.k_sh, adk, a.scale, lane);
    store_rows<DH>((bf16*)a.dv + (int64_t)b * a.v_sb + (int64_t)key * a.v_st + (int64_t)kvh * a.v_sh, adv, 1.0f, lane);
  }
}

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, 1) void win_dq_bf16_kernel(WinArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  dq_rows<DH, NW>(a, smem, (int)blockIdx.x);
}
template <int DH, int KG, int QH, bool FAR>
__global__ __launch_bounds__(64 * KG * QH, KG * QH == 8 ? 1 : 2) void win_dkdv_bf16_kernel(WinArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  dkdv_keys<DH, KG, QH, FAR>(a, smem, (int)blockIdx.x);
}
// dK dV in blocks of 64 keys, by the first nkv workgroups, and dQ in blocks of 128 rows by the others: neither needs the
// other, and short runs leave a chip that one of them alone does not fill (4 x 1000 tokens, 12 heads of 64, window 256: 39
// us, in two launches 50, launch gaps included). Heads of 64: three workgroups on a CU, at two stages for dQ and 24 bytes of spills a
// lane (16384 tokens, 16 heads, window 2048: 590 us, two workgroups 645).
template <int DH>
__global__ __launch_bounds__(256, DH == 64 ? 3 : 2) void win_bwd_bf16_kernel(WinArgs a, int nkv) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int id = (int)blockIdx.x;
  if (id < nkv) dkdv_keys<DH, 2, 2, false>(a, smem, id);
  else dq_rows<DH, 4>(a, smem, id - nkv);
}

template <class K>
static hipError_t launch(K k, int64_t blocks, int threads, int lds, const WinArgs& a, hipStream_t s) {
  hipError_t e = set_lds(k, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(threads), lds, s, a);
  return hipGetLastError();
}
template <int DH>
static hipError_t bwd(const WinArgs& a, hipStream_t s) {
  // dK dV: long runs of tiles that fill the chip twice over in blocks of 256 keys (full attention of 32768 tokens, 32 heads of 128:
  // 16.1 ms, blocks of 64 17.7). Else of 64, two to three workgroups on a CU, one at its start or end while others work: 4000
  // tokens, 16 heads, window 512 66 us (74); heads of 64 at any length: 16384 tokens, window 2048 289 (331), full attention of
  // 32768 tokens, 16 heads 4.24 ms (4.37).
  const int64_t heads = (int64_t)a.Hkv * a.B, wide = ((int64_t)a.Skv + 255) / 256 * heads;
  const bool wide_kv = DH == 128 && !a.window && wide >= 512, wide_q = win_wide(a.Sq, a);
  hipError_t e = hipSuccess;
  if constexpr (DH == 128)
    if (a.dk && wide_kv) e = launch(win_dkdv_bf16_kernel<DH, 8, 1, false>, wide, 512, WinKvCfg<DH, 8, 1>::LDS, a, s);
  if (e == hipSuccess && a.dq && wide_q)
    e = launch(win_dq_bf16_kernel<DH, 8>, ((int64_t)a.Sq * a.G + 255) / 256 * heads, 512, WinDqCfg<DH, 8>::LDS, a, s);
  const int64_t nkv = a.dk && !wide_kv ? ((int64_t)a.Skv + 63) / 64 * a.chunks * heads : 0;
  const int64_t nq = a.dq && !wide_q ? ((int64_t)a.Sq * a.G + 127) / 128 * heads : 0;
  if (e != hipSuccess || nkv + nq == 0) return e;
  auto k = win_bwd_bf16_kernel<DH>;
  constexpr int lds = std::max(WinKvCfg<DH, 2, 2>::LDS, WinDqCfg<DH, 4>::LDS);
  if ((e = set_lds(k, lds)) != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)(nkv + nq)), dim3(256), lds, s, a, (int)nkv);
  return hipGetLastError();
}
template <int DH>
static hipError_t far(const WinArgs& a, hipStream_t s) {
  return launch(win_dkdv_bf16_kernel<DH, 1, 2, true>, (int64_t)a.far * ((std::min(a.sinks, a.Skv) + 31) / 32) * a.Hkv * a.B, 128,
                WinKvCfg<DH, 1, 2>::LDS, a, s);
}

hipError_t win_bwd_bf16(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? bwd<64>(a, s) : bwd<128>(a, s); }
hipError_t win_far_bf16(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? far<64>(a, s) : far<128>(a, s); }

}  // namespace bpt
