// Attention with a sliding window and sinks, bf16 backward: dQ (rows outside, key tiles inside) and dK, dV
// (keys outside, query tiles of all the kv head's query heads inside).
#include "win_tiles.h"

namespace bpt {

// S^T = K Q^T, dP^T = V dO^T, dS^T = P^T (dP^T - Delta), dQ^T += K^T dS^T; P from the saved
// log-sum-exp. Rows and ring as in the forward.
template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void win_dq_bf16_kernel(WinArgs a) {
  using C = WinCfg<DH, NW>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nblk = (a.Sq * a.G + C::ROWS - 1) / C::ROWS;
  int hh, blk;
  xcd_map((int)blockIdx.x, a.Hkv * a.B, hh, blk);
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
    const float nl = a.nlse2[sidx], ndl = a.ndelta[sidx];
    settle(nl);
    settle(ndl);
    const RingOff<DH, NW> roff = ring_offsets<DH, NW>(a.k_st, a.v_st, wave, lane);
    auto issue = [&](int j) {
      issue_keys<DH, NW>(smem + (j % C::NS) * C::STAGE, Kb, a.k_st, Vb, a.v_st, tiles.key0(j), w.run, roff, wave, lane);
    };
    auto tile = [&](int j) {
      const int k0 = tiles.key0(j);
      const char* kt = smem + (j % C::NS) * C::STAGE;
      const char* vt = kt + C::TB;
      f32x16 s[2] = {f32x16{}, f32x16{}}, dp[2];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[mt][r] = ndl;  // the MFMAs leave dP^T - Delta
#pragma unroll
        for (int kk = 0; kk < C::KSTEPS; ++kk) {
          s[mt] = mfma32x32x16(frag_rows<DH>(kt, 32 * mt, 2 * kk, lane), qf[kk], s[mt]);
          dp[mt] = mfma32x32x16(frag_rows<DH>(vt, 32 * mt, 2 * kk, lane), dof[kk], dp[mt]);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[mt][r] = fast_exp2(fmaf(s[mt][r], c, nl)) * dp[mt][r];
      }
      if (!w.all(k0)) w.mask(s, k0, lane, 0.0f);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const bf16x8 sb = acc_to_b(s[mt], hf);
#pragma unroll
          for (int t = 0; t < C::DT; ++t)
            acc[t] = mfma32x32x16(frag_tr<DH>(kt, 32 * mt + 16 * hf, 32 * t, lane), sb, acc[t]);
        }
    };
    ring_loop<C, C::DPS>(tiles.n, issue, [&](int j) {
      if (!w.none(tiles.key0(j))) tile(j);
    });
  }
  if (w.i < a.Sq)
    store_rows<DH>((bf16*)a.dq + (int64_t)b * a.q_sb + (int64_t)w.i * a.q_st + (int64_t)h * a.q_sh, acc, a.scale, lane);
}

// Ring of the dK dV kernel: tiles of 64 queries (Q, dO) and their -lse (base 2) and -Delta
template <int DH, int NWAVES>
struct WinKvCfg {
  static constexpr int KSTEPS = DH / 16, DT = DH / 32;
  static constexpr int NW = NWAVES, KEYS = 32 * NW;
  static constexpr int TB = RmTile<DH>::BYTES, STAGE = 2 * TB + 2 * 64 * 4;
  static constexpr int NS = NW == 8 || DH == 64 ? 4 : 2;
  static constexpr int LDS = NS * STAGE;
  static constexpr int DPS = Ring2<DH, NW>::DPW + 2;
};

// NW waves of 32 keys of one kv head. S = Q K^T and dP = dO V^T have the key on the lane axis, so P and dS feed dV^T += dO^T P
// and dK^T += Q^T dS directly. The tiles of the kv head's query heads follow one another.
template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void win_dkdv_bf16_kernel(WinArgs a) {
  using C = WinKvCfg<DH, NW>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int hh, blk;
  xcd_map((int)blockIdx.x, a.Hkv * a.B, hh, blk);
  const int kvh = hh % a.Hkv, b = hh / a.Hkv;
  const Seq sq = seq_of(a, b);
  const int k0 = blk * C::KEYS, kw = k0 + 32 * wave, key = kw + (lane & 31);
  const float c = a.scale * LOG2E;

  f32x16 adv[C::DT], adk[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t) adv[t] = adk[t] = f32x16{};
  QVis run{0, -1};
  if (k0 < sq.nk) run = qvis_of(a, sq, k0, min(k0 + C::KEYS, sq.nk) - 1, false);
  const int t0 = run.lo / 64, nt = run.hi >= run.lo ? run.hi / 64 + 1 - t0 : 0;
  if (nt > 0) {
    QVis mine = qvis_of(a, sq, key, key, false), first{0, -1}, last{0, -1};
    if (key >= sq.nk) mine.hi = -1;
    if (kw < sq.nk) first = qvis_of(a, sq, kw, kw, false);
    const int kl = min(kw + 31, sq.nk - 1);
    if (kw < sq.nk) last = qvis_of(a, sq, kl, kl, false);
    // the queries that all of the wave's keys see: the first key behind the sinks has the lowest end
    const int ks = kw < a.sinks && a.sinks <= kl ? a.sinks : kw;
    const int all_lo = max(first.lo, last.lo), all_hi = kw < sq.nk ? min(qvis_of(a, sq, ks, ks, false).hi, last.hi) : -1;
    const bool full = kw + 31 < sq.nk;
    bf16x8 kf[C::KSTEPS], vf[C::KSTEPS];
    {
      const int64_t kr = min(key, sq.nk - 1);
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
    auto issue = [&](int it) {
      const int h = kvh * a.G + it / nt, q0 = 64 * (t0 + it % nt);
      char* st = smem + (it % C::NS) * C::STAGE;
      issue_picked<DH, NW>(st, (const bf16*)a.q + (int64_t)b * a.q_sb + (int64_t)h * a.q_sh, a.q_st,
                           (const bf16*)a.dout + (int64_t)b * a.o_sb + (int64_t)h * a.o_sh, a.o_st, q0, wave, lane,
                           [&](int q) { return min(max(q, run.lo), run.hi); });
      const int64_t sidx = ((int64_t)b * a.Hq + h) * a.Sqp + q0;       // Sqp % 64 == 0: in bounds
      dma4s(scalar_ptr(a.nlse2 + sidx), 4u * lane, st + 2 * C::TB);
      dma4s(scalar_ptr(a.ndelta + sidx), 4u * lane, st + 2 * C::TB + 256);
    };
    auto tile = [&](int it, int q0) {
      const char* qs = smem + (it % C::NS) * C::STAGE;
      const char* ds = qs + C::TB;
      const float* ls = (const float*)(qs + 2 * C::TB);
      // a tile that all the wave's keys see in full needs no mask
      const bool all = full && q0 >= all_lo && q0 + 63 <= all_hi;
      const int lo = mine.lo - q0 - 4 * (lane >> 5), hi = mine.hi - q0 - 4 * (lane >> 5);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        f32x16 s = {}, dp;
        f32x4 l4[4];
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
          const int qi = 32 * mt + 8 * rg + 4 * (lane >> 5);
          l4[rg] = *(const f32x4*)(ls + qi);
          const f32x4 d4 = *(const f32x4*)(ls + 64 + qi);
#pragma unroll
          for (int e = 0; e < 4; ++e) dp[4 * rg + e] = d4[e];   // the MFMAs leave dP - Delta
        }
#pragma unroll
        for (int kk = 0; kk < C::KSTEPS; ++kk) {
          s = mfma32x32x16(frag_rows<DH>(qs, 32 * mt, 2 * kk, lane), kf[kk], s);
          dp = mfma32x32x16(frag_rows<DH>(ds, 32 * mt, 2 * kk, lane), vf[kk], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fast_exp2(fmaf(s[r], c, l4[r >> 2][r & 3]));
        if (!all) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int q = 32 * mt + 8 * (r >> 2) + (r & 3);
            s[r] = q >= lo && q <= hi ? s[r] : 0.0f;
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = s[r] * dp[r];       // dS: rows read are real ones, dP is finite
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const bf16x8 pb = acc_to_b(s, hf), sb = acc_to_b(dp, hf);
#pragma unroll
          for (int t = 0; t < C::DT; ++t) {
            adv[t] = mfma32x32x16(frag_tr<DH>(ds, 32 * mt + 16 * hf, 32 * t, lane), pb, adv[t]);
            adk[t] = mfma32x32x16(frag_tr<DH>(qs, 32 * mt + 16 * hf, 32 * t, lane), sb, adk[t]);
          }
        }
      }
    };
    ring_loop<C, C::DPS>(nt * a.G, issue, [&](int it) {
      const int q0 = 64 * (t0 + it % nt);
      if (q0 <= max(first.hi, last.hi) && q0 + 63 >= min(first.lo, last.lo) && kw < sq.nk) tile(it, q0);
    });
  }
  if (key < a.Skv) {
    store_rows<DH>((bf16*)a.dk + (int64_t)b * a.k_sb + (int64_t)key * a.k_st + (int64_t)kvh * a.k_sh, adk, a.scale, lane);
    store_rows<DH>((bf16*)a.dv + (int64_t)b * a.v_sb + (int64_t)key * a.v_st + (int64_t)kvh * a.v_sh, adv, 1.0f, lane);
  }
}

template <int DH, int NW>
static hipError_t launch_dkdv(const WinArgs& a, hipStream_t s) {
  using C = WinKvCfg<DH, NW>;
  auto k = win_dkdv_bf16_kernel<DH, NW>;
  hipError_t e = set_lds(k, C::LDS);
  if (e != hipSuccess) return e;
  const int64_t nblk = ((int64_t)a.Skv + C::KEYS - 1) / C::KEYS;
  hipLaunchKernelGGL(k, dim3((unsigned)(nblk * a.Hkv * a.B)), dim3(64 * NW), C::LDS, s, a);
  return hipGetLastError();
}
template <int DH, int NW>
static hipError_t launch_dq(const WinArgs& a, hipStream_t s) {
  using C = WinCfg<DH, NW>;
  auto k = win_dq_bf16_kernel<DH, NW>;
  hipError_t e = set_lds(k, C::LDS);
  if (e != hipSuccess) return e;
  const int64_t nblk = ((int64_t)a.Sq * a.G + C::ROWS - 1) / C::ROWS;
  hipLaunchKernelGGL(k, dim3((unsigned)(nblk * a.Hkv * a.B)), dim3(64 * NW), C::LDS, s, a);
  return hipGetLastError();
}

hipError_t win_dkdv_bf16(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? launch_dkdv<64, 8>(a, s) : launch_dkdv<128, 8>(a, s); }
hipError_t win_dq_bf16(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? launch_dq<64, 8>(a, s) : launch_dq<128, 8>(a, s); }

}  // namespace bpt
