// Attention with a sliding window and sinks, bf16 forward.
#include "win_tiles.h"

namespace bpt {

// Online softmax over key tiles of 64, scores transposed (S^T = K Q^T: a lane owns one row of the list
// r = token * G + head, so its maximum and sum are register reductions and one exchange), P^T straight from the accumulators into
// O^T += V^T P^T. NW waves of 32 rows share the K and V tiles of an LDS ring. The scores are scaled
// in fp32 (the FMA that subtracts the reference), so q is used as it is.
template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void win_fwd_bf16_kernel(WinArgs a) {
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
  float ref = NEG_INF, l_run = 0.0f;                // the row's reference maximum, base 2
  if (tiles.n > 0) {
    bf16x8 qf[C::KSTEPS];
    {
      const bf16* q = (const bf16*)a.q + (int64_t)b * a.q_sb + (int64_t)w.safe(sq) * a.q_st + (int64_t)h * a.q_sh;
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk) {
        qf[kk] = __builtin_bit_cast(bf16x8, ld16(q + 16 * kk + 8 * (lane >> 5)));
        settle(qf[kk]);
      }
    }
    const RingOff<DH, NW> roff = ring_offsets<DH, NW>(a.k_st, a.v_st, wave, lane);
    auto issue = [&](int j) {
      issue_keys<DH, NW>(smem + (j % C::NS) * C::STAGE, Kb, a.k_st, Vb, a.v_st, tiles.key0(j), w.run, roff, wave, lane);
    };
    auto tile = [&](int j) {
      const int k0 = tiles.key0(j);
      const char* kt = smem + (j % C::NS) * C::STAGE;
      const char* vt = kt + C::TB;
      f32x16 t[2] = {f32x16{}, f32x16{}};
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) t[mt] = mfma32x32x16(frag_rows<DH>(kt, 32 * mt, 2 * kk, lane), qf[kk], t[mt]);
      if (!w.all(k0)) w.mask(t, k0, lane, NEG_INF);
      float mx = NEG_INF;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, t[mt][r]);
      mx = max_halves(mx) * c;
      const float m_new = fmaxf(ref, mx);
      const float m_use = m_new == NEG_INF ? 0.0f : m_new;
      if (__ballot(m_new > ref)) {
        const float corr = fast_exp2(ref - m_use);
        l_run *= corr;
#pragma unroll
        for (int d = 0; d < C::DT; ++d) acc[d] *= corr;
        ref = m_new;
      }
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          t[mt][r] = fast_exp2(fmaf(t[mt][r], c, -m_use));
          l_run += t[mt][r];
        }
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const bf16x8 pb = acc_to_b(t[mt], hf);
#pragma unroll
          for (int d = 0; d < C::DT; ++d)
            acc[d] = mfma32x32x16(frag_tr<DH>(vt, 32 * mt + 16 * hf, 32 * d, lane), pb, acc[d]);
        }
    };
    ring_loop<C, C::DPS>(tiles.n, issue, [&](int j) {
      if (!w.none(tiles.key0(j))) tile(j);
    });
  }
  const float l = sum_halves(l_run);
  if (w.i < a.Sq) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;   // a row that sees nothing: 0
    store_rows<DH>((bf16*)a.o + (int64_t)b * a.o_sb + (int64_t)w.i * a.o_st + (int64_t)h * a.o_sh, acc, inv, lane);
    if (lane < 32) a.lse[((int64_t)b * a.Hq + h) * a.lse_ld + w.i] = l > 0.0f ? (ref + log2f(l)) * LN2 : NEG_INF;
  }
}

template <int DH, int NW>
static hipError_t launch_fwd(const WinArgs& a, hipStream_t s) {
  using C = WinCfg<DH, NW>;
  auto k = win_fwd_bf16_kernel<DH, NW>;
  hipError_t e = set_lds(k, C::LDS);
  if (e != hipSuccess) return e;
  const int64_t nblk = ((int64_t)a.Sq * a.G + C::ROWS - 1) / C::ROWS;
  hipLaunchKernelGGL(k, dim3((unsigned)(nblk * a.Hkv * a.B)), dim3(64 * NW), C::LDS, s, a);
  return hipGetLastError();
}

hipError_t win_fwd_bf16(const WinArgs& a, hipStream_t s) {
  return a.dh == 64 ? launch_fwd<64, 8>(a, s) : launch_fwd<128, 8>(a, s);
}

}  // namespace bpt
