// Attention with a sliding window and sinks, bf16 forward.
#include "win_tiles.h"

namespace bpt {

// Online softmax over key tiles of 64, scores transposed (S^T = K Q^T: a lane owns one row of the list
// r = token * G + head, so its maximum and sum are register reductions and one exchange), P^T straight from the accumulators into
// O^T += V^T P^T. NW waves of 32 rows share the K and V tiles of an LDS ring. The scores are scaled
// in fp32 (the FMA that subtracts the reference), so q is used as it is.
// Weights are rounded to bf16 where they become an MFMA's operand, as in the layer's attention: products of fp32 operands run at a
// sixteenth of the rate. The sum that divides them stays fp32 and unrounded. Outputs are 2.2e-3 off (fp32 weights and the output's own
// rounding: 1.6e-3).
// 16384 tokens, 16 heads of 128, 8 key heads, window 4096: 502 us, 970 TFLOP/s (full attention of 32768 tokens, 32 heads: 8.5-8.7 ms,
// 1010-1030; heads of 64, 16 of them: 2.7-3.0 ms, 730-820). Bound by issue: beside 32 MFMAs a tile costs a wave 32 exponentials, FMAs, sums,
// maxima and 16 conversions, and as many LDS fragments. Window 1024, 8192 tokens: 94 us, 690, tiles at both ends of the
// window half used and a workgroup's start and end for 18 tiles.
// Two stages for 4 waves: heads of 64 then have three workgroups on a CU (16384 tokens, window 2048: 211 -> 190 us).
template <int DH, int NW>
using WinFwdCfg = WinCfg<DH, NW, NW == 8 ? 4 : 2>;

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void win_fwd_bf16_kernel(WinArgs a) {
  using C = WinFwdCfg<DH, NW>;
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
    const RingOff<DH, NW> roff = ring_offsets<DH, NW>(a.k_st, a.v_st, wave, lane);
    auto issue = [&](int j) {
      issue_keys<DH, NW>(smem + (j % C::NS) * C::STAGE, Kb, a.k_st, Vb, a.v_st, tiles.key0(j), w.run, roff, wave, lane);
    };
    ring_start<C>(tiles.n, issue);                     // on their way before anything is waited for
    bf16x8 qf[C::KSTEPS];
    {
      const bf16* q = (const bf16*)a.q + (int64_t)b * a.q_sb + (int64_t)w.safe(sq) * a.q_st + (int64_t)h * a.q_sh;
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk) {
        qf[kk] = __builtin_bit_cast(bf16x8, ld16(q + 16 * kk + 8 * (lane >> 5)));
        settle(qf[kk]);
      }
    }
    OnlineRows<C::DT> sm{c};
    auto scores = [&](int j, f32x16 (&t)[2]) {
      const char* kt = smem + (j % C::NS) * C::STAGE;
      t[0] = t[1] = f32x16{};
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) t[mt] = mfma32x32x16(frag_rows<DH>(kt, 32 * mt, 2 * kk, lane), qf[kk], t[mt]);
    };
    auto add_values = [&](int j, const f32x16 (&t)[2]) {
      const char* vt = smem + (j % C::NS) * C::STAGE + C::TB;
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
    auto tile = [&](int j) {
      const int k0 = tiles.key0(j);
      if (w.none(k0)) return;
      f32x16 t[2];
      scores(j, t);
      if (!w.all(k0)) w.mask(t, k0, lane, NEG_INF);
      sm.weights(t, acc);
      add_values(j, t);
    };
    ring_loop<C, C::DPS>(tiles.n, issue, tile);
    ref = sm.ref;
    l_run = sm.sum;
  }
  const float l = sum_halves(l_run);
  if (w.i < a.Sq) {
    const bool sees = l != 0.0f && w.exists;         // a row that sees nothing: 0 (a NaN stays one)
    const float inv = sees ? 1.0f / l : 0.0f;
    if (!sees) {
#pragma unroll
      for (int d = 0; d < C::DT; ++d) acc[d] = f32x16{};
    }
    store_rows<DH>((bf16*)a.o + (int64_t)b * a.o_sb + (int64_t)w.i * a.o_st + (int64_t)h * a.o_sh, acc, inv, lane);
    if (lane < 32) a.lse[((int64_t)b * a.Hq + h) * a.lse_ld + w.i] = sees ? (ref + log2f(l)) * LN2 : NEG_INF;
  }
}

// Few rows (new tokens, short pieces of a prompt): 32 rows per workgroup and one of a.nsplit slices of the key tiles, so
// that the cache is read by the whole chip. Bound by that read: each of the 4 waves streams tiles of 32 keys (every fourth of the
// slice) through two LDS stages of its own, without a barrier, 80 KB of a CU's LDS in flight while the other 80 KB
// are worked on; waves and slices are merged as two runs of an online softmax are. 24 sequences of up to 16384 keys, 32 heads of 128,
// 8 key heads, all keys visible: 285 us, 5.7 TB/s; one of 65536: 57 us, 4.7 TB/s with the join.
template <int DH>
struct WinTokCfg {
  static constexpr int KSTEPS = DH / 16, DT = DH / 32, NW = 4;
  static constexpr int PITCH = RmTile<DH>::PITCH, SLOTS = RmTile<DH>::SLOTS;
  static constexpr int BL = (32 * PITCH + 1023) / 1024, TB = BL * 1024;   // copies and bytes of 32 rows (the last copy runs past them)
  static constexpr int STAGE = 2 * TB, LDS = NW * 2 * STAGE;
  static constexpr int OP = DH + 4;                   // pitch of a merged row, floats
  static_assert(NW * 32 * OP * 4 + 2 * NW * 32 * 4 <= LDS, "the merge reuses the stages");
};

template <int DH>
__global__ __launch_bounds__(256, 1) void win_token_kernel(WinArgs a) {
  using C = WinTokCfg<DH>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = a.Sq * a.G, nblk = (rows + 31) / 32;
  int hh, blk;
  xcd_map((int)blockIdx.x, a.Hkv * a.B, hh, blk);
  const int kvh = hh % a.Hkv, b = hh / a.Hkv, slice = blk / nblk, r0 = blk % nblk * 32;
  const Seq sq = seq_of(a, b);
  const Rows w(a, sq, r0, 0, 32, lane);
  const int h = kvh * a.G + w.head;
  const bf16* Kb = (const bf16*)a.k + (int64_t)b * a.k_sb + (int64_t)kvh * a.k_sh;
  const bf16* Vb = (const bf16*)a.v + (int64_t)b * a.v_sb + (int64_t)kvh * a.v_sh;
  const Tiles<32> tiles(w.run);
  const int per = (tiles.n + a.nsplit - 1) / a.nsplit, j0 = slice * per, j1 = min(j0 + per, tiles.n);

  f32x16 acc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t) acc[t] = f32x16{};
  OnlineRows<C::DT> sm{a.scale * LOG2E};
  if (j0 + wave < j1) {
    bf16x8 qf[C::KSTEPS];
    {
      const bf16* q = (const bf16*)a.q + (int64_t)b * a.q_sb + (int64_t)w.safe(sq) * a.q_st + (int64_t)h * a.q_sh;
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk) {
        qf[kk] = __builtin_bit_cast(bf16x8, ld16(q + 16 * kk + 8 * (lane >> 5)));
        settle(qf[kk]);
      }
    }
    char* mine = smem + wave * 2 * C::STAGE;
    auto issue = [&](int j, int at) {
      const int k0 = tiles.key0(j);
      const Vis seen = seen_in(w.run, k0, 32);
      const bf16 *ko = Kb + (int64_t)k0 * a.k_st, *vo = Vb + (int64_t)k0 * a.v_st;
#pragma unroll
      for (int i = 0; i < C::BL; ++i) {
        const int slot = 64 * i + lane, col = slot % C::SLOTS, k = k0 + slot / C::SLOTS;
        const int row = seen.clamp(k) - k0, c8 = (col < DH / 8 ? col : 0) * 8;
        dma16s(scalar_ptr(ko), 2u * (uint32_t)(row * a.k_st + c8), mine + at * C::STAGE + i * 1024);
        dma16s(scalar_ptr(vo), 2u * (uint32_t)(row * a.v_st + c8), mine + at * C::STAGE + C::TB + i * 1024);
      }
    };
    int at = 0;
    issue(j0 + wave, 0);
    for (int j = j0 + wave; j < j1; j += 4, at ^= 1) {
      if (j + 4 < j1) {
        issue(j + 4, at ^ 1);
        wait_vmcnt<2 * C::BL>();
      } else {
        wait_vmcnt<0>();
      }
      const int k0 = tiles.key0(j);
      const char* kt = mine + at * C::STAGE;
      f32x16 t[1] = {f32x16{}};
#pragma unroll
      for (int kk = 0; kk < C::KSTEPS; ++kk) t[0] = mfma32x32x16(frag_rows<DH>(kt, 0, 2 * kk, lane), qf[kk], t[0]);
      w.mask(t, k0, lane, NEG_INF);
      sm.weights(t, acc);
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const bf16x8 pb = acc_to_b(t[0], hf);
#pragma unroll
        for (int d = 0; d < C::DT; ++d) acc[d] = mfma32x32x16(frag_tr<DH>(kt + C::TB, 16 * hf, 32 * d, lane), pb, acc[d]);
      }
      wait_lgkm();                                    // the stage is read before the next copies overwrite it
    }
  }
  // merge the waves in order: numerators row by row in LDS, with maximum and sum
  __syncthreads();
  float* red = (float*)smem;
  float *red_m = red + C::NW * 32 * C::OP, *red_l = red_m + C::NW * 32;
  const float l = sum_halves(sm.sum);
  float* my = red + (wave * 32 + (lane & 31)) * C::OP;
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg)
      *(f32x4*)(my + 32 * t + 8 * rg + 4 * (lane >> 5)) = f32x4{acc[t][4 * rg], acc[t][4 * rg + 1], acc[t][4 * rg + 2], acc[t][4 * rg + 3]};
  if (lane < 32) {
    red_m[wave * 32 + lane] = sm.ref;
    red_l[wave * 32 + lane] = l;
  }
  __syncthreads();
  for (int e = tid; e < 32 * (DH / 4); e += 256) {
    const int ri = e / (DH / 4), d = 4 * (e % (DH / 4)), rr = r0 + ri;
    if (rr >= rows) break;
    float m = NEG_INF, lt = 0.0f;
#pragma unroll
    for (int v = 0; v < C::NW; ++v) m = fmaxf(m, red_m[v * 32 + ri]);
    f32x4 o = {};
#pragma unroll
    for (int v = 0; v < C::NW; ++v) {                 // a wave without keys: zeros (or a NaN)
      const float f = red_m[v * 32 + ri] == NEG_INF ? 1.0f : fast_exp2(red_m[v * 32 + ri] - m);
      lt = fmaf(red_l[v * 32 + ri], f, lt);
      o += f * *(const f32x4*)(red + (v * 32 + ri) * C::OP + d);
    }
    if (rr / a.G >= sq.nq) {
      m = NEG_INF;
      lt = 0.0f;
      o = f32x4{};
    }
    if (a.nsplit > 1) {
      const int64_t p = ((int64_t)slice * a.B * a.Hkv + (int64_t)b * a.Hkv + kvh) * rows + rr;
      *(f32x4*)(a.part_o + p * DH + d) = o;
      if (d == 0) {
        a.part_ml[2 * p] = m;
        a.part_ml[2 * p + 1] = lt;
      }
      continue;
    }
    const int i = rr / a.G, hq = kvh * a.G + rr % a.G;
    const float inv = lt != 0.0f ? 1.0f / lt : 0.0f;  // a row that sees nothing: 0
    bf16x4 x;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = (bf16)(lt != 0.0f ? o[k] * inv : 0.0f);   // beside rows that see a NaN too
    *(bf16x4*)((bf16*)a.o + (int64_t)b * a.o_sb + (int64_t)i * a.o_st + (int64_t)hq * a.o_sh + d) = x;
    if (d == 0) a.lse[((int64_t)b * a.Hq + hq) * a.lse_ld + i] = lt != 0.0f ? (m + log2f(lt)) * LN2 : NEG_INF;
  }
}

template <int DH, int NW>
static hipError_t launch_fwd(const WinArgs& a, hipStream_t s) {
  using C = WinFwdCfg<DH, NW>;
  auto k = win_fwd_bf16_kernel<DH, NW>;
  hipError_t e = set_lds(k, C::LDS);
  if (e != hipSuccess) return e;
  const int64_t nblk = ((int64_t)a.Sq * a.G + C::ROWS - 1) / C::ROWS;
  hipLaunchKernelGGL(k, dim3((unsigned)(nblk * a.Hkv * a.B)), dim3(64 * NW), C::LDS, s, a);
  return hipGetLastError();
}
template <int DH>
static hipError_t launch_token(const WinArgs& a, hipStream_t s) {
  using C = WinTokCfg<DH>;
  auto k = win_token_kernel<DH>;
  hipError_t e = set_lds(k, C::LDS);
  if (e != hipSuccess) return e;
  const int64_t nblk = ((int64_t)a.Sq * a.G + 31) / 32;
  hipLaunchKernelGGL(k, dim3((unsigned)(nblk * a.nsplit * a.Hkv * a.B)), dim3(256), C::LDS, s, a);
  return hipGetLastError();
}

template <int DH>
static hipError_t fwd(const WinArgs& a, hipStream_t s) {
  if (a.few) return launch_token<DH>(a, s);
  return win_wide(a.Sq, a) ? launch_fwd<DH, 8>(a, s) : launch_fwd<DH, 4>(a, s);
}
hipError_t win_fwd_bf16(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? fwd<64>(a, s) : fwd<128>(a, s); }

}  // namespace bpt
