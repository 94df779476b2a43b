// Attention with a sliding window and sinks, fp32: forward (whole, or one of several slices of
// the keys), its join, and the backward. Matrix products on v_mfma_f32_16x16x4_f32 (attn_common.h:
// row and column fragments straight from memory, 4 waves, in the backward 8, sharing 16 rows).
//
// The query heads of a kv head and their tokens are one list of rows, r = token * G + head: a
// workgroup's 16 rows then cover few tokens, see nearly the same keys, and a single token's heads
// fill one workgroup.
//
// Bound by latency where few rows leave each workgroup alone on its CU: 512 tokens, 4 heads of 64, window 128: forward 7.6 us, backward
// 19, each a chain of a few tiles (fragments from L2, dh / 4 dependent fp32 MFMAs, exponentials), a start and a merge.
#include <algorithm>

#include "win_attn.h"

namespace bpt {

namespace {

// Column fragment of rows given by a clamp of the key index
template <int DH>
BPT_DEV ColFrag<DH> col_frag_vis(const float* X, int64_t ld, int key0, const Vis& v, int g, int c16) {
  ColFrag<DH> f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t row = v.clamp(key0 + 4 * g + r);
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) f.v[r][t] = X[row * ld + 16 * t + c16];
  }
  return f;
}

}  // namespace

// 16 rows of one kv head; wave w takes the key tiles of 32 w, w + 4, ... of the slice, with its own
// running maximum and sum (both in units of the raw products; -inf and 0 until a row has seen a
// key), merged at the end in wave order. Several slices: the unnormalised numerator, maximum and sum go to
// the workspace, for win_join.
template <int DH>
__global__ __launch_bounds__(256) void win_fwd_f32_kernel(WinArgs a) {
  constexpr int NC = DH / 16;
  __shared__ __attribute__((aligned(16))) float red[4][16][DH + 4];
  __shared__ float red_m[4][16], red_l[4][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
  const int rows = a.Sq * a.G, nblk = (rows + 15) / 16;
  const int slice = blockIdx.x / nblk, blk = nblk - 1 - blockIdx.x % nblk;   // most keys first
  const int kvh = blockIdx.y, b = blockIdx.z;
  const Seq sq = seq_of(a, b);
  const int r0 = blk * 16;
  const int i0 = r0 / a.G, i1 = min((r0 + 15) / a.G, sq.nq - 1);
  const int row = r0 + c16, i = row / a.G, h = kvh * a.G + row % a.G;
  const float c = a.scale * LOG2E;

  Vis mine{0, -1, 0}, run{0, -1, 0};
  if (i < sq.nq) mine = vis_of(a, sq, sq.off + i, sq.off + i);
  if (i0 <= i1) run = vis_run(a, sq, sq.off + i0, sq.off + i1);
  const Tiles<32> tiles(run);
  const int per = (tiles.n + a.nsplit - 1) / a.nsplit, j0 = slice * per, j1 = min(j0 + per, tiles.n);

  const float* Kb = (const float*)a.k + (int64_t)b * a.k_sb + (int64_t)kvh * a.k_sh;
  const float* Vb = (const float*)a.v + (int64_t)b * a.v_sb + (int64_t)kvh * a.v_sh;
  f32x4 acc[NC];
#pragma unroll
  for (int t = 0; t < NC; ++t) acc[t] = f32x4{};
  float m_run = NEG_INF, l_run = 0.0f;
  if (j0 < j1) {                                   // the run has a query: row i1 exists
    const int qi = min(i, sq.nq - 1);
    const RowFrag<DH> qf = row_frag<DH>((const float*)a.q + (int64_t)b * a.q_sb + (int64_t)qi * a.q_st + (int64_t)h * a.q_sh, g);
    for (int j = j0 + wave; j < j1; j += 4) {
      const int k0 = tiles.key0(j);
      f32x4 s[2];
      ColFrag<DH> vf[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const RowFrag<DH> kf = row_frag<DH>(Kb + (int64_t)run.clamp(k0 + 16 * u + c16) * a.k_st, g);
        s[u] = dot_frags<DH>(kf, qf);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) vf[u] = col_frag_vis<DH>(Vb, a.v_st, k0 + 16 * u, run, g, c16);
      float mx = NEG_INF;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (!mine.sees(k0 + 16 * u + 4 * g + r)) s[u][r] = NEG_INF;
          else s[u][r] *= c;
          mx = fmaxf(mx, s[u][r]);
        }
      const float m_new = fmaxf(m_run, max_groups(mx));
      const float m_use = m_new == NEG_INF ? 0.0f : m_new;
      const float corr = m_run == NEG_INF ? 0.0f : fast_exp2(m_run - m_use);
      l_run *= corr;
#pragma unroll
      for (int t = 0; t < NC; ++t) acc[t] *= corr;
      m_run = m_new;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[u][r] = fast_exp2(s[u][r] - m_use);
          l_run += s[u][r];
        }
#pragma unroll
      for (int u = 0; u < 2; ++u) add_outer<DH>(acc, vf[u], s[u]);
    }
  }
  l_run = sum_groups(l_run);
  if (g == 0) {
    red_m[wave][c16] = m_run;
    red_l[wave][c16] = l_run;
  }
#pragma unroll
  for (int t = 0; t < NC; ++t) *(f32x4*)&red[wave][c16][16 * t + 4 * g] = acc[t];
  __syncthreads();
  for (int e = tid; e < 16 * (DH / 4); e += 256) {
    const int ri = e / (DH / 4), d = 4 * (e % (DH / 4)), rr = r0 + ri;
    if (rr >= rows) continue;
    float m = NEG_INF, l = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, red_m[w][ri]);
    f32x4 o = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = red_m[w][ri] == NEG_INF ? 1.0f : fast_exp2(red_m[w][ri] - m);   // without keys: zeros (or a NaN)
      l = fmaf(red_l[w][ri], f, l);
      o += f * *(const f32x4*)&red[w][ri][d];
    }
    if (a.nsplit > 1) {
      const int64_t at = ((int64_t)slice * a.B * a.Hkv + (int64_t)b * a.Hkv + kvh) * rows + rr;
      *(f32x4*)(a.part_o + at * DH + d) = o;
      if (d == 0) {
        a.part_ml[2 * at] = m;
        a.part_ml[2 * at + 1] = l;
      }
      continue;
    }
    const int ii = rr / a.G, hh = kvh * a.G + rr % a.G;
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;  // a row that sees nothing: 0 (a NaN stays one)
    *(f32x4*)((float*)a.o + (int64_t)b * a.o_sb + (int64_t)ii * a.o_st + (int64_t)hh * a.o_sh + d) = l != 0.0f ? o * inv : f32x4{};
    if (d == 0) a.lse[((int64_t)b * a.Hq + hh) * a.lse_ld + ii] = l != 0.0f ? (m + log2f(l)) * LN2 : NEG_INF;
  }
}

// Joins the slices of a row: one wave per row; lane z holds the maximum and sum of slice z, numerators are added in order.
template <typename T>
__global__ __launch_bounds__(256) void win_join_kernel(WinArgs a) {
  const int lane = threadIdx.x & 63;
  const int rows = a.Sq * a.G;
  const int rr = blockIdx.x * 4 + (threadIdx.x >> 6), kvh = blockIdx.y, b = blockIdx.z;
  if (rr >= rows) return;
  const int64_t all = (int64_t)a.B * a.Hkv * rows, at = ((int64_t)b * a.Hkv + kvh) * rows + rr;
  const int d = a.dh == 128 ? 2 * lane : lane;
  float mz = NEG_INF, l = 0.0f;                      // of slice `lane`; at most 64
  if (lane < a.nsplit) {
    const float* ml = a.part_ml + 2 * (lane * all + at);
    mz = ml[0];
    l = ml[1];
  }
  float m = mz;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float fz = mz == NEG_INF ? 1.0f : fast_exp2(mz - m);   // without keys: zeros (or a NaN)
  l *= fz;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) l += __shfl_xor(l, o, 64);
  float o0 = 0.0f, o1 = 0.0f;
#pragma unroll 8
  for (int z = 0; z < a.nsplit; ++z) {
    const float f = __shfl(fz, z, 64);
    const float* p = a.part_o + (z * all + at) * a.dh + d;
    o0 = fmaf(p[0], f, o0);
    if (a.dh == 128) o1 = fmaf(p[1], f, o1);
  }
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  const int i = rr / a.G, h = kvh * a.G + rr % a.G;
  T* o = (T*)a.o + (int64_t)b * a.o_sb + (int64_t)i * a.o_st + (int64_t)h * a.o_sh + d;
  o[0] = from_f32<T>(l != 0.0f ? o0 * inv : 0.0f);   // a row that sees nothing: 0, beside rows that see a NaN too
  if (a.dh == 128) o[1] = from_f32<T>(l != 0.0f ? o1 * inv : 0.0f);
  if (lane == 0) a.lse[((int64_t)b * a.Hq + h) * a.lse_ld + i] = l != 0.0f ? (m + log2f(l)) * LN2 : NEG_INF;
}

// -Delta = -sum_d dO O and -lse / scale (what the raw products are reduced by) of every row, [B, Hq, Sqp]; 0 where a row
// sees nothing, and behind the rows. 8 features a lane, dh / 8 lanes a row.
//
// bf16: the rounding of O leaves Delta off by about 2^-9 |dO| |O|, which matters beside dS where few keys are averaged
// (|O| falls as 1 / sqrt(keys), and dS cancels: a row with one key has dS = 0). A row that sees at most 8 keys takes Delta =
// sum_k P dP instead, which is as exact as the products: the gradients' error over a batch of 4 x 1000 tokens, window 256, falls from 2.5e-3
// to that of the rounded P and dS alone, 2.35e-3. Else bound by the read of O and dO: 8192 tokens, 16 heads of 128 13 us, 5 TB/s.
constexpr int kExactKeys = 8;

struct Row8 {                                       // 8 features
  float v[8];
  Row8() = default;
  BPT_DEV explicit Row8(const float* p) {
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  }
  BPT_DEV explicit Row8(const bf16* p) {
    const bf16x8 a = *(const bf16x8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
  }
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void win_delta_kernel(WinArgs a) {
  constexpr int LPR = DH / 8;                       // lanes per row
  const int d = 8 * (threadIdx.x % LPR);
  const int i = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, h = blockIdx.y, b = blockIdx.z;   // Sqp % (256 / LPR) == 0
  const int64_t at = ((int64_t)b * a.Hq + h) * a.Sqp + i;
  const Seq sq = seq_of(a, b);
  auto dot = [&](const Row8& x, const Row8& y) {     // over the row's lanes
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x.v[e], y.v[e], s);
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
    return s;
  };
  float s = 0.0f, nl = 0.0f;
  if (i < sq.nq) {                                  // the same for all lanes of a row
    const int64_t o = (int64_t)b * a.o_sb + (int64_t)i * a.o_st + (int64_t)h * a.o_sh + d;
    const Row8 g((const T*)a.dout + o), out((const T*)a.o + o);
    const float lse = a.lse[((int64_t)b * a.Hq + h) * a.lse_ld + i];
    const bool sees = lse != NEG_INF;
    nl = sees ? -lse / a.scale : 0.0f;
    const Vis v = vis_of(a, sq, sq.off + i, sq.off + i);
    const int from = max(v.lo, v.se), n = v.se + max(v.hi + 1 - from, 0);   // keys 0 .. se - 1 and from .. hi
    if (sizeof(T) == 2 && n <= kExactKeys) {
      const Row8 q((const T*)a.q + (int64_t)b * a.q_sb + (int64_t)i * a.q_st + (int64_t)h * a.q_sh + d);
      const T* K = (const T*)a.k + (int64_t)b * a.k_sb + (int64_t)(h / a.G) * a.k_sh + d;
      const T* V = (const T*)a.v + (int64_t)b * a.v_sb + (int64_t)(h / a.G) * a.v_sh + d;
#pragma unroll 1
      for (int j0 = 0; j0 < n; j0 += 2) {            // two keys' rows on their way at once
        Row8 kr[2], vr[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int j = min(j0 + u, n - 1);
          const int64_t k = j < v.se ? j : from + j - v.se;
          kr[u] = Row8(K + k * a.k_st);
          vr[u] = Row8(V + k * a.v_st);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float p = fast_exp2((dot(q, kr[u]) + nl) * a.scale * LOG2E), dp = dot(g, vr[u]);
          s = j0 + u < n ? fmaf(p, dp, s) : s;
        }
      }
    } else {
      s = dot(g, out);
      s = sees ? s : 0.0f;
    }
  }
  if (d == 0) {
    a.ndelta[at] = -s;
    a.nlse[at] = nl;
  }
}

// Sums of 8 waves' 16 x DH results (rows on lanes), in LDS: red[0 .. 3] are left to be added
template <int DH>
BPT_DEV void add_eight(float (&red)[4][16][DH + 4], const f32x4 (&x)[DH / 16], int wave, int g, int c16) {
  __syncthreads();
  if (wave >= 4)
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) *(f32x4*)&red[wave - 4][c16][16 * t + 4 * g] = x[t];
  __syncthreads();
  if (wave < 4)
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) {
      f32x4* at = (f32x4*)&red[wave][c16][16 * t + 4 * g];
      *at = x[t] + *at;
    }
  __syncthreads();
}
template <int DH>
BPT_DEV f32x4 add_four(const float (&red)[4][16][DH + 4], int row, int d) {
  return ((*(const f32x4*)&red[0][row][d] + *(const f32x4*)&red[1][row][d]) + *(const f32x4*)&red[2][row][d]) +
         *(const f32x4*)&red[3][row][d];
}

// dQ: 16 rows as in the forward, each of 8 waves takes every eighth key tile of 16; dS^T has the row on the
// lane axis and is the B operand of dQ^T += K^T dS^T.
template <int DH>
BPT_DEV void dq_f32(const WinArgs& a, float (&red)[4][16][DH + 4], int blk) {
  constexpr int NC = DH / 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
  const int rows = a.Sq * a.G, r0 = blk * 16;
  const int kvh = blockIdx.y, b = blockIdx.z;
  const Seq sq = seq_of(a, b);
  const int i0 = r0 / a.G, i1 = min((r0 + 15) / a.G, sq.nq - 1);
  const int row = r0 + c16, i = row / a.G, h = kvh * a.G + row % a.G;
  const float c = a.scale * LOG2E;
  Vis mine{0, -1, 0}, run{0, -1, 0};
  if (i < sq.nq) mine = vis_of(a, sq, sq.off + i, sq.off + i);
  if (i0 <= i1) run = vis_run(a, sq, sq.off + i0, sq.off + i1);
  const Tiles<16> tiles(run);
  const float* Kb = (const float*)a.k + (int64_t)b * a.k_sb + (int64_t)kvh * a.k_sh;
  const float* Vb = (const float*)a.v + (int64_t)b * a.v_sb + (int64_t)kvh * a.v_sh;
  f32x4 dq[NC];
#pragma unroll
  for (int t = 0; t < NC; ++t) dq[t] = f32x4{};
  if (tiles.n > 0) {
    const int qi = min(i, sq.nq - 1);
    const RowFrag<DH> qf = row_frag<DH>((const float*)a.q + (int64_t)b * a.q_sb + (int64_t)qi * a.q_st + (int64_t)h * a.q_sh, g);
    const RowFrag<DH> of = row_frag<DH>((const float*)a.dout + (int64_t)b * a.o_sb + (int64_t)qi * a.o_st + (int64_t)h * a.o_sh, g);
    const int64_t sidx = ((int64_t)b * a.Hq + h) * a.Sqp + qi;
    const float nl = a.nlse[sidx], ndl = a.ndelta[sidx];
    for (int j = wave; j < tiles.n; j += 8) {
      const int k0 = tiles.key0(j);
      const int64_t kr = run.clamp(k0 + c16);
      const RowFrag<DH> kf = row_frag<DH>(Kb + kr * a.k_st, g), vf = row_frag<DH>(Vb + kr * a.v_st, g);
      const ColFrag<DH> kc = col_frag_vis<DH>(Kb, a.k_st, k0, run, g, c16);
      const f32x4 s = dot_frags<DH>(kf, qf);
      f32x4 ds = dot_frags<DH>(vf, of);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        ds[r] = mine.sees(k0 + 4 * g + r) ? fast_exp2((s[r] + nl) * c) * (ds[r] + ndl) : 0.0f;
      add_outer<DH>(dq, kc, ds);
    }
  }
  if (!mine.any()) {                                 // nothing seen: 0, beside rows that see a NaN too
#pragma unroll
    for (int t = 0; t < NC; ++t) dq[t] = f32x4{};
  }
  add_eight<DH>(red, dq, wave, g, c16);
  for (int e = tid; e < 16 * (DH / 4); e += 512) {
    const int ri = e / (DH / 4), d = 4 * (e % (DH / 4)), rr = r0 + ri;
    if (rr >= rows) continue;
    const f32x4 x = add_four<DH>(red, ri, d);
    const int ii = rr / a.G, hh = kvh * a.G + rr % a.G;
    *(f32x4*)((float*)a.dq + (int64_t)b * a.q_sb + (int64_t)ii * a.q_st + (int64_t)hh * a.q_sh + d) = x * a.dq_scale;
  }
}

// dK, dV: 16 keys (FAR: 16 sinks and a chunk of the queries beyond their window, as in the bf16 kernel); each of 8 waves takes every eighth (query head, tile of 16 queries) pair of the kv head, in order. P
// and dS have the key on the lane axis and are the B operands of dV^T += dO^T P, dK^T += Q^T dS.
template <int DH, bool FAR>
BPT_DEV void dkdv_f32(const WinArgs& a, float (&red)[4][16][DH + 4], int blk) {
  constexpr int NC = DH / 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
  const int chunks = FAR ? a.far : a.chunks, chunk = blk % chunks;
  const int kvh = blockIdx.y, b = blockIdx.z, k0 = blk / chunks * 16, key = k0 + c16;
  const Seq sq = seq_of(a, b);
  const bool near = FAR || a.far > 0;
  const int kend = FAR ? min(sq.nk, a.sinks) : sq.nk;
  const float c = a.scale * LOG2E;
  f32x4 dk[NC], dv[NC];
#pragma unroll
  for (int t = 0; t < NC; ++t) dk[t] = dv[t] = f32x4{};
  if (k0 < kend) {
    const int kr = min(key, kend - 1);
    QVis mine = qvis_of(a, sq, key, key, near);
    if (key >= sq.nk) mine.hi = -1;
    QVis run = qvis_of(a, sq, k0, min(k0 + 15, kend - 1), near);
    if (FAR) run = QVis{a.causal ? max(k0 + a.window - sq.off, 0) : 0, sq.nq - 1};
    const RowFrag<DH> kf = row_frag<DH>((const float*)a.k + (int64_t)b * a.k_sb + (int64_t)kvh * a.k_sh + (int64_t)kr * a.k_st, g);
    const RowFrag<DH> vf = row_frag<DH>((const float*)a.v + (int64_t)b * a.v_sb + (int64_t)kvh * a.v_sh + (int64_t)kr * a.v_st, g);
    const int t0 = run.lo / 16, nt = run.hi >= run.lo ? run.hi / 16 + 1 - t0 : 0;
    const int per = (nt * a.G + chunks - 1) / chunks;
    for (int it = chunk * per + wave; it < min((chunk + 1) * per, nt * a.G); it += 8) {
      const int h = kvh * a.G + it / nt, q0 = 16 * (t0 + it % nt);
      const float* Qb = (const float*)a.q + (int64_t)b * a.q_sb + (int64_t)h * a.q_sh;
      const float* dOb = (const float*)a.dout + (int64_t)b * a.o_sb + (int64_t)h * a.o_sh;
      const int64_t qr = min(max(q0 + c16, run.lo), run.hi);
      const RowFrag<DH> qf = row_frag<DH>(Qb + qr * a.q_st, g), of = row_frag<DH>(dOb + qr * a.o_st, g);
      const int64_t sidx = ((int64_t)b * a.Hq + h) * a.Sqp + q0 + 4 * g;   // Sqp % 64 == 0
      const f32x4 l4 = *(const f32x4*)(a.nlse + sidx), d4 = *(const f32x4*)(a.ndelta + sidx);
      const Vis qv{run.lo, run.hi, 0};
      ColFrag<DH> oc, qc;                            // fetched with the rest where registers allow
      if constexpr (DH == 64) {
        oc = col_frag_vis<DH>(dOb, a.o_st, q0, qv, g, c16);
        qc = col_frag_vis<DH>(Qb, a.q_st, q0, qv, g, c16);
        __builtin_amdgcn_sched_barrier(0);
      }
      f32x4 p = dot_frags<DH>(qf, kf), ds = dot_frags<DH>(of, vf);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int q = q0 + 4 * g + r;
        const bool in = q >= mine.lo && q <= mine.hi;
        const bool ok = !FAR ? in : q <= run.hi && (a.causal ? q > mine.hi : !in);
        p[r] = ok ? fast_exp2((p[r] + l4[r]) * c) : 0.0f;
        ds[r] = ok ? p[r] * (ds[r] + d4[r]) : 0.0f;
      }
      if constexpr (DH != 64) oc = col_frag_vis<DH>(dOb, a.o_st, q0, qv, g, c16);
      add_outer<DH>(dv, oc, p);
      if constexpr (DH != 64) qc = col_frag_vis<DH>(Qb, a.q_st, q0, qv, g, c16);
      add_outer<DH>(dk, qc, ds);
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    f32x4 (&x)[NC] = which ? dv : dk;
    add_eight<DH>(red, x, wave, g, c16);
    const int64_t base = which ? (int64_t)b * a.v_sb + (int64_t)kvh * a.v_sh : (int64_t)b * a.k_sb + (int64_t)kvh * a.k_sh;
    float* out = (float*)(which ? a.dv : a.dk) + base;
    for (int e = tid; e < 16 * (DH / 4); e += 512) {
      const int ki = e / (DH / 4), d = 4 * (e % (DH / 4));
      const int ns = win_slot_keys(a);
      if (k0 + ki >= (FAR ? ns : a.Skv)) continue;
      const f32x4 x = add_four<DH>(red, ki, d);
      if (k0 + ki < ns) {
        const int64_t at = ((int64_t)(FAR ? 1 + chunk : chunk) * a.B * a.Hkv + (int64_t)b * a.Hkv + kvh) * ns + k0 + ki;
        *(f32x4*)(a.part_s + (2 * at + which) * DH + d) = x;
        continue;
      }
      *(f32x4*)(out + (int64_t)(k0 + ki) * (which ? a.v_st : a.k_st) + d) = x * (which ? 1.0f : a.scale);
    }
  }
}

// dK dV by the first nkv workgroups of a kv head, dQ by the others: neither needs the other
template <int DH>
__global__ __launch_bounds__(512) void win_bwd_f32_kernel(WinArgs a, int nkv) {
  __shared__ __attribute__((aligned(16))) float red[4][16][DH + 4];
  if ((int)blockIdx.x < nkv) dkdv_f32<DH, false>(a, red, blockIdx.x);
  else dq_f32<DH>(a, red, gridDim.x - 1 - blockIdx.x);
}
template <int DH>
__global__ __launch_bounds__(512) void win_far_f32_kernel(WinArgs a) {
  __shared__ __attribute__((aligned(16))) float red[4][16][DH + 4];
  dkdv_f32<DH, true>(a, red, blockIdx.x);
}

template <int DH>
static hipError_t fwd_f32(const WinArgs& a, hipStream_t s) {
  const unsigned nblk = (unsigned)(((int64_t)a.Sq * a.G + 15) / 16);
  hipLaunchKernelGGL(win_fwd_f32_kernel<DH>, dim3(nblk * a.nsplit, a.Hkv, a.B), dim3(256), 0, s, a);
  return hipGetLastError();
}
// dK and dV of the sinks: the window's part and the chunks'. A workgroup per (sink, dK or dV): its groups of DH / 4 lanes take
// every n-th slot, in order, and are added in order.
template <typename T, int DH>
__global__ __launch_bounds__(256) void win_sinks_kernel(WinArgs a, int slots) {
  constexpr int L = DH / 4, N = 256 / L;
  __shared__ f32x4 red[N][L];
  const int ns = min(a.sinks, a.Skv), grp = threadIdx.x / L, l = threadIdx.x % L;
  const int64_t row = blockIdx.x, stride = (int64_t)gridDim.x * DH;
  const int which = (int)(row % 2), key = (int)(row / 2 % ns);
  const int64_t bh = row / 2 / ns, b = bh / a.Hkv, kvh = bh % a.Hkv;
  f32x4 x = {};
  if (key < seq_of(a, (int)b).nk) {
    const float* p = a.part_s + row * DH + 4 * l;
#pragma unroll 4
    for (int z = grp; z < slots; z += N) x += *(const f32x4*)(p + z * stride);
  }
  red[grp][l] = x;
  __syncthreads();
  if (grp) return;
  for (int g = 1; g < N; ++g) x += red[g][l];
  if (!which) x *= a.scale;
  T* out = which ? (T*)a.dv + b * a.v_sb + (int64_t)key * a.v_st + kvh * a.v_sh : (T*)a.dk + b * a.k_sb + (int64_t)key * a.k_st + kvh * a.k_sh;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[4 * l + e] = from_f32<T>(x[e]);
}

// dK and dV of all keys from a few slots, in order: 4 features a thread.
template <typename T>
__global__ __launch_bounds__(256) void win_chunks_kernel(WinArgs a) {
  const int L = a.dh / 4, at = blockIdx.x * 256 + threadIdx.x, key = at / (2 * L), which = at / L % 2, d = 4 * (at % L);
  const int kvh = blockIdx.y, b = blockIdx.z;
  if (key >= a.Skv) return;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.Skv * 2, row = (((int64_t)b * a.Hkv + kvh) * a.Skv + key) * 2 + which;
  f32x4 x = {};
  if (key < seq_of(a, b).nk)
    for (int z = 0; z < a.chunks; ++z) x += *(const f32x4*)(a.part_s + (z * rows + row) * a.dh + d);
  if (!which) x *= a.scale;
  T* out = which ? (T*)a.dv + b * a.v_sb + (int64_t)key * a.v_st + kvh * a.v_sh : (T*)a.dk + b * a.k_sb + (int64_t)key * a.k_st + kvh * a.k_sh;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[d + e] = from_f32<T>(x[e]);
}

template <int DH>
static hipError_t bwd_f32(const WinArgs& a, hipStream_t s) {
  const int nkv = a.dk ? (a.Skv + 15) / 16 * a.chunks : 0, nq = a.dq ? (int)(((int64_t)a.Sq * a.G + 15) / 16) : 0;
  if (nkv + nq == 0) return hipSuccess;
  hipLaunchKernelGGL(win_bwd_f32_kernel<DH>, dim3(nkv + nq, a.Hkv, a.B), dim3(512), 0, s, a, nkv);
  return hipGetLastError();
}
template <int DH>
static hipError_t far_f32(const WinArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(win_far_f32_kernel<DH>, dim3((std::min(a.sinks, a.Skv) + 15) / 16 * a.far, a.Hkv, a.B), dim3(512), 0, s, a);
  return hipGetLastError();
}
hipError_t win_fwd_f32(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? fwd_f32<64>(a, s) : fwd_f32<128>(a, s); }
hipError_t win_bwd_f32(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? bwd_f32<64>(a, s) : bwd_f32<128>(a, s); }
hipError_t win_far_f32(const WinArgs& a, hipStream_t s) { return a.dh == 64 ? far_f32<64>(a, s) : far_f32<128>(a, s); }

hipError_t win_join(Dt t, const WinArgs& a, hipStream_t s) {
  auto k = t == BF16 ? win_join_kernel<bf16> : win_join_kernel<float>;
  hipLaunchKernelGGL(k, dim3((unsigned)(((int64_t)a.Sq * a.G + 3) / 4), a.Hkv, a.B), dim3(256), 0, s, a);
  return hipGetLastError();
}
hipError_t win_chunks(Dt t, const WinArgs& a, hipStream_t s) {
  auto k = t == BF16 ? win_chunks_kernel<bf16> : win_chunks_kernel<float>;
  hipLaunchKernelGGL(k, dim3((unsigned)(((int64_t)a.Skv * a.dh / 2 + 255) / 256), a.Hkv, a.B), dim3(256), 0, s, a);
  return hipGetLastError();
}
hipError_t win_sinks(Dt t, const WinArgs& a, int slots, hipStream_t s) {
  const int64_t n = (int64_t)a.B * a.Hkv * std::min(a.sinks, a.Skv) * 2;
  auto k = t == BF16 ? (a.dh == 64 ? win_sinks_kernel<bf16, 64> : win_sinks_kernel<bf16, 128>)
                     : (a.dh == 64 ? win_sinks_kernel<float, 64> : win_sinks_kernel<float, 128>);
  hipLaunchKernelGGL(k, dim3((unsigned)n), dim3(256), 0, s, a, slots);
  return hipGetLastError();
}
hipError_t win_delta(Dt t, const WinArgs& a, hipStream_t s) {
  auto k = t == BF16 ? (a.dh == 64 ? win_delta_kernel<bf16, 64> : win_delta_kernel<bf16, 128>)
                     : (a.dh == 64 ? win_delta_kernel<float, 64> : win_delta_kernel<float, 128>);
  hipLaunchKernelGGL(k, dim3((unsigned)(a.Sqp * (a.dh / 8) / 256), a.Hq, a.B), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace bpt
