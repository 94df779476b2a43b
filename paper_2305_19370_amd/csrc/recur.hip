// A gated linear recurrence along the sequence, per channel:
//   r = sigma(gr), i = sigma(gi), l = -c softplus(lambda) r, a = e^l, m = sqrt(1 - a^2), u = i x,
//   h_t = a_t h_{t-1} + m_t u_t.
// Its gradient, e_t the gradient that reaches h_{t-1} through step t: d_t = dy_t + e_{t+1}, e_t = a_t d_t, and with
// w_t = l_t d_t (a_t h_{t-1} - a_t^2 / m_t u_t) (d loss / d log l_t):
//   dgr = w (1 - r), dlambda = sigma(lambda) / softplus(lambda) sum_t w, dx = d m i, dgi = d m u (1 - i), dh0 = e_0.
// l / m tends to 0 with l, so a gate that is closed, whose m is 0, divides by nothing.
//
// A run of steps maps h to A h + B (A the product of its a); runs join as (A1, B1), (A2, B2) -> (A1 A2, A2 B1 + B2), and the
// gradient's e does the same from the right. A thread takes M steps of four channels, the four threads of a wave that share the channels
// and the waves of a workgroup join theirs, and a workgroup walks along the sequence, its state in registers. States every
// 128 steps are kept for the backward, which rebuilds those between: y is not read again, and a bf16 y
// costs the gradients nothing.
#include <algorithm>

#include "common.h"
#include "internal.h"

namespace bpt {

namespace {

constexpr int kLanes = kRecurCh / 4;                 // threads of a wave side by side on the channels
constexpr int kTs = 64 / kLanes;                     // and behind one another on the steps
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr int kMaxWaves = 8;

// four elements as they are in memory, and as numbers
template <typename T> struct Raw4;
template <> struct Raw4<bf16> {
  u32x2 v;
  BPT_DEV void load(const bf16* p) { v = *(const u32x2*)p; }
  BPT_DEV float operator[](int e) const {
    const uint32_t w = v[e >> 1];
    return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
  }
};
template <> struct Raw4<float> {
  f32x4 v;
  BPT_DEV void load(const float* p) { v = *(const f32x4*)p; }
  BPT_DEV float operator[](int e) const { return v[e]; }
};
BPT_DEV void store4(float* p, const float* v) { *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]}; }
BPT_DEV void store4(bf16* p, const float* v) {
  bf16x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = (bf16)v[e];
  *(bf16x4*)p = x;
}

// softplus(x) log2(e) c, negative: the base-2 logarithm of a is this times r. And sigma(x) / softplus(x), which tends
// to 1 for x -> -inf.
BPT_DEV float softplus(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))); }
BPT_DEV float decay2(float lam, float c) { return -c * softplus(lam) * kLog2e; }
BPT_DEV float sigma_over_softplus(float lam) {
  if (lam < -20.0f) return 1.0f;                     // 1 - e^lam / 2
  return 1.0f / (1.0f + expf(-lam)) / softplus(lam);
}

BPT_DEV float sigma(float g) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * g)); }
// sigma(g) and sigma(-g), both to a few units of their last place
BPT_DEV void sigma_both(float g, float& s, float& rest) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(g)), q = __builtin_amdgcn_rcpf(1.0f + e), p = e * q;
  s = g >= 0.0f ? q : p;
  rest = g >= 0.0f ? p : q;
}
// 1 - a^2 for a = e^l, w = 2 l <= 0: near 0 the series of -expm1, whose next term is under 2^-29 of it; a^2 carries 2^-22 of
// 1, so the difference is good to 2^-18 where the series ends
BPT_DEV float one_minus_a2(float a, float w) {
  const float series = -w * fmaf(w, fmaf(w, fmaf(w, fmaf(w, 1.0f / 120.0f, 1.0f / 24.0f), 1.0f / 6.0f), 0.5f), 1.0f);
  return w > -0.0625f ? series : fmaf(-a, a, 1.0f);
}

// value of the thread `o` lanes before (after) this one; kept where there is none
BPT_DEV float up(float v, int o) { return __shfl_up(v, (unsigned)o, 64); }
BPT_DEV float down(float v, int o) { return __shfl_down(v, (unsigned)o, 64); }

BPT_DEV int64_t steps_of(const RecurArgs& p, int b) {
  return p.lens ? min(max((int64_t)p.lens[b], (int64_t)0), p.S) : p.S;
}

}  // namespace

// ------------------------------------------------------------------ forward
// Steps [chunk L, chunk L + L), L = waves * kTs * M. Steps behind a sequence's length leave the state as it is (a = 1, no
// input), whatever their elements hold; their y is 0.
template <typename T, int M>
__global__ __launch_bounds__(64 * kMaxWaves) void recur_fwd_kernel(RecurArgs p) {
  __shared__ __attribute__((aligned(16))) float sa[kMaxWaves][kRecurCh], sb[kMaxWaves][kRecurCh], sh[kMaxWaves][kRecurCh];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nw = blockDim.x >> 6;
  const int cl = lane % kLanes, ts = lane / kLanes;
  const int L = nw * kTs * M;
  const int b = blockIdx.x / p.nct, ct = blockIdx.x % p.nct;
  const int ch = ct * kRecurCh + 4 * cl;               // this thread's channels
  const int chr = min(ch, p.D - 4);                    // those it reads: the last ones instead of none
  const int cw = ct * kRecurCh + lane, cwr = min(cw, p.D - 1);   // wave 0: a channel per lane
  const int64_t n = steps_of(p, b);
  const T *x = (const T*)p.x + b * p.x_sb + chr, *gr = (const T*)p.r + b * p.r_sb + chr, *gi = (const T*)p.i + b * p.i_sb + chr;
  T* y = (T*)p.y + b * p.y_sb + chr;
  float k2[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k2[e] = decay2(p.lam[chr + e], p.c);
  float state = wave == 0 && p.h0 ? p.h0[(int64_t)b * p.D + cwr] : 0.0f;

  for (int64_t chunk = 0; chunk < p.nchunks; ++chunk) {
    const int64_t t0 = chunk * L + (wave * kTs + ts) * M;
    Raw4<T> rx[M], rr[M], ri[M];
#pragma unroll
    for (int j = 0; j < M; ++j) {
      const int64_t t = min(t0 + j, max(n - 1, (int64_t)0));
      rx[j].load(x + t * p.x_st);
      rr[j].load(gr + t * p.r_st);
      ri[j].load(gi + t * p.i_st);
    }
    float a[M][4], u[M][4], A[4] = {1, 1, 1, 1}, B[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < M; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float l2 = k2[e] * sigma(rr[j][e]);
        const float al = __builtin_amdgcn_exp2f(l2);
        const float m = __builtin_amdgcn_sqrtf(one_minus_a2(al, 2.0f * kLn2 * l2));
        const bool live = t0 + j < n;
        a[j][e] = live ? al : 1.0f;
        u[j][e] = live ? m * (sigma(ri[j][e]) * rx[j][e]) : 0.0f;
        B[e] = fmaf(a[j][e], B[e], u[j][e]);
        A[e] *= a[j][e];
      }
    // the threads before this one in the wave, then the waves before this one
    float Ax[4], Bx[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int o = kLanes; o < 64; o *= 2) {
        const float A1 = up(A[e], o), B1 = up(B[e], o);
        if (lane >= o) {
          B[e] = fmaf(A[e], B1, B[e]);
          A[e] *= A1;
        }
      }
      Ax[e] = up(A[e], kLanes);
      Bx[e] = up(B[e], kLanes);
      if (ts == 0) Ax[e] = 1.0f, Bx[e] = 0.0f;
    }
    if (ts == kTs - 1) {
      store4(&sa[wave][4 * cl], A);
      store4(&sb[wave][4 * cl], B);
    }
    __syncthreads();
    if (wave == 0) {
      for (int w = 0; w < nw; ++w) {
        sh[w][lane] = state;
        const int64_t t = chunk * L + (int64_t)w * kTs * M;
        if (p.saved && t % kRecurKeep == 0 && t > 0 && t < p.S && cw < p.D)
          p.saved[((int64_t)b * ((p.S - 1) / kRecurKeep) + t / kRecurKeep - 1) * p.D + cw] = state;
        state = fmaf(sa[w][lane], state, sb[w][lane]);
      }
    }
    __syncthreads();
    float h[4];
    {
      const f32x4 hw = *(const f32x4*)&sh[wave][4 * cl];
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = fmaf(Ax[e], hw[e], Bx[e]);
    }
#pragma unroll
    for (int j = 0; j < M; ++j) {
      float out[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        h[e] = fmaf(a[j][e], h[e], u[j][e]);
        out[e] = t0 + j < n ? h[e] : 0.0f;
      }
      if (t0 + j < p.S && ch < p.D) store4(y + (t0 + j) * p.y_st, out);
    }
  }
  if (wave == 0 && p.hT && cw < p.D) p.hT[(int64_t)b * p.D + cw] = state;
}

// ------------------------------------------------------------------ backward
// The chunks from the last one down, e in registers. States within a chunk of 128 steps from the one kept before it.
template <typename T, int M>
__global__ __launch_bounds__(64 * kMaxWaves) void recur_bwd_kernel(RecurArgs p) {
  __shared__ __attribute__((aligned(16))) float sa[kMaxWaves][kRecurCh], sb[kMaxWaves][kRecurCh], se[kMaxWaves][kRecurCh];
  __shared__ __attribute__((aligned(16))) float sh[kMaxWaves][kRecurCh], sd[kMaxWaves][kRecurCh], sw[kMaxWaves][kRecurCh];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nw = blockDim.x >> 6;
  const int cl = lane % kLanes, ts = lane / kLanes;
  const int L = nw * kTs * M;                          // at most kRecurKeep
  const int b = blockIdx.x / p.nct, ct = blockIdx.x % p.nct;
  const int ch = ct * kRecurCh + 4 * cl, chr = min(ch, p.D - 4);
  const int cw = ct * kRecurCh + lane, cwr = min(cw, p.D - 1);
  const int64_t n = steps_of(p, b), row = (int64_t)b * p.D + cwr, kept = (p.S - 1) / kRecurKeep;
  const T *x = (const T*)p.x + b * p.x_sb + chr, *gr = (const T*)p.r + b * p.r_sb + chr, *gi = (const T*)p.i + b * p.i_sb + chr;
  const T* dy = (const T*)p.dy + b * p.y_sb + chr;
  T *dx = (T*)p.dx + b * p.x_sb + chr, *dr = (T*)p.dr + b * p.r_sb + chr, *di = (T*)p.di + b * p.i_sb + chr;
  float k2[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k2[e] = decay2(p.lam[chr + e], p.c);
  float back = wave == 0 && p.dhT ? p.dhT[row] : 0.0f;   // e of the step behind the chunk

  for (int64_t chunk = p.nchunks - 1; chunk >= 0; --chunk) {
    const int64_t t0 = chunk * L + (wave * kTs + ts) * M;
    Raw4<T> rx[M], rr[M], ri[M], ry[M];
#pragma unroll
    for (int j = 0; j < M; ++j) {
      const int64_t t = min(t0 + j, max(n - 1, (int64_t)0));
      rr[j].load(gr + t * p.r_st);
      ri[j].load(gi + t * p.i_st);
      rx[j].load(x + t * p.x_st);
      ry[j].load(dy + t * p.y_st);
    }
    float state = 0.0f;
    if (wave == 0) state = chunk > 0 ? p.saved[((int64_t)b * kept + chunk - 1) * p.D + cwr] : p.h0 ? p.h0[row] : 0.0f;
    // per step: a, the state before it, dy, and the factors of d (and of d h) in the results
    float a[M][4], h[M][4], d[M][4], l[M][4], q[M][4], r1[M][4], fx[M][4], fi[M][4];
    float A[4] = {1, 1, 1, 1}, B[4] = {0, 0, 0, 0}, E[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < M; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool live = t0 + j < n;
        float r, i, i1;
        sigma_both(rr[j][e], r, r1[j][e]);
        sigma_both(ri[j][e], i, i1);
        const float l2 = k2[e] * r, al = __builtin_amdgcn_exp2f(l2), s = one_minus_a2(al, 2.0f * kLn2 * l2);
        // 1 / m; an s below the normal numbers counts as 0 (m < 2^-63): l / m is smaller still
        const float im = s >= 1.17549435e-38f ? __builtin_amdgcn_rsqf(s) : 0.0f, m = s * im, xe = rx[j][e], u = i * xe;
        l[j][e] = live ? kLn2 * l2 * al : 0.0f;                       // w = d (l a h - q)
        q[j][e] = live ? al * al * u * (kLn2 * l2 * im) : 0.0f;
        fx[j][e] = live ? m * i : 0.0f;
        fi[j][e] = live ? m * u * i1 : 0.0f;
        a[j][e] = live ? al : 1.0f;
        h[j][e] = live ? m * u : 0.0f;
        d[j][e] = live ? ry[j][e] : 0.0f;
        if (!live) r1[j][e] = 0.0f;
        B[e] = fmaf(a[j][e], B[e], h[j][e]);
        A[e] *= a[j][e];
      }
#pragma unroll
    for (int j = M - 1; j >= 0; --j)
#pragma unroll
      for (int e = 0; e < 4; ++e) E[e] = a[j][e] * (d[j][e] + E[e]);
    float Ax[4], Bx[4], Az[4], Ez[4];                  // the threads of the wave before this one, and behind it
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float Ad = A[e];
#pragma unroll
      for (int o = kLanes; o < 64; o *= 2) {
        const float A1 = up(A[e], o), B1 = up(B[e], o), A2 = down(Ad, o), E2 = down(E[e], o);
        if (lane >= o) {
          B[e] = fmaf(A[e], B1, B[e]);
          A[e] *= A1;
        }
        if (lane < 64 - o) {
          E[e] = fmaf(Ad, E2, E[e]);
          Ad *= A2;
        }
      }
      Ax[e] = up(A[e], kLanes);
      Bx[e] = up(B[e], kLanes);
      Az[e] = down(Ad, kLanes);
      Ez[e] = down(E[e], kLanes);
      if (ts == 0) Ax[e] = 1.0f, Bx[e] = 0.0f;
      if (ts == kTs - 1) Az[e] = 1.0f, Ez[e] = 0.0f;
    }
    if (ts == kTs - 1) {
      store4(&sa[wave][4 * cl], A);
      store4(&sb[wave][4 * cl], B);
    }
    if (ts == 0) store4(&se[wave][4 * cl], E);
    __syncthreads();
    if (wave == 0) {
      for (int w = 0; w < nw; ++w) {
        sh[w][lane] = state;
        state = fmaf(sa[w][lane], state, sb[w][lane]);
      }
      for (int w = nw - 1; w >= 0; --w) {
        sd[w][lane] = back;
        back = fmaf(sa[w][lane], back, se[w][lane]);
      }
    }
    __syncthreads();
    float hh[4], ee[4], ws[4] = {0, 0, 0, 0};
    {
      const f32x4 hw = *(const f32x4*)&sh[wave][4 * cl], ew = *(const f32x4*)&sd[wave][4 * cl];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        hh[e] = fmaf(Ax[e], hw[e], Bx[e]);
        ee[e] = fmaf(Az[e], ew[e], Ez[e]);
      }
    }
#pragma unroll
    for (int j = 0; j < M; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float before = hh[e];
        hh[e] = fmaf(a[j][e], hh[e], h[j][e]);
        h[j][e] = before;
      }
#pragma unroll
    for (int j = M - 1; j >= 0; --j) {
      float ox[4], og[4], oi[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float g = d[j][e] + ee[e], w = t0 + j < n ? g * (l[j][e] * h[j][e] - q[j][e]) : 0.0f;
        ws[e] += w;
        og[e] = w * r1[j][e];
        ox[e] = t0 + j < n ? g * fx[j][e] : 0.0f;
        oi[e] = t0 + j < n ? g * fi[j][e] : 0.0f;
        ee[e] = a[j][e] * g;
      }
      if (t0 + j < p.S && ch < p.D) {
        store4(dx + (t0 + j) * p.x_st, ox);
        store4(dr + (t0 + j) * p.r_st, og);
        store4(di + (t0 + j) * p.i_st, oi);
      }
    }
    // sum of w over the chunk, in the order of the steps' threads and waves
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int o = kLanes; o < 64; o *= 2) ws[e] += __shfl_xor(ws[e], o, 64);
    }
    if (ts == 0) store4(&sw[wave][4 * cl], ws);
    __syncthreads();
    if (wave == 0 && cw < p.D) {
      float sum = 0.0f;
      for (int w = 0; w < nw; ++w) sum += sw[w][lane];
      p.part[((int64_t)b * p.nchunks + chunk) * p.D + cw] = sum;
    }
  }
  if (wave == 0 && p.dh0 && cw < p.D) p.dh0[row] = back;
}

// dlambda from the sums of w of the chunks, [rows, D], added in a fixed order: 16 runs of rows, then those
__global__ __launch_bounds__(1024) void recur_dlam_kernel(const float* part, int64_t rows, int D, const float* lam, float* dlam) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (c < D)
    for (int64_t i = g; i < rows; i += 16) sum += part[i * D + c];
  s[g][lane] = sum;
  __syncthreads();
  if (g == 0 && c < D) {
    for (int k = 1; k < 16; ++k) sum += s[k][lane];
    dlam[c] = sum * sigma_over_softplus(lam[c]);
  }
}

// ------------------------------------------------------------------ launchers
namespace {
constexpr int kFwdM = 8, kBwdM = 4;
int waves_for(int64_t S, int per) { return (int)std::min<int64_t>(kMaxWaves, (S + per - 1) / per); }
}  // namespace

int64_t recur_bwd_chunks(int64_t S) { return (S + kRecurKeep - 1) / kRecurKeep; }

hipError_t recur_fwd(Dt t, RecurArgs p, hipStream_t s) {
  const int nw = waves_for(p.S, kTs * kFwdM);
  p.nct = (p.D + kRecurCh - 1) / kRecurCh;
  p.nchunks = (p.S + nw * kTs * kFwdM - 1) / (nw * kTs * kFwdM);
  const dim3 grid((unsigned)(p.B * p.nct)), block((unsigned)(64 * nw));
  if (t == F32) hipLaunchKernelGGL((recur_fwd_kernel<float, kFwdM>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((recur_fwd_kernel<bf16, kFwdM>), grid, block, 0, s, p);
  return hipGetLastError();
}

hipError_t recur_bwd(Dt t, RecurArgs p, hipStream_t s) {
  static_assert(kMaxWaves * kTs * kBwdM == kRecurKeep, "a chunk starts at a state that was kept");
  const int nw = waves_for(p.S, kTs * kBwdM);
  p.nct = (p.D + kRecurCh - 1) / kRecurCh;
  p.nchunks = recur_bwd_chunks(p.S);
  const dim3 grid((unsigned)(p.B * p.nct)), block((unsigned)(64 * nw));
  if (t == F32) hipLaunchKernelGGL((recur_bwd_kernel<float, kBwdM>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((recur_bwd_kernel<bf16, kBwdM>), grid, block, 0, s, p);
  return hipGetLastError();
}

hipError_t recur_dlam(const RecurArgs& p, float* dlam, hipStream_t s) {
  hipLaunchKernelGGL(recur_dlam_kernel, dim3((unsigned)((p.D + 63) / 64)), dim3(1024), 0, s, p.part,
                     p.B * recur_bwd_chunks(p.S), p.D, p.lam, dlam);
  return hipGetLastError();
}

}  // namespace bpt
