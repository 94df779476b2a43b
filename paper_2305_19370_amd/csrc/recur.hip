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
// and the waves of a workgroup join theirs. States every 64 steps are kept for the backward, which rebuilds those between: y is
// not read again, and a bf16 y costs the gradients nothing.
//
// Every chunk of steps is a workgroup: it reads its steps, makes its (A, B) known, learns the state before it from those of up to 15
// chunks before it and the state before those, and goes on, so that elements are read once whatever the split. A word
// that is made known holds its number and a mark in 64 bits, written and read at once: no fence is needed. Workgroups
// draw their chunks from a counter, in order: whatever a workgroup waits for, a workgroup that has started before it gives without waiting
// for later ones, so every wait ends. States join in the order of the steps, always the same.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace bpt {

namespace {

constexpr int kLanes = kRecurCh / 4;                 // threads of a wave side by side on the channels
constexpr int kTs = 64 / kLanes;                     // and behind one another on the steps
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr int kFwdWaves = 8, kBwdWaves = 4;          // of a workgroup

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
// sigma(g) and sigma(-g), both to a few units of their last place; far below 0, where e is infinite, both 0: all that the second
// one multiplies has the first as a factor
BPT_DEV void sigma_both(float g, float& s, float& rest) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * g);
  s = __builtin_amdgcn_rcpf(1.0f + e);
  rest = s * fminf(e, 3.0e38f);                        // not 0 times infinity; a NaN stays one in s
}
// 1 - a^2 for a = 2^l2, l2 <= 0: where a^2 > 15/16 the series of 1 - e^w, w = 2 ln(2) l2, whose next term is under 2^-29 of it;
// a^2 carries 2^-22 of 1, so the difference is good to 2^-18 where the series ends
BPT_DEV float one_minus_a2(float a, float l2) {
  constexpr float c = 2.0f * kLn2;
  const float series = l2 * fmaf(l2, fmaf(l2, fmaf(l2, fmaf(l2, -c * c * c * c * c / 120.0f, -c * c * c * c / 24.0f), -c * c * c / 6.0f),
                                          -c * c / 2.0f), -c);
  return l2 > -0.0625f / c ? series : fmaf(-a, a, 1.0f);
}

// Keeps the compiler from forming values later, where they are used: it would hold what they are formed from, in more registers
BPT_DEV void formed(float& x, float& y, float& z) { asm volatile("" : "+v"(x), "+v"(y), "+v"(z)); }
// A load is over: what it read may be overwritten (hT may be h0, dh0 may be dhT)
BPT_DEV void loaded(float& x) { asm volatile("" : "+v"(x) : : "memory"); }

// value of the thread `o` lanes before this one
BPT_DEV float up(float v, int o) { return __shfl_up(v, (unsigned)o, 64); }

// A number and its mark, made known to (learned from) other workgroups
typedef unsigned long long Word;
BPT_DEV void tell(Word* p, float v) {
  __hip_atomic_store(p, (Word)1 << 32 | __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
BPT_DEV Word look(const Word* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
BPT_DEV bool known(Word w) { return (w >> 32) != 0; }
BPT_DEV float number(Word w) { return __uint_as_float((uint32_t)w); }

// What chunk `at` of a chain (of one sequence and 64 channels) learns from those before it, a channel per lane: wave w of NW joins 16 / NW
// chunks of its group as far as they lie before it; wave 0 also takes the state before the group (start: before the chain).
constexpr int kGroup = 16;
constexpr int kTries = 1 << 24;        // some ten seconds; what is not known by then becomes NaN
template <int NW>
BPT_DEV void learn(const Word* runs, const Word* groups, int lane, int wave, int at, float start, float& a, float& b, float& state) {
  constexpr int C = kGroup / NW;                       // chunks of a wave
  const int first = at - at % kGroup + C * wave, before = min(at - first, C);
  a = 1.0f;
  b = 0.0f;
  state = start;
  const bool ask = wave == 0 && at >= kGroup;
  if (before <= 0 && !ask) return;
  const Word* g = groups + (int64_t)(at / kGroup - 1) * 64 + lane;
  Word wa[C], wb[C], ws = (Word)1 << 32;
  bool all = false;
  for (int tries = 0; !all && tries < kTries; ++tries) {
    all = true;
    if (ask) ws = look(g);
#pragma unroll
    for (int k = 0; k < C; ++k)
      if (k < before) {
        const Word* p = runs + (int64_t)(first + k) * 128 + lane;
        wa[k] = look(p);
        wb[k] = look(p + 64);
      }
    all = known(ws);
#pragma unroll
    for (int k = 0; k < C; ++k)
      if (k < before) all = all && known(wa[k]) && known(wb[k]);
    all = __all(all);
    if (!all) __builtin_amdgcn_s_sleep(1);
  }
#pragma unroll
  for (int k = 0; k < C; ++k)
    if (k < before) {
      b = fmaf(number(wa[k]), b, number(wb[k]));
      a *= number(wa[k]);
    }
  if (ask) state = number(ws);
  if (!all) b = __builtin_nanf("");
}

// A tensor's rows of one chunk: a base that is the same for all threads and 32-bit offsets (strides are under 2^21 elements)
template <typename T>
struct Rows {
  const char* base;
  uint32_t st, col;                    // bytes
  BPT_DEV Rows(const void* t, int64_t sb, int64_t stride, int b, int64_t first, int ch)
      : base((const char*)t + (b * sb + first * stride) * (int64_t)sizeof(T)), st((uint32_t)stride * sizeof(T)), col((uint32_t)ch * sizeof(T)) {}
  BPT_DEV T* at(int row) const { return (T*)(base + (uint32_t)(row * st + col)); }
};

BPT_DEV int64_t steps_of(const RecurArgs& p, int b) {
  return p.lens ? min(max((int64_t)p.lens[b], (int64_t)0), p.S) : p.S;
}

}  // namespace

// ------------------------------------------------------------------ forward
// Steps [chunk L, chunk L + L), L = waves * kTs * M. Steps behind a sequence's length leave the state as it is (a = 1, no
// input), whatever their elements hold; their y is 0.
//
// 256 steps of 64 channels (fp32: 128), two workgroups on a CU. Bound by HBM with the vector units more than half busy (33
// instructions and 6 of them exponentials, reciprocals or roots an element): 96000 steps of width 1024, bf16 177 us, 4.4 TB/s; fp32
// 163840 steps 480 us, 5.6 TB/s. Chunks of 128 steps with 4 waves of 168 registers 200; a workgroup that takes chunk after
// chunk, the next one's elements under way, 239; one state that goes from group to group of 256 chunks 205; halves of a
// chunk's threads in loops without selects 195.
template <typename T, int M, bool CHAIN>
__global__ __launch_bounds__(64 * kFwdWaves, 4) void recur_fwd_kernel(RecurArgs p) {
  __shared__ __attribute__((aligned(16))) float sa[kFwdWaves][kRecurCh], sb[kFwdWaves][kRecurCh], sh[kFwdWaves][kRecurCh];
  __shared__ float fa[kFwdWaves][kRecurCh], fb[kFwdWaves][kRecurCh];
  __shared__ uint32_t drawn;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int cl = lane % kLanes, ts = lane / kLanes;
  const int L = nw * kTs * M;
  uint32_t bc = blockIdx.x;                            // sequence and channels
  int64_t chunk = 0;                                   // the only one, unless CHAIN
  if constexpr (CHAIN) {
    if (tid == 0) drawn = atomicAdd(p.counter, 1u);
    __syncthreads();
    const uint32_t chains = (uint32_t)(p.B * p.nct);
    const uint32_t at = __builtin_amdgcn_readfirstlane(drawn);
    bc = at % chains;
    chunk = at / chains;
  }
  const int b = bc / p.nct, ct = bc % p.nct;
  const int ch = ct * kRecurCh + 4 * cl;               // this thread's channels
  const int chr = min(ch, p.D - 4);                    // those it reads: the last ones instead of none
  const int cw = ct * kRecurCh + lane, cwr = min(cw, p.D - 1);   // where a lane is one channel
  const int row0 = (wave * kTs + ts) * M;
  const int64_t n = steps_of(p, b), first = chunk * L;
  float k2[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k2[e] = CHAIN ? p.k2[chr + e] : decay2(p.lam[chr + e], p.c);
  float state = wave == 0 && p.h0 ? p.h0[(int64_t)b * p.D + cwr] : 0.0f;

  const Rows<T> x(p.x, p.x_sb, p.x_st, b, first, chr), gr(p.r, p.r_sb, p.r_st, b, first, chr), gi(p.i, p.i_sb, p.i_st, b, first, chr);
  const int have = (int)min(max(n - first, (int64_t)0), (int64_t)L);   // steps of the chunk that exist
  Raw4<T> rx[M], rr[M], ri[M];
#pragma unroll
  for (int j = 0; j < M; ++j) {
    const int t = max(min(row0 + j, have - 1), 0);
    rx[j].load(x.at(t));
    rr[j].load(gr.at(t));
    ri[j].load(gi.at(t));
  }
  float a[M][4], u[M][4], A[4] = {1, 1, 1, 1}, B[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < M; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float l2 = k2[e] * sigma(rr[j][e]);
      const float al = __builtin_amdgcn_exp2f(l2);
      const float m = __builtin_amdgcn_sqrtf(one_minus_a2(al, l2));
      const bool live = row0 + j < have;
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
  loaded(state);
  __syncthreads();
  if constexpr (CHAIN) {
    Word *runs = p.runs + (int64_t)bc * p.nchunks * 128, *groups = p.groups + (int64_t)bc * p.ngroups * 64;
    const int at = (int)chunk, last = (int)p.nchunks - 1;
    float At = 1.0f, Bt = 0.0f;
    if (wave == 0) {
      for (int w = 0; w < kFwdWaves; ++w) {
        Bt = fmaf(sa[w][lane], Bt, sb[w][lane]);
        At *= sa[w][lane];
      }
      if (at < last && (at + 1) % kGroup) {
        tell(runs + (int64_t)at * 128 + lane, At);
        tell(runs + (int64_t)at * 128 + 64 + lane, Bt);
      }
    }
    learn<kFwdWaves>(runs, groups, lane, wave, at, state, fa[wave][lane], fb[wave][lane], state);
    __syncthreads();
    if (wave == 0) {
      for (int w = 0; w < kFwdWaves; ++w) state = fmaf(fa[w][lane], state, fb[w][lane]);
      if (at < last && (at + 1) % kGroup == 0) tell(groups + (int64_t)(at / kGroup) * 64 + lane, fmaf(At, state, Bt));
    }
  }
  if (wave == 0) {
    for (int w = 0; w < nw; ++w) {
      sh[w][lane] = state;
      const int64_t t = first + (int64_t)w * kTs * M;
      if (p.saved && t % kRecurKeep == 0 && t > 0 && t < p.S && cw < p.D)
        p.saved[((int64_t)b * ((p.S - 1) / kRecurKeep) + t / kRecurKeep - 1) * p.D + cw] = state;
      state = fmaf(sa[w][lane], state, sb[w][lane]);
    }
    if (p.hT && cw < p.D && chunk == p.nchunks - 1) p.hT[(int64_t)b * p.D + cw] = state;
  }
  __syncthreads();
  float h[4];
  {
    const f32x4 hw = *(const f32x4*)&sh[wave][4 * cl];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = fmaf(Ax[e], hw[e], Bx[e]);
  }
  const Rows<T> y(p.y, p.y_sb, p.y_st, b, first, ch);
#pragma unroll
  for (int j = 0; j < M; ++j) {
    float out[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      h[e] = fmaf(a[j][e], h[e], u[j][e]);
      out[e] = row0 + j < have ? h[e] : 0.0f;
    }
    if (first + row0 + j < p.S && ch < p.D) store4(y.at(row0 + j), out);
  }
}

// Few steps (new tokens of many sequences): a thread walks along the steps of four channels, and over a few sequences, for which
// it forms the channels' decay once. Bound by the launch and one access there and back for a handful of
// sequences, by the copy for many.
template <typename T>
__global__ __launch_bounds__(64) void recur_few_kernel(RecurArgs p, int per) {
  const int ch = blockIdx.x * 256 + 4 * (int)threadIdx.x;
  if (ch >= p.D) return;
  float k2[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k2[e] = decay2(p.lam[ch + e], p.c);
  const int b0 = blockIdx.y * per, b1 = min(b0 + per, p.B);
  for (int b = b0; b < b1; ++b) {
    const int n = (int)steps_of(p, b);
    f32x4 h = {0, 0, 0, 0};
    if (p.h0) h = *(const f32x4*)(p.h0 + (int64_t)b * p.D + ch);
    for (int t = 0; t < (int)p.S; ++t) {
      Raw4<T> rx, rr, ri;
      rx.load((const T*)p.x + b * p.x_sb + t * p.x_st + ch);
      rr.load((const T*)p.r + b * p.r_sb + t * p.r_st + ch);
      ri.load((const T*)p.i + b * p.i_sb + t * p.i_st + ch);
      float out[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float l2 = k2[e] * sigma(rr[e]), a = __builtin_amdgcn_exp2f(l2);
        const float m = __builtin_amdgcn_sqrtf(one_minus_a2(a, l2));
        const float next = fmaf(a, h[e], m * (sigma(ri[e]) * rx[e]));
        h[e] = t < n ? next : h[e];
        out[e] = t < n ? next : 0.0f;
      }
      store4((T*)p.y + b * p.y_sb + t * p.y_st + ch, out);
    }
    if (p.hT) *(f32x4*)(p.hT + (int64_t)b * p.D + ch) = h;
  }
}

// ------------------------------------------------------------------ backward
// The chunks of 64 steps from the last one down; the states within one from the one kept before it.
//
// A thread's 16 elements take five registers each between the two passes over them and 8 bytes of LDS, three workgroups of four
// waves on a CU. Bound by that: half of the time the vector units are busy (65 instructions an element), elements under way for
// 70 % of HBM's rate. 96000 steps of width 1024, bf16 365 us, 3.8 TB/s; fp32 163840 steps 985 us, 4.8 TB/s. Runs joined by
// lane exchanges instead of through LDS 372; 8 waves with half as many elements a thread 407; with selects for
// steps that do not exist in whole chunks too 408.
template <typename T, int M, bool CHAIN>
__global__ __launch_bounds__(64 * kBwdWaves, sizeof(T) == 4 ? 2 : 3) void recur_bwd_kernel(RecurArgs p) {
  extern __shared__ __attribute__((aligned(16))) f32x4 keep[];   // per thread and step: factors of d in dx and di
  __shared__ uint32_t drawn;
  __shared__ __attribute__((aligned(16))) float run[kBwdWaves][3][kTs][kRecurCh];   // (A, B) and E of the threads' runs; h before, e behind
  __shared__ float sa[kBwdWaves][kRecurCh], sb[kBwdWaves][kRecurCh], se[kBwdWaves][kRecurCh];
  __shared__ float sw[kBwdWaves][kRecurCh], fa[kBwdWaves][kRecurCh], fb[kBwdWaves][kRecurCh], fs[kRecurCh];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int cl = lane % kLanes, ts = lane / kLanes;
  const int L = nw * kTs * M;                          // kRecurKeep, unless there is one chunk
  uint32_t bc = blockIdx.x;
  int64_t chunk = 0;
  if constexpr (CHAIN) {
    if (tid == 0) drawn = atomicAdd(p.counter, 1u);
    __syncthreads();
    const uint32_t chains = (uint32_t)(p.B * p.nct);
    const uint32_t at = __builtin_amdgcn_readfirstlane(drawn);
    bc = at % chains;
    chunk = p.nchunks - 1 - at / chains;
  }
  const int b = bc / p.nct, ct = bc % p.nct;
  const int ch = ct * kRecurCh + 4 * cl, chr = min(ch, p.D - 4);
  const int cw = ct * kRecurCh + lane, cwr = min(cw, p.D - 1);
  const int row0 = (wave * kTs + ts) * M;
  const int64_t n = steps_of(p, b), row = (int64_t)b * p.D + cwr, kept = (p.S - 1) / kRecurKeep;
  float k2[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k2[e] = CHAIN ? p.k2[chr + e] : decay2(p.lam[chr + e], p.c);

  float back = p.dhT ? p.dhT[row] : 0.0f;              // e of the step behind the chunk

  const int64_t first = chunk * L;
  const Rows<T> x(p.x, p.x_sb, p.x_st, b, first, chr), gr(p.r, p.r_sb, p.r_st, b, first, chr), gi(p.i, p.i_sb, p.i_st, b, first, chr),
      dy(p.dy, p.y_sb, p.y_st, b, first, chr);
  const int have = (int)min(max(n - first, (int64_t)0), (int64_t)L);
  Raw4<T> rx[M], rr[M], ri[M], ry[M];
#pragma unroll
  for (int j = 0; j < M; ++j) {
    const int t = max(min(row0 + j, have - 1), 0);
    rr[j].load(gr.at(t));
    ri[j].load(gi.at(t));
    rx[j].load(x.at(t));
    ry[j].load(dy.at(t));
  }
  // per step: a, the state before it, and the factors of d (and of d h) in the results
  float a[M][4], h[M][4], l[M][4], q[M][4], r1[M][4];
  float A[4], B[4], E[4];
  auto form = [&](auto whole) {
#pragma unroll
    for (int j = 0; j < M; ++j) {
      float fx[4], fi[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float r, i, i1;
        sigma_both(rr[j][e], r, r1[j][e]);
        sigma_both(ri[j][e], i, i1);
        const float l2 = k2[e] * r, al = __builtin_amdgcn_exp2f(l2), s = one_minus_a2(al, l2);
        // 1 / m; an s below the normal numbers counts as 0 (m < 2^-63): l / m is smaller still
        const float im = s >= 1.17549435e-38f ? __builtin_amdgcn_rsqf(s) : 0.0f, v = i * rx[j][e] * im;
        a[j][e] = al;
        h[j][e] = s * v;                             // m u
        l[j][e] = kLn2 * l2 * al;                    // w = d (l a h - q)
        q[j][e] = al * (kLn2 * l2 * al) * v;
        fx[e] = s * im * i;
        fi[e] = h[j][e] * i1;
        if constexpr (!decltype(whole)::value) {
          const bool live = row0 + j < have;
          a[j][e] = live ? a[j][e] : 1.0f;
          h[j][e] = live ? h[j][e] : 0.0f;
        }
        B[e] = j ? fmaf(a[j][e], B[e], h[j][e]) : h[j][e];
        A[e] = j ? A[e] * a[j][e] : a[j][e];
      }
      store4((float*)(keep + (2 * j) * blockDim.x + tid), fx);
      store4((float*)(keep + (2 * j + 1) * blockDim.x + tid), fi);
#pragma unroll
      for (int e = 0; e < 4; ++e) formed(l[j][e], q[j][e], r1[j][e]);
    }
#pragma unroll
    for (int j = M - 1; j >= 0; --j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = decltype(whole)::value || row0 + j < have ? ry[j][e] : 0.0f;
        E[e] = a[j][e] * (j < M - 1 ? d + E[e] : d);
      }
  };
  if (have == L) form(std::true_type{});
  else form(std::false_type{});
  // a lane is a channel, as in the forward
  store4(&run[wave][0][ts][4 * cl], A);
  store4(&run[wave][1][ts][4 * cl], B);
  store4(&run[wave][2][ts][4 * cl], E);
  wave_sync();
  float Aw = 1.0f, Bw = 0.0f, Ew = 0.0f;
#pragma unroll
  for (int k = 0; k < kTs; ++k) {
    const float Ak = run[wave][0][k][lane];
    Bw = fmaf(Ak, Bw, run[wave][1][k][lane]);
    Aw *= Ak;
  }
#pragma unroll
  for (int k = kTs - 1; k >= 0; --k) Ew = fmaf(run[wave][0][k][lane], Ew, run[wave][2][k][lane]);
  sa[wave][lane] = Aw;
  sb[wave][lane] = Bw;
  se[wave][lane] = Ew;
  loaded(back);
  __syncthreads();
  float state = chunk > 0 ? p.saved[((int64_t)b * kept + chunk - 1) * p.D + cwr] : p.h0 ? p.h0[row] : 0.0f;
  float At = 1.0f, Et = 0.0f;
  if constexpr (CHAIN) {
    Word *runs = p.runs + (int64_t)bc * p.nchunks * 128, *groups = p.groups + (int64_t)bc * p.ngroups * 64;
    const int at = (int)(p.nchunks - 1 - chunk), last = (int)p.nchunks - 1;
    if (wave == 0) {
#pragma unroll
      for (int w = kBwdWaves - 1; w >= 0; --w) {
        Et = fmaf(sa[w][lane], Et, se[w][lane]);
        At *= sa[w][lane];
      }
      if (at < last && (at + 1) % kGroup) {
        tell(runs + (int64_t)at * 128 + lane, At);
        tell(runs + (int64_t)at * 128 + 64 + lane, Et);
      }
    }
    learn<kBwdWaves>(runs, groups, lane, wave, at, back, fa[wave][lane], fb[wave][lane], back);
    if (wave == 0) fs[lane] = back;
    __syncthreads();
    back = fs[lane];
#pragma unroll
    for (int w = 0; w < kBwdWaves; ++w) back = fmaf(fa[w][lane], back, fb[w][lane]);
    if (wave == 0 && at < last && (at + 1) % kGroup == 0) tell(groups + (int64_t)(at / kGroup) * 64 + lane, fmaf(At, back, Et));
  }
  for (int w = 0; w < wave; ++w) state = fmaf(sa[w][lane], state, sb[w][lane]);
  for (int w = nw - 1; w > wave; --w) back = fmaf(sa[w][lane], back, se[w][lane]);
#pragma unroll
  for (int k = 0; k < kTs; ++k) {
    const float Bk = run[wave][1][k][lane];
    run[wave][1][k][lane] = state;
    state = fmaf(run[wave][0][k][lane], state, Bk);
  }
#pragma unroll
  for (int k = kTs - 1; k >= 0; --k) {
    const float Ek = run[wave][2][k][lane];
    run[wave][2][k][lane] = back;
    back = fmaf(run[wave][0][k][lane], back, Ek);
  }
  if (wave == 0 && p.dh0 && cw < p.D && chunk == 0) p.dh0[row] = back;
  wave_sync();
  float hh[4], ee[4], ws[4] = {0, 0, 0, 0};
  {
    const f32x4 hw = *(const f32x4*)&run[wave][1][ts][4 * cl], ew = *(const f32x4*)&run[wave][2][ts][4 * cl];
#pragma unroll
    for (int e = 0; e < 4; ++e) hh[e] = hw[e], ee[e] = ew[e];
  }
  const Rows<T> dx(p.dx, p.x_sb, p.x_st, b, first, ch), dr(p.dr, p.r_sb, p.r_st, b, first, ch), di(p.di, p.i_sb, p.i_st, b, first, ch);
  auto give = [&](auto whole) {
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
      const f32x4 fx = keep[(2 * j) * blockDim.x + tid], fi = keep[(2 * j + 1) * blockDim.x + tid];
      const bool live = decltype(whole)::value || row0 + j < have;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float g = (live ? ry[j][e] : 0.0f) + ee[e], w = live ? g * fmaf(l[j][e], h[j][e], -q[j][e]) : 0.0f;
        ws[e] += w;
        og[e] = live ? w * r1[j][e] : 0.0f;
        ox[e] = live ? g * fx[e] : 0.0f;
        oi[e] = live ? g * fi[e] : 0.0f;
        ee[e] = a[j][e] * g;
      }
      if ((decltype(whole)::value || first + row0 + j < p.S) && ch < p.D) {
        store4(dx.at(row0 + j), ox);
        store4(dr.at(row0 + j), og);
        store4(di.at(row0 + j), oi);
      }
    }
  };
  if (have == L) give(std::true_type{});
  else give(std::false_type{});
  // sum of w over the chunk, in the order of its runs
  store4(&run[wave][2][ts][4 * cl], ws);
  wave_sync();
  float part = 0.0f;
#pragma unroll
  for (int k = 0; k < kTs; ++k) part += run[wave][2][k][lane];
  sw[wave][lane] = part;
  __syncthreads();
  if (wave == 0 && cw < p.D) {
    float sum = 0.0f;
    for (int w = 0; w < nw; ++w) sum += sw[w][lane];
    p.part[((int64_t)b * p.nchunks + chunk) * p.D + cw] = sum * (CHAIN ? p.ratio[cw] : sigma_over_softplus(p.lam[cw]));
  }
}

// Before the chained kernels: nothing is known yet; per channel log2 a of a fully open gate, and what dlambda's sum is multiplied by
__global__ __launch_bounds__(256) void recur_start_kernel(RecurArgs p, int64_t words) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  if (i == 0) *p.counter = 0;
  if (i < p.D) {
    p.k2[i] = decay2(p.lam[i], p.c);
    p.ratio[i] = sigma_over_softplus(p.lam[i]);
  }
  for (int64_t k = i; k < words / 2; k += step) ((u32x4*)p.runs)[k] = u32x4{0, 0, 0, 0};
}

// dlambda from the chunks' sums, [rows, D], added in a fixed order: a workgroup's 256 runs of rows of 16 channels, 16 of them, then
// those by exchanges
__global__ __launch_bounds__(1024) void recur_dlam_kernel(const float* part, int64_t rows, int D, float* dlam) {
  __shared__ f32x4 s[256][4];
  const int q = threadIdx.x & 3, g = threadIdx.x >> 2, c = blockIdx.x * 16 + 4 * q;
  f32x4 sum = {0, 0, 0, 0};
  if (c < D) {
#pragma unroll 4
    for (int64_t i = g; i < rows; i += 256) sum += *(const f32x4*)(part + i * D + c);
  }
  s[g][q] = sum;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  sum = s[16 * g][q];
#pragma unroll
  for (int k = 1; k < 16; ++k) sum += s[16 * g + k][q];
#pragma unroll
  for (int o = 4; o < 64; o *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], o, 64);
  if (g == 0 && c < D) *(f32x4*)(dlam + c) = sum;
}

// ------------------------------------------------------------------ launchers
namespace {
constexpr int kFwdM = 8, kBwdM = 4;                  // steps of a thread
constexpr int kFewSteps = 8;           // of the forward in which a thread walks alone

int64_t words_of(const RecurArgs& p) { return (int64_t)p.B * p.nct * (p.nchunks * 128 + p.ngroups * 64); }

// chunks, their number of waves, and whether they are chained
int plan(RecurArgs& p, Dt t, bool backward) {
  const int per = kTs * (backward ? kBwdM : t == F32 ? kFwdM / 2 : kFwdM);
  const int nw = (int)std::min<int64_t>(backward ? kBwdWaves : kFwdWaves, (p.S + per - 1) / per);
  p.nct = (p.D + kRecurCh - 1) / kRecurCh;
  p.nchunks = (p.S + nw * per - 1) / (nw * per);
  p.ngroups = (p.nchunks + kGroup - 1) / kGroup;
  return nw;
}
bool chains(const RecurArgs& p) { return p.nchunks > 1; }

hipError_t start(RecurArgs& p, hipStream_t s) {
  p.runs = (unsigned long long*)p.chain;
  p.groups = p.runs + (int64_t)p.B * p.nct * p.nchunks * 128;
  p.k2 = (float*)(p.runs + words_of(p));
  p.ratio = p.k2 + p.D;
  p.counter = (uint32_t*)(p.ratio + p.D);
  const int64_t blocks = std::max<int64_t>((p.D + 255) / 256, std::min<int64_t>((words_of(p) + 511) / 512, 2048));
  hipLaunchKernelGGL(recur_start_kernel, dim3((unsigned)blocks), dim3(256), 0, s, p, words_of(p));
  return hipGetLastError();
}
}  // namespace

int64_t recur_bwd_chunks(int64_t S) { return (S + kRecurKeep - 1) / kRecurKeep; }

int64_t recur_chain_bytes(Dt t, RecurArgs p, int backward) {
  plan(p, t, backward);
  return chains(p) ? words_of(p) * 8 + (2 * (int64_t)p.D + 4) * 4 : 0;
}

hipError_t recur_fwd(Dt t, RecurArgs p, hipStream_t s) {
  if (p.S <= kFewSteps) {
    const int gx = (p.D + 255) / 256, per = std::max((int)(((int64_t)p.B * gx + 8191) / 8192), (p.B + 65534) / 65535);
    const dim3 grid((unsigned)gx, (unsigned)((p.B + per - 1) / per));
    if (t == F32) hipLaunchKernelGGL((recur_few_kernel<float>), grid, dim3(64), 0, s, p, per);
    else hipLaunchKernelGGL((recur_few_kernel<bf16>), grid, dim3(64), 0, s, p, per);
    return hipGetLastError();
  }
  const int nw = plan(p, t, false);
  const bool chain = chains(p);
  if (chain) {
    const hipError_t e = start(p, s);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)(p.B * p.nct * (chain ? p.nchunks : 1))), block((unsigned)(64 * nw));
  if (t == F32) {
    if (chain) hipLaunchKernelGGL((recur_fwd_kernel<float, kFwdM / 2, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((recur_fwd_kernel<float, kFwdM / 2, false>), grid, block, 0, s, p);
  } else {
    if (chain) hipLaunchKernelGGL((recur_fwd_kernel<bf16, kFwdM, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((recur_fwd_kernel<bf16, kFwdM, false>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

namespace {
template <typename T, bool CHAIN>
hipError_t launch_bwd(const RecurArgs& p, int nw, hipStream_t s) {
  // with what the kernel declares under 64 KiB of LDS, which a launch may have as it is
  static_assert(2 * kBwdM * 64 * kBwdWaves * 16 <= 32768, "keep, beside 19 KiB");
  hipLaunchKernelGGL((recur_bwd_kernel<T, kBwdM, CHAIN>), dim3((unsigned)(p.B * p.nct * (CHAIN ? p.nchunks : 1))), dim3((unsigned)(64 * nw)),
                     2 * kBwdM * 64 * nw * 16, s, p);
  return hipGetLastError();
}
}  // namespace

hipError_t recur_bwd(Dt t, RecurArgs p, hipStream_t s) {
  static_assert(kBwdWaves * kTs * kBwdM == kRecurKeep, "a chunk starts at a state that was kept");
  const int nw = plan(p, t, true);
  const bool chain = chains(p);
  if (chain) {
    const hipError_t e = start(p, s);
    if (e != hipSuccess) return e;
  }
  if (t == F32) return chain ? launch_bwd<float, true>(p, nw, s) : launch_bwd<float, false>(p, nw, s);
  return chain ? launch_bwd<bf16, true>(p, nw, s) : launch_bwd<bf16, false>(p, nw, s);
}

// Up to 2048 rows in one launch, more by col_sum's two: 256 rows of 2048 4.7 us (two launches 9.5 and a gap), 1500 of 1024 7.6 (9.6)
int64_t recur_dlam_floats(int64_t rows, int64_t D) { return rows > 2048 ? std::min<int64_t>(rows / 16, 512) * D : 0; }
hipError_t recur_dlam(const RecurArgs& p, float* dlam, float* partial, hipStream_t s) {
  const int64_t rows = p.B * recur_bwd_chunks(p.S), n = recur_dlam_floats(rows, p.D);
  if (n > 0) return col_sum(F32, p.part, p.D, rows, p.D, dlam, partial, n, s);
  hipLaunchKernelGGL(recur_dlam_kernel, dim3((unsigned)((p.D + 15) / 16)), dim3(1024), 0, s, p.part, rows, p.D, dlam);
  return hipGetLastError();
}

}  // namespace bpt
