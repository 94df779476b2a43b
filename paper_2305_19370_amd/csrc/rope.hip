// Rotary positions: pair (a, b) of a head at position p becomes (c a - s b, s a + c b), c and s the cosine and
// sine of p times the pair's frequency, times mscale; the gradient is the rotation by the opposite angle.
//
// A workgroup takes a few rows (tokens): it forms their cosines and sines once, in LDS, for all heads, then streams the heads
// through, 16 bytes per access. The angle is reduced in full turns in 64 bits (positions of a million
// leave no digits of it in 32), the remainder of a turn in fp32. Bound by the copy: 16384 tokens, 32 heads of 128, bf16
// 52 us, 5.1 TB/s (a large copy: 5.2).
#include <algorithm>

#include "common.h"
#include "internal.h"

namespace bpt {

namespace {

constexpr int kRopeRows = 4;             // rows of a workgroup, at most
constexpr int kMaxPairs = 64;

template <int N> BPT_DEV void ld(const float* p, float* v) {
  if constexpr (N == 1) {
    v[0] = p[0];
  } else {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      const f32x4 x = *(const f32x4*)(p + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = x[e];
    }
  }
}
template <int N> BPT_DEV void ld(const bf16* p, float* v) {
  if constexpr (N == 1) {
    v[0] = (float)p[0];
  } else {
    const bf16x8 x = *(const bf16x8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)x[e];
  }
}
template <int N> BPT_DEV void st(float* p, const float* v) {
  if constexpr (N == 1) {
    p[0] = v[0];
  } else {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) *(f32x4*)(p + 4 * q) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
  }
}
template <int N> BPT_DEV void st(bf16* p, const float* v) {
  if constexpr (N == 1) {
    p[0] = (bf16)v[0];
  } else {
    bf16x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (bf16)v[e];
    *(bf16x8*)p = x;
  }
}

}  // namespace

// Units of a head: half layout, N elements of the first half of the rotated part and their partners; interleaved,
// N elements (a pair for N = 1); behind the rotated part, N elements that are copied. N = 8 or 1.
template <typename T, int N, bool INTER>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, int rows_per) {
  __shared__ float2 cs[kRopeRows][kMaxPairs];
  const int tid = threadIdx.x, pairs = a.rot / 2;
  const int64_t r0 = (int64_t)blockIdx.x * rows_per;
  const int nr = (int)(a.rows - r0 < rows_per ? a.rows - r0 : rows_per);
  for (int e = tid; e < nr * pairs; e += 256) {
    const int r = e / pairs, i = e - r * pairs;
    const int64_t p = a.positions ? (int64_t)a.positions[r0 + r] : a.pos0 + (r0 + r) % a.S;
    const double t = (double)p * a.turns[i];
    float s, c;
    sincospif(2.0f * (float)(t - rint(t)), &s, &c);
    cs[r][i] = float2{c * a.mscale, s * a.mscale * a.sign};
  }
  __syncthreads();
  const int turned = INTER ? (N == 1 ? pairs : a.rot / N) : pairs / N;
  const int units = turned + (a.x == a.y ? 0 : (a.dh - a.rot) / N);
  const T* X = (const T*)a.x + r0 * a.ldx;
  T* Y = (T*)a.y + r0 * a.ldy;
  const int per_row = units * a.H;
  for (int e = tid; e < nr * per_row; e += 256) {
    const int r = e / per_row, f = e - r * per_row, h = f / units, u = f - h * units;
    const T* x = X + r * a.ldx + (int64_t)h * a.dh;
    T* y = Y + r * a.ldy + (int64_t)h * a.dh;
    if (u >= turned) {
      const int d = a.rot + (u - turned) * N;
      float v[N];
      ld<N>(x + d, v);
      st<N>(y + d, v);
    } else if (!INTER) {
      float v[N], w[N], p[N], q[N];
      ld<N>(x + N * u, v);
      ld<N>(x + pairs + N * u, w);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float2 z = cs[r][N * u + k];
        p[k] = z.x * v[k] - z.y * w[k];
        q[k] = z.x * w[k] + z.y * v[k];
      }
      st<N>(y + N * u, p);
      st<N>(y + pairs + N * u, q);
    } else if (N == 1) {
      const float2 z = cs[r][u];
      const float v = to_f32<T>(x[2 * u]), w = to_f32<T>(x[2 * u + 1]);
      y[2 * u] = from_f32<T>(z.x * v - z.y * w);
      y[2 * u + 1] = from_f32<T>(z.x * w + z.y * v);
    } else {
      float v[N];
      ld<N>(x + N * u, v);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        const float2 z = cs[r][N / 2 * u + k];
        const float p = v[2 * k], q = v[2 * k + 1];
        v[2 * k] = z.x * p - z.y * q;
        v[2 * k + 1] = z.x * q + z.y * p;
      }
      st<N>(y + N * u, v);
    }
  }
}

// Feature-major, in place (the gradient of a layer's projection, without a window): a thread turns 8 consecutive tokens of one pair in every
// head, its cosines and sines formed once. 16384 tokens, 32 heads of 128, bf16 48 us (token-major 45); 2048 tokens 22 (10), 64 workgroups
// of pairs by 1 of tokens, each a chain over the heads.
template <typename T>
__global__ __launch_bounds__(256) void rope_t_kernel(RopeArgs a, int64_t Sp) {
  const int i = blockIdx.y, pairs = a.rot / 2;
  const int64_t c0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;   // column, within one sequence: Sp % 8 == 0
  if (c0 >= a.rows / a.S * Sp) return;
  float cs[8], sn[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const double t = (double)(a.pos0 + (c0 + k) % Sp) * a.turns[i];
    sincospif(2.0f * (float)(t - rint(t)), &sn[k], &cs[k]);
    cs[k] *= a.mscale;
    sn[k] *= a.mscale * a.sign;
  }
  T* x = (T*)a.y + (int64_t)(a.interleaved ? 2 * i : i) * a.ldx + c0;
  const int64_t other = (a.interleaved ? 1 : pairs) * a.ldx, head = a.dh * a.ldx;
  for (int h = 0; h < a.H; ++h, x += head) {
    float v[8], w[8], p[8], q[8];
    ld<8>(x, v);
    ld<8>(x + other, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      p[k] = cs[k] * v[k] - sn[k] * w[k];
      q[k] = cs[k] * w[k] + sn[k] * v[k];
    }
    st<8>(x, p);
    st<8>(x + other, q);
  }
}

hipError_t rope_t(Dt t, const RopeArgs& a, int64_t Sp, hipStream_t s) {
  const int64_t cols = a.rows / a.S * Sp;
  auto k = t == BF16 ? rope_t_kernel<bf16> : rope_t_kernel<float>;
  hipLaunchKernelGGL(k, dim3((unsigned)((cols / 8 + 255) / 256), a.rot / 2), dim3(256), 0, s, a, Sp);
  return hipGetLastError();
}

// Launches of at most 2^25 rows (2^26, four to a workgroup, would be 2^32 threads, which are refused). Where rows stand at pos0 + row %
// S, a launch takes whole runs of S or a part of one, pos0 moved to its start.
template <typename T, int N, bool INTER>
static hipError_t launch(const RopeArgs& a, hipStream_t s) {
  const int rows_per = a.rows >= 4096 ? kRopeRows : 1;   // few rows: one per workgroup
  const int64_t most = (int64_t)1 << 25;
  for (int64_t r = 0, n; r < a.rows; r += n) {
    const int64_t at = r % a.S;
    n = std::min(a.rows - r, most);
    if (a.rows > most) n = at == 0 && n >= a.S ? n / a.S * a.S : std::min(n, a.S - at);
    RopeArgs b = a;
    b.rows = n;
    b.x = (const T*)a.x + r * a.ldx;
    b.y = (T*)a.y + r * a.ldy;
    if (a.positions) b.positions = a.positions + r;
    b.pos0 = a.pos0 + at;
    hipLaunchKernelGGL((rope_kernel<T, N, INTER>), dim3((unsigned)((n + rows_per - 1) / rows_per)), dim3(256), 0, s, b, rows_per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename T>
static hipError_t launch_t(const RopeArgs& a, hipStream_t s) {
  const bool wide = a.rot % (a.interleaved ? 8 : 16) == 0;   // 16-byte pieces; dh and the row strides are multiples of 8
  if (a.interleaved) return wide ? launch<T, 8, true>(a, s) : launch<T, 1, true>(a, s);
  return wide ? launch<T, 8, false>(a, s) : launch<T, 1, false>(a, s);
}

hipError_t rope(Dt t, const RopeArgs& a, hipStream_t s) { return t == BF16 ? launch_t<bf16>(a, s) : launch_t<float>(a, s); }

}  // namespace bpt
