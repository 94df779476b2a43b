// Distillation of a language-model head from a teacher's largest logits: what stands around the products.
// Token t has student logits z over the vocabulary and a list of (v_j, k_j); q = softmax(v / tau) over the list, p_tau =
// softmax(z / tau):
//   kl_t = sum_j q_j log(q_j / p_tau(k_j)),  ce_t = -log p_1(y_t),  loss = sum_t w_t (soft tau^2 kl_t + hard ce_t)
//   d loss / d z = w (soft tau (p_tau - q) + hard (p_1 - onehot(y)))
// The list (and the target, an entry of q = 0) is sorted by index first. The product that forms the logits then reduces them to
// maximum and sums of 64 columns in its epilogue and picks the listed ones out (a table says which entries fall into which 64
// columns). The backward writes the gradient of a token without a list from the logits that the forward kept, or else in the epilogue
// of their product formed again, transposed; the listed elements are overwritten afterwards from the picked logits, so that p - q is
// rounded once: to the type of the operands of dh = G W^T and dW = h^T G, which in bf16 puts those 2.2e-3 to 2.5e-3 from 64 bits, where
// the rounding of dh and dW themselves is 1.7e-3 and that of G alone 1.5e-3. Twice the products would take G in two parts.
// A weight is exp2((z - max) scale - log2(sum)): a small tau makes z / tau large, and a difference of two such numbers, z / tau and
// their log-sum-exp, would be off by the rounding of |z| / tau (2e-3 of p at tau = 1e-3 and logits of 20).
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace bpt {

namespace {
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kNone = 0x7FFFFFFF;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;
constexpr int kPiece = 1024;                         // of a token's row of `seg`

BPT_DEV float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
}  // namespace

// One wave per token: valid entries sorted by index, an index that is given twice once with the sum of its probabilities; the
// target's place among them; the token's factors. With seg, also where the entries of every 64 columns are.
// The order comes from counting smaller indices: K steps over LDS for each of a lane's entries, a comparison and an addition each.
template <int kPer>                                    // entries of a lane
__global__ __launch_bounds__(256) void distill_prep_kernel(DistillArgs a) {
  __shared__ __attribute__((aligned(16))) int skey[4][64 * kPer];
  __shared__ __attribute__((aligned(16))) float sq[4][64 * kPer];
  __shared__ __attribute__((aligned(16))) uint16_t sseg[4][kPiece];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * 4 + wv;      // a wave past the end works on the last token and stores nothing
  const bool real = t < a.T;
  const int64_t tt = real ? t : a.T - 1;
  const int K = a.K, K1 = a.K1;
  int key[kPer];
  float q[kPer], mx = -__builtin_inff();
  const int y = a.targets ? a.targets[tt] : -1;
  const bool has_y = y >= 0 && y < a.V;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int j = lane + 64 * e;
    key[e] = kNone;
    q[e] = -__builtin_inff();
    if (j < K) {
      const int k = a.index[tt * K + j];
      const float v = a.values[tt * K + j];
      if (k >= 0 && k < a.V && !(v == -__builtin_inff())) {
        key[e] = k;
        q[e] = v;
        mx = fmaxf(mx, v);
      }
    } else if (j < K1 && has_y) {
      key[e] = y;
    }
  }
  mx = wave_max(mx);
  float sum = 0.0f;
  bool mine = false;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int j = lane + 64 * e;
    const bool listed = j < K && key[e] != kNone;
    q[e] = listed ? __builtin_amdgcn_exp2f((q[e] - mx) * a.scale) : 0.0f;
    sum += q[e];
    mine |= listed;
  }
  sum = warp_sum(sum);
  const bool some = __any(mine);
  const float inv = some ? 1.0f / sum : 0.0f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    q[e] = q[e] * inv;
    skey[wv][lane + 64 * e] = key[e];
    sq[wv][lane + 64 * e] = q[e];
  }
  wave_sync();
  // places in the sorted list: smaller indices, and equal ones that come before
  int rank[kPer], valid = 0, n = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) rank[e] = 0;
#pragma unroll
  for (int b = 0; b < kPer; ++b) {
    const int end = K1 < 64 * b + 64 ? K1 : 64 * b + 64;   // kNone behind the last entry: smaller than nothing
#pragma unroll 2
    for (int i = 64 * b; i < end; i += 4) {
      const i32x4 k = *(const i32x4*)&skey[wv][i];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          if (b == e) rank[e] += k[u] - (i + u - 64 * b < lane) < key[e];
          else rank[e] += b < e ? k[u] <= key[e] : k[u] < key[e];
        }
    }
  }
  wave_sync();
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const bool counts = key[e] != kNone;
    if (counts) {
      skey[wv][rank[e]] = key[e];
      sq[wv][rank[e]] = q[e];
    }
    valid += __popcll(__ballot(counts));
  }
  wave_sync();
  // the first of equal ones takes the sum of their probabilities
  bool first[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int at = lane + 64 * e;
    first[e] = at < valid && (at == 0 || skey[wv][at - 1] != skey[wv][at]);
    if (first[e]) {
      key[e] = skey[wv][at];
      q[e] = sq[wv][at];
      for (int j = at + 1; j < valid && skey[wv][j] == key[e]; ++j) q[e] += sq[wv][j];
    }
  }
  wave_sync();
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const unsigned long long mask = __ballot(first[e]);
    const int at = n + __popcll(mask & ((1ull << lane) - 1));
    n += __popcll(mask);
    if (!first[e]) continue;
    skey[wv][at] = key[e];
    if (real) {
      a.sidx[t * K1 + at] = key[e];
      a.sq[t * K1 + at] = q[e];
      if (a.targets && key[e] == y) a.ypos[t] = at;
    }
  }
  wave_sync();
  if (!real) return;
  if (lane == 0) {
    const float w = a.weights ? a.weights[t] : a.weight;
    a.count[t] = n;
    if (!has_y) a.ypos[t] = -1;
    a.gs[t] = some ? w * a.soft * a.tau : 0.0f;
    a.gh[t] = has_y ? w * a.hard : 0.0f;
    a.w[t] = w;
  }
  if (a.seg) {
    // pieces of the row in LDS: zeros, then from the first entry of every 64 columns that have any
    uint16_t* piece = sseg[wv];
    for (int64_t g0 = 0; g0 < a.ng; g0 += kPiece) {
      const int len = (int)std::min<int64_t>(a.ldseg - g0, kPiece);   // a multiple of 8
      for (int c = 8 * lane; c < len; c += 512) *(u32x4*)(piece + c) = u32x4{0, 0, 0, 0};
      wave_sync();
      for (int e = lane; e < n; e += 64) {
        const int g = skey[wv][e] >> 6;
        if (g < g0 || g >= g0 + len || (e > 0 && skey[wv][e - 1] >> 6 == g)) continue;
        int many = 1;
        while (e + many < n && skey[wv][e + many] >> 6 == g) ++many;
        piece[g - g0] = (uint16_t)(e << 7 | many);
      }
      wave_sync();
      u32x4* out = (u32x4*)(a.seg + (t - a.t0) * a.ldseg + g0);
      for (int c = lane; c < len / 8; c += 64) out[c] = ((const u32x4*)piece)[c];
      wave_sync();
    }
  }
}

namespace {
// (m, l) of two sets: l = sum of 2^((z - m) s)
BPT_DEV void join(float& m, float& l, float& l1, float m2, float l2, float l12, float s) {
  const float M = fmaxf(m, m2);
  if (M == -__builtin_inff()) {                        // sums of nothing, 0, or of NaN, which a maximum does not show
    l += l2;
    l1 += l12;
    return;
  }
  const float f = __builtin_amdgcn_exp2f((m - M) * s), f2 = __builtin_amdgcn_exp2f((m2 - M) * s);
  const float g = __builtin_amdgcn_exp2f((m - M) * kLog2e), g2 = __builtin_amdgcn_exp2f((m2 - M) * kLog2e);
  l = l * f + l2 * f2;
  l1 = l1 * g + l12 * g2;
  m = M;
}

// the token's log-sum-exps and losses, by its wave
BPT_DEV void finish(const DistillArgs& a, int64_t t, int lane, float m, float l, float l1) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) join(m, l, l1, __shfl_xor(m, o, 64), __shfl_xor(l, o, 64), __shfl_xor(l1, o, 64), a.scale);
  // maximum and logarithms apart: with a small tau z / tau is large, and one number would hold of ll what is left behind z / tau
  const float ll = logf(l), lo = a.two ? logf(l1) : ll;
  float kl = 0.0f;
  for (int j = lane; j < a.count[t]; j += 64) {
    const float q = a.sq[t * a.K1 + j];
    if (q != 0.0f) kl += q * (logf(q) + (m - a.sz[t * a.K1 + j]) / a.tau + ll);
  }
  kl = warp_sum(kl);
  if (lane) return;
  const int y = a.ypos[t];
  const bool in = a.w[t] != 0.0f;                      // a token of no weight is left out, whatever it holds
  a.mx[t] = m;
  a.lt[t] = ll;
  a.l1[t] = lo;
  a.tokens[t] = in ? kl : 0.0f;
  a.tokens[a.Tall + t] = in && y >= 0 ? (m - a.sz[t * a.K1 + y]) + lo : 0.0f;
}
}  // namespace

// bf16: from the summaries of 64 columns, [rows, ng] of (max, sum) and with two temperatures the second sums
__global__ __launch_bounds__(256) void distill_merge_kernel(DistillArgs a, const float* part, const float* part1) {
  const int lane = threadIdx.x & 63;
  const int64_t t = a.t0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.T) return;
  float m = -__builtin_inff(), l = 0.0f, l1 = 0.0f;
  for (int64_t j0 = lane; j0 < a.ng; j0 += 512) {      // eight in flight
    u32x2 v[8];
    float v1[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t j = j0 + 64 * k, at = (t - a.t0) * a.ng + j;
      v[k] = j < a.ng ? *(const u32x2*)(part + 2 * at) : u32x2{0xFF800000u, 0u};   // -inf, 0
      v1[k] = a.two && j < a.ng ? part1[at] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) join(m, l, l1, __uint_as_float(v[k][0]), __uint_as_float(v[k][1]), v1[k], a.scale);
  }
  finish(a, t, lane, m, l, l1);
}

// fp32: from the logits [rows, ld], ld a multiple of 64, by one workgroup per token: maximum, then sums and the listed logits, the
// second time from the L2. (A wave per token walked 200 steps of 14302 logits.)
__global__ __launch_bounds__(256) void distill_rows_kernel(DistillArgs a, const float* z, int64_t ld) {
  __shared__ float part[3][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = a.t0 + blockIdx.x, whole = a.V / 4 * 4;
  const float* row = z + (t - a.t0) * ld;
  float m = -__builtin_inff(), l = 0.0f, l1 = 0.0f;
#pragma unroll 4
  for (int64_t j = 4 * tid; j < whole; j += 1024) {
    const f32x4 v = *(const f32x4*)(row + j);
    m = fmaxf(m, fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
  }
  for (int64_t j = whole + tid; j < a.V; j += 256) m = fmaxf(m, row[j]);
  m = wave_max(m);
  if (lane == 0) part[0][wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
  auto add = [&](float v) {
    l += __builtin_amdgcn_exp2f((v - m) * a.scale);
    if (a.two) l1 += __builtin_amdgcn_exp2f((v - m) * kLog2e);
  };
#pragma unroll 2
  for (int64_t j = 4 * tid; j < whole; j += 1024) {
    const f32x4 v = *(const f32x4*)(row + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) add(v[e]);
  }
  for (int64_t j = whole + tid; j < a.V; j += 256) add(row[j]);
  l = warp_sum(l);
  l1 = warp_sum(l1);
  if (lane == 0) part[1][wave] = l, part[2][wave] = l1;
  __syncthreads();
  if (wave > 0) return;
  const int n = a.count[t];
  for (int j = lane; j < n; j += 64) a.sz[t * a.K1 + j] = row[a.sidx[t * a.K1 + j]];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");   // finish() reads them by other lanes
  // lane 0 holds the whole, the others nothing
  l = (part[1][0] + part[1][1]) + (part[1][2] + part[1][3]);
  l1 = (part[2][0] + part[2][1]) + (part[2][2] + part[2][3]);
  finish(a, t, lane, lane ? -__builtin_inff() : m, lane ? 0.0f : l, lane ? 0.0f : l1);
}

// loss = (sum w (soft tau^2 kl + hard ce), sum w kl, sum w ce), in a fixed order by one workgroup
__global__ __launch_bounds__(1024) void distill_loss_kernel(DistillArgs a, float* loss) {
  __shared__ float part[2][1024];
  const int tid = threadIdx.x;
  float kl = 0.0f, ce = 0.0f;
  for (int64_t t = tid; t < a.Tall; t += 1024) {
    const float w = a.w[t];
    if (w != 0.0f) {
      kl += w * a.tokens[t];
      ce += w * a.tokens[a.Tall + t];
    }
  }
  part[0][tid] = kl;
  part[1][tid] = ce;
  __syncthreads();
  for (int o = 512; o >= 1; o >>= 1) {
    if (tid < o) {
      part[0][tid] += part[0][tid + o];
      part[1][tid] += part[1][tid + o];
    }
    __syncthreads();
  }
  if (tid == 0) {
    loss[0] = a.soft * a.tau * a.tau * part[0][0] + a.hard * part[1][0];
    loss[1] = part[0][0];
    loss[2] = part[1][0];
  }
}

// The gradient of a token without a list from the logits that the forward kept, transposed as the products read it: tiles of 64 logits by
// 256 bytes of tokens. A thread takes four logits of four tokens; in LDS a row of the tile holds pieces of four tokens, its piece c
// at c ^ f(row / 4), so that both the writes of a wave (16 rows, four pieces) and its reads (whole rows) use every bank.
// A workgroup does `steps` tiles of the same tokens, whose factors it loads once.
// Bound by memory: 8192 tokens, 50304 columns 503 us, 4.9 TB/s (the product formed again 1540).
template <typename T>
__global__ __launch_bounds__(256) void distill_grad_kernel(DistillArgs a, float dloss, const float* z, T* G, int64_t ld, int tiles, int steps) {
  constexpr int kTok = 256 / sizeof(T), kGroups = kTok / 64;
  typedef typename std::conditional<sizeof(T) == 4, u32x4, u32x2>::type Piece;   // four tokens
  __shared__ __attribute__((aligned(16))) char tile[64 * 256];
  const int q = threadIdx.x & 15, tg = threadIdx.x >> 4;   // logits 4 q .. 4 q + 3, tokens 4 tg .. of each 64
  const int part = (tiles + steps - 1) / steps;
  const int64_t n0 = (int64_t)(blockIdx.x / part) * kTok, rows = a.T - a.t0, ldz = a.ng * 64;
  const int first = (int)(blockIdx.x % part) * steps, last = first + steps < tiles ? first + steps : tiles;
  float mx[kGroups][4], l2[kGroups][4], g[kGroups][4], l21[kGroups][4], g1[kGroups][4];
#pragma unroll
  for (int k = 0; k < kGroups; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t n = n0 + 64 * k + 4 * tg + e, t = a.t0 + (n < rows ? n : rows - 1);
      mx[k][e] = a.mx[t];
      l2[k][e] = a.lt[t] * kLog2e;
      g[k][e] = a.gs[t];
      g1[k][e] = a.gh[t];
      l21[k][e] = a.two ? a.l1[t] * kLog2e : 0.0f;
      if (!a.two) g[k][e] += g1[k][e], g1[k][e] = 0.0f;
      if (n >= rows) g[k][e] = g1[k][e] = 0.0f;
      g[k][e] *= dloss;
      g1[k][e] *= dloss;
    }
  for (int i = first; i < last; ++i) {
    const int64_t v0 = (int64_t)i * 64;
    f32x4 v[kGroups][4];
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t n = n0 + 64 * k + 4 * tg + e;
        v[k][e] = *(const f32x4*)(z + (n < rows ? n : rows - 1) * ldz + v0 + 4 * q);
      }
    if (i > first) __syncthreads();
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        __attribute__((aligned(16))) T out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float d = v[k][e][c] - mx[k][e];
          float r = g[k][e] * __builtin_amdgcn_exp2f(fmaf(d, a.scale, -l2[k][e]));
          if (a.two) r = fmaf(g1[k][e], __builtin_amdgcn_exp2f(fmaf(d, kLog2e, -l21[k][e])), r);
          const bool none = (g[k][e] == 0.0f && g1[k][e] == 0.0f) || v0 + 4 * q + c >= a.V;
          out[e] = from_f32<T>(none ? 0.0f : r);
        }
        const int piece = (16 * k + tg) ^ (kGroups * q);   // pairs of pieces stay together in 16 bits
        *(Piece*)(tile + (4 * q + c) * 256 + piece * sizeof(Piece)) = *(const Piece*)out;
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = 16 * k + tg;
      const int64_t n = n0 + q * (16 / sizeof(T));
      if (n < (rows + 63) / 64 * 64)
        *(u32x4*)(G + (v0 + row) * ld + n) = *(const u32x4*)(tile + row * 256 + ((q * 16) ^ (row / 4 * kGroups * (int)sizeof(Piece))));
    }
  }
}

// Workgroups from `first` on: the listed elements of the logits' gradient, transposed [V, ld] with the block's tokens as columns. Those
// before it: h of the tokens that have a gradient, zeros for the others, so that what those hold does not reach dW.
template <typename T>
__global__ __launch_bounds__(256) void distill_listed_kernel(DistillArgs a, float dloss, T* G, int64_t ld, const T* h, T* out, int64_t D,
                                                             uint32_t first) {
  const int64_t rows = a.T - a.t0;
  if (blockIdx.x < first) {
    constexpr int N = 16 / sizeof(T);
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, t = e / (D / N);
    if (t >= rows) return;
    const bool in = a.gs[a.t0 + t] != 0.0f || a.gh[a.t0 + t] != 0.0f;
    ((u32x4*)out)[e] = in ? ((const u32x4*)h)[e] : u32x4{0, 0, 0, 0};
    return;
  }
  // neighbouring threads take neighbouring tokens: their lists' columns of G are neighbours
  const int64_t e = (int64_t)(blockIdx.x - first) * 256 + threadIdx.x, j = e / rows, t = a.t0 + e % rows;
  if (j >= a.K1 || j >= a.count[t]) return;
  const float gs = a.gs[t], gh = a.gh[t], d = a.sz[t * a.K1 + j] - a.mx[t];
  if (gs == 0.0f && gh == 0.0f) return;
  const float p = __builtin_amdgcn_exp2f(fmaf(d, a.scale, -a.lt[t] * kLog2e)), p1 = a.two ? __builtin_amdgcn_exp2f(fmaf(d, kLog2e, -a.l1[t] * kLog2e)) : p;
  const float g = gs * (p - a.sq[t * a.K1 + j]) + gh * (a.ypos[t] == j ? p1 - 1.0f : p1);
  G[(int64_t)a.sidx[t * a.K1 + j] * ld + (t - a.t0)] = from_f32<T>(dloss * g);
}

// ------------------------------------------------------------------ launchers
hipError_t distill_prep(const DistillArgs& a, hipStream_t s) {
  // tokens t0 .. T: pointers of whole tensors
  DistillArgs b = a;
  const int64_t n = a.T - a.t0;
  b.index += a.t0 * a.K; b.values += a.t0 * a.K;
  if (b.targets) b.targets += a.t0;
  if (b.weights) b.weights += a.t0;
  b.sidx += a.t0 * a.K1; b.sq += a.t0 * a.K1; b.ypos += a.t0; b.count += a.t0; b.gs += a.t0; b.gh += a.t0; b.w += a.t0;
  b.T = n; b.t0 = 0;
  const dim3 grid((unsigned)((n + 3) / 4));
  static_assert(kDistillMaxK + 1 <= 64 * 5, "entries of a lane");
  if (a.K1 <= 64) hipLaunchKernelGGL((distill_prep_kernel<1>), grid, dim3(256), 0, s, b);
  else if (a.K1 <= 128) hipLaunchKernelGGL((distill_prep_kernel<2>), grid, dim3(256), 0, s, b);
  else if (a.K1 <= 192) hipLaunchKernelGGL((distill_prep_kernel<3>), grid, dim3(256), 0, s, b);
  else hipLaunchKernelGGL((distill_prep_kernel<5>), grid, dim3(256), 0, s, b);
  return hipGetLastError();
}
hipError_t distill_merge(const DistillArgs& a, const float* part, const float* part1, hipStream_t s) {
  hipLaunchKernelGGL(distill_merge_kernel, dim3((unsigned)((a.T - a.t0 + 3) / 4)), dim3(256), 0, s, a, part, part1);
  return hipGetLastError();
}
hipError_t distill_rows(const DistillArgs& a, const float* z, int64_t ld, hipStream_t s) {
  hipLaunchKernelGGL(distill_rows_kernel, dim3((unsigned)(a.T - a.t0)), dim3(256), 0, s, a, z, ld);
  return hipGetLastError();
}
hipError_t distill_loss(const DistillArgs& a, float* loss, hipStream_t s) {
  hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(1024), 0, s, a, loss);
  return hipGetLastError();
}
hipError_t distill_grad(Dt t, const DistillArgs& a, float dloss, const float* z, void* G, int64_t ld, hipStream_t s) {
  const int64_t rows = a.T - a.t0, n = t == F32 ? (rows + 63) / 64 : (rows + 127) / 128;
  const int steps = n * a.ng >= 8192 ? 4 : 1;          // where that many workgroups are left
  const dim3 grid((unsigned)(n * ((a.ng + steps - 1) / steps)));
  if (t == F32) hipLaunchKernelGGL((distill_grad_kernel<float>), grid, dim3(256), 0, s, a, dloss, z, (float*)G, ld, (int)a.ng, steps);
  else hipLaunchKernelGGL((distill_grad_kernel<bf16>), grid, dim3(256), 0, s, a, dloss, z, (bf16*)G, ld, (int)a.ng, steps);
  return hipGetLastError();
}
hipError_t distill_listed(Dt t, const DistillArgs& a, float dloss, void* G, int64_t ld, const void* h, void* out, int64_t D,
                          hipStream_t s) {
  const int64_t rows = a.T - a.t0, n = out ? (rows * D / (t == F32 ? 4 : 8) + 255) / 256 : 0;
  const dim3 grid((unsigned)(n + (rows * a.K1 + 255) / 256));
  if (t == F32)
    hipLaunchKernelGGL((distill_listed_kernel<float>), grid, dim3(256), 0, s, a, dloss, (float*)G, ld, (const float*)h, (float*)out, D, (uint32_t)n);
  else
    hipLaunchKernelGGL((distill_listed_kernel<bf16>), grid, dim3(256), 0, s, a, dloss, (bf16*)G, ld, (const bf16*)h, (bf16*)out, D, (uint32_t)n);
  return hipGetLastError();
}

}  // namespace bpt
