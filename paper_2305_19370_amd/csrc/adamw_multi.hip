// AdamW over a list of tensors, moments in 32 or in 8 bits.
//
// A block is 256 consecutive elements of one tensor: one wave, 4 elements a lane. The list is part of the kernel's
// arguments; a wave finds its tensor by the blocks in front of it.
//
// 8-bit moments: the first moment m and the root r = sqrt(v) of the second as e4m3 codes, scaled by a power of two per block so
// that the largest value lies in [128, 256). Codes are rounded up with the probability of the value's
// place between two codes (16 bits of a mix of element, tensor, step and seed): a moment that moves by
// less than a step per update, as r does with beta2 near 1, still follows its expectation, where
// rounding to nearest would never move it. A root above zero keeps a code above zero, so m / r stays bounded.
//
// Bound by the copy (16 bytes an access and lane; a list costs one launch per kAdamTensors tensors): 50 million elements, 30 bytes
// each with 32-bit moments and a bf16 copy 283 us, 5.3 TB/s; 142 million, 16 bytes each with 8-bit ones, bf16 gradients
// and a bf16 copy 435 us, 5.2 TB/s. There the arithmetic is nearly as long: with the library's root (two of them) and division 480 us,
// with maxima of a wave by exchanges through LDS 450.
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace bpt {

namespace {

BPT_DEV uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0x6A09E667u;
  return x ^ (x >> 16);
}

// The largest of a wave's values: rows of 16 lanes by neighbours, pairs, mirrored halves and rows, then one of each.
BPT_DEV uint32_t wave_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));    // quad_perm [1, 0, 3, 2]
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));    // quad_perm [2, 3, 0, 1]
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));   // row_half_mirror
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));   // row_mirror
  auto of = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); };
  return max(max(of(0), of(16)), max(of(32), of(48)));
}
BPT_DEV float pow2(int e) { return __uint_as_float((uint32_t)e << 23); }   // 2^(e - 127)

// e4m3 code of 0 <= y < 256: 16 random bits below the third mantissa bit, then truncation. Below 2^-6, where steps are
// all 2^-9, y + 2^-6 has those steps.
BPT_DEV uint32_t e4m3_code(float y, uint32_t rnd16) {
  const bool small = y < 0.015625f;
  const uint32_t bits = __float_as_uint(small ? y + 0.015625f : y) + (rnd16 << 4);
  return (bits >> 20) - (small ? 968u : 960u);
}

// The root of w, 2^-100 <= w < inf or 0, rounded to nearest. The hardware's s is at most a step off; the root lies above the
// midpoint of s and its neighbour s' iff w > s s', since w and s s' are multiples of a step^2 and the midpoint's square is
// s s' + step^2 / 4.
BPT_DEV float root(float w) {
  const float s = __builtin_amdgcn_sqrtf(w);
  const float dn = __uint_as_float(__float_as_uint(s) - 1u), up = __uint_as_float(__float_as_uint(s) + 1u);
  const float r = fmaf(-dn, s, w) <= 0.0f ? dn : s;
  return fmaf(-up, s, w) > 0.0f ? up : r;
}
// n / d of finite numbers, d normal: the quotient by the reciprocal, corrected by its remainder; off by half a step and 2^-20 of one.
BPT_DEV float quotient(float n, float d) {
  const float y = __builtin_amdgcn_rcpf(d), q = n * y;
  return fmaf(fmaf(-q, d, n), y, q);
}

template <typename T> BPT_DEV void ld4(const T* p, int n, float (&v)[4]) {   // n elements exist
  if (n >= 4) {
    if constexpr (sizeof(T) == 4) {
      const f32x4 x = *(const f32x4*)p;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = x[e];
    } else {
      const bf16x4 x = *(const bf16x4*)p;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (float)x[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < n ? to_f32<T>(p[e]) : 0.0f;
  }
}
template <typename T> BPT_DEV void st4(T* p, int n, const float (&v)[4]) {
  if (n >= 4) {
    if constexpr (sizeof(T) == 4) {
      *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
    } else {
      bf16x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (bf16)v[e];
      *(bf16x4*)p = x;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  }
}
BPT_DEV uint32_t ld_codes(const uint8_t* p, int n) {
  if (n >= 4) return *(const uint32_t*)p;
  uint32_t x = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) x |= (uint32_t)p[e] << (8 * e);
  return x;
}
BPT_DEV void st_codes(uint8_t* p, int n, uint32_t x) {
  if (n >= 4) {
    *(uint32_t*)p = x;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) p[e] = (uint8_t)(x >> (8 * e));
}
BPT_DEV void decode(uint32_t x, float scale, float (&v)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  v[0] = lo[0] * scale;
  v[1] = lo[1] * scale;
  v[2] = hi[0] * scale;
  v[3] = hi[1] * scale;
}

}  // namespace

template <typename TG, typename TL, int BITS>
__global__ __launch_bounds__(256) void adamw_multi_kernel(AdamArgs a) {
#pragma clang fp contract(off)   // every operation rounds as the formula is written
  const int lane = threadIdx.x & 63;
  const uint32_t blk = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blk >= a.blocks) return;
  int ti = 0;
  for (int step = 32; step >= 1; step >>= 1)
    if (ti + step < a.count && a.t[ti + step].first <= blk) ti += step;
  const AdamTensor& t = a.t[ti];
  const int64_t b = blk - t.first, at = b * 256 + 4 * lane;
  const int n = (int)(t.n - at < 4 ? (t.n - at < 0 ? 0 : t.n - at) : 4);
  float p[4] = {}, g[4] = {}, m[4] = {}, v[4] = {}, r[4];
  uint32_t em = 0, er = 0;
  if (n > 0) {
    ld4<float>(t.p + at, n, p);
    ld4<TG>((const TG*)t.g + at, n, g);
    if constexpr (BITS == 32) {
      ld4<float>((const float*)t.m + at, n, m);
      ld4<float>((const float*)t.v + at, n, v);
    } else {
      const uint32_t mc = ld_codes((const uint8_t*)t.m + at, n), rc = ld_codes((const uint8_t*)t.v + at, n);
      decode(mc, pow2(max((int)t.exps[2 * b] - 7, 0)), m);
      decode(rc, pow2(max((int)t.exps[2 * b + 1] - 7, 0)), r);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = r[e] * r[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    m[e] = a.b1 * m[e] + a.nb1 * g[e];
    v[e] = a.b2 * v[e] + a.nb2 * (g[e] * g[e]);
  }
  if constexpr (BITS == 32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = p[e] * t.decay - a.lr * (m[e] * a.c1) / (sqrtf(v[e] * a.c2) + a.eps);
    if (n > 0) {
      st4<float>((float*)t.m + at, n, m);
      st4<float>((float*)t.v + at, n, v);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      em = max(em, __float_as_uint(m[e]) & 0x7FFFFFFFu);
      er = max(er, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    }
    em = wave_max(em);
    er = wave_max(er);
    const bool finite = max(em, er) < 0x7F800000u;
    em = min(max(em >> 23, 27u), 254u);
    er = ((er >> 23) + 127u) >> 1;
    const float sm = pow2(261 - (int)em);
    // roots are formed of v 4^k, which puts the block's largest near 2^62 (k kept where 4^k is an fp32 number and nothing is scaled down):
    // what then lies below 2^-100 has the least code, and a root far below eps
    const int k = min(max(157 - (int)er, 0), 63);
    const float scale = pow2(2 * k + 127), rc2 = a.rc2 * pow2(127 - k), sr = pow2(261 - (int)er - k);
    uint32_t mc = 0, rc = 0;
    auto update = [&](auto ordinary) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float num = a.lr * (m[e] * a.c1);
        r[e] = ordinary ? root(v[e] * scale) : sqrtf(v[e] * scale);
        const float den = r[e] * rc2 + a.eps;
        p[e] = p[e] * t.decay - (ordinary ? quotient(num, den) : num / den);
        const float ym = fabsf(m[e]) * sm, yr = r[e] * sr;
        const uint32_t rnd = mix32((uint32_t)(at + e) ^ t.key);
        uint32_t cm = e4m3_code(ym, rnd & 0xFFFFu), cr = e4m3_code(yr, rnd >> 16);
        if (!ordinary) {                              // the code of NaN for what is not finite
          cm = ym < 512.0f ? cm : 0x7Fu;
          cr = yr < 512.0f ? cr : 0x7Fu;
        }
        cm |= m[e] < 0.0f ? 0x80u : 0u;
        cr = max(cr, v[e] > 0.0f ? 1u : 0u);
        mc |= cm << (8 * e);
        rc |= cr << (8 * e);
      }
    };
    if (finite) update(std::true_type{});
    else update(std::false_type{});
    if (n > 0) {
      st_codes((uint8_t*)t.m + at, n, mc);
      st_codes((uint8_t*)t.v + at, n, rc);
    }
    if (lane == 0) *(uint16_t*)(t.exps + 2 * b) = (uint16_t)(em | er << 8);
  }
  if (n > 0) {
    st4<float>(t.p + at, n, p);
    if (t.low) st4<TL>((TL*)t.low + at, n, p);
  }
}

template <typename TG, typename TL, int BITS>
static hipError_t launch(const AdamArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((adamw_multi_kernel<TG, TL, BITS>), dim3((a.blocks + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename TG, typename TL>
static hipError_t launch_b(int bits, const AdamArgs& a, hipStream_t s) {
  return bits == 8 ? launch<TG, TL, 8>(a, s) : launch<TG, TL, 32>(a, s);
}

hipError_t adamw_multi(Dt tg, Dt tl, int bits, const AdamArgs& a, hipStream_t s) {
  if (tg == BF16) return tl == BF16 ? launch_b<bf16, bf16>(bits, a, s) : launch_b<bf16, float>(bits, a, s);
  return tl == BF16 ? launch_b<float, bf16>(bits, a, s) : launch_b<float, float>(bits, a, s);
}

}  // namespace bpt
