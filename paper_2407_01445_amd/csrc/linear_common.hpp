// Epilogue and tile order shared by the linear layers' kernels.
#pragma once
#include "mfma_common.hpp"
#include "operators.hpp"

namespace fc {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));    // four floats at any address of a float

// Phi(z) = (1 + erf(z / sqrt 2)) / 2 and, times `density`, the normal density at z.  The complementary error function by the
// rational approximation 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions: absolute error 1.5e-7, an ulp of
// fp32 at one, for one exponential - which the density shares - and one reciprocal.
__device__ __forceinline__ float normal_cdf(float z, float* density) {
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
  const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);     // exp(-z^2 / 2)
  float s = fmaf(1.061405429f, t, -1.453152027f);
  s = fmaf(s, t, 1.421413741f);
  s = fmaf(s, t, -0.284496736f);
  s = fmaf(s, t, 0.254829592f);
  const float tail = 0.5f * s * t * e;
  *density = e * 0.3989422804014327f;
  return z < 0.f ? tail : 1.f - tail;
}
// 1 / (1 + exp(-1.702 z))
__device__ __forceinline__ float quick_gate(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * (-1.702f * 1.4426950408889634f)));
}
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == FASTCLIP_ACT_GELU) {
    float density;
    const float r = z * normal_cdf(z, &density);
    return z < -38.f ? 0.f : r;                    // there Phi is zero in fp32; -inf times zero is not the limit
  } else if constexpr (ACT == FASTCLIP_ACT_QUICK_GELU) {
    return z < -80.f ? 0.f : z * quick_gate(z);
  } else {
    return z;
  }
}
template <int ACT>
__device__ __forceinline__ float activation_slope(float z) {
  if constexpr (ACT == FASTCLIP_ACT_GELU) {
    float density;
    const float p = normal_cdf(z, &density);
    return fabsf(z) > 38.f ? (z > 0.f ? 1.f : 0.f) : fmaf(z, density, p);
  } else if constexpr (ACT == FASTCLIP_ACT_QUICK_GELU) {
    const float p = quick_gate(z);
    return fabsf(z) > 80.f ? (z > 0.f ? 1.f : 0.f) : fmaf(1.702f * z * p, 1.f - p, p);
  } else {
    return 1.f;
  }
}

template <int V>
__device__ __forceinline__ void load_bf16(float (&x)[V], const bf16_t* p) {
  if constexpr (V == 8) {
    const u32x4 w = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = bf2f(p[i]);
  }
}
template <int V>
__device__ __forceinline__ void store_bf16(bf16_t* p, const float (&x)[V]) {
  if constexpr (V == 8) {
    const u32x4 w = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    *(u32x4*)p = w;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = f2bf(x[i]);
  }
}
template <int V>
__device__ __forceinline__ void load_f32(float (&x)[V], const float* p) {
  if constexpr (V == 8) {
    const f32x4_any a = *(const f32x4_any*)p, b = *(const f32x4_any*)(p + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < 4 ? a[i & 3] : b[i & 3];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = p[i];
  }
}
template <int V>
__device__ __forceinline__ void store_f32(float* p, const float (&x)[V]) {
  if constexpr (V == 8) {
    *(f32x4_any*)p = f32x4_any{x[0], x[1], x[2], x[3]};
    *(f32x4_any*)(p + 4) = f32x4_any{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = x[i];
  }
}

// What a layer does with V neighbouring sums of row m, columns n .. n + V - 1 (inside the matrix): bias, the value before the
// activation kept, activation or the derivative's factor, residual, one rounding.  BF16: type of pre.
template <bool BF16, int ACT, int V>
__device__ __forceinline__ void finish_values_act(const LinearArgs& a, float (&z)[V], int64_t m, int64_t n) {
  float t[V];
  if (a.bias) {
    load_f32<V>(t, a.bias + n);
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] += t[i];
  }
  if (a.pre_out) {
    if constexpr (BF16) store_bf16<V>((bf16_t*)a.pre_out + m * a.ld_pre + n, z);
    else store_f32<V>((float*)a.pre_out + m * a.ld_pre + n, z);
  }
  if constexpr (ACT != FASTCLIP_ACT_NONE) {
    if (a.pre_in) {
      if constexpr (BF16) load_bf16<V>(t, (const bf16_t*)a.pre_in + m * a.ld_pre + n);
      else load_f32<V>(t, (const float*)a.pre_in + m * a.ld_pre + n);
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] *= activation_slope<ACT>(t[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] = activate<ACT>(z[i]);
    }
  }
  if (a.residual) {
    if (a.out_bf16) load_bf16<V>(t, (const bf16_t*)a.residual + m * a.ld_res + n);
    else load_f32<V>(t, (const float*)a.residual + m * a.ld_res + n);
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] += t[i];
  }
  if (a.out_bf16) store_bf16<V>((bf16_t*)a.out + m * a.ld_out + n, z);
  else store_f32<V>((float*)a.out + m * a.ld_out + n, z);
}
template <bool BF16, int V>
__device__ __forceinline__ void finish_values(const LinearArgs& a, float (&z)[V], int64_t m, int64_t n) {
  if (a.act == FASTCLIP_ACT_GELU) finish_values_act<BF16, FASTCLIP_ACT_GELU, V>(a, z, m, n);
  else if (a.act == FASTCLIP_ACT_QUICK_GELU) finish_values_act<BF16, FASTCLIP_ACT_QUICK_GELU, V>(a, z, m, n);
  else finish_values_act<BF16, FASTCLIP_ACT_NONE, V>(a, z, m, n);
}

// Which output tile and split a workgroup takes.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: those of
// one XCD take neighbouring tiles, eight rows of tiles by as many columns as there are.
struct TilePlace { int64_t m, n; int split; };
__device__ __forceinline__ TilePlace tile_place(uint32_t id, uint32_t groups, uint32_t rows, uint32_t cols) {
  const uint32_t tiles = rows * cols, xcd = id & 7, per = groups >> 3, more = groups & 7;
  const uint32_t at = xcd * per + (xcd < more ? xcd : more) + (id >> 3);
  const uint32_t split = at / tiles, t = at - split * tiles;
  const uint32_t band = t / (8 * cols), in = t - band * 8 * cols;
  const uint32_t height = rows - band * 8 < 8 ? rows - band * 8 : 8;
  return {(int64_t)(band * 8 + in % height), (int64_t)(in / height), (int)split};
}

}  // namespace fc
