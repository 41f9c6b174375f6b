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

// ---- the epilogue of a wavefront's part of a tile --------------------------------------------------------------------------
//
// Eight neighbouring values of an output row at a time, groups h = 0 .. G - 1 side by side in a row of blocks.  Vector memory
// operations complete in the order of their issue, stores too: a load behind stores waits for them.  So everything that the
// epilogue reads is requested ahead of the stores: the bias before the first, residual and pre three groups
// ahead.
struct Held8 { u32x4 lo, hi; };                 // eight bf16 (lo) or fp32 values as they lie in memory
__device__ __forceinline__ void hold(Held8& x, const void* p, int64_t at, bool bf16) {
  if (bf16) {
    x.lo = *(const u32x4*)((const bf16_t*)p + at);
  } else {
    x.lo = *(const u32x4*)((const float*)p + at);
    x.hi = *(const u32x4*)((const float*)p + at + 4);
  }
}
__device__ __forceinline__ float held_value(const Held8& x, int i, bool bf16) {
  const float wide = __uint_as_float(i < 4 ? x.lo[i & 3] : x.hi[i & 3]);
  const uint32_t w = x.lo[i >> 1];
  return bf16 ? __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16) : wide;
}
// values(j, h, v): the eight sums of group h of row of blocks j, this lane's; its output row is m_of(j), its first column n_of(h).
template <int ACT, int ROWS, int G, typename Values, typename MOf, typename NOf>
__device__ __forceinline__ void finish_tile_act(const LinearArgs& a, Values&& values, MOf&& m_of, NOf&& n_of) {
  const bool slope = ACT != FASTCLIP_ACT_NONE && a.pre_in, out_bf16 = a.out_bf16;
  float bias[G][8];
#pragma unroll
  for (int h = 0; h < G; ++h) {
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[h][e] = 0.f;
    if (a.bias) load_f32<8>(bias[h], a.bias + (n_of(h) < a.N ? n_of(h) : a.N - 8));
  }
  constexpr int kAhead = 3;                      // groups
  Held8 extra[kAhead + 1];                       // pre_in or residual: a call has at most one of the two
  auto request = [&](int t) {
    const int64_t m = m_of(t / G) < a.M ? m_of(t / G) : a.M - 1, n = n_of(t % G) < a.N ? n_of(t % G) : a.N - 8;
    if (slope) hold(extra[t % (kAhead + 1)], a.pre_in, m * a.ld_pre + n, true);
    else if (a.residual) hold(extra[t % (kAhead + 1)], a.residual, m * a.ld_res + n, out_bf16);
  };
#pragma unroll
  for (int t = 0; t < kAhead && t < ROWS * G; ++t) request(t);
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    const int64_t m = m_of(j);
    char* out = (char*)a.out + (m * a.ld_out) * (out_bf16 ? 2 : 4);
    bf16_t* pre = (bf16_t*)a.pre_out + m * a.ld_pre;
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const int t = j * G + h;
      if (t + kAhead < ROWS * G) request(t + kAhead);
      const Held8& with = extra[t % (kAhead + 1)];
      const int64_t n = n_of(h);
      float v[8];
      values(j, h, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += bias[h][e];
      const bool in = m < a.M && n < a.N;
      if (a.pre_out && in) store_bf16<8>(pre + n, v);
      if (slope) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= activation_slope<ACT>(held_value(with, e, true));
      } else if constexpr (ACT != FASTCLIP_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = activate<ACT>(v[e]);
      }
      if (a.residual) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += held_value(with, e, out_bf16);
      }
      if (in) {
        if (out_bf16) store_bf16<8>((bf16_t*)out + n, v);
        else store_f32<8>((float*)out + n, v);
      }
      FC_PIN();      // the sums of one group at a time in registers of their own
    }
  }
}
template <bool HAS_ACT, int ROWS, int G, typename Values, typename MOf, typename NOf>
__device__ __forceinline__ void finish_tile(const LinearArgs& a, Values&& values, MOf&& m_of, NOf&& n_of) {
  if (HAS_ACT && a.act == FASTCLIP_ACT_GELU) finish_tile_act<FASTCLIP_ACT_GELU, ROWS, G>(a, values, m_of, n_of);
  else if (HAS_ACT && a.act == FASTCLIP_ACT_QUICK_GELU) finish_tile_act<FASTCLIP_ACT_QUICK_GELU, ROWS, G>(a, values, m_of, n_of);
  else finish_tile_act<FASTCLIP_ACT_NONE, ROWS, G>(a, values, m_of, n_of);
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
