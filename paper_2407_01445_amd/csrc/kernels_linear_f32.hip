// Products of linear layers in fp32 (gfx950, wave64, MFMA 32x32x2 f32): the accuracy path of kernels_linear.hip, any width and
// stride.
//
//   out[m, n] = sum_k P[m, k] Q[n, k]
//
// A workgroup of four wavefronts forms a 64 x 64 tile, 32 of k a stage: the next stage comes into registers while the matrix
// cores work on the present one in LDS, guarded, so that what lies outside the matrices is zero.  The order of k inside a stage
// is free as long as both operands keep to it: lanes below 32 take k = 8 s .. 8 s + 3, the others 8 s + 4 .. 8 s + 7, which an
// operand by rows reads as 16 bytes for four products.  P gives the MFMA's rows, so that 32 lanes hold neighbouring columns and
// a store is whole lines whatever the alignment.
#include "linear_common.hpp"

namespace fc {

constexpr int kTile32 = 64, kDepth32 = 32;
constexpr int kRowFloats = 36;      // by rows: 32 of k and 4 more, so that the 16 rows of a read cover the banks
constexpr int kDepthFloats = 72;    // by depth: 64 columns and 8 more, so that rows of k four apart lie in different halves of the banks
constexpr int kPanelFloats = 64 * kRowFloats;     // either layout

template <bool BY_DEPTH>
struct Operand32 {
  const float* base;
  int64_t ld;
  int left;            // rows (columns) of the tile that exist
  bool wide;           // 16-byte loads
  int tid;
  float r[2][4];
  __device__ __forceinline__ void open(const void* matrix, int64_t ld_, int64_t first, int64_t count, int tid_) {
    ld = ld_; tid = tid_;
    base = (const float*)matrix + (BY_DEPTH ? first : first * ld);
    left = (int)(count - first < kTile32 ? count - first : kTile32);
    wide = !((uintptr_t)matrix & 15) && ld % 4 == 0;
  }
  __device__ __forceinline__ void request(int64_t k0, int64_t end) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // four words of this thread: columns c .. c + 3 of line `line` (a row, or a row of k)
      const int line = BY_DEPTH ? (tid >> 4) + 16 * i : (tid >> 3) + 32 * i;
      const int c = BY_DEPTH ? (tid & 15) * 4 : (tid & 7) * 4;
      const float* at = base + (BY_DEPTH ? (k0 + line) * ld + c : line * ld + k0 + c);
      const bool in = BY_DEPTH ? k0 + line < end : line < left;
      const int64_t rest = BY_DEPTH ? left - c : end - k0 - c;      // words from c on that exist
      if (in && wide && rest >= 4) {
        const float4 v = *(const float4*)at;
        r[i][0] = v.x; r[i][1] = v.y; r[i][2] = v.z; r[i][3] = v.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r[i][e] = in && e < rest ? at[e] : 0.f;
      }
    }
  }
  __device__ __forceinline__ void deposit(float* panel) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int line = BY_DEPTH ? (tid >> 4) + 16 * i : (tid >> 3) + 32 * i;
      const int c = BY_DEPTH ? (tid & 15) * 4 : (tid & 7) * 4;
      *(float4*)(panel + line * (BY_DEPTH ? kDepthFloats : kRowFloats) + c) = make_float4(r[i][0], r[i][1], r[i][2], r[i][3]);
    }
  }
  // k = 8 s + 4 h .. + 3 of row (column) `at`
  static __device__ __forceinline__ void read(const float* panel, int at, int h, int s, float (&x)[4]) {
    if constexpr (BY_DEPTH) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = panel[(8 * s + 4 * h + j) * kDepthFloats + at];
    } else {
      const float4 v = *(const float4*)(panel + at * kRowFloats + 8 * s + 4 * h);
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    }
  }
};

template <bool PD, bool QD>
__global__ void __launch_bounds__(256) k_linear_f32(LinearArgs a, uint32_t tiles_m, uint32_t tiles_n, int64_t slice) {
  __shared__ __attribute__((aligned(16))) float panels[2][2][kPanelFloats];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave & 1, wn = wave >> 1, lr = lane & 31, hk = lane >> 5;
  const TilePlace place = tile_place(blockIdx.x, gridDim.x, tiles_m, tiles_n);
  const int64_t m0 = place.m * kTile32, n0 = place.n * kTile32, k0 = place.split * slice;
  const int64_t end = k0 + slice < a.K ? k0 + slice : a.K;
  const int stages = (int)((end - k0 + kDepth32 - 1) / kDepth32);
  Operand32<PD> p;
  Operand32<QD> q;
  p.open(a.p, a.ldp, m0, a.M, tid);
  q.open(a.q, a.ldq, n0, a.N, tid);
  f32x16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.f;
  const bool sums = PD && QD && a.dbias && place.n == 0 && wn == 0;
  float total = 0.f;

  p.request(k0, end);
  q.request(k0, end);
  p.deposit(panels[0][0]);
  q.deposit(panels[0][1]);
  __syncthreads();
  for (int g = 0; g < stages; ++g) {
    const bool more = g + 1 < stages;
    if (more) {
      p.request(k0 + (int64_t)(g + 1) * kDepth32, end);
      q.request(k0 + (int64_t)(g + 1) * kDepth32, end);
    }
    const float* panel_p = panels[g & 1][0];
    const float* panel_q = panels[g & 1][1];
    float some = 0.f;
#pragma unroll
    for (int s = 0; s < kDepth32 / 8; ++s) {
      float x[4], y[4];
      Operand32<PD>::read(panel_p, wm * 32 + lr, hk, s, x);
      Operand32<QD>::read(panel_q, wn * 32 + lr, hk, s, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], y[j], acc, 0, 0, 0);
      if constexpr (PD && QD) some += (x[0] + x[1]) + (x[2] + x[3]);
    }
    total += some;
    if (more) {
      p.deposit(panels[(g + 1) & 1][0]);
      q.deposit(panels[(g + 1) & 1][1]);
    }
    __syncthreads();
  }

  const bool split = gridDim.x > tiles_m * tiles_n;
  if (sums) {
    const float s = total + __shfl_xor(total, 32);
    const int64_t m = m0 + wm * 32 + lr;
    float* to = split ? a.partial + (int64_t)(gridDim.x / (tiles_m * tiles_n)) * a.M * a.N + place.split * a.M : a.dbias;
    if (hk == 0 && m < a.M) to[m] = s;
  }
  const int64_t n = n0 + wn * 32 + lr;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int64_t m = m0 + wm * 32 + 8 * (v >> 2) + 4 * hk + (v & 3);
    if (m < a.M && n < a.N) {
      float z[1] = {acc[v]};
      if (split) a.partial[((int64_t)place.split * a.M + m) * a.N + n] = z[0];
      else finish_values<false, 1>(a, z, m, n);
    }
  }
}

template <bool PD, bool QD>
static void launch_form_f32(const LinearArgs& a, const LinearPlan& plan, hipStream_t s) {
  const uint32_t tm = (uint32_t)((a.M + kTile32 - 1) / kTile32), tn = (uint32_t)((a.N + kTile32 - 1) / kTile32);
  hipLaunchKernelGGL((k_linear_f32<PD, QD>), dim3(tm * tn * (uint32_t)plan.splits), dim3(256), 0, s, a, tm, tn, plan.slice);
}

void launch_linear_f32(const LinearArgs& a, const LinearPlan& plan, hipStream_t s) {
  if (a.p_by_depth) launch_form_f32<true, true>(a, plan, s);
  else if (a.q_by_depth) launch_form_f32<false, true>(a, plan, s);
  else launch_form_f32<false, false>(a, plan, s);
}

}  // namespace fc
