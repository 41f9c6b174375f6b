// Products of linear layers in fp32 (gfx950, wave64, MFMA 32x32x2 f32): the accuracy path of kernels_linear.hip, any width and
// stride.
//
//   out[m, n] = sum_k P[m, k] Q[n, k]
//
// The fp32 matrix cores take 64 cycles for the 128 operand words of a product, so that one wavefront needs little data at a time,
// and wavefronts need not meet: each forms 32 x 32 of the output from LDS of its own, 32 of k (a line of an operand by rows) at a
// time, the next block on its way from memory by direct-to-LDS loads while the present one is multiplied.  Where there are tiles
// enough, a workgroup's four wavefronts have four of them, 64 x 64 in all, and no barrier; where there are few, they share one,
// every fourth block of k each, and add up at the end, each finishing a quarter.  (Operands straight from memory
// into registers instead, as the products want them, fetch 32 bytes of each of 32 lines per load and took twice as long.)  The
// order of k inside a block is free as long as both operands keep to it: lanes below 32 take k = 8 s .. 8 s + 3, the others
// 8 s + 4 .. 8 s + 7, which by rows is one 16-byte read for four products.  P gives the MFMA's rows, so that 32 lanes hold
// neighbouring columns and a store is whole lines whatever the alignment.
//
// Edges: rows beyond M (columns beyond N) repeat the last one, and what they produce is not stored; depth beyond K comes from a
// block of zeros.
//
// Measured on one MI355X: 1000 rows, 760 -> 760, forward with a residual 17 us, 68 TFLOP/s; the matrix cores alone would take 8 us
// for its 768 tiles, three a compute unit, and each of their wavefronts waits for its six blocks one after another.
#include "linear_common.hpp"

namespace fc {

constexpr int kBlock32 = 32;                     // of k
constexpr uint32_t kPanel32 = 32 * 128;          // bytes of 32 rows (columns) of a block
__device__ __align__(16) uint32_t g_zero_f32[4] = {0, 0, 0, 0};

// 4 or 16 bytes per lane from an address of its own into LDS
template <bool WIDE>
__device__ __forceinline__ void dma_from(const void* lane_address, uint32_t lds_byte_addr) {
  if constexpr (WIDE)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 : : "v"(lane_address), "s"(__builtin_amdgcn_readfirstlane(lds_byte_addr)) : "memory");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
                 : : "v"(lane_address), "s"(__builtin_amdgcn_readfirstlane(lds_byte_addr)) : "memory");
}

typedef float Words32[4][4];       // [s][j]: k = 8 s + 4 h + j of a row (column)

// 32 rows (columns) of an operand from `first` on.  LDS image by rows: 128 bytes a row, 16-byte chunk c of
// row r at c ^ ((r >> 1) & 7); by depth: 128 bytes a row of k, row k at k ^ ((k >> 2) & 1), so that the rows k and k + 4 that the
// halves of a wavefront read lie in different halves of the banks.  WIDE: 16 bytes a lane and load, else 4.
template <bool BY_DEPTH, bool WIDE>
struct Operand32 {
  static constexpr int kLoads = WIDE ? 4 : 16;     // wave loads of a block of k
  const char* base;
  int64_t line;                    // bytes from one row (row of k) to the next
  uint32_t off[kLoads];            // this lane's bytes from there at depth 0
  int lane;
  // k of this lane's (first) word of load i, inside a block
  __device__ __forceinline__ int depth_of(int i) const {
    const int r = WIDE ? 8 * i + (lane >> 3) : 2 * i + (lane >> 5);
    if constexpr (BY_DEPTH) return r ^ ((r >> 2) & 1);
    if constexpr (WIDE) return 4 * ((lane & 7) ^ ((r >> 1) & 7));
    return 4 * (((lane >> 2) & 7) ^ ((r >> 1) & 7)) + (lane & 3);
  }
  __device__ __forceinline__ void open(const void* matrix, int64_t ld, int64_t first, int64_t count, int lane_) {
    line = ld * 4; lane = lane_;
    base = (const char*)matrix + (BY_DEPTH ? first * 4 : first * line);
    const int left = (int)(count - first < 32 ? count - first : 32);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int r;                       // row, or column (the first of four)
      if constexpr (BY_DEPTH) {
        r = WIDE ? 4 * (lane & 7) : lane & 31;
        r = r < left ? r : left - (WIDE ? 4 : 1);
        off[i] = (uint32_t)depth_of(i) * (uint32_t)line + (uint32_t)r * 4u;
      } else {
        r = WIDE ? 8 * i + (lane >> 3) : 2 * i + (lane >> 5);
        r = r < left ? r : left - 1;
        off[i] = (uint32_t)r * (uint32_t)line + (uint32_t)depth_of(i) * 4u;
      }
    }
  }
  // requests the block of k from k0 on (wave-uniform)
  __device__ __forceinline__ void request(int64_t k0, int64_t end, uint32_t lds) const {
    const char* at = wave_uniform(base + (BY_DEPTH ? k0 * line : k0 * 4));
    constexpr uint32_t kStep = WIDE ? 1024 : 256;
    if (k0 + kBlock32 <= end) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if constexpr (WIDE) dma16(at, off[i], lds + (uint32_t)i * kStep);
        else dma4(at, off[i], lds + (uint32_t)i * kStep);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        dma_from<WIDE>(k0 + depth_of(i) < end ? at + off[i] : (const char*)g_zero_f32, lds + (uint32_t)i * kStep);
    }
  }
  static __device__ __forceinline__ void read(Words32& x, const char* panel, int lr, int h) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if constexpr (BY_DEPTH) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = 8 * s + 4 * h + j;
          x[s][j] = *(const float*)(panel + (k ^ ((k >> 2) & 1)) * 128 + lr * 4);
        }
      } else {
        const float4 v = *(const float4*)(panel + lr * 128 + (((2 * s + h) ^ ((lr >> 1) & 7)) << 4));
        x[s][0] = v.x; x[s][1] = v.y; x[s][2] = v.z; x[s][3] = v.w;
      }
    }
  }
};

// SHARED: the four wavefronts share a tile.
template <bool PD, bool QD, bool WIDE, bool SHARED>
__global__ void __launch_bounds__(256) k_linear_f32(LinearArgs a, uint32_t rows, uint32_t cols, int splits, int64_t slice) {
  typedef Operand32<PD, WIDE> OpP;
  typedef Operand32<QD, WIDE> OpQ;
  constexpr uint32_t kBuffer = 2 * kPanel32;
  constexpr int kRequests = OpP::kLoads + OpQ::kLoads;
  // Per wavefront the blocks on their way, then the parts of the sums.  A shared tile's wavefront has one: a block is in registers
  // before the next takes its place, and four workgroups instead of two share a compute unit and cover the wait (1000 rows of 760
  // -> 760 19.6 -> 15.7 us).  Requests of single words hold registers for two only, and want two blocks (a weight's gradient of 650 x
  // 600 from 8000 rows 84 us, 91 with one).
  constexpr bool kOne = SHARED && WIDE;
  constexpr int kBuffers = kOne ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) char ring[4 * kBuffers * kBuffer];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 31, hk = lane >> 5;
  const TilePlace place = tile_place(blockIdx.x, gridDim.x, rows, cols);
  const int64_t m0 = SHARED ? place.m * 32 : place.m * 64 + 32 * (wave & 1), n0 = SHARED ? place.n * 32 : place.n * 64 + 32 * (wave >> 1);
  if (!SHARED && (m0 >= a.M || n0 >= a.N)) return;
  const int64_t k0 = place.split * slice, end = k0 + slice < a.K ? k0 + slice : a.K;
  OpP p;
  OpQ q;
  p.open(a.p, a.ldp, m0, a.M, lane);
  q.open(a.q, a.ldq, n0, a.N, lane);
  f32x16 acc[2];               // two chains of sums: a product does not wait for the one in front
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
  const bool sums = PD && QD && a.dbias && n0 == 0;           // this tile also sums P over the depth
  float total = 0.f;

  constexpr int64_t kStep = (SHARED ? 4 : 1) * kBlock32;
  const char* mine = ring + wave * kBuffers * kBuffer;
  const uint32_t mine_at = lds_addr(mine);
  auto request = [&](int64_t k, uint32_t buffer) {
    p.request(k, end, mine_at + buffer);
    q.request(k, end, mine_at + buffer + kPanel32);
  };
  uint32_t here = 0;
  const int64_t first = k0 + (SHARED ? wave * kBlock32 : 0);
  if (first < end) request(first, 0);
  for (int64_t k = first; k < end; k += kStep) {
    if (!kOne && k + kStep < end) {
      request(k + kStep, here ^ kBuffer);
      wait_vmcnt<kRequests>();                   // the older block's have landed
    } else {
      FC_WAIT_VMCNT0();
    }
    FC_FENCE();
    __builtin_amdgcn_wave_barrier();
    Words32 x, y;
    OpP::read(x, mine + here, lr, hk);
    OpQ::read(y, mine + here + kPanel32, lr, hk);
    if constexpr (kOne) {                        // the block is in registers: the next takes its place
      FC_FENCE();
      __builtin_amdgcn_s_waitcnt(0xc07f);        // lgkmcnt 0
      __builtin_amdgcn_wave_barrier();
      FC_FENCE();
      if (k + kStep < end) request(k + kStep, 0);
      FC_FENCE();
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j & 1] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[s][j], y[s][j], acc[j & 1], 0, 0, 0);
    if constexpr (PD && QD) {
      if (sums) {
        float some = 0.f;
#pragma unroll
        for (int s = 0; s < 4; ++s) some += (x[s][0] + x[s][1]) + (x[s][2] + x[s][3]);
        total += some;
      }
    }
    if constexpr (!kOne) {
      FC_FENCE();                                // the block's reads are over before the next request takes its place
      __builtin_amdgcn_wave_barrier();
      here ^= kBuffer;
    }
  }

  float* bias_to = splits > 1 ? a.partial + (int64_t)splits * a.M * a.N + (int64_t)place.split * a.M : a.dbias;
  const int64_t n = n0 + lr;
  const bool in = n < a.N;
  const float bias = a.bias && in ? a.bias[n] : 0.f;
  if constexpr (!SHARED) {
    if (sums) {
      total += __shfl_xor(total, 32);
      if (hk == 0 && m0 + lr < a.M) bias_to[m0 + lr] = total;
    }
    auto row_of = [&](int v) { return m0 + 8 * (v >> 2) + 4 * hk + (v & 3); };
    float extra[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) extra[v] = splits == 1 && in && row_of(v) < a.M ? single_extra(a, row_of(v), n) : 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int64_t m = row_of(v);
      if (in && m < a.M) {
        if (splits > 1) a.partial[((int64_t)place.split * a.M + m) * a.N + n] = acc[0][v] + acc[1][v];
        else finish_single(a, acc[0][v] + acc[1][v], bias, extra[v], m, n);
      }
    }
  } else {
    __syncthreads();
    float(*parts)[16][64] = (float(*)[16][64])ring;
    if (sums) {
      parts[wave][0][lane] = total + __shfl_xor(total, 32);
      __syncthreads();
      if (tid < 32 && m0 + tid < a.M)
        bias_to[m0 + tid] = (parts[0][0][tid] + parts[1][0][tid]) + (parts[2][0][tid] + parts[3][0][tid]);
      __syncthreads();
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) parts[wave][v][lane] = acc[0][v] + acc[1][v];
    __syncthreads();
    // this wavefront finishes the accumulators number v with v mod 4 its own
    auto row_of = [&](int t) { return m0 + 8 * t + 4 * hk + wave; };
    float extra[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) extra[t] = splits == 1 && in && row_of(t) < a.M ? single_extra(a, row_of(t), n) : 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int v = 4 * t + wave;
      const int64_t m = row_of(t);
      const float z = (parts[0][v][lane] + parts[1][v][lane]) + (parts[2][v][lane] + parts[3][v][lane]);
      if (in && m < a.M) {
        if (splits > 1) a.partial[((int64_t)place.split * a.M + m) * a.N + n] = z;
        else finish_single(a, z, bias, extra[t], m, n);
      }
    }
  }
}

// 16-byte loads: aligned lines of whole words, also at an operand's edges (by rows the depth, by depth the columns)
static bool wide_f32(const void* p, int64_t ld, int64_t width) { return !((uintptr_t)p & 15) && ld % 4 == 0 && width % 4 == 0; }

template <bool PD, bool QD>
static void launch_form_f32(const LinearArgs& a, const LinearPlan& plan, hipStream_t s) {
  const uint32_t rows = (uint32_t)((a.M + plan.tile - 1) / plan.tile), cols = (uint32_t)((a.N + plan.tile - 1) / plan.tile);
  const dim3 grid(rows * cols * (uint32_t)plan.splits);
  const bool wide = wide_f32(a.p, a.ldp, PD ? a.M : a.K) && wide_f32(a.q, a.ldq, QD ? a.N : a.K);
#define FC_F32(WIDE, SHARED) \
  hipLaunchKernelGGL((k_linear_f32<PD, QD, WIDE, SHARED>), grid, dim3(256), 0, s, a, rows, cols, plan.splits, plan.slice)
  if (plan.tile == 32) {
    if (wide) FC_F32(true, true);
    else FC_F32(false, true);
  } else {
    if (wide) FC_F32(true, false);
    else FC_F32(false, false);
  }
#undef FC_F32
}

void launch_linear_f32(const LinearArgs& a, const LinearPlan& plan, hipStream_t s) {
  if (a.p_by_depth) launch_form_f32<true, true>(a, plan, s);
  else if (a.q_by_depth) launch_form_f32<false, true>(a, plan, s);
  else launch_form_f32<false, false>(a, plan, s);
}

}  // namespace fc
