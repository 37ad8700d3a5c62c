// The gated block H = silu(X W_gate^T) * (X W_up^T) for few tokens, and what its gradients need beside matrix products:
//   dU = dH silu(G),  dG = dH U silu'(G),  silu'(g) = s (1 + g (1 - s)) with s = 1 / (1 + exp(-g))
// The three products dX = dG W_gate + dU W_up, dW_gate = dG^T X, dW_up = dU^T X run on the grouped contraction, whose operands are
// both K-contiguous.  So dG and dU are written as rows (the left operand of dX, K = channels) and transposed (the left operands
// of dW, K = tokens), and W_gate, W_up and X are transposed; the copies are padded with zeros to whole K tiles.
// What this file does itself is bound by memory, the products by the matrix pipe.  8192 tokens, 20480 x 3584: the operands 857 us for
// 3.7 GB (4.3 TB/s; pieces of 128 bytes in rows far apart: with tiles of 128 x 64 780 us, but 19 us instead of 14 where a block is
// small), the products 1.63 and 1.59 ms (1.47 and 1.51 PFLOP/s), the forward product 1.66 ms, with the projections kept in float32
// (1.34 GB more) 1.85, between the others 1.91.  Kept as bf16 they would be half of that, and every gradient would carry two roundings more.
// bf16: dG and dU are rounded, half a step, because the matrix instructions take no wider operand: gradients are 0.0023 off in the
// 2-norm where the final rounding alone makes 0.0017.  As a sum of two bf16 each they would not be, in twice the K of every product.
#include <algorithm>

#include "camera_internal.h"

namespace camera {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kTile = 64;      // rows and columns of a tile
constexpr int kThreads = 256;

// exp2 and rcp are single hardware instructions (about 1 ulp each)
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
}

// ---- operands of the backward pass ---------------------------------------------------------------------------------
template <class T>
struct alignas(16) Chunk {
  static constexpr int N = 16 / sizeof(T);
  T v[N];
};

// A 64 x 64 tile on its way to its transpose: element (row, col) at [col][row].  A thread puts N columns of a row and takes N rows
// of a column.
template <class T>
struct Turn {
  static constexpr int N = Chunk<T>::N;
  static constexpr int kLd = kTile + N;  // 16-byte aligned columns
  T (*cell)[kLd];
  __device__ __forceinline__ void put(int row, int col, const T* v) const {
#pragma unroll
    for (int i = 0; i < N; ++i) cell[col + i][row] = v[i];
  }
  __device__ __forceinline__ Chunk<T> take(int row, int col) const { return *reinterpret_cast<const Chunk<T>*>(&cell[col][row]); }
};
template <class T>
using Cells = T[2][kTile][Turn<T>::kLd];

// dst[c][r] = src[r][c] of one tile; zero for r >= rows.  dst's rows are whole tiles long.
template <class T>
__device__ __forceinline__ void transpose_tile(const T* src, int64_t rows, int64_t cols, int64_t lds, T* dst, int64_t ldd, int64_t r0,
                                               int64_t c0, Cells<T>& cells) {
  constexpr int N = Chunk<T>::N, kPer = kTile / N, kStep = kThreads / kPer;
  const Turn<T> turn{cells[0]};
  const int at = threadIdx.x % kPer * N;
#pragma unroll
  for (int r = threadIdx.x / kPer; r < kTile; r += kStep) {
    Chunk<T> v{};
    if (r0 + r < rows && c0 + at < cols) v = *reinterpret_cast<const Chunk<T>*>(src + (r0 + r) * lds + c0 + at);
    turn.put(r, at, v.v);
  }
  __syncthreads();
#pragma unroll
  for (int c = threadIdx.x / kPer; c < kTile; c += kStep)
    if (c0 + c < cols) *reinterpret_cast<Chunk<T>*>(dst + (c0 + c) * ldd + r0 + at) = turn.take(at, c);
}

// N values of a row that may start at any element, `left` of them there (zeros behind).
template <class T>
__device__ __forceinline__ Chunk<T> load_ragged(const T* p, int64_t left) {
  Chunk<T> v{};
  if (left >= Chunk<T>::N) {
    __builtin_memcpy(&v, p, sizeof(v));
  } else {
    for (int i = 0; i < left; ++i) v.v[i] = p[i];
  }
  return v;
}

template <class T>
__device__ __forceinline__ void gradient_tile(const GatedOperands& a, int64_t r0, int64_t c0, Cells<T>& cells) {
  constexpr int N = Chunk<T>::N, kPer = kTile / N, kStep = kThreads / kPer;
  const Turn<T> turn_g{cells[0]}, turn_u{cells[1]};
  const int at = threadIdx.x % kPer * N;
  const int64_t c = c0 + at;
  T* rows = static_cast<T*>(a.rows);
#pragma unroll
  for (int r = threadIdx.x / kPer; r < kTile; r += kStep) {
    Chunk<T> dg{}, du{};
    const int64_t row = r0 + r;
    if (row < a.n && c < a.d_ff) {  // pre's rows are readable to the next multiple of 8 columns
      const float* g = a.pre + row * 2 * a.pre_ld + c;
      const Chunk<T> dh = load_ragged(static_cast<const T*>(a.dH) + row * a.lddh + c, a.d_ff - c);
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const f32x4 gs = *reinterpret_cast<const f32x4*>(g + i), us = *reinterpret_cast<const f32x4*>(g + a.pre_ld + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (c + i + j >= a.d_ff) continue;
          const float d = (float)dh.v[i + j], s = sigmoid(gs[j]);
          du.v[i + j] = (T)(d * (gs[j] * s));
          dg.v[i + j] = (T)(d * us[j] * (s * fmaf(gs[j], 1.0f - s, 1.0f)));
        }
      }
    }
    if (rows != nullptr && row < a.n) {
      *reinterpret_cast<Chunk<T>*>(rows + row * 2 * a.f_pad + c) = dg;
      *reinterpret_cast<Chunk<T>*>(rows + row * 2 * a.f_pad + a.f_pad + c) = du;
    }
    turn_g.put(r, at, dg.v);
    turn_u.put(r, at, du.v);
  }
  if (a.cols == nullptr) return;
  __syncthreads();
#pragma unroll
  for (int k = threadIdx.x / kPer; k < kTile; k += kStep) {
    if (c0 + k >= a.d_ff) continue;
    T* out = static_cast<T*>(a.cols) + (c0 + k) * a.n_pad + r0 + at;
    *reinterpret_cast<Chunk<T>*>(out) = turn_g.take(at, k);
    *reinterpret_cast<Chunk<T>*>(out + a.d_ff * a.n_pad) = turn_u.take(at, k);
  }
}

// Tiles of the four matrices, one workgroup each: dG and dU, W_gate, W_up, X.
struct OperandTiles {
  int64_t gradient, weight, x;  // of each
};
__host__ __device__ __forceinline__ OperandTiles operand_tiles(const GatedOperands& a) {
  const int64_t d = (a.d_model + kTile - 1) / kTile;
  return {a.n_pad / kTile * (a.f_pad / kTile), a.w_t != nullptr ? a.f_pad / kTile * d : 0, a.x_t != nullptr ? a.n_pad / kTile * d : 0};
}
template <class T>
__global__ __launch_bounds__(kThreads) void gated_operands_kernel(GatedOperands a) {
  __shared__ __align__(16) Cells<T> cells;
  const OperandTiles tiles = operand_tiles(a);
  int64_t id = linear_block();
  const int64_t across_n = a.n_pad / kTile, across_f = a.f_pad / kTile;
  if (id < tiles.gradient) return gradient_tile<T>(a, id % across_n * kTile, id / across_n * kTile, cells);
  id -= tiles.gradient;
  if (id < 2 * tiles.weight) {
    const bool up = id >= tiles.weight;
    if (up) id -= tiles.weight;
    T* dst = static_cast<T*>(a.w_t) + (up ? a.f_pad : 0);
    return transpose_tile<T>(static_cast<const T*>(up ? a.W_up : a.W_gate), a.d_ff, a.d_model, a.d_model, dst, 2 * a.f_pad,
                             id % across_f * kTile, id / across_f * kTile, cells);
  }
  id -= 2 * tiles.weight;
  if (id < tiles.x)
    transpose_tile<T>(static_cast<const T*>(a.X), a.n, a.d_model, a.ldx, static_cast<T*>(a.x_t), a.n_pad, id % across_n * kTile,
                      id / across_n * kTile, cells);
}

// Four columns a thread, a row (of all groups) or more a workgroup.
template <class T>
__global__ __launch_bounds__(kThreads) void sum_parts_kernel(const float* __restrict__ part, int parts, int64_t part_stride, int64_t rows,
                                                             int64_t group_rows, int64_t cols, T* __restrict__ out, int64_t ld,
                                                             int64_t expert_gap) {
  const int64_t quads = cols / 4;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * quads; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / quads, c = (i - row * quads) * 4;
    f32x4 sum = *reinterpret_cast<const f32x4*>(part + row * cols + c);
    for (int p = 1; p < parts; ++p) sum += *reinterpret_cast<const f32x4*>(part + p * part_stride + row * cols + c);
    struct alignas(4 * sizeof(T)) Quad {
      T v[4];
    } q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q.v[j] = (T)sum[j];
    *reinterpret_cast<Quad*>(out + row / group_rows * expert_gap + row * ld + c) = q;
  }
}

__global__ __launch_bounds__(kThreads) void zero_kernel(uint4* __restrict__ dst, int64_t vectors) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * kThreads) dst[i] = uint4{0, 0, 0, 0};
}

// ---- few tokens ----------------------------------------------------------------------------------------------------
// Bound by reading the weights once: a workgroup has 16 channels, its eight waves an eighth of K each, and a wave loads the
// operands of kSteps matrix instructions of K = 32 before it multiplies.  Lane 16 q + r holds K elements [8 q, 8 q + 8) of row r:
// the weights are the left operand (16 channels), the tokens the right one (NT tiles of 16).  The waves' partial sums meet in LDS
// and are added in wave order.  One token: 2560 x 3584 10.3 us (3.6 TB/s, 160 workgroups, all of their loads in flight at once),
// 14336 x 4096 41 us (5.7 TB/s; small tiles 35).
constexpr int kRowsWaves = 8;
constexpr int kChannels = 16;

template <int NT>
__global__ __launch_bounds__(kRowsWaves * kWave) void gated_rows_kernel(const __bf16* __restrict__ X, int64_t ldx, int n, int d_model,
                                                                        const __bf16* __restrict__ W_gate,
                                                                        const __bf16* __restrict__ W_up, int64_t d_ff,
                                                                        __bf16* __restrict__ H, int64_t ldh, float* __restrict__ pre,
                                                                        int64_t pre_ld) {
  constexpr int kSteps = NT == 1 ? 8 : 4;
  __shared__ float red[kRowsWaves][2][4][kWave];
  const int tid = threadIdx.x, lane = tid % kWave, r = lane % 16, q = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int64_t c0 = (int64_t)blockIdx.x * kChannels;
  const int64_t c = min(c0 + r, d_ff - 1);  // rows past the end read the last one again
  const int steps = (d_model + 31) / 32, first = steps * wave / kRowsWaves, last = steps * (wave + 1) / kRowsWaves;
  const __bf16 *g = W_gate + c * d_model + 8 * q, *u = W_up + c * d_model + 8 * q;
  const __bf16* x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) x[t] = X + (int64_t)min(16 * t + r, n - 1) * ldx + 8 * q;
  f32x4 acc_g[NT] = {}, acc_u[NT] = {};
  for (int s0 = first; s0 < last; s0 += kSteps) {
    bf16x8 ag[kSteps] = {}, au[kSteps] = {}, b[kSteps][NT] = {};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int k = 32 * (s0 + i);
      if (s0 + i < last && k + 8 * q < d_model) {  // d_model is a multiple of 8: a lane's eight elements are all there or none
        ag[i] = *reinterpret_cast<const bf16x8*>(g + k);
        au[i] = *reinterpret_cast<const bf16x8*>(u + k);
#pragma unroll
        for (int t = 0; t < NT; ++t) b[i][t] = *reinterpret_cast<const bf16x8*>(x[t] + k);
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc_g[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ag[i], b[i][t], acc_g[t], 0, 0, 0);
        acc_u[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(au[i], b[i][t], acc_u[t], 0, 0, 0);
      }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t > 0) __syncthreads();  // the previous tile's sums have been read
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // accumulator element e: channel 4 q + e, token r
      red[wave][0][e][lane] = acc_g[t][e];
      red[wave][1][e][lane] = acc_u[t][e];
    }
    __syncthreads();
    const int channel = tid % 16, token = tid / 16;
    if (token < 16 && 16 * t + token < n) {
      const int from = channel / 4 * 16 + token;
      float sg = 0.0f, su = 0.0f;
#pragma unroll
      for (int w = 0; w < kRowsWaves; ++w) {
        sg += red[w][0][channel % 4][from];
        su += red[w][1][channel % 4][from];
      }
      const int64_t at = c0 + channel, row = 16 * t + token;
      const bool inside = at < d_ff;
      if (H != nullptr && at < ((d_ff + 7) & ~(int64_t)7)) H[row * ldh + at] = (__bf16)(inside ? sg * sigmoid(sg) * su : 0.0f);
      if (pre != nullptr && inside) {
        pre[row * 2 * pre_ld + at] = sg;
        pre[row * 2 * pre_ld + pre_ld + at] = su;
      }
    }
  }
}

}  // namespace

hipError_t launch_gated_operands(hipStream_t stream, int dtype, const GatedOperands& a) {
  if (a.f_pad % kTile != 0 || a.n_pad % kTile != 0 || a.d_ff > a.f_pad || a.n > a.n_pad) return hipErrorInvalidValue;
  const OperandTiles tiles = operand_tiles(a);
  const int64_t blocks = tiles.gradient + 2 * tiles.weight + tiles.x;
  if (blocks >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  if (dtype == CAMERA_BF16) hipLaunchKernelGGL((gated_operands_kernel<__bf16>), launch_grid(blocks), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((gated_operands_kernel<float>), launch_grid(blocks), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_sum_parts(hipStream_t stream, int dtype, const float* part, int parts, int64_t part_stride, int groups, int64_t group_rows,
                            int64_t cols, void* out, int64_t ld, int64_t expert_gap) {
  const int64_t rows = groups * group_rows;
  const int64_t blocks = std::min<int64_t>((rows * (cols / 4) + kThreads - 1) / kThreads, 8192);
  if (blocks < 1 || cols % 4 != 0) return hipErrorInvalidValue;
  if (dtype == CAMERA_BF16)
    hipLaunchKernelGGL((sum_parts_kernel<__bf16>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, part, parts, part_stride, rows,
                       group_rows, cols, static_cast<__bf16*>(out), ld, expert_gap);
  else
    hipLaunchKernelGGL((sum_parts_kernel<float>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, part, parts, part_stride, rows,
                       group_rows, cols, static_cast<float*>(out), ld, expert_gap);
  return hipGetLastError();
}

hipError_t launch_zero(hipStream_t stream, void* dst, int64_t vectors) {
  const int64_t blocks = std::min<int64_t>((vectors + kThreads - 1) / kThreads, 2048);
  hipLaunchKernelGGL(zero_kernel, dim3((unsigned)std::max<int64_t>(blocks, 1)), dim3(kThreads), 0, stream, static_cast<uint4*>(dst), vectors);
  return hipGetLastError();
}

hipError_t launch_gated_rows(hipStream_t stream, const void* X, int64_t ldx, int64_t n, int64_t d_model, const void* W_gate,
                             const void* W_up, int64_t d_ff, void* H, int64_t ldh, float* pre, int64_t pre_ld) {
  if (n < 1 || n > kGatedRowsMost) return hipErrorInvalidValue;
  auto kern = n <= 16 ? gated_rows_kernel<1> : n <= 32 ? gated_rows_kernel<2> : gated_rows_kernel<4>;
  static_assert(kGatedRowsMost == 64, "four tiles of tokens");
  hipLaunchKernelGGL(kern, dim3((unsigned)((d_ff + kChannels - 1) / kChannels)), dim3(kRowsWaves * kWave), 0, stream,
                     static_cast<const __bf16*>(X), ldx, (int)n, (int)d_model, static_cast<const __bf16*>(W_gate),
                     static_cast<const __bf16*>(W_up), d_ff, static_cast<__bf16*>(H), ldh, pre, pre_ld);
  return hipGetLastError();
}

}  // namespace camera
