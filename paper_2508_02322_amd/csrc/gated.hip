// What the gradients of the gated block H = silu(X W_gate^T) * (X W_up^T) need beside matrix products:
//   dU = dH silu(G),  dG = dH U silu'(G),  silu'(g) = s (1 + g (1 - s)) with s = 1 / (1 + exp(-g))
// The three products dX = dG W_gate + dU W_up, dW_gate = dG^T X, dW_up = dU^T X run on the grouped contraction, whose operands are
// both K-contiguous.  So dG and dU are written as rows (the left operand of dX, K = channels) and transposed (the left operands
// of dW, K = tokens), and W_gate, W_up and X are transposed; the copies are padded with zeros to whole K tiles.
// All of it is bound by memory.
#include <algorithm>

#include "camera_internal.h"

namespace camera {
namespace {

constexpr int kTile = 64;      // rows and columns of a tile
constexpr int kThreads = 256;

template <class T>
struct Elems;
template <>
struct Elems<float> {
  static constexpr int N = 4;
};
template <>
struct Elems<__bf16> {
  static constexpr int N = 8;
};
template <class T>
struct alignas(16) Chunk {
  T v[Elems<T>::N];
};

// A 64 x 64 tile on its way to its transpose: element (row, col) at [col][row].  A thread puts N columns of a row and takes N rows
// of a column.
template <class T>
struct Turn {
  static constexpr int N = Elems<T>::N;
  static constexpr int kLd = kTile + N;  // 16-byte aligned columns
  T (*cell)[kLd];
  __device__ __forceinline__ void put(int row, int col, const T* v) const {
#pragma unroll
    for (int i = 0; i < N; ++i) cell[col + i][row] = v[i];
  }
  __device__ __forceinline__ Chunk<T> take(int row, int col) const { return *reinterpret_cast<const Chunk<T>*>(&cell[col][row]); }
};

template <class T>
__global__ __launch_bounds__(kThreads) void transpose_kernel(const T* __restrict__ src, int64_t rows, int64_t cols, int64_t lds,
                                                             T* __restrict__ dst, int64_t ldd) {
  constexpr int N = Elems<T>::N, kPer = kTile / N, kStep = kThreads / kPer;
  __shared__ __align__(16) T cell[kTile][Turn<T>::kLd];
  const Turn<T> turn{cell};
  const int64_t r0 = (int64_t)blockIdx.x * kTile, c0 = (int64_t)blockIdx.y * kTile;
  const int at = threadIdx.x % kPer * N;
  for (int r = threadIdx.x / kPer; r < kTile; r += kStep) {
    Chunk<T> v{};
    if (r0 + r < rows && c0 + at < cols) v = *reinterpret_cast<const Chunk<T>*>(src + (r0 + r) * lds + c0 + at);
    turn.put(r, at, v.v);
  }
  __syncthreads();
  for (int c = threadIdx.x / kPer; c < kTile; c += kStep)
    if (c0 + c < cols) *reinterpret_cast<Chunk<T>*>(dst + (c0 + c) * ldd + r0 + at) = turn.take(at, c);
}

template <class T>
__global__ __launch_bounds__(kThreads) void gated_grad_kernel(const float* __restrict__ pre, int64_t pre_ld, const T* __restrict__ dH,
                                                              int64_t lddh, int64_t n, int64_t d_ff, T* __restrict__ rows_out,
                                                              int64_t f_pad, T* __restrict__ cols_out, int64_t n_pad) {
  constexpr int N = Elems<T>::N, kPer = kTile / N, kStep = kThreads / kPer;
  __shared__ __align__(16) T cell[2][kTile][Turn<T>::kLd];
  const Turn<T> turn_g{cell[0]}, turn_u{cell[1]};
  const int64_t r0 = (int64_t)blockIdx.x * kTile, c0 = (int64_t)blockIdx.y * kTile;
  const int at = threadIdx.x % kPer * N;
  const int64_t c = c0 + at;
  for (int r = threadIdx.x / kPer; r < kTile; r += kStep) {
    Chunk<T> dg{}, du{};
    const int64_t row = r0 + r;
    if (row < n && c < d_ff) {  // pre's rows are readable to the next multiple of 8 columns
      const float* g = pre + row * 2 * pre_ld + c;
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const float4 gv = *reinterpret_cast<const float4*>(g + i), uv = *reinterpret_cast<const float4*>(g + pre_ld + i);
        const float gs[4] = {gv.x, gv.y, gv.z, gv.w}, us[4] = {uv.x, uv.y, uv.z, uv.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (c + i + j >= d_ff) continue;
          const float dh = (float)dH[row * lddh + c + i + j];
          const float s = 1.0f / (1.0f + __expf(-gs[j]));
          du.v[i + j] = (T)(dh * (gs[j] * s));
          dg.v[i + j] = (T)(dh * us[j] * (s * fmaf(gs[j], 1.0f - s, 1.0f)));
        }
      }
    }
    if (rows_out != nullptr && row < n && c < f_pad) {
      *reinterpret_cast<Chunk<T>*>(rows_out + row * 2 * f_pad + c) = dg;
      *reinterpret_cast<Chunk<T>*>(rows_out + row * 2 * f_pad + f_pad + c) = du;
    }
    turn_g.put(r, at, dg.v);
    turn_u.put(r, at, du.v);
  }
  if (cols_out == nullptr) return;
  __syncthreads();
  for (int k = threadIdx.x / kPer; k < kTile; k += kStep) {
    if (c0 + k >= d_ff) continue;
    T* out = cols_out + (c0 + k) * n_pad + r0 + at;
    *reinterpret_cast<Chunk<T>*>(out) = turn_g.take(at, k);
    *reinterpret_cast<Chunk<T>*>(out + d_ff * n_pad) = turn_u.take(at, k);
  }
}

__global__ __launch_bounds__(kThreads) void zero_kernel(uint4* __restrict__ dst, int64_t vectors) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * kThreads) dst[i] = uint4{0, 0, 0, 0};
}

int64_t tiles(int64_t x) { return (x + kTile - 1) / kTile; }

template <class T>
hipError_t transpose(hipStream_t stream, const void* src, int64_t rows, int64_t cols, int64_t lds, void* dst, int64_t ldd, int64_t rows_pad) {
  hipLaunchKernelGGL((transpose_kernel<T>), dim3((unsigned)tiles(rows_pad), (unsigned)tiles(cols)), dim3(kThreads), 0, stream,
                     static_cast<const T*>(src), rows, cols, lds, static_cast<T*>(dst), ldd);
  return hipGetLastError();
}
template <class T>
hipError_t gated_grad(hipStream_t stream, const float* pre, int64_t pre_ld, const void* dH, int64_t lddh, int64_t n, int64_t d_ff,
                      void* rows_out, int64_t f_pad, void* cols_out, int64_t n_pad) {
  hipLaunchKernelGGL((gated_grad_kernel<T>), dim3((unsigned)tiles(n_pad), (unsigned)tiles(f_pad)), dim3(kThreads), 0, stream, pre, pre_ld,
                     static_cast<const T*>(dH), lddh, n, d_ff, static_cast<T*>(rows_out), f_pad, static_cast<T*>(cols_out), n_pad);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_transpose(hipStream_t stream, int dtype, const void* src, int64_t rows, int64_t cols, int64_t lds, void* dst,
                            int64_t ldd, int64_t rows_pad) {
  if (rows_pad % kTile != 0 || rows > rows_pad || ldd < rows_pad || tiles(cols) > 65535) return hipErrorInvalidValue;
  return dtype == CAMERA_BF16 ? transpose<__bf16>(stream, src, rows, cols, lds, dst, ldd, rows_pad)
                              : transpose<float>(stream, src, rows, cols, lds, dst, ldd, rows_pad);
}

hipError_t launch_zero(hipStream_t stream, void* dst, int64_t vectors) {
  const int64_t blocks = std::min<int64_t>((vectors + kThreads - 1) / kThreads, 2048);
  hipLaunchKernelGGL(zero_kernel, dim3((unsigned)std::max<int64_t>(blocks, 1)), dim3(kThreads), 0, stream, static_cast<uint4*>(dst), vectors);
  return hipGetLastError();
}

hipError_t launch_gated_grad(hipStream_t stream, int dtype, const float* pre, int64_t pre_ld, const void* dH, int64_t lddh, int64_t n,
                             int64_t d_ff, void* rows_out, int64_t f_pad, void* cols_out, int64_t n_pad) {
  if (f_pad % kTile != 0 || n_pad % kTile != 0 || d_ff > f_pad || n > n_pad || tiles(f_pad) > 65535) return hipErrorInvalidValue;
  return dtype == CAMERA_BF16 ? gated_grad<__bf16>(stream, pre, pre_ld, dH, lddh, n, d_ff, rows_out, f_pad, cols_out, n_pad)
                              : gated_grad<float>(stream, pre, pre_ld, dH, lddh, n, d_ff, rows_out, f_pad, cols_out, n_pad);
}

}  // namespace camera
