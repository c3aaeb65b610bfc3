// Elementwise kernels around the products of netmax_product.cuh: operands laid out for the tensor cores, column sums, norms and
// momentum.  All of them are bound by memory; sums are taken in a fixed order, so results do not change from run to run.
#pragma once
#include "netmax_product.cuh"

namespace netmax {

constexpr int kElementThreads = 256;
constexpr int kMaxParts = 64;       // partial maxima of a matrix
constexpr int kPiece = 4096;        // elements of a replica that one CTA of the step's kernels works on
constexpr int kSumRows = 256;       // rows of a part of a column sum

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double parts[kElementThreads / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kElementThreads / 32; ++w) s += parts[w];
  return s;
}
__device__ __forceinline__ float block_max(float v) {
  __shared__ float parts[kElementThreads / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  __syncthreads();
  if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int w = 0; w < kElementThreads / 32; ++w) s = fmaxf(s, parts[w]);
  return s;
}

// An operand on its way to the tensor cores: `count` matrices of rows x cols; with z, dy act'(z).
struct OperandJob {
  const void* src = nullptr;
  int64_t row = 0, batch = 0;
  const void* z = nullptr;
  int64_t z_row = 0, z_batch = 0;
  int32_t activation = 0;
  int32_t rows = 0, cols = 0, count = 0, parts = 0;
  void* dst = nullptr;
  int64_t dst_row = 0, dst_batch = 0, dst_plane = 0;
  float* maxima = nullptr;  // [count][parts]
  int32_t* exponent = nullptr;
};
struct OperandParams {
  OperandJob job[3];
  unsigned int* error = nullptr;
  int32_t clear_error = 0;
};

template <typename T>
__device__ __forceinline__ float operand_value(const OperandJob& j, int q, uint32_t row, uint32_t col) {
  float v = (float)((const T*)j.src)[q * j.batch + row * j.row + col];
  if (j.z) v *= activation_slope((float)((const T*)j.z)[q * j.z_batch + row * j.z_row + col], j.activation);
  return v;
}

// Largest finite magnitude of every matrix, in parts.
__global__ __launch_bounds__(kElementThreads) void operand_maxima_kernel(const __grid_constant__ OperandParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *p.error = 0;
  const OperandJob& j = p.job[blockIdx.z];
  if ((int)blockIdx.x >= j.parts) return;
  const uint32_t total = (uint32_t)j.rows * (uint32_t)j.cols, cols = (uint32_t)j.cols;
  for (int q = blockIdx.y; q < j.count; q += gridDim.y) {
    float most = 0.0f;
    for (uint32_t e = blockIdx.x * kElementThreads + threadIdx.x; e < total; e += (uint32_t)j.parts * kElementThreads) {
      const uint32_t row = e / cols;
      const float v = fabsf(operand_value<float>(j, q, row, e - row * cols));
      if (v <= 3.402823466e38f) most = fmaxf(most, v);
    }
    most = block_max(most);
    if (threadIdx.x == 0) j.maxima[q * j.parts + blockIdx.x] = most;
  }
}

// fp32 as two fp16 planes of the values times a power of two that brings the largest to [2^14, 2^15); bfloat16 as it is.
template <typename T>
__global__ __launch_bounds__(kElementThreads) void operand_kernel(const __grid_constant__ OperandParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *p.error = 0;
  const OperandJob& j = p.job[blockIdx.z];
  const uint32_t total = (uint32_t)j.rows * (uint32_t)j.cols, cols = (uint32_t)j.cols;
  for (int q = blockIdx.y; q < j.count; q += gridDim.y) {
    int exponent = 0;
    if (sizeof(T) == 4) {
      float most = 0.0f;
      for (int k = threadIdx.x; k < j.parts; k += kElementThreads) most = fmaxf(most, j.maxima[q * j.parts + k]);
      most = block_max(most);
      if (most > 0.0f) exponent = min(14 - ilogbf(most), 126);  // (from 2^-112 on the largest lies lower; such values vanish beside any bias)
      if (blockIdx.x == 0 && threadIdx.x == 0) j.exponent[q] = exponent;
    }
    const float scale = ldexpf(1.0f, exponent);
    for (uint32_t e = blockIdx.x * kElementThreads + threadIdx.x; e < total; e += gridDim.x * kElementThreads) {
      const uint32_t row = e / cols, col = e - row * cols;
      const float v = operand_value<T>(j, q, row, col);
      const int64_t at = q * j.dst_batch + row * j.dst_row + col;
      if (sizeof(T) == 4) {
        __half hi, lo;
        split(v * scale, hi, lo);
        ((__half*)j.dst)[at] = hi;
        ((__half*)j.dst)[at + j.dst_plane] = lo;
      } else {
        ((__nv_bfloat16*)j.dst)[at] = __float2bfloat16_rn(v);
      }
    }
  }
}

// Column sums of dy act'(z): parts of kSumRows rows each, 64 columns per CTA, four rows at a time.
template <typename T>
__global__ __launch_bounds__(kElementThreads) void column_sums_kernel(const __grid_constant__ OperandJob j, float* parts, int n_parts, unsigned int* clear) {
  __shared__ float sums[4][64];
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (clear && blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *clear = 0;
  const int lane = threadIdx.x % 64, group = threadIdx.x / 64, col = blockIdx.x * 64 + lane;
  for (int q = blockIdx.z; q < j.count; q += gridDim.z) {
    for (int part = blockIdx.y; part < n_parts; part += gridDim.y) {
      const int first = part * kSumRows, last = min(j.rows, first + kSumRows);
      float s = 0.0f;
      if (col < j.cols)
        for (int row = first + group; row < last; row += 4) s += operand_value<T>(j, q, row, col);
      sums[group][lane] = s;
      __syncthreads();
      if (group == 0 && col < j.cols) parts[((int64_t)q * n_parts + part) * j.cols + col] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
      __syncthreads();
    }
  }
}
template <typename T>
__global__ __launch_bounds__(kElementThreads) void column_totals_kernel(const float* parts, int n_parts, int cols, int count, T* out, int64_t batch) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  const int64_t total = (int64_t)count * cols;
  for (int64_t e = (int64_t)blockIdx.x * kElementThreads + threadIdx.x; e < total; e += (int64_t)gridDim.x * kElementThreads) {
    const int64_t q = e / cols, col = e - q * cols;
    double s = 0.0;
    for (int k = 0; k < n_parts; ++k) s += (double)parts[(q * n_parts + k) * cols + col];
    out[q * batch + col] = (T)(float)s;
  }
}

// ---- Newton-Schulz: norms and the first iterate ------------------------------------------------
struct NormParams {  // `count` matrices of rows x cols on their own
  const void* u = nullptr;
  int64_t row = 0, batch = 0;
  int32_t rows = 0, cols = 0, count = 0, pieces = 0;
  double* parts = nullptr;  // [count][pieces] sums of squares
  __half* planes = nullptr;
  int64_t dst_row = 0, dst_batch = 0, dst_plane = 0;
  unsigned int* error = nullptr;
  int32_t clear_error = 0;
};
__device__ __forceinline__ void first_iterate(float u, double inverse, __half* at, int64_t plane) {
  __half hi, lo;
  split((float)((double)u * inverse), hi, lo);
  at[0] = hi;
  at[plane] = lo;
}
// 2^14 / norm; 0 for a matrix of zeros.  A norm that is not finite makes the whole matrix NaN, as the products would.
__device__ __forceinline__ double inverse_norm(double squares) {
  if (squares == 0.0) return 0.0;
  if (!(squares <= 1.7e308)) return squares - squares;
  return (double)kPlaneScale / sqrt(squares);
}

template <typename T>
__global__ __launch_bounds__(kElementThreads) void norm_parts_kernel(const __grid_constant__ NormParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *p.error = 0;
  const uint32_t total = (uint32_t)p.rows * (uint32_t)p.cols, cols = (uint32_t)p.cols;
  for (int q = blockIdx.y; q < p.count; q += gridDim.y) {
    double s = 0.0;
    const uint32_t first = blockIdx.x * kPiece, last = min(total, first + kPiece);
    for (uint32_t e = first + threadIdx.x; e < last; e += kElementThreads) {
      const uint32_t row = e / cols;
      const double v = (double)(float)((const T*)p.u)[q * p.batch + row * p.row + (e - row * cols)];
      s += v * v;
    }
    s = block_sum(s);
    if (threadIdx.x == 0) p.parts[(int64_t)q * p.pieces + blockIdx.x] = s;
  }
}
template <typename T>
__global__ __launch_bounds__(kElementThreads) void first_iterate_kernel(const __grid_constant__ NormParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  const uint32_t total = (uint32_t)p.rows * (uint32_t)p.cols, cols = (uint32_t)p.cols;
  for (int q = blockIdx.y; q < p.count; q += gridDim.y) {
    double s = 0.0;
    for (int k = threadIdx.x; k < p.pieces; k += kElementThreads) s += p.parts[(int64_t)q * p.pieces + k];
    const double inverse = inverse_norm(block_sum(s));
    const uint32_t first = blockIdx.x * kPiece, last = min(total, first + kPiece);
    for (uint32_t e = first + threadIdx.x; e < last; e += kElementThreads) {
      const uint32_t row = e / cols, col = e - row * cols;
      first_iterate((float)((const T*)p.u)[q * p.batch + row * p.row + col], inverse, p.planes + q * p.dst_batch + row * p.dst_row + col, p.dst_plane);
    }
  }
}

// ---- the step: momentum, norms, and everything that no matrix covers ---------------------------
struct StepSegment {
  uint32_t first_piece, offset, length;
  int32_t matrix;  // -1: between matrices
};
struct StepMatrix {
  __half* planes;  // of worker 0
  int64_t row, worker, plane;
  uint32_t cols;
  uint32_t pad;
};
constexpr int kMaxSegments = 2 * kMaxMatrices + 1;
struct StepParams {
  StepSegment segment[kMaxSegments];
  const void* gradient = nullptr;
  int64_t gradient_row = 0;
  const float* momentum = nullptr;
  float* momentum_next = nullptr;
  int64_t momentum_row = 0, momentum_next_row = 0;
  float mu = 0;
  int32_t nesterov = 0, segments = 0, pieces = 0, workers = 0;
  double* parts = nullptr;  // [workers][pieces]
  PullParams pull;
  unsigned int* error = nullptr;
  int32_t clear_error = 0;
};
struct StepIterateParams {
  StepMatrix matrix[kMaxMatrices];
};
__device__ __forceinline__ int find_segment(const StepParams& p, uint32_t piece) {
  int lo = 0, hi = p.segments - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (p.segment[mid].first_piece <= piece) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// m' = mu m + g, u = g + mu m' or m'; sums of squares of u inside matrices, the whole update outside them.
template <typename T>
__global__ __launch_bounds__(kElementThreads) void step_momentum_kernel(const __grid_constant__ StepParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *p.error = 0;
  const StepSegment seg = p.segment[find_segment(p, blockIdx.x)];
  const uint32_t first = seg.offset + (blockIdx.x - seg.first_piece) * kPiece, last = min(seg.offset + seg.length, first + kPiece);
  for (int i = blockIdx.y; i < p.workers; i += gridDim.y) {
    const T* g = (const T*)p.gradient + i * p.gradient_row;
    const float* m = p.momentum + i * p.momentum_row;
    float* m_next = p.momentum_next + i * p.momentum_next_row;
    const int peer = p.pull.peers[i * p.pull.draw_stride];
    const bool pull = peer != i && (uint32_t)peer < (uint32_t)p.workers;
    const float w = pull ? p.pull.weights[i * p.pull.draw_stride] : 0.0f;
    const T* own = (const T*)p.pull.x + i * p.pull.x_row;
    const T* other = (const T*)p.pull.x + (pull ? peer : i) * p.pull.x_row;
    T* next = (T*)p.pull.x_next + i * p.pull.next_row;
    double s = 0.0;
    for (uint32_t e = first + threadIdx.x; e < last; e += kElementThreads) {
      const float grad = (float)g[e], after = fmaf(p.mu, m[e], grad);
      m_next[e] = after;
      const float u = p.nesterov ? fmaf(p.mu, after, grad) : after;
      if (seg.matrix >= 0) {
        s += (double)u * (double)u;
      } else {
        const float x = (float)own[e], h = fmaf(-p.pull.lr, fmaf(p.pull.decay, x, u), x);
        next[e] = (T)(pull ? fmaf(-w, h - (float)other[e], h) : h);
      }
    }
    if (seg.matrix >= 0) {
      s = block_sum(s);
      if (threadIdx.x == 0) p.parts[(int64_t)i * p.pieces + blockIdx.x] = s;
    }
  }
}
template <typename T>
__global__ __launch_bounds__(kElementThreads) void step_first_iterate_kernel(const __grid_constant__ StepParams p, const __grid_constant__ StepIterateParams tables) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  const int at = find_segment(p, blockIdx.x);
  const StepSegment seg = p.segment[at];
  if (seg.matrix < 0) return;
  const StepMatrix& to = tables.matrix[seg.matrix];
  const uint32_t pieces = (seg.length + kPiece - 1) / kPiece;
  const uint32_t begin = (blockIdx.x - seg.first_piece) * kPiece, end = min(seg.length, begin + kPiece), cols = to.cols;
  for (int i = blockIdx.y; i < p.workers; i += gridDim.y) {
    double s = 0.0;
    for (uint32_t k = threadIdx.x; k < pieces; k += kElementThreads) s += p.parts[(int64_t)i * p.pieces + seg.first_piece + k];
    const double inverse = inverse_norm(block_sum(s));
    const T* g = (const T*)p.gradient + i * p.gradient_row + seg.offset;
    const float* m_next = p.momentum_next + i * p.momentum_next_row + seg.offset;
    for (uint32_t e = begin + threadIdx.x; e < end; e += kElementThreads) {
      const float after = m_next[e], u = p.nesterov ? fmaf(p.mu, after, (float)g[e]) : after;
      const uint32_t row = e / cols;
      first_iterate(u, inverse, to.planes + i * to.worker + row * to.row + (e - row * cols), to.plane);
    }
  }
}

}  // namespace netmax
