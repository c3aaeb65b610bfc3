// The layer for batches of a few rows: bound by reading the weights once, so they go through the FMA units as they are.  A warp takes
// kOutputs outputs at a time, its lanes share out k, and all rows of the batch use a weight while it is in a register; more than eight rows
// read the weights twice.  The tensor cores' path reads fp32 weights once, writes them as planes and reads those.  us for 8 workers, this /
// that path, at 4096 x 4096 (fp32 weights are read in 82, bfloat16 in 41), 2048 x 2048 and 512 x 512:
//   layer, fp32                 1 row  87 / 307, 28 / 84, 3.0 / 14.4;    8 rows 140 / 308, 38 / 84, 6.2 / 14.5;   16 rows 250 / 308, 73 / 84, 9.7 / 14.6
//   bfloat16                    1 row  50 / 68, 9.2 / 18.9, 2.4 / 7.7;   4 rows 68 / 60, 14.7 / 18.9, 3.6 / 7.7;   5 rows 125 / 60, 30 / 19, 4.6 / 7.7
//   bfloat16, to be laid out    1 row 118 / 229, 30 / 67, 5.0 / 13.4;    4 rows 252 / 228, 48 / 67, 9.5 / 13.4;    5 rows 504 / 229, 101 / 67, 17 / 14
//   gradient, fp32              1 row 181 / 673, 65 / 199, 12 / 26;      8 rows 313 / 674, 95 / 192, 26 / 24;     16 rows 524 / 675, 153 / 192, 39 / 25
//   gradient, bfloat16          1 row 213 / 200, 70 / 57, 12 / 11;       4 rows 241 / 189, 84 / 56, 16 / 11;       5 rows 280 / 189, 79 / 56, 19 / 11
//   the same, to be laid out    1 row 560 / 438, 225 / 117, 23 / 18;     4 rows 480 / 431, 187 / 117, 24 / 18;     5 rows 536 / 431, 154 / 117, 32 / 18
// The bfloat16 gradient takes this path for its dz, which the other one rounds to bfloat16 where there is an activation.
#pragma once
#include "netmax_operators.cuh"

namespace netmax {

// Up to so many rows.
constexpr int kFewRowsF32 = 16, kFewRowsBf16 = 4;

struct FewRowsParams {
  const void *x = nullptr, *weight = nullptr, *bias = nullptr, *residual = nullptr;
  void *y = nullptr, *z = nullptr;
  int64_t x_row = 0, x_batch = 0, weight_row = 0, weight_batch = 0, bias_batch = 0, residual_row = 0, residual_batch = 0, y_row = 0, y_batch = 0, z_row = 0,
          z_batch = 0;
  int32_t n = 0, n_in = 0, n_out = 0, activation = 0;
  int32_t pieces = 0;  // rows of x and of the weights start on 16-byte boundaries
  unsigned int* error = nullptr;
};

template <typename T, int kRows, int kOutputs>
__global__ __launch_bounds__(kElementThreads) void few_rows_kernel(const __grid_constant__ FewRowsParams p) {
  constexpr int kN = 16 / sizeof(T);  // values of a load
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *p.error = 0;
  const int lane = threadIdx.x % 32, first = (blockIdx.x * (kElementThreads / 32) + threadIdx.x / 32) * kOutputs;
  if (first >= p.n_out) return;
  const int64_t q = blockIdx.y;
  const int rows_before = blockIdx.z * kRows, n = min(kRows, p.n - rows_before);
  const T* x = (const T*)p.x + q * p.x_batch + rows_before * p.x_row;
  const T* w = (const T*)p.weight + q * p.weight_batch + first * p.weight_row;
  float sum[kOutputs][kRows] = {};
  auto step = [&](int k, int count, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    float a[kOutputs][kN];
#pragma unroll
    for (int o = 0; o < kOutputs; ++o) {
      // (outputs past the last one repeat it: their sums are not stored)
      const int64_t row = first + o < p.n_out ? o : p.n_out - 1 - first;
      load_values<T, kWhole, kN>(w + row * p.weight_row + k, count, a[o]);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      float b[kN];
      load_values<T, kWhole, kN>(x + (r < n ? r : n - 1) * p.x_row + k, count, b);
#pragma unroll
      for (int o = 0; o < kOutputs; ++o)
#pragma unroll
        for (int e = 0; e < kN; ++e) sum[o][r] = fmaf(a[o][e], b[e], sum[o][r]);
    }
  };
  int k = lane * kN;
  if (p.pieces) {
#pragma unroll 2
    for (; k + kN <= p.n_in; k += 32 * kN) step(k, kN, std::true_type());
  }
  for (; k < p.n_in; k += 32 * kN) step(k, min(kN, p.n_in - k), std::false_type());
#pragma unroll
  for (int h = 0; h < kOutputs * kRows; h += 32) {
  float mine = 0.0f;  // lane o * kRows + r - h has output `first + o` of row r
#pragma unroll
  for (int o = 0; o < kOutputs; ++o)
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (o * kRows + r < h || o * kRows + r >= h + 32) continue;
      float s = sum[o][r];
#pragma unroll
      for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
      if (lane == o * kRows + r - h) mine = s;
    }
  const int e = h + lane, o = first + e / kRows;
  if (e >= kOutputs * kRows || o >= p.n_out || e % kRows >= n) continue;
  const int64_t r = rows_before + e % kRows;
  if (p.bias) mine += (float)((const T*)p.bias)[q * p.bias_batch + o];
  if (p.z) ((T*)p.z)[q * p.z_batch + r * p.z_row + o] = (T)mine;
  mine = activate(mine, p.activation);
  if (p.residual) mine += (float)((const T*)p.residual)[q * p.residual_batch + r * p.residual_row + o];
  ((T*)p.y)[q * p.y_batch + r * p.y_row + o] = (T)mine;
  }
}

// ---- the gradient of such batches: bound by writing dW and reading W once ----------------------
// A thread has kN neighbouring columns of n_in, `1 << shift` threads a row; dz of 64 outputs at a time goes through shared memory.
constexpr int kFewOutputs = 64;
struct FewRowsBackParams {
  const void *dy = nullptr, *z = nullptr, *x = nullptr, *weight = nullptr;
  void *dx = nullptr, *dweight = nullptr, *dbias = nullptr;
  int64_t dy_row = 0, dy_batch = 0, z_row = 0, z_batch = 0, x_row = 0, x_batch = 0, weight_row = 0, weight_batch = 0, dx_row = 0, dx_batch = 0, dweight_row = 0,
          dweight_batch = 0, dbias_batch = 0;
  int32_t M = 0, n = 0, n_in = 0, n_out = 0, activation = 0;
  int32_t shift = 0, col_tiles = 1, outputs_per_block = kFewOutputs, chunks = 1;
  float* parts = nullptr;  // [chunks][M][n][n_in] of dx
  unsigned int* error = nullptr;
  int32_t clear_error = 0;
};

template <typename T>
__device__ __forceinline__ void stage_dz(const FewRowsBackParams& p, int64_t q, int first, float (*dz)[kFewOutputs]) {
  for (int e = threadIdx.x; e < p.n * kFewOutputs; e += kElementThreads) {
    const int r = e / kFewOutputs, o = first + e % kFewOutputs;
    float v = 0.0f;
    if (o < p.n_out) {
      v = (float)((const T*)p.dy)[q * p.dy_batch + r * p.dy_row + o];
      if (p.z) v *= activation_slope((float)((const T*)p.z)[q * p.z_batch + r * p.z_row + o], p.activation);
    }
    dz[r][e % kFewOutputs] = v;
  }
}

// dW and the sums of dz.
template <typename T, int kRows>
__global__ __launch_bounds__(kElementThreads) void few_rows_dweight_kernel(const __grid_constant__ FewRowsBackParams p) {
  constexpr int kN = 16 / sizeof(T);
  __shared__ float dz[kRows][kFewOutputs];
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *p.error = 0;
  const int64_t q = blockIdx.y;
  const int tile = blockIdx.x % p.col_tiles, first = blockIdx.x / p.col_tiles * kFewOutputs;
  const int col = ((tile << p.shift) + (threadIdx.x & ((1 << p.shift) - 1))) * kN, count = min(kN, p.n_in - col);
  stage_dz<T>(p, q, first, dz);
  __syncthreads();
  if (p.dbias && tile == 0)
    for (int o = threadIdx.x; o < kFewOutputs && first + o < p.n_out; o += kElementThreads) {
      float s = 0.0f;
      for (int r = 0; r < p.n; ++r) s += dz[r][o];
      ((T*)p.dbias)[q * p.dbias_batch + first + o] = (T)s;
    }
  if (!p.dweight || count <= 0) return;
  float x[kRows][kN];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
#pragma unroll
    for (int k = 0; k < kN; ++k) x[r][k] = 0.0f;
    if (r < p.n) load_values<T, false, kN>((const T*)p.x + q * p.x_batch + r * p.x_row + col, count, x[r]);
  }
  const int step = kElementThreads >> p.shift, n = p.n;
  T* out = (T*)p.dweight + q * p.dweight_batch + first * p.dweight_row + col;
  const int64_t row = p.dweight_row;
  for (int o = threadIdx.x >> p.shift; o < kFewOutputs && first + o < p.n_out; o += step) {
    float v[kN] = {};
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (r >= n) break;
      const float d = dz[r][o];
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] = fmaf(d, x[r][k], v[k]);
    }
    store_values<T, false, kN>(out + o * row, count, v);
  }
}

// dx, or its part of a block's outputs.
template <typename T, int kRows>
__global__ __launch_bounds__(kElementThreads) void few_rows_dx_kernel(const __grid_constant__ FewRowsBackParams p) {
  constexpr int kN = 16 / sizeof(T);
  __shared__ float dz[kRows][kFewOutputs];
  __shared__ float sums[kElementThreads][kN];
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *p.error = 0;
  const int64_t q = blockIdx.y;
  const int tile = blockIdx.x % p.col_tiles, chunk = blockIdx.x / p.col_tiles, begin = chunk * p.outputs_per_block, end = min(p.n_out, begin + p.outputs_per_block);
  const int lanes = 1 << p.shift, lane = threadIdx.x & (lanes - 1), at = threadIdx.x >> p.shift, step = kElementThreads >> p.shift;
  const int col = ((tile << p.shift) + lane) * kN, count = min(kN, p.n_in - col), n = p.n;
  float acc[kRows][kN] = {};
  const T* w = (const T*)p.weight + q * p.weight_batch + col;
  const int64_t row = p.weight_row;
  for (int first = begin; first < end; first += kFewOutputs) {
    __syncthreads();
    stage_dz<T>(p, q, first, dz);
    __syncthreads();
    if (count <= 0) continue;
    const int last = min(kFewOutputs, end - first);
    for (int o = at; o < last; o += 4 * step) {
      float a[4][kN];
#pragma unroll
      for (int u = 0; u < 4; ++u)  // (outputs past the last one repeat it, with a zero for dz)
        load_values<T, false, kN>(w + (int64_t)(first + min(o + u * step, last - 1)) * row, count, a[u]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool live = o + u * step < last;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          if (r >= n) break;
          const float d = live ? dz[r][o + u * step] : 0.0f;
          if (!live) break;
#pragma unroll
          for (int k = 0; k < kN; ++k) acc[r][k] = fmaf(d, a[u][k], acc[r][k]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= n) break;
    if (step > 1) {  // rows of threads, in their order
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kN; ++k) sums[threadIdx.x][k] = acc[r][k];
      __syncthreads();
      if (at == 0)
        for (int y = 1; y < step; ++y)
#pragma unroll
          for (int k = 0; k < kN; ++k) acc[r][k] += sums[y * lanes + lane][k];
    }
    if (at != 0 || count <= 0) continue;
    if (p.chunks > 1) store_values<float, false, kN>(p.parts + (((int64_t)chunk * p.M + q) * n + r) * p.n_in + col, count, acc[r]);
    else store_values<T, false, kN>((T*)p.dx + q * p.dx_batch + r * p.dx_row + col, count, acc[r]);
  }
}
template <typename T>
__global__ __launch_bounds__(kElementThreads) void few_rows_total_kernel(const __grid_constant__ FewRowsBackParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  const int64_t row_length = p.n_in, each = (int64_t)p.n * row_length, total = each * p.M;
  for (int64_t e = (int64_t)blockIdx.x * kElementThreads + threadIdx.x; e < total; e += (int64_t)gridDim.x * kElementThreads) {
    float s = 0.0f;
#pragma unroll 8
    for (int c = 0; c < p.chunks; ++c) s += p.parts[c * total + e];
    const int64_t q = e / each, r = (e - q * each) / row_length, col = e - q * each - r * row_length;
    ((T*)p.dx)[q * p.dx_batch + r * p.dx_row + col] = (T)s;
  }
}

}  // namespace netmax
