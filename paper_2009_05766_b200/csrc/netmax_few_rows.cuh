// The layer for batches of a few rows: bound by reading the weights once, so they go through the FMA units as they are.  A warp takes
// kOutputs outputs at a time, its lanes share out k, and all rows of the batch use a weight while it is in a register.  The tensor
// cores' path reads fp32 weights twice and writes them as planes first.  us for 8 workers' 4096 x 4096 layers, this / that path: fp32 (read
// in 82) 1 row 82, 4 rows 123, 8 rows 140 / 431, 16 rows in two passes; bfloat16 (41) 1 row 45, 4 rows 66 / 63, 8 rows 117 / 63.
#pragma once
#include "netmax_operators.cuh"

namespace netmax {

// Up to so many rows: fp32; bfloat16 that the tensor cores can read in place; bfloat16 that would have to be laid out first.
constexpr int kFewRowsF32 = 16, kFewRowsBf16 = 4, kFewRowsBf16Laid = 8;

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
  float mine = 0.0f;  // lane o * kRows + r has output `first + o` of row r
#pragma unroll
  for (int o = 0; o < kOutputs; ++o)
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      float s = sum[o][r];
#pragma unroll
      for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
      if (lane == o * kRows + r) mine = s;
    }
  const int o = first + lane / kRows;
  if (lane >= kOutputs * kRows || o >= p.n_out || lane % kRows >= n) return;
  const int64_t r = rows_before + lane % kRows;
  if (p.bias) mine += (float)((const T*)p.bias)[q * p.bias_batch + o];
  if (p.z) ((T*)p.z)[q * p.z_batch + r * p.z_row + o] = (T)mine;
  mine = activate(mine, p.activation);
  if (p.residual) mine += (float)((const T*)p.residual)[q * p.residual_batch + r * p.residual_row + o];
  ((T*)p.y)[q * p.y_batch + r * p.y_row + o] = (T)mine;
}

}  // namespace netmax
