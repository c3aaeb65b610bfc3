// Elementwise kernels around the products of netmax_product.cuh: operands laid out for the tensor cores, column sums, norms and
// momentum.  All of them are bound by memory; sums are taken in a fixed order, so results do not change from run to run.
#pragma once
#include "netmax_product.cuh"

namespace netmax {

constexpr int kElementThreads = 256;
constexpr int kPiece = 8192;        // elements of a replica that one CTA of the step's kernels works on
template <typename T>
constexpr int kUnroll = sizeof(T) == 4 ? 2 : 4;  // rows that a thread has in flight: 32 registers of them, and 32 of z

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

// How the elementwise kernels go over a matrix: a thread takes eight neighbouring columns, `1 << shift` threads a row, and a CTA
// `rows_per_block` rows of a tile that wide.
struct Sweep {
  int32_t rows = 0, cols = 0, count = 0;
  int32_t shift = 0, col_tiles = 1, row_blocks = 1, rows_per_block = 1;
};
struct SweepAt {
  int col, count, row, last, step, row_block;  // `count` live columns from `col` on; rows row, row + step, ... below last
};
__device__ __forceinline__ SweepAt sweep_at(const Sweep& s, int block) {
  SweepAt a;
  const int lane = threadIdx.x & ((1 << s.shift) - 1);
  a.row_block = block / s.col_tiles;
  a.col = (((block - a.row_block * s.col_tiles) << s.shift) + lane) * 8;
  a.count = min(8, s.cols - a.col);
  a.step = kElementThreads >> s.shift;
  a.row = a.row_block * s.rows_per_block + ((int)threadIdx.x >> s.shift);
  a.last = min(s.rows, (a.row_block + 1) * s.rows_per_block);
  return a;
}

// An operand on its way to the tensor cores: `count` matrices of rows x cols; with z, dy act'(z).
struct OperandJob {
  Sweep sweep;
  const void* src = nullptr;
  int64_t row = 0, batch = 0;
  const void* z = nullptr;
  int64_t z_row = 0, z_batch = 0;
  int32_t activation = 0;
  void* dst = nullptr;  // NULL: not laid out
  int64_t dst_row = 0, dst_batch = 0, dst_plane = 0;
  float* maxima = nullptr;  // [count][blocks]
  int32_t* exponent = nullptr;
  float* sums = nullptr;    // [count][row blocks][cols]: column sums of the blocks; NULL: not wanted
};
struct OperandParams {
  OperandJob job[4];
  unsigned int* error = nullptr;
  int32_t clear_error = 0;
};

// Eight values as they lie in memory, so that the loads of several rows are under way before the first one's arithmetic.
template <typename T>
struct Eight {
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* at, int count, bool whole) {
    if (whole) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
        const uint4 a = ((const uint4*)at)[k];
        w[4 * k] = a.x, w[4 * k + 1] = a.y, w[4 * k + 2] = a.z, w[4 * k + 3] = a.w;
      }
    } else if (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < (int)sizeof(T) * 2) w[k] = k < count ? ((const uint32_t*)at)[k] : 0;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t lo = 2 * k < count ? ((const unsigned short*)at)[2 * k] : 0, hi = 2 * k + 1 < count ? ((const unsigned short*)at)[2 * k + 1] : 0;
        w[k] = lo | hi << 16;
      }
    }
  }
  __device__ __forceinline__ float get(int k) const {
    if (sizeof(T) == 4) return __uint_as_float(w[k]);
    return __uint_as_float(k % 2 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
  }
};
template <typename T>
__device__ __forceinline__ bool whole_rows(const T* base, int64_t row, int count) {
  return count == 8 && (((uintptr_t)base | (uintptr_t)(row * (int64_t)sizeof(T))) & 15) == 0;
}

// A thread's rows of matrix q, kUnroll<T> at a time: use(row, values).
template <typename T, typename Use>
__device__ __forceinline__ void sweep_rows(const OperandJob& j, const SweepAt& a, int q, const Use& use) {
  if (a.count <= 0) return;
  const T* src = (const T*)j.src + q * j.batch + a.col;
  const T* z = j.z ? (const T*)j.z + q * j.z_batch + a.col : nullptr;
  const bool whole = whole_rows(src, j.row, a.count), whole_z = z && whole_rows(z, j.z_row, a.count);
  const int64_t row_stride = j.row, z_stride = j.z_row;
  const int activation = j.activation;
#pragma unroll 1
  for (int row = a.row; row < a.last; row += kUnroll<T> * a.step) {
    Eight<T> raw[kUnroll<T>], raw_z[kUnroll<T>];
#pragma unroll
    for (int u = 0; u < kUnroll<T>; ++u) {  // (rows past the last one repeat it: their values are not used)
      const int64_t r = min(row + u * a.step, a.last - 1);
      raw[u].load(src + r * row_stride, a.count, whole);
      if (z) raw_z[u].load(z + r * z_stride, a.count, whole_z);
    }
#pragma unroll
    for (int u = 0; u < kUnroll<T>; ++u) {
      if (row + u * a.step >= a.last) break;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = raw[u].get(k);
      if (z) {
        if (activation == kActRelu) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] *= activation_slope(raw_z[u].get(k), kActRelu);
        } else if (activation == kActGelu) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] *= activation_slope(raw_z[u].get(k), kActGelu);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] *= activation_slope(raw_z[u].get(k), kActSilu);
        }
      }
      use(row + u * a.step, v);
    }
  }
}

// A block's column sums: every thread's rows first, then the threads of a column in order.
__device__ __forceinline__ void write_sums(const OperandJob& j, const SweepAt& a, int q, const float (&sum)[8]) {
  __shared__ float parts[kElementThreads * 8];
  const int width = 8 << j.sweep.shift, lane = threadIdx.x & ((1 << j.sweep.shift) - 1);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) parts[((int)threadIdx.x >> j.sweep.shift) * width + lane * 8 + k] = sum[k];
  __syncthreads();
  const int tile = a.col - lane * 8;
  for (int c = threadIdx.x; c < width && tile + c < j.sweep.cols; c += kElementThreads) {
    float s = 0.0f;
    for (int r = 0; r < a.step; ++r) s += parts[r * width + c];
    j.sums[((int64_t)q * j.sweep.row_blocks + a.row_block) * j.sweep.cols + tile + c] = s;
  }
}

// fp32: the largest finite magnitude of every block, and the column sums.
__global__ __launch_bounds__(kElementThreads) void operand_maxima_kernel(const __grid_constant__ OperandParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *p.error = 0;
  const OperandJob j = p.job[blockIdx.z];  // (a copy: read in place, its fields are indexed loads from the constant bank, over and over)
  const int blocks = j.sweep.col_tiles * j.sweep.row_blocks;
  if ((int)blockIdx.x >= blocks) return;
  const SweepAt a = sweep_at(j.sweep, blockIdx.x);
  for (int q = blockIdx.y; q < j.sweep.count; q += gridDim.y) {
    float most = 0.0f, sum[8] = {};
    sweep_rows<float>(j, a, q, [&](int, const float (&v)[8]) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float m = fabsf(v[k]);
        if (m <= 3.402823466e38f) most = fmaxf(most, m);
        sum[k] += v[k];
      }
    });
    if (j.sums) write_sums(j, a, q, sum);
    if (j.maxima) {
      most = block_max(most);
      if (threadIdx.x == 0) j.maxima[q * blocks + blockIdx.x] = most;
    }
  }
}

// fp32 as two fp16 planes of the values times a power of two that brings the largest to [2^14, 2^15); bfloat16 as it is, with the
// column sums.
template <typename T>
__global__ __launch_bounds__(kElementThreads) void operand_kernel(const __grid_constant__ OperandParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *p.error = 0;
  const OperandJob j = p.job[blockIdx.z];
  const int blocks = j.sweep.col_tiles * j.sweep.row_blocks;
  if ((int)blockIdx.x >= blocks || (sizeof(T) == 4 && !j.dst)) return;
  const SweepAt a = sweep_at(j.sweep, blockIdx.x);
  for (int q = blockIdx.y; q < j.sweep.count; q += gridDim.y) {
    int exponent = 0;
    if (sizeof(T) == 4) {
      float most = 0.0f;
      for (int k = threadIdx.x; k < blocks; k += kElementThreads) most = fmaxf(most, j.maxima[q * blocks + k]);
      most = block_max(most);
      if (most > 0.0f) exponent = min(14 - ilogbf(most), 126);  // (from 2^-112 on the largest lies lower; such values vanish beside any bias)
      if (blockIdx.x == 0 && threadIdx.x == 0) j.exponent[q] = exponent;
    }
    const float scale = ldexpf(1.0f, exponent);
    float sum[8] = {};
    char* dst = (char*)j.dst + (q * j.dst_batch + a.col) * 2;
    const int64_t dst_row = j.dst_row * 2, dst_plane = j.dst_plane * 2;
    const bool laid = j.dst != nullptr;
    sweep_rows<T>(j, a, q, [&](int row, float (&v)[8]) {
      char* at = dst + row * dst_row;  // (rows are padded to eight columns)
      if (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= scale;
        uint4 hi, lo;
        split8(v, hi, lo);
        *(uint4*)at = hi;
        *(uint4*)(at + dst_plane) = lo;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += v[k];
        if (laid) store_values<__nv_bfloat16, true, 8>((__nv_bfloat16*)at, 8, v);
      }
    });
    if (sizeof(T) == 2 && j.sums) write_sums(j, a, q, sum);
  }
}

// fp32 rows as two fp16 planes, each row times a power of two of its own.  kLanes threads a row, as many as hold it with up to
// 32 values each in registers; rows longer than 8,192 are read again from L2.
template <int kLanes>
__global__ __launch_bounds__(kElementThreads) void operand_rows_kernel(const __grid_constant__ OperandParams p) {
  constexpr int kHeld = 4;  // groups of eight values
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *p.error = 0;
  const OperandJob j = p.job[blockIdx.z];
  const int asked = blockIdx.x * (kElementThreads / kLanes) + threadIdx.x / kLanes, lane = threadIdx.x % kLanes, cols = j.sweep.cols;
  if (blockIdx.x * (kElementThreads / kLanes) >= j.sweep.rows) return;
  const bool live = asked < j.sweep.rows;  // (rows past the last one go through its motions, up to the stores)
  const int row = live ? asked : j.sweep.rows - 1;
  __shared__ float parts[kElementThreads / 32];
  for (int q = blockIdx.y; q < j.sweep.count; q += gridDim.y) {
    const float* src = (const float*)j.src + q * j.batch + row * j.row;
    const int whole = ((uintptr_t)src & 15) == 0 ? cols / 8 * 8 : 0;  // columns that go in 16-byte pieces
    float most = 0.0f, held[kHeld][8];
    auto look = [&](float v) {
      v = fabsf(v);
      if (v <= 3.402823466e38f) most = fmaxf(most, v);
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int c = (i * kLanes + lane) * 8;
      if (c >= whole) break;
      load_values<float, true, 8>(src + c, 8, held[i]);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if ((i * kLanes + lane) * 8 >= whole) break;
#pragma unroll
      for (int k = 0; k < 8; ++k) look(held[i][k]);
    }
    for (int c = (kHeld * kLanes + lane) * 8; c < whole; c += kLanes * 8) {
      float v[8];
      load_values<float, true, 8>(src + c, 8, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) look(v[k]);
    }
    for (int c = whole + lane; c < cols; c += kLanes) look(src[c]);
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    if (kLanes > 32) {
      __syncthreads();
      if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = most;
      __syncthreads();
      const int first = threadIdx.x / kLanes * (kLanes / 32);
#pragma unroll
      for (int w = 0; w < kLanes / 32; ++w) most = fmaxf(most, parts[first + w]);
    }
    if (!live) continue;
    const int exponent = most > 0.0f ? min(14 - ilogbf(most), 126) : 0;
    if (lane == 0) j.exponent[(int64_t)q * j.sweep.rows + row] = exponent;
    const float scale = ldexpf(1.0f, exponent);
    __half* dst = (__half*)j.dst + q * j.dst_batch + row * j.dst_row;
    auto put = [&](int c, float (&v)[8]) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= scale;
      uint4 hi, lo;
      split8(v, hi, lo);
      *(uint4*)(dst + c) = hi;
      *(uint4*)(dst + c + j.dst_plane) = lo;
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int c = (i * kLanes + lane) * 8;
      if (c >= whole) break;
      put(c, held[i]);
    }
    for (int c = (kHeld * kLanes + lane) * 8; c < whole; c += kLanes * 8) {
      float v[8];
      load_values<float, true, 8>(src + c, 8, v);
      put(c, v);
    }
    for (int c = whole + lane; c < cols; c += kLanes) {
      const float v[4] = {src[c] * scale, 0.0f, 0.0f, 0.0f};
      uint32_t hi[2], lo[2];
      split_values<4>(v, hi, lo);
      dst[c] = __ushort_as_half((unsigned short)hi[0]);
      dst[c + j.dst_plane] = __ushort_as_half((unsigned short)lo[0]);
    }
  }
}

// The blocks' column sums added up, in double.
template <typename T>
__global__ __launch_bounds__(kElementThreads) void column_totals_kernel(const float* parts, int n_parts, int cols, int count, T* out, int64_t batch) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  const int64_t total = (int64_t)count * cols;
  for (int64_t e = (int64_t)blockIdx.x * kElementThreads + threadIdx.x; e < total; e += (int64_t)gridDim.x * kElementThreads) {
    const int64_t q = e / cols, col = e - q * cols;
    double s = 0.0;
#pragma unroll 8
    for (int k = 0; k < n_parts; ++k) s += (double)parts[(q * n_parts + k) * cols + col];
    out[q * batch + col] = (T)(float)s;
  }
}

// ---- Newton-Schulz: norms and the first iterate ------------------------------------------------
struct NormParams {  // matrices on their own
  Sweep sweep;
  const void* u = nullptr;
  int64_t row = 0, batch = 0;
  double* parts = nullptr;  // [count][blocks] sums of squares
  __half* planes = nullptr;
  int64_t dst_row = 0, dst_batch = 0, dst_plane = 0;
  unsigned int* error = nullptr;
  int32_t clear_error = 0;
};
// 2^14 / norm as two factors, so that neither they nor the product with one of them leave fp32's range where the iterate does not; zeros
// for a matrix of zeros.  A norm that is not finite makes the whole matrix NaN, as the products would.
struct Inverse {
  float a, b;
};
__device__ __forceinline__ Inverse inverse_norm(double squares) {
  if (squares == 0.0) return {0.0f, 0.0f};
  if (!(squares <= 1.7e308)) return {__int_as_float(0x7FC00000), 1.0f};
  const double inverse = (double)kPlaneScale / sqrt(squares);
  const int e = ilogb(inverse) / 2;
  return {ldexpf(1.0f, e), (float)ldexp(inverse, -e)};
}

template <typename T>
__global__ __launch_bounds__(kElementThreads) void norm_parts_kernel(const __grid_constant__ NormParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *p.error = 0;
  const SweepAt a = sweep_at(p.sweep, blockIdx.x);
  OperandJob job;
  for (int q = blockIdx.y; q < p.sweep.count; q += gridDim.y) {
    double s = 0.0;
    job.src = p.u;
    job.row = p.row;
    job.batch = p.batch;
    sweep_rows<T>(job, a, q, [&](int, const float (&v)[8]) {
#pragma unroll
      for (int k = 0; k < 8; ++k) s += (double)v[k] * (double)v[k];
    });
    s = block_sum(s);
    if (threadIdx.x == 0) p.parts[(int64_t)q * gridDim.x + blockIdx.x] = s;
  }
}
template <typename T>
__global__ __launch_bounds__(kElementThreads) void first_iterate_kernel(const __grid_constant__ NormParams p) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  const SweepAt a = sweep_at(p.sweep, blockIdx.x);
  OperandJob job;
  for (int q = blockIdx.y; q < p.sweep.count; q += gridDim.y) {
    double s = 0.0;
    for (int k = threadIdx.x; k < (int)gridDim.x; k += kElementThreads) s += p.parts[(int64_t)q * gridDim.x + k];
    const Inverse inverse = inverse_norm(block_sum(s));
    job.src = p.u;
    job.row = p.row;
    job.batch = p.batch;
    __half* dst = p.planes + q * p.dst_batch + a.col;
    sweep_rows<T>(job, a, q, [&](int row, float (&v)[8]) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = v[k] * inverse.a * inverse.b;
      uint4 hi, lo;
      split8(v, hi, lo);
      *(uint4*)(dst + row * p.dst_row) = hi;
      *(uint4*)(dst + row * p.dst_row + p.dst_plane) = lo;
    });
  }
}

// S from its parts: the 32 x 32 blocks on and below the diagonal, added up in the parts' order, as planes, the others mirrored.
struct CombineGroup {
  const float* parts = nullptr;  // [matrix][split][side][row]
  __half* out = nullptr;
  int64_t row = 0, part_batch = 0, out_batch = 0, out_plane = 0;
  int32_t side = 0, splits = 1, first_block = 0;  // blocks of all its matrices, from first_block on
};
struct CombineParams {
  CombineGroup group[kMaxGroups];
  int32_t groups = 0, planes = 1;
};
__global__ __launch_bounds__(kElementThreads) void combine_kernel(const __grid_constant__ CombineParams p) {
  __shared__ uint32_t turned[32][33];
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  int k = 0;
  while (k + 1 < p.groups && p.group[k + 1].first_block <= (int)blockIdx.x) ++k;
  const CombineGroup g = p.group[k];
  const int edge = (g.side + 31) / 32, per = edge * (edge + 1) / 2;
  int t = (int)blockIdx.x - g.first_block;
  const int q = t / per;
  t -= q * per;
  int i = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
  while (i * (i + 1) / 2 > t) --i;
  while ((i + 1) * (i + 2) / 2 <= t) ++i;
  const int j = t - i * (i + 1) / 2, r = threadIdx.x / 8, c = threadIdx.x % 8 * 4, m = i * 32 + r, n = j * 32 + c;
  uint32_t hi[2] = {}, lo[2] = {};
  const bool live = m < g.side && n < g.side;
  if (live) {
    float v[4] = {};
    const float* at = g.parts + (int64_t)q * g.splits * g.part_batch + (int64_t)m * g.row + n;
    for (int s = 0; s < g.splits; ++s) {
      const float4 a = *(const float4*)(at + s * g.part_batch);
      v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= kPlaneUnscale;
    split_values<4>(v, hi, lo);
    __half* out = g.out + q * g.out_batch + (int64_t)m * g.row + n;
    store_words(out, hi);
    if (p.planes == 2) store_words(out + g.out_plane, lo);
  }
  if (i == j) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) turned[c + e][r] = (hi[e / 2] >> (16 * (e % 2)) & 0xFFFF) | (lo[e / 2] >> (16 * (e % 2))) << 16;
  __syncthreads();
  const int m2 = j * 32 + r, n2 = i * 32 + c;
  if (m2 >= g.side || n2 >= g.side) return;
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = turned[r][c + e];
  const uint32_t h[2] = {__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410)}, l[2] = {__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632)};
  __half* out = g.out + q * g.out_batch + (int64_t)m2 * g.row + n2;
  store_words(out, h);
  if (p.planes == 2) store_words(out + g.out_plane, l);
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

// A piece of a segment: elements [first, last), taken four at a time from the multiple of eight at or before `first` on, so that every
// full group lies on a 16-byte boundary where fp32 arrays do (and a warp's stores fill whole sectors).
struct Piece {
  uint32_t first, last, group;
};
__device__ __forceinline__ Piece piece_of(const StepSegment& s, uint32_t block) {
  Piece p;
  const uint32_t base = s.offset & ~7u, begin = base + (block - s.first_piece) * kPiece;
  p.first = max(begin, s.offset);
  p.last = min(begin + kPiece, s.offset + s.length);
  p.group = begin + threadIdx.x * 4;
  return p;
}
// Four elements from `at` on, of which those in [first, last) exist.
template <typename T>
__device__ __forceinline__ void load_group(const T* base, uint32_t at, const Piece& p, float (&v)[4]) {
  if (at >= p.first && at + 4 <= p.last) return load_values<T, false, 4>(base + at, 4, v);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = at + k >= p.first && at + k < p.last ? (float)base[at + k] : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_group(T* base, uint32_t at, const Piece& p, const float (&v)[4]) {
  if (at >= p.first && at + 4 <= p.last) return store_values<T, false, 4>(base + at, 4, v);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (at + k >= p.first && at + k < p.last) base[at + k] = (T)v[k];
}
constexpr int kGroupsPerThread = kPiece / (4 * kElementThreads);

// m' = mu m + g, u = g + mu m' or m'; sums of squares of u inside matrices, the whole update outside them.
template <typename T>
__global__ __launch_bounds__(kElementThreads) void step_momentum_kernel(const __grid_constant__ StepParams p) {
  ptx::wait_for_predecessor();
  ptx::let_successor_start();  // (in this order: see SmallParams::behind_rest)
  if (p.clear_error && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *p.error = 0;
  const StepSegment seg = p.segment[find_segment(p, blockIdx.x)];
  const Piece piece = piece_of(seg, blockIdx.x);
  for (int i = blockIdx.y; i < p.workers; i += gridDim.y) {
    const T* g = (const T*)p.gradient + i * p.gradient_row;
    const float* m = p.momentum + i * p.momentum_row;
    float* m_next = p.momentum_next + i * p.momentum_next_row;
    double s = 0.0;
    float grad[kGroupsPerThread][4], mom[kGroupsPerThread][4];
#pragma unroll
    for (int u = 0; u < kGroupsPerThread; ++u) {
      const uint32_t at = piece.group + u * 4 * kElementThreads;
      if (at >= piece.last) break;
      load_group(g, at, piece, grad[u]);
      load_group(m, at, piece, mom[u]);
    }
#pragma unroll
    for (int u = 0; u < kGroupsPerThread; ++u) {
      const uint32_t at = piece.group + u * 4 * kElementThreads;
      if (at >= piece.last) break;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        mom[u][k] = fmaf(p.mu, mom[u][k], grad[u][k]);
        grad[u][k] = p.nesterov ? fmaf(p.mu, mom[u][k], grad[u][k]) : mom[u][k];  // (elements outside the piece are zeros)
        s += (double)grad[u][k] * (double)grad[u][k];
      }
      store_group(m_next, at, piece, mom[u]);
    }
    if (seg.matrix >= 0) {
      s = block_sum(s);
      if (threadIdx.x == 0) p.parts[(int64_t)i * p.pieces + blockIdx.x] = s;
      continue;
    }
    const int peer = p.pull.peers[i * p.pull.draw_stride];
    const bool pull = peer != i && (uint32_t)peer < (uint32_t)p.workers;
    const float w = pull ? p.pull.weights[i * p.pull.draw_stride] : 0.0f;
    const T* own = (const T*)p.pull.x + i * p.pull.x_row;
    const T* other = (const T*)p.pull.x + (pull ? peer : i) * p.pull.x_row;
    T* next = (T*)p.pull.x_next + i * p.pull.next_row;
#pragma unroll
    for (int u = 0; u < kGroupsPerThread; ++u) {
      const uint32_t at = piece.group + u * 4 * kElementThreads;
      if (at >= piece.last) break;
      float x[4], xm[4];
      load_group(own, at, piece, x);
      load_group(other, at, piece, xm);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float h = fmaf(-p.pull.lr, fmaf(p.pull.decay, x[k], grad[u][k]), x[k]);
        x[k] = pull ? fmaf(-w, h - xm[k], h) : h;
      }
      store_group(next, at, piece, x);
    }
  }
}
template <typename T>
__global__ __launch_bounds__(kElementThreads) void step_first_iterate_kernel(const __grid_constant__ StepParams p, const __grid_constant__ StepIterateParams tables) {
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  const StepSegment seg = p.segment[find_segment(p, blockIdx.x)];
  if (seg.matrix < 0) return;
  const StepMatrix to = tables.matrix[seg.matrix];
  const Piece piece = piece_of(seg, blockIdx.x);
  const uint32_t pieces = ((seg.offset & 7) + seg.length + kPiece - 1) / kPiece, cols = to.cols;
  const bool whole = ((seg.offset | cols) & 3) == 0;  // groups of four do not cross rows
  for (int i = blockIdx.y; i < p.workers; i += gridDim.y) {
    const T* g = (const T*)p.gradient + i * p.gradient_row;
    const float* m_next = p.momentum_next + i * p.momentum_next_row;
    float grad[kGroupsPerThread][4], mom[kGroupsPerThread][4];
#pragma unroll
    for (int u = 0; u < kGroupsPerThread; ++u) {
      const uint32_t at = piece.group + u * 4 * kElementThreads;
      if (at >= piece.last) break;
      load_group(m_next, at, piece, mom[u]);
      if (p.nesterov) load_group(g, at, piece, grad[u]);
    }
    double s = 0.0;
    for (uint32_t k = threadIdx.x; k < pieces; k += kElementThreads) s += p.parts[(int64_t)i * p.pieces + seg.first_piece + k];
    const Inverse inverse = inverse_norm(block_sum(s));
    __half* planes = to.planes + i * to.worker;
#pragma unroll
    for (int u = 0; u < kGroupsPerThread; ++u) {
      const uint32_t at = piece.group + u * 4 * kElementThreads;
      if (at >= piece.last) break;
#pragma unroll
      for (int k = 0; k < 4; ++k) mom[u][k] = (p.nesterov ? fmaf(p.mu, mom[u][k], grad[u][k]) : mom[u][k]) * inverse.a * inverse.b;
      uint32_t hi[2], lo[2];
      split_values<4>(mom[u], hi, lo);
      if (whole) {  // (then a group lies inside the segment or outside it)
        if (at < piece.first) continue;
        const uint32_t e = at - seg.offset, row = e / cols;
        __half* to4 = planes + row * to.row + (e - row * cols);
        store_words(to4, hi);
        store_words(to4 + to.plane, lo);
      } else {
        const uint32_t begin = max(at, piece.first) - seg.offset;
        uint32_t row = begin / cols, col = begin - row * cols;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (at + k < piece.first || at + k >= piece.last) continue;
          __half* to1 = planes + row * to.row + col;
          to1[0] = __ushort_as_half((unsigned short)(hi[k / 2] >> (16 * (k % 2))));
          to1[to.plane] = __ushort_as_half((unsigned short)(lo[k / 2] >> (16 * (k % 2))));
          if (++col == cols) {
            col = 0;
            ++row;
          }
        }
      }
    }
  }
}

}  // namespace netmax
