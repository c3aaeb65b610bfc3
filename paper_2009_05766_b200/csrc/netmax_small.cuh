// Newton-Schulz orthogonalisation of small and of long, thin matrices (smaller side up to 64 with a larger one up to 8192; up to 128 and
// 4096): a CTA or a cluster of CTAs per matrix, everything in one launch.
//
// The general path is 15 products and two sweeps, each a launch of 5-7 us whose work is far below a microsecond for small sizes (four
// 64 x 64 matrices: 112 us); of long, thin ones its sums over the length run on one CTA (three of 27 x 4024: 205 us).  Here the iterate
// stays in shared memory as two fp16 planes in the tensor cores' own layout (blocks of 64 columns, rows of 128 bytes, 16-byte pieces
// swizzled by the row), S = X X^T and the polynomial beside it, accumulators in TMEM; a step is three rounds of products, wait, 16 columns
// a thread, barrier.  The one layout serves as k-contiguous operand (X X^T, S S, P) and as n-contiguous one (X in P X).  Tall matrices are
// transposed on their way in and out.  All products take the three terms of two-plane factors, whatever the storage: they cost little here.
// Sums over more than 128 columns of X go to accumulators of their own, added in fp32.
//
// The CTAs of a cluster share out the columns of X.  Each adds up one part of the rows of S over all of them, in their order, through
// distributed shared memory, and gives every CTA its planes; what follows from S they all work out for themselves.
#pragma once
#include "netmax_operators.cuh"

namespace netmax {

constexpr int kSmallThreads = 512;

struct SmallMatrix {
  uint32_t offset, rows, cols;
  float scale;
};
struct SmallParams {
  // matrices on their own
  const void* u = nullptr;
  int64_t row = 0, batch = 0;
  void* out = nullptr;
  int64_t out_row = 0, out_batch = 0;
  // or inside replicas: matrix q / workers of worker q % workers, for the q-th cluster
  const void* gradient = nullptr;
  int64_t gradient_row = 0;
  const float* momentum = nullptr;
  float* momentum_next = nullptr;
  int64_t momentum_row = 0, momentum_next_row = 0;
  float mu = 0;
  int32_t nesterov = 0;
  PullParams pull;
  SmallMatrix matrix[kMaxMatrices];
  int32_t rows = 0, cols = 0, steps = 0;
  int32_t ctas = 1;  // of a cluster
  uint32_t tmem_columns = 0;
  float ca = 0, cb = 0, cc = 0;
  unsigned int* error = nullptr;
  int32_t clear_error = 0;
  // The launch before is the step's for everything outside small matrices.  It lets this one start when it has itself waited for what came
  // before both, and they touch different elements: so this kernel waits for it only at its end, for the sake of the launch behind.
  int32_t behind_rest = 0;
};

// Shared memory of a matrix: two planes of the iterate, two of S, and a block behind them (a product's 128 rows of A run past 64-row
// blocks; what they find there reaches only rows of the accumulator that nobody reads).
__host__ __device__ inline uint32_t small_side(uint32_t rows, uint32_t cols) { return (rows < cols ? rows : cols) <= 64 ? 64 : 128; }
// Columns of the iterate that a CTA of a cluster holds.
__host__ __device__ inline uint32_t small_slice(uint32_t rows, uint32_t cols, uint32_t ctas) {
  return (((rows < cols ? cols : rows) + ctas - 1) / ctas + 63) / 64 * 64;
}
constexpr uint32_t kMostCtas = 16;
__host__ __device__ inline uint32_t most_columns(uint32_t side) { return side == 64 ? 512 : 256; }
inline uint32_t least_ctas(uint32_t rows, uint32_t cols) {
  uint32_t c = 1;
  while (small_slice(rows, cols, c) > most_columns(small_side(rows, cols))) c *= 2;
  return c;
}
// Whether matrices take this path (us, this / the general path, five steps of fp32: 24 of 128 x 1152 199 / 234, 32 of 128 x 4096 600 / 783).
inline bool is_small(int64_t rows, int64_t cols) {
  const int64_t side = rows < cols ? rows : cols, length = rows < cols ? cols : rows;
  return side <= 128 && length <= (int64_t)kMostCtas * most_columns(side <= 64 ? 64 : 128);
}
// Of these, the ones that a step leaves to the general path where that has larger matrices to run anyway: adding up 128 x 128 parts costs a
// cluster about as much as the rest of its work, and in launches that are there already they cost less (the update of 8 ResNet18-sized
// replicas 3850 us, with these apart 3990).
inline bool joins_larger(int64_t rows, int64_t cols) { return (rows < cols ? rows : cols) > 64 && least_ctas((uint32_t)rows, (uint32_t)cols) > 1; }
// CTAs for each of `count` matrices: as many as hold one; with sides up to 64 more while SMs would be idle and slices are long, but of
// clusters of sixteen no more than surely run at once (nine of 3726 x 11 in eights 78 us, in sixteens 116).
inline uint32_t small_ctas(int64_t count, uint32_t rows, uint32_t cols, int sms) {
  uint32_t c = least_ctas(rows, cols);
  while (small_side(rows, cols) == 64 && c < kMostCtas && small_slice(rows, cols, c) > 128 && count * c * 2 <= (c < 8 ? sms : 64)) c *= 2;
  return c;
}
inline size_t small_smem(uint32_t rows, uint32_t cols, uint32_t ctas) {
  const size_t r = small_side(rows, cols), l = small_slice(rows, cols, ctas);
  return 1024 + 2 * r * l * 2 + 2 * r * r * 2 + kBoxBytes;
}
inline uint32_t small_tmem(uint32_t rows, uint32_t cols, uint32_t ctas) {
  const uint32_t r = small_side(rows, cols), l = small_slice(rows, cols, ctas), need = l > (l + 127) / 128 * r ? l : (l + 127) / 128 * r;
  uint32_t c = 32;
  while (c < need) c *= 2;
  return c;
}

// Another CTA's shared memory.
__device__ __forceinline__ float4 load_remote(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void store_remote(uint32_t at, uint4 v) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void store_remote(uint32_t at, double v) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(v) : "memory"); }
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&v)[16]) {
  uint32_t r[16];
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
// Byte of element (row, column) in a plane of `side` rows.
__device__ __forceinline__ uint32_t small_at(uint32_t side, uint32_t row, uint32_t col) {
  return (col / 64) * side * 128 + row * 128 + ((((col % 64) / 8) ^ (row & 7)) * 16) + (col % 8) * 2;
}

template <typename T, bool kStep>
__global__ __launch_bounds__(kSmallThreads, 1) void small_schulz_kernel(const __grid_constant__ SmallParams p) {
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t bar;
  __shared__ uint32_t tmem_at;
  __shared__ double squares[kSmallThreads / 32], norms[kMostCtas];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  unsigned char* const base = raw + (((ptx::smem(raw) + 1023) & ~1023u) - ptx::smem(raw));
  const uint32_t ctas = p.ctas, rank = blockIdx.x % ctas, matrix = blockIdx.x / ctas;
  const int worker = kStep ? matrix % p.pull.workers : 0, which = kStep ? matrix / p.pull.workers : 0;
  const uint32_t rows = kStep ? p.matrix[which].rows : (uint32_t)p.rows, cols = kStep ? p.matrix[which].cols : (uint32_t)p.cols;
  const bool tall = rows > cols;
  const uint32_t side = small_side(rows, cols), length = small_slice(rows, cols, ctas);
  const uint32_t begin = rank * length, whole_length = tall ? rows : cols;           // this CTA's columns of the iterate
  const uint32_t own = begin < whole_length ? min(length, whole_length - begin) : 0;  // that exist
  const uint32_t x_plane = side * length * 2, s_plane = side * side * 2;
  unsigned char* const x = base;
  unsigned char* const s = base + 2 * x_plane;
  if (threadIdx.x == 0) {
    ptx::barrier_init(ptx::smem(&bar), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) ptx::tmem_alloc<1>(ptx::smem(&tmem_at), p.tmem_columns);
  for (uint32_t at = threadIdx.x * 16; at < 2 * x_plane; at += kSmallThreads * 16) *(uint4*)(x + at) = make_uint4(0, 0, 0, 0);
  ptx::fence_before();
  __syncthreads();
  ptx::fence_after();
  const uint32_t tmem = tmem_at;
  // Only now that this CTA holds its TMEM: a CTA of the successor that takes an SM's columns first and waits for this grid, beside one of
  // this grid that waits for columns, would never end.
  ptx::let_successor_start();
  if (!p.behind_rest) ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x == 0 && threadIdx.x == 0) *p.error = 0;

  // ---- the matrix, its norm, and the first iterate
  const uint32_t own_rows = tall ? own : rows, own_cols = tall ? cols : own, first_row = tall ? begin : 0, first_col = tall ? 0 : begin;
  const uint32_t groups_per_row = max(1u, (own_cols + 7) / 8), groups = own_cols ? own_rows * groups_per_row : 0;  // at most 4096 of eight columns
  float u[8][8];
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t group = i * kSmallThreads + threadIdx.x;
    if (group >= groups) break;
    const uint32_t row = group / groups_per_row, col = (group - row * groups_per_row) * 8;
    const int count = min(8u, own_cols - col);
    if (kStep) {
      const int64_t at = (int64_t)p.matrix[which].offset + (first_row + row) * cols + first_col + col;
      float grad[8];
      load8((const T*)p.gradient + worker * p.gradient_row + at, count, grad);
      load8(p.momentum + worker * p.momentum_row + at, count, u[i]);
#pragma unroll
      for (int k = 0; k < 8; ++k) u[i][k] = fmaf(p.mu, u[i][k], grad[k]);
      store8(p.momentum_next + worker * p.momentum_next_row + at, count, u[i]);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (p.nesterov) u[i][k] = fmaf(p.mu, u[i][k], grad[k]);
    } else {
      load8((const T*)p.u + matrix * p.batch + (first_row + row) * p.row + first_col + col, count, u[i]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += (double)u[i][k] * (double)u[i][k];  // (columns that are not there are zeros)
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) squares[warp] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kSmallThreads / 32; ++w) sum += squares[w];
  if (ctas > 1) {
    ptx::cluster_sync();  // (every CTA of the cluster runs)
    if (threadIdx.x < ctas) store_remote(ptx::map_to(ptx::smem(&norms[rank]), threadIdx.x), sum);
    ptx::cluster_sync();
    sum = 0.0;
    for (uint32_t r = 0; r < ctas; ++r) sum += norms[r];
  }
  const Inverse inverse = inverse_norm(sum);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t group = i * kSmallThreads + threadIdx.x;
    if (group >= groups) break;
    const uint32_t row = group / groups_per_row, col = (group - row * groups_per_row) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) u[i][k] = u[i][k] * inverse.a * inverse.b;
    uint4 hi, lo;
    split8(u[i], hi, lo);
    if (!tall) {
      *(uint4*)(x + small_at(side, row, col)) = hi;
      *(uint4*)(x + x_plane + small_at(side, row, col)) = lo;
    } else {
      const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (col + k >= own_cols) break;
        const uint32_t at = small_at(side, col + k, row);
        *(unsigned short*)(x + at) = (unsigned short)(h[k / 2] >> (16 * (k % 2)));
        *(unsigned short*)(x + x_plane + at) = (unsigned short)(l[k / 2] >> (16 * (k % 2)));
      }
    }
  }

  // ---- the steps
  const uint32_t idesc = 1u << 4 | (128 / 16) << 24;  // fp16, sums in fp32, 128 rows
  const uint32_t m = (warp % 4) * 32 + lane;          // this thread's row, and every fourth 16 columns
  const uint32_t from = tmem + ((warp % 4) * 32 << 16);
  const bool live = (warp % 4) * 32 < (int)side;
  const uint32_t parts = (length + 127) / 128;
  // descriptors' low words: X and S k-contiguous, X n-contiguous; offsets in 16 bytes
  const uint32_t low_x = ptx::descriptor_low(ptx::smem(x), 16), low_s = ptx::descriptor_low(ptx::smem(s), 16), low_xn = ptx::descriptor_low(ptx::smem(x), side * 128);
  const uint32_t block = side * 8, plane_x = x_plane >> 4, plane_s = s_plane >> 4;
  bool ok = true;
  uint32_t phase = 0;
  auto products_done = [&] {  // (a thread that gave up once waits no more; all go through the same barriers whatever happens)
    ok = ok && ptx::wait(ptx::smem(&bar), phase & 1);
    ++phase;
    ptx::fence_after();
  };
  auto written = [&] {  // what threads have stored is there for the tensor cores
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    ptx::fence_before();
    __syncthreads();
    ptx::fence_after();
  };
  // S's parts before they are added up: fp32, in the place of its planes, 16-byte pieces swizzled by the row.
  auto part_at = [&](uint32_t row, uint32_t piece) { return row * side * 4 + ((piece ^ (row & 7)) * 16); };
  written();
  for (int step = 0; step < p.steps; ++step) {
    const bool last = step + 1 == p.steps;
    if (warp == 0 && ptx::elect()) {  // S = X X^T
      for (uint32_t part = 0; part < parts; ++part) {
        const uint32_t d = tmem + part * side, i = idesc | side / 8 << 17, blocks = min(2u, (length - part * 128) / 64);
#pragma unroll
        for (int term = 0; term < 3; ++term) {
          uint32_t a = low_x + (term == 1 ? plane_x : 0) + part * 2 * block, b = low_x + (term == 0 ? plane_x : 0) + part * 2 * block;
          for (uint32_t k = 0; k < blocks; ++k, a += block, b += block)
#pragma unroll
            for (int u = 0; u < 4; ++u) ptx::mma<1>(d, ptx::descriptor(a + 2 * u), ptx::descriptor(b + 2 * u), i, term + u > 0 || k > 0);
        }
      }
      ptx::commit<1>(ptx::smem(&bar));
    }
    __syncwarp();
    products_done();
    if (live) {
      for (uint32_t c = (warp / 4) * 16; c < side; c += 64) {
        float v[16], w[16];
        tmem_load16(from + c, v);
        for (uint32_t part = 1; part < parts; ++part) {
          tmem_load16(from + part * side + c, w);
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] += w[k];
        }
        if (ctas > 1) {
#pragma unroll
          for (int k = 0; k < 4; ++k) *(float4*)(s + part_at(m, c / 4 + k)) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
          continue;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float t[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] = v[8 * h + k] * kPlaneUnscale;
          uint4 hi, lo;
          split8(t, hi, lo);
          *(uint4*)(s + small_at(side, m, c + 8 * h)) = hi;
          *(uint4*)(s + s_plane + small_at(side, m, c + 8 * h)) = lo;
        }
      }
    }
    if (ctas > 1) {  // rows rank * side / ctas ... of S, eight columns a thread
      const uint32_t share = side / ctas * (side / 8);
      float t[2][8] = {};  // (two CTAs share out 128 x 128: two pieces a thread, otherwise at most one)
      ptx::fence_before();
      ptx::cluster_sync();  // all parts are there
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t piece = i * kSmallThreads + threadIdx.x;
        if (piece >= share) break;
        const uint32_t row = rank * (side / ctas) + piece / (side / 8), col = piece % (side / 8) * 8;
        for (uint32_t r = 0; r < ctas; ++r) {
          const float4 a = load_remote(ptx::map_to(ptx::smem(s) + part_at(row, col / 4), r)), b = load_remote(ptx::map_to(ptx::smem(s) + part_at(row, col / 4 + 1), r));
          t[i][0] += a.x, t[i][1] += a.y, t[i][2] += a.z, t[i][3] += a.w, t[i][4] += b.x, t[i][5] += b.y, t[i][6] += b.z, t[i][7] += b.w;
        }
      }
      ptx::cluster_sync();  // all have been read
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t piece = i * kSmallThreads + threadIdx.x;
        if (piece >= share) break;
        const uint32_t row = rank * (side / ctas) + piece / (side / 8), col = piece % (side / 8) * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) t[i][k] *= kPlaneUnscale;
        uint4 hi, lo;
        split8(t[i], hi, lo);
        for (uint32_t r = 0; r < ctas; ++r) {
          const uint32_t at = ptx::map_to(ptx::smem(s) + small_at(side, row, col), r);
          store_remote(at, hi);
          store_remote(at + s_plane, lo);
        }
      }
      asm volatile("fence.proxy.async;" ::: "memory");
      ptx::cluster_sync();  // every CTA has all of S
      asm volatile("fence.proxy.async;" ::: "memory");
      ptx::fence_after();
    } else {
      written();
    }
    if (warp == 0 && ptx::elect()) {  // S S
      const uint32_t i = idesc | side / 8 << 17;
#pragma unroll
      for (int term = 0; term < 3; ++term) {
        uint32_t a = low_s + (term == 1 ? plane_s : 0), b = low_s + (term == 0 ? plane_s : 0);
        for (uint32_t k = 0; k < side / 64; ++k, a += block, b += block)
#pragma unroll
          for (int u = 0; u < 4; ++u) ptx::mma<1>(tmem, ptx::descriptor(a + 2 * u), ptx::descriptor(b + 2 * u), i, term + u > 0 || k > 0);
      }
      ptx::commit<1>(ptx::smem(&bar));
    }
    __syncwarp();
    products_done();
    if (live) {
      for (uint32_t c = (warp / 4) * 16; c < side; c += 64) {  // P = b S + c S S in S's place: every thread reads what it writes
        float v[16];
        tmem_load16(from + c, v);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4* at = (uint4*)(s + small_at(side, m, c + 8 * h));
          uint4* at_lo = (uint4*)((unsigned char*)at + s_plane);
          float t[8], f[8];
          unpack_half(*at, t);
          unpack_half(*at_lo, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] = fmaf(p.cc, v[8 * h + k] * kPlaneUnscale, p.cb * (t[k] + f[k]));
          uint4 hi, lo;
          split8(t, hi, lo);
          *at = hi;
          *at_lo = lo;
        }
      }
    }
    written();
    if (warp == 0 && ptx::elect()) {  // P X
      for (uint32_t n = 0; n < length; n += 256) {
        const uint32_t i = idesc | 1u << 16 | min(256u, length - n) / 8 << 17;
#pragma unroll
        for (int term = 0; term < 3; ++term) {
          uint32_t a = low_s + (term == 1 ? plane_s : 0), b = low_xn + (term == 0 ? plane_x : 0) + n / 64 * block;
          for (uint32_t k = 0; k < side / 64; ++k, a += block, b += 64 * 8)
#pragma unroll
            for (int u = 0; u < 4; ++u) ptx::mma<1>(tmem + n, ptx::descriptor(a + 2 * u), ptx::descriptor(b + u * 128), i, term + u > 0 || k > 0);
        }
      }
      ptx::commit<1>(ptx::smem(&bar));
    }
    __syncwarp();
    products_done();
    if (live) {
      for (uint32_t c = (warp / 4) * 16; c < length; c += 64) {
        float v[16];
        tmem_load16(from + c, v);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4* at = (uint4*)(x + small_at(side, m, c + 8 * h));
          uint4* at_lo = (uint4*)((unsigned char*)at + x_plane);
          float t[8], f[8];
          unpack_half(*at, t);
          unpack_half(*at_lo, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] = fmaf(p.ca, t[k] + f[k], v[8 * h + k] * kPlaneUnscale);
          if (!last) {
            uint4 hi, lo;
            split8(t, hi, lo);
            *at = hi;
            *at_lo = lo;
            continue;
          }
          // row m, columns c + 8 h ... of the iterate: a row of the matrix, or a piece of eight of its rows' column m
          if (m >= (tall ? cols : rows) || c + 8 * h >= own) continue;
          const int count = min(8u, own - (c + 8 * h));
          const uint32_t col = begin + c + 8 * h;
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] *= kPlaneUnscale;
          if (!kStep) {
            T* out = (T*)p.out + matrix * p.out_batch;
            if (!tall) {
              store8(out + m * p.out_row + col, count, t);
            } else {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (k < count) out[(int64_t)(col + k) * p.out_row + m] = (T)t[k];
            }
            continue;
          }
          const int64_t first = (int64_t)p.matrix[which].offset + (tall ? (int64_t)col * cols + m : (int64_t)m * cols + col);
          const float scale = p.matrix[which].scale;
          const int peer = p.pull.peers[worker * p.pull.draw_stride];
          const bool pull = peer != worker && (uint32_t)peer < (uint32_t)p.pull.workers;
          const float weight = pull ? p.pull.weights[worker * p.pull.draw_stride] : 0.0f;
          const T* own = (const T*)p.pull.x + worker * p.pull.x_row + first;
          const T* other = (const T*)p.pull.x + (pull ? peer : worker) * p.pull.x_row + first;
          T* next = (T*)p.pull.x_next + worker * p.pull.next_row + first;
          float xi[8], xm[8];
          if (!tall) {
            load8(own, count, xi);
            load8(other, count, xm);
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              xi[k] = k < count ? (float)own[k * cols] : 0.0f;
              xm[k] = k < count ? (float)other[k * cols] : 0.0f;
            }
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float y = fmaf(-p.pull.lr, fmaf(p.pull.decay, xi[k], scale * t[k]), xi[k]);
            t[k] = pull ? fmaf(-weight, y - xm[k], y) : y;
          }
          if (!tall) {
            store8(next, count, t);
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (k < count) next[k * cols] = (T)t[k];
          }
        }
      }
    }
    written();
  }
  if (!ok) {
    *(volatile unsigned int*)p.error = 1;
    __threadfence_system();
  }
  ptx::fence_before();
  __syncthreads();
  if (ctas > 1) ptx::cluster_sync();  // (no CTA's shared memory goes while another one may still use it)
  ptx::fence_after();
  if (warp == 0) ptx::tmem_free<1>(tmem, p.tmem_columns);
  if (p.behind_rest) ptx::wait_for_predecessor();
}

}  // namespace netmax
