// Batched matrix products on the tensor cores (tcgen05, accumulators in TMEM, operands by TMA), one kernel for all of the
// operators that train real weights in the replicas.
//
//   D[m][n] = sum_k A[m][k] B[n][k]        m = the output's rows, n = its contiguous columns
//
// Both operands are 16-bit (fp16 or bf16) and lie in memory either with k contiguous or with m (n) contiguous; the descriptors of the
// tensor cores and the order of the TMA coordinates say which, so no operand is ever transposed.  fp32 operands come as two
// fp16 planes, hi = fp16(s v) and lo = fp16(s v - hi) with s a power of two: 22 bits, so that
//   hi hi + hi lo + lo hi = s^2 A B^T (1 + O(2^-22))
// costs three products in one accumulator instead of one (the term lo lo is below the fp32 accumulator's own rounding).
//
// One CTA pair (cta_group::2) works on a tile of 256 x 256 (two planes: 256 x 128), each CTA with its own 128 rows of A and half the rows
// of B in shared memory: a tile of k = 64 then costs an SM 32 KB from L2 for 512 cycles of tensor work, 48 KB if every CTA worked for
// itself.  Problems that would leave SMs without a tile that way take one CTA per tile of 128 x 64 or 128 x 128.  With two planes the epilogue
// warps hold fp32 sums (see kPromote): of 128 columns they are 32 registers a thread, and sixteen warps finish a tile under the
// products of the next; of 256 columns eight warps held 128 each and the tensor cores waited for them (fp32 layer of 8 x (512 x 512 x 2048):
// 50 us).  The first warps are the
// epilogue, one issues the TMA loads, one the products; the accumulators are double-buffered so that the epilogue of a tile
// runs under the products of the next.
//
// A thread of the epilogue reads one row of 32 columns from TMEM.  Handled as they come, loads and stores of such rows touch 32 lines each
// (and with the roles of rows and columns exchanged 64 bytes each, 22 instructions per 32 elements: the iterates of 8 matrices of 512 x 4608
// took 104 us a product).  So a warp turns its 32 x 32 values around in 4 KB of shared memory: afterwards a lane has eight columns of every
// eighth row, everything in global memory moves in 16-byte pieces of whole 64- or 128-byte lines, and the arithmetic has independent
// elements to interleave.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

namespace netmax {

constexpr int kEpilogueWarps = 16;        // behind them one warp loads and one multiplies
constexpr int kProductThreads = (kEpilogueWarps + 2) * 32;
constexpr int kSlotBytes = 4096;          // of an epilogue warp: 32 x 32 fp32
constexpr int kProductBox = 64;           // a TMA box: 64 rows of 64 16-bit values (128 bytes, the swizzle's width)
constexpr int kBoxBytes = kProductBox * 128;
constexpr int kMaxGroups = 12;            // groups of equal matrices in one launch
constexpr int kMaxMatrices = 256;         // matrices of one replica in one launch
constexpr int kMaxStages = 8;
// Accumulators in TMEM's 512 columns: two of 256, or four of 128.
__host__ __device__ constexpr int accumulators(int planes) { return planes == 2 ? 4 : 2; }
constexpr float kPlaneScale = 16384.0f;   // 2^14: what the planes of Newton-Schulz iterates are scaled by (all |v| < 2.9)
constexpr float kPlaneUnscale = 1.0f / 16384.0f;

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };
enum Epilogue {
  kLayerF32, kLayerBf16,  // y = act(D + bias) + residual, z = D + bias
  kGram,                  // planes of D (symmetric)
  kPolynomial,            // planes of b A + c D (symmetric), A from planes
  kUpdate,                // planes of a X + D, X from planes
  kLastF32, kLastBf16,    // the same, out as fp32 / bf16
  kStepF32, kStepBf16,    // the same, into a worker's local step and its pull
  kPartial,               // D over a part of k, as fp32 (symmetric; combine_kernel adds the parts up)
};

struct ProductGroup {
  CUtensorMap a, b;  // {contiguous, other, matrix, plane}
  int32_t tile_begin = 0, tiles_m = 0, tiles_n = 0;
  int32_t M = 0, N = 0, K = 0;
  int32_t symmetric = 0;       // only tiles up to the diagonal, the others mirrored: a tile's rows over its columns (1 or 2); 0: no
  int32_t a_mn = 0, b_mn = 0;  // m (n) contiguous instead of k
  int32_t a_box = 64, b_box = 64;  // rows of a box
  int32_t splits = 1;          // parts of k, each with a tile of its own
  int32_t bn = 0;              // columns of a tile
  int32_t a_batched = 1, b_batched = 1;  // 0: one matrix for all
  uint32_t idesc = 0;
  // epilogue: element (m, n) of matrix q at base + q * batch + m * row + n
  void* out = nullptr;
  int64_t out_row = 0, out_batch = 0, out_plane = 0;
  void* z = nullptr;
  int64_t z_row = 0, z_batch = 0;
  const void* bias = nullptr;
  int64_t bias_batch = 0;
  const void* residual = nullptr;  // or the planes of A (kPolynomial) and X (kUpdate, kLast*, kStep*)
  int64_t residual_row = 0, residual_batch = 0, residual_plane = 0;
  int32_t activation = 0;
  const int32_t *exp_a = nullptr, *exp_b = nullptr;  // planes hold 2^exp times the values: per matrix, or per row of it
  int32_t exp_a_rows = 0, exp_b_rows = 0;            // rows of a matrix that have exponents of their own; 0: per matrix
  int32_t first_matrix = 0;                          // of the step's table
  int32_t pieces = 0;                                // every row of every view above starts on a 16-byte boundary, and N is a multiple of 8
};

struct PullParams {  // a worker's local step and pull, behind the last product
  const void* x = nullptr;
  void* x_next = nullptr;
  int64_t x_row = 0, next_row = 0;
  const int32_t* peers = nullptr;
  const float* weights = nullptr;
  int32_t draw_stride = 1;  // peers[draw_stride i] and weights[draw_stride i] are worker i's
  float lr = 0, decay = 0;
  int32_t workers = 0;
};

struct ProductParams {
  ProductGroup group[kMaxGroups];
  PullParams step;
  uint32_t matrix_offset[kMaxMatrices];
  float matrix_scale[kMaxMatrices];
  int32_t groups = 0, tiles = 0, planes = 1, stages = 2;
  uint32_t stage_bytes = 0, a_bytes = 0, b_bytes = 0;  // of a stage; of one plane of A and of B in it
  float ca = 0, cb = 0, cc = 0;        // the quintic's coefficients
  unsigned int* error = nullptr;       // raised by a wait that ran out
  int32_t clear_error = 0;
};

// ---- the few instructions that have no CUDA C++ form ------------------------------------------
namespace ptx {
__device__ __forceinline__ uint32_t smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool elect() {
  uint32_t pred;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(pred));
  return pred != 0;
}
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {  // bar: an address of the cluster's window
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t map_to(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// False if the phase did not end within 2^32 cycles (about two seconds) or 2^28 looks, whichever comes first.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) {
  if (try_wait(bar, parity)) return true;
  const long long start = clock64();
  for (uint32_t i = 0; i < (1u << 28); ++i) {
    if (try_wait(bar, parity)) return true;
    if ((i & 1023) == 1023 && clock64() - start > (1ll << 32)) return false;
  }
  return false;
}
template <int kCtas>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
  if (kCtas == 2)
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  if (kCtas == 2)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// Arrives at `bar` (in both CTAs of a pair) when every product issued so far has been done.
template <int kCtas>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (kCtas == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns) {
  if (kCtas == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <int kCtas>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
  if (kCtas == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tmem_load32(uint32_t at, float (&v)[32]) {
  uint32_t r[32];
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_successor_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// Shared-memory descriptor of an operand tile in 128-byte swizzled rows: the low word holds the address and the leading offset, both in
// 16 bytes, so a place further on is a sum of low words.  k contiguous: groups of eight rows are 1024 bytes apart.  m (n) contiguous: a
// row is 64 values of one k; groups of eight k are 1024 bytes apart, blocks of 64 m `leading` bytes.
constexpr uint32_t kDescriptorHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t descriptor_low(uint32_t at, uint32_t leading) { return (at & 0x3FFFF) >> 4 | (leading >> 4) << 16; }
__device__ __forceinline__ uint64_t descriptor(uint32_t low) { return (uint64_t)kDescriptorHigh << 32 | low; }
}  // namespace ptx

// Phi(z) and exp(-z^2 / 2) by formula 7.1.26 of Abramowitz and Stegun's handbook, within 1.5e-7: one exponential and one reciprocal for both
// (with erff and an exponential of its own the gradient's layout of 67 M gelu values took 171 us).
__device__ __forceinline__ float gauss(float z, float& e) {
  const float h = fabsf(z) * 0.70710678118654752f, t = __fdividef(1.0f, fmaf(0.3275911f, h, 1.0f));
  e = __expf(-h * h);
  const float tail = 0.5f * e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
  return z < 0.0f ? tail : 1.0f - tail;
}
// Both within a few units of 2^-24 of 1 + |z|, which is what a sum's rounding leaves of z.
__device__ __forceinline__ float activate(float z, int activation) {
  float e;
  if (activation == kActRelu) return z > 0.0f ? z : (z != z ? z : 0.0f);
  if (activation == kActGelu) return z * gauss(z, e);
  if (activation == kActSilu) return __fdividef(z, 1.0f + __expf(-z));
  return z;
}
__device__ __forceinline__ float activation_slope(float z, int activation) {
  if (activation == kActRelu) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);  // (NaN stays NaN)
  if (activation == kActGelu) {
    float e;
    const float p = gauss(z, e);
    return fmaf(z * 0.39894228040143268f, e, p);
  }
  const float s = __fdividef(1.0f, 1.0f + __expf(-z));
  return s * (1.0f + z * (1.0f - s));
}

struct Tile {
  int g, q, s, i, j;  // group, matrix, part of k, tile row (m) and column (n)
};
__device__ __forceinline__ Tile find_tile(const ProductParams& p, int t) {
  Tile out;
  out.g = 0;
  while (out.g + 1 < p.groups && p.group[out.g + 1].tile_begin <= t) ++out.g;
  const ProductGroup& g = p.group[out.g];
  t -= g.tile_begin;
  if (g.symmetric) {  // row i has the tiles up to the diagonal's: (i + 1) r, the last row as many as there are
    const int r = g.symmetric, per = r * (g.tiles_m * (g.tiles_m - 1) / 2) + g.tiles_n;
    out.q = t / per;
    t -= out.q * per;
    int i = (int)((sqrtf(8.0f * (float)(t / r) + 1.0f) - 1.0f) * 0.5f);  // (at most one off: i is small)
    while (r * (i * (i + 1) / 2) > t) --i;
    while (r * ((i + 1) * (i + 2) / 2) <= t) ++i;
    out.i = i;
    out.j = t - r * (i * (i + 1) / 2);
  } else {
    const int per = g.tiles_m * g.tiles_n;
    out.q = t / per;
    t -= out.q * per;
    out.j = t / g.tiles_m;
    out.i = t - out.j * g.tiles_m;
  }
  out.s = out.q % g.splits;
  out.q /= g.splits;
  return out;
}
// The steps of 64 k of a tile's part.
__device__ __forceinline__ int first_step(const ProductGroup& g, const Tile& t) { return t.s * (((g.K + 63) / 64 + g.splits - 1) / g.splits); }
__device__ __forceinline__ int steps_of(const ProductGroup& g, const Tile& t) {
  const int all = (g.K + 63) / 64, per = (all + g.splits - 1) / g.splits;
  return min(per, all - t.s * per);
}

// Two or four words of packed 16-bit values.
template <int kWords>
__device__ __forceinline__ void load_words(const void* at, uint32_t (&w)[kWords]) {
  if constexpr (kWords == 4) {
    const uint4 a = *(const uint4*)at;
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
  } else {
    const uint2 a = *(const uint2*)at;
    w[0] = a.x, w[1] = a.y;
  }
}
template <int kWords>
__device__ __forceinline__ void store_words(void* at, const uint32_t (&w)[kWords]) {
  if constexpr (kWords == 4) *(uint4*)at = make_uint4(w[0], w[1], w[2], w[3]);
  else *(uint2*)at = make_uint2(w[0], w[1]);
}
// kN values of a type (four or eight), in pieces of up to 16 bytes where the address allows it (kWhole: it does); `count` of them exist.
template <typename T, bool kWhole, int kN>
__device__ __forceinline__ void load_values(const T* at, int count, float (&v)[kN]) {
  constexpr int kPieceBytes = kN * (int)sizeof(T) < 16 ? kN * (int)sizeof(T) : 16;
  if (kWhole || (count == kN && ((uintptr_t)at & (kPieceBytes - 1)) == 0)) {
    if (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < kN; k += 4) {
        const float4 a = *(const float4*)(at + k);
        v[k] = a.x, v[k + 1] = a.y, v[k + 2] = a.z, v[k + 3] = a.w;
      }
    } else {
      uint32_t w[kN / 2];
      load_words(at, w);
#pragma unroll
      for (int k = 0; k < kN / 2; ++k) {
        v[2 * k] = __uint_as_float(w[k] << 16);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = k < count ? (float)at[k] : 0.0f;
  }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *(const uint32_t*)&h;
}
template <typename T, bool kWhole, int kN>
__device__ __forceinline__ void store_values(T* at, int count, const float (&v)[kN]) {
  constexpr int kPieceBytes = kN * (int)sizeof(T) < 16 ? kN * (int)sizeof(T) : 16;
  if (kWhole || (count == kN && ((uintptr_t)at & (kPieceBytes - 1)) == 0)) {
    if (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < kN; k += 4) *(float4*)(at + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    } else {
      uint32_t w[kN / 2];
#pragma unroll
      for (int k = 0; k < kN / 2; ++k) w[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
      store_words(at, w);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kN; ++k)
      if (k < count) at[k] = (T)v[k];
  }
}
template <typename T>
__device__ __forceinline__ void load8(const T* at, int count, float (&v)[8]) { load_values<T, false, 8>(at, count, v); }
template <typename T>
__device__ __forceinline__ void store8(T* at, int count, const float (&v)[8]) { store_values<T, false, 8>(at, count, v); }

// Words of two fp16 each.
template <int kN>
__device__ __forceinline__ void unpack_half(const uint32_t (&w)[kN / 2], float (&v)[kN]) {
#pragma unroll
  for (int k = 0; k < kN / 2; ++k) {
    const float2 f = __half22float2(*(const __half2*)&w[k]);
    v[2 * k] = f.x;
    v[2 * k + 1] = f.y;
  }
}
template <int kN>
__device__ __forceinline__ void pack_half(const float (&v)[kN], uint32_t (&w)[kN / 2]) {
#pragma unroll
  for (int k = 0; k < kN / 2; ++k) {
    const __half2 a = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
    w[k] = *(const uint32_t*)&a;
  }
}
// Values as two planes; what is not finite stays so, once.
template <int kN>
__device__ __forceinline__ void split_values(const float (&v)[kN], uint32_t (&hi)[kN / 2], uint32_t (&lo)[kN / 2]) {
#pragma unroll
  for (int k = 0; k < kN / 2; ++k) {
    const __half2 a = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
    const float2 f = __half22float2(a);
    const __half2 b = __floats2half2_rn(fabsf(f.x) <= 65504.0f ? v[2 * k] - f.x : 0.0f, fabsf(f.y) <= 65504.0f ? v[2 * k + 1] - f.y : 0.0f);
    hi[k] = *(const uint32_t*)&a;
    lo[k] = *(const uint32_t*)&b;
  }
}
__device__ __forceinline__ void unpack_half(const uint4& a, float (&v)[8]) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  unpack_half<8>(w, v);
}
__device__ __forceinline__ void split8(const float (&v)[8], uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
  split_values<8>(v, h, l);
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
// Columns that a lane takes of a row of a staged chunk: eight where 16-bit values are stored, four where fp32 is (16 bytes either way;
// with eight, two stores would each fill halves of their sectors).  32 / kN lanes a row, kN rows at a time, 32 / kN times.
__host__ __device__ constexpr int lane_columns(int epilogue) { return epilogue == kLayerF32 || epilogue == kLastF32 || epilogue == kStepF32 || epilogue == kPartial ? 4 : 8; }

// What an epilogue reads besides the accumulator, both planes, as it will go over the chunk.
template <int kN>
struct Residual {
  uint32_t hi[32 / kN][kN / 2], lo[32 / kN][kN / 2];
};
template <int kEpilogue, int kPlanes>
__device__ __forceinline__ void load_residual(const ProductGroup& g, int q, int m0, int n0, int lane, Residual<lane_columns(kEpilogue)>& r) {
  if (kEpilogue < kPolynomial || kEpilogue >= kStepF32) return;  // (the step reads them along with the replicas)
  constexpr int kN = lane_columns(kEpilogue), kLanes = 32 / kN;
  const int n = n0 + kN * (lane % kLanes), row = lane / kLanes, rows = n < g.N ? g.M - m0 - row : 0;  // (planes' rows are padded to eight columns)
  const __half* at = (const __half*)g.residual + q * g.residual_batch + (int64_t)(m0 + row) * g.residual_row + n;
  const int64_t step = kN * g.residual_row;
#pragma unroll
  for (int i = 0; i < 32 / kN; ++i, at += step) {
#pragma unroll
    for (int k = 0; k < kN / 2; ++k) r.hi[i][k] = r.lo[i][k] = 0;
    if (kN * i < rows) {
      load_words(at, r.hi[i]);
      if (kEpilogue > kPolynomial || kPlanes == 2) load_words(at + g.residual_plane, r.lo[i]);
    }
  }
}

// A thread's 32 columns into its row of the warp's 4 KB: 16-byte pieces, the row's number folded in, so that neither direction meets a
// bank twice.
__device__ __forceinline__ void stage_row(float* slot, const float (&acc)[32]) {
  const int lane = threadIdx.x % 32;
#pragma unroll
  for (int c = 0; c < 8; ++c)
    *(float4*)(slot + lane * 32 + (c ^ (lane & 7)) * 4) = make_float4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
}

template <int kN>
__device__ __forceinline__ void activate_all(float (&v)[kN], int activation) {
  if (activation == kActRelu) {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = activate(v[k], kActRelu);
  } else if (activation == kActGelu) {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = activate(v[k], kActGelu);
  } else if (activation == kActSilu) {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = activate(v[k], kActSilu);
  }
}
// A lane's columns kN c ... of row `row` of the staged chunk.
template <int kN>
__device__ __forceinline__ void read_slot(const float* slot, int row, int c, float (&v)[kN]) {
#pragma unroll
  for (int k = 0; k < kN; k += 4) {
    const float4 a = *(const float4*)(slot + row * 32 + ((kN / 4 * c + k / 4) ^ (row & 7)) * 4);
    v[k] = a.x, v[k + 1] = a.y, v[k + 2] = a.z, v[k + 3] = a.w;
  }
}

// What a chunk's function reads of its group over and over, once in registers: read in place, every use is an indexed load from the
// constant bank that the stores in between make the compiler repeat (a ragged chunk took 5 us so).
struct LayerRows {
  int64_t out, z, residual;
  bool has_z, has_residual, has_bias;
  int activation;
  __device__ __forceinline__ explicit LayerRows(const ProductGroup& g)
      : out(g.out_row), z(g.z_row), residual(g.residual_row), has_z(g.z != nullptr), has_residual(g.residual != nullptr), has_bias(g.bias != nullptr),
        activation(g.activation) {}
};
// 2^e for e in [-126, 127].
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
// v 2^e for e in [-252, 252], in two factors, so that neither leaves fp32's range.
__device__ __forceinline__ float times_power(float v, int e) { return v * power_of_two(e >> 1) * power_of_two(e - (e >> 1)); }
// The exponents of rows and columns of a chunk, NULL where the whole matrix has one.
struct Exponents {
  const int32_t *rows = nullptr, *columns = nullptr;
  __device__ __forceinline__ Exponents(const ProductGroup& g, int q) {
    if (g.exp_a_rows) rows = g.exp_a + (int64_t)(g.a_batched ? q : 0) * g.exp_a_rows;
    if (g.exp_b_rows) columns = g.exp_b + (int64_t)(g.b_batched ? q : 0) * g.exp_b_rows;
  }
};
// y and z of a chunk whose 32 x 32 elements all exist, in 16-byte pieces.
template <typename T>
__device__ __forceinline__ void layer_chunk(const ProductGroup& g, int q, int m0, int n0, int exponent, const float* slot) {
  constexpr int kN = sizeof(T) == 4 ? 4 : 8, kLanes = 32 / kN;
  const int lane = threadIdx.x % 32, c = lane % kLanes, n = n0 + kN * c, row = lane / kLanes;
  const LayerRows g1(g);
  float bias[kN];
  if (g1.has_bias) {
    const T* b = (const T*)g.bias + q * g.bias_batch + n;
#pragma unroll
    for (int k = 0; k < kN; ++k) bias[k] = (float)b[k];
  }
  int column_exponent[kN], row_exponent[32 / kN];
  if (sizeof(T) == 4) {
    const Exponents e(g, q);
#pragma unroll
    for (int k = 0; k < kN; ++k) column_exponent[k] = exponent - (e.columns ? e.columns[n + k] : 0);
#pragma unroll
    for (int i = 0; i < 32 / kN; ++i) row_exponent[i] = e.rows ? e.rows[m0 + row + kN * i] : 0;
  }
  const T* r = (const T*)g.residual + q * g.residual_batch + (int64_t)(m0 + row) * g1.residual + n;
  T* z = (T*)g.z + q * g.z_batch + (int64_t)(m0 + row) * g1.z + n;
  T* y = (T*)g.out + q * g.out_batch + (int64_t)(m0 + row) * g1.out + n;
#pragma unroll
  for (int i = 0; i < 32 / kN; ++i, r += kN * g1.residual, z += kN * g1.z, y += kN * g1.out) {
    float v[kN], add[kN];
    if (g1.has_residual) load_values<T, true>(r, kN, add);
    read_slot(slot, kN * i + row, c, v);
    if (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] = times_power(v[k], column_exponent[k] - row_exponent[i]);
    }
    if (g1.has_bias) {
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] += bias[k];
    }
    if (g1.has_z) store_values<T, true>(z, kN, v);
    activate_all(v, g1.activation);
    if (g1.has_residual) {
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] += add[k];
    }
    store_values<T, true>(y, kN, v);
  }
}
// Of any chunk: a column a lane, so that a row's elements still go out together whatever their alignment.
template <typename T>
__device__ __forceinline__ void ragged_layer_chunk(const ProductGroup& g, int q, int m0, int n0, int exponent, const float* slot) {
  const int lane = threadIdx.x % 32, n = n0 + lane, rows = n < g.N ? min(32, g.M - m0) : 0;
  const LayerRows g1(g);
  const float bias = g1.has_bias && rows > 0 ? (float)((const T*)g.bias)[q * g.bias_batch + n] : 0.0f;
  const Exponents e(g, q);
  if (sizeof(T) == 4 && e.columns && rows > 0) exponent -= e.columns[n];
  const T* r = (const T*)g.residual + q * g.residual_batch + (int64_t)m0 * g1.residual + n;
  T* z = (T*)g.z + q * g.z_batch + (int64_t)m0 * g1.z + n;
  T* y = (T*)g.out + q * g.out_batch + (int64_t)m0 * g1.out + n;
#pragma unroll 1
  for (int i0 = 0; i0 < 32; i0 += 8, r += 8 * g1.residual, z += 8 * g1.z, y += 8 * g1.out) {
    float v[8], add[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u;
      v[u] = slot[i * 32 + ((lane / 4) ^ (i & 7)) * 4 + lane % 4];
      if (sizeof(T) == 4) v[u] = times_power(v[u], exponent - (e.rows && i < rows ? e.rows[m0 + i] : 0));
      v[u] += bias;
    }
    if (g1.has_residual) {
#pragma unroll
      for (int u = 0; u < 8; ++u) add[u] = i0 + u < rows ? (float)r[u * g1.residual] : 0.0f;
    }
    if (g1.has_z) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u < rows) z[u * g1.z] = (T)v[u];
    }
    activate_all(v, g1.activation);
    if (g1.has_residual) {
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] += add[u];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u < rows) y[u * g1.out] = (T)v[u];
  }
}

// The local step and the pull of a chunk of a worker's matrix.
template <typename T, int kN, int kAhead>
__device__ __forceinline__ void step_chunk(const ProductParams& p, const ProductGroup& g, int q, int m0, int n0, const float* slot) {
  constexpr int kLanes = 32 / kN;
  const int lane = threadIdx.x % 32, c = lane % kLanes, n = n0 + kN * c, row = lane / kLanes, count = min(kN, g.N - n), rows = count > 0 ? g.M - m0 - row : 0;
  const PullParams& s = p.step;
  const int matrix = g.first_matrix + q / s.workers, worker = q % s.workers;
  const float scale = p.matrix_scale[matrix] * kPlaneUnscale;
  const int peer = s.peers[worker * s.draw_stride];
  const bool pull = peer != worker && (uint32_t)peer < (uint32_t)s.workers;
  const float w = pull ? s.weights[worker * s.draw_stride] : 0.0f;
  const int64_t at = (int64_t)p.matrix_offset[matrix] + (int64_t)(m0 + row) * g.out_row + n, step = kN * g.out_row;
  const T* own = (const T*)s.x + worker * s.x_row + at;
  const T* other = (const T*)s.x + (pull ? peer : worker) * s.x_row + at;
  T* next = (T*)s.x_next + worker * s.next_row + at;
  const bool whole = count == kN && (((uintptr_t)own | (uintptr_t)other | (uintptr_t)next | (uintptr_t)(step * sizeof(T))) & 15) == 0;
  const int64_t plane = g.residual_plane, plane_step = kN * g.residual_row;
  const float ca = p.ca, lr = s.lr, decay = s.decay;
  const __half* planes = (const __half*)g.residual + q * g.residual_batch + (int64_t)(m0 + row) * g.residual_row + n;
#pragma unroll
  for (int i0 = 0; i0 < 32 / kN; i0 += kAhead) {  // kAhead rows in flight
    float xi[kAhead][kN], xm[kAhead][kN];
    uint32_t hi[kAhead][kN / 2], lo[kAhead][kN / 2];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (kN * (i0 + u) >= rows) break;
      load_words(planes + (i0 + u) * plane_step, hi[u]);
      load_words(planes + (i0 + u) * plane_step + plane, lo[u]);
      if (whole) {
        load_values<T, true>(own + (i0 + u) * step, kN, xi[u]);
        load_values<T, true>(other + (i0 + u) * step, kN, xm[u]);
      } else {
        load_values<T, false>(own + (i0 + u) * step, count, xi[u]);
        load_values<T, false>(other + (i0 + u) * step, count, xm[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u;
      if (kN * i >= rows) break;
      float v[kN], x[kN], xl[kN];
      read_slot(slot, kN * i + row, c, v);
      unpack_half<kN>(hi[u], x);
      unpack_half<kN>(lo[u], xl);
#pragma unroll
      for (int k = 0; k < kN; ++k) {
        const float o = scale * fmaf(ca, x[k] + xl[k], v[k] * kPlaneUnscale);
        const float h = fmaf(-lr, fmaf(decay, xi[u][k], o), xi[u][k]);
        v[k] = pull ? fmaf(-w, h - xm[u][k], h) : h;
      }
      if (whole) store_values<T, true>(next + i * step, kN, v);
      else store_values<T, false>(next + i * step, count, v);
    }
  }
}

// Rows m0 ... m0 + 31 and columns n0 ... n0 + 31 of the accumulator, which the warp has staged.  Called from one place in a loop: unrolled
// over a tile's chunks the code outgrew the instruction cache (the 8 x (4096 x 4096 x 4096) layer with silu: 1715 us).
template <int kEpilogue, int kPlanes>
__device__ __forceinline__ void epilogue_chunk(const ProductParams& p, const ProductGroup& g, const Tile& t, int m0, int n0, int exponent, float* slot,
                                               const Residual<lane_columns(kEpilogue)>& residual) {
  const int lane = threadIdx.x % 32;
  __syncwarp();
  if (kEpilogue == kLayerF32 || kEpilogue == kLayerBf16) {
    using T = typename std::conditional<kEpilogue == kLayerF32, float, __nv_bfloat16>::type;
    if (g.pieces && m0 + 32 <= g.M && n0 + 32 <= g.N) layer_chunk<T>(g, t.q, m0, n0, exponent, slot);
    else ragged_layer_chunk<T>(g, t.q, m0, n0, exponent, slot);
    return;
  }
  if (kEpilogue == kStepF32 || kEpilogue == kStepBf16) {
    using T = typename std::conditional<kEpilogue == kStepF32, float, __nv_bfloat16>::type;
    step_chunk<T, lane_columns(kEpilogue), kPlanes == 2 ? 2 : 1>(p, g, t.q, m0, n0, slot);
    return;
  }
  constexpr int kN = lane_columns(kEpilogue), kLanes = 32 / kN;
  const int c = lane % kLanes, n = n0 + kN * c, row = lane / kLanes, count = min(kN, g.N - n), rows = count > 0 ? g.M - m0 - row : 0;
  const int64_t out_step = kN * g.out_row, out_plane = g.out_plane;  // (in registers: see LayerRows)
  const float ca = p.ca, cb = p.cb, cc = p.cc;
  if (kEpilogue == kPartial) {
    float* out = (float*)g.out + (int64_t)(t.q * g.splits + t.s) * g.out_batch + (int64_t)(m0 + row) * g.out_row + n;
#pragma unroll
    for (int i = 0; i < 32 / kN; ++i, out += out_step) {
      if (kN * i >= rows) break;
      float v[kN];
      read_slot(slot, kN * i + row, c, v);
      store_values<float, true>(out, kN, v);  // (rows are padded to eight columns)
    }
    return;
  }
  if (kEpilogue == kLastF32 || kEpilogue == kLastBf16) {
    using T = typename std::conditional<kEpilogue == kLastF32, float, __nv_bfloat16>::type;
    T* out = (T*)g.out + t.q * g.out_batch + (int64_t)(m0 + row) * g.out_row + n;
    const bool pieces = g.pieces;
#pragma unroll
    for (int i = 0; i < 32 / kN; ++i, out += out_step) {
      if (kN * i >= rows) break;
      float v[kN], x[kN], lo[kN];
      read_slot(slot, kN * i + row, c, v);
      unpack_half<kN>(residual.hi[i], x);
      unpack_half<kN>(residual.lo[i], lo);
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] = kPlaneUnscale * fmaf(ca, x[k] + lo[k], v[k] * kPlaneUnscale);
      if (pieces) store_values<T, true>(out, kN, v);
      else store_values<T, false>(out, count, v);
    }
    return;
  }
  const bool mirrored = kEpilogue != kUpdate && t.j < g.symmetric * t.i;
  __half* out = (__half*)g.out + t.q * g.out_batch + (int64_t)(m0 + row) * g.out_row + n;
#pragma unroll
  for (int i = 0; i < 4; ++i, out += out_step) {
    if (8 * i >= rows) break;
    float v[kN], x[kN], lo[kN];
    read_slot(slot, 8 * i + row, c, v);
    if (kEpilogue >= kPolynomial) {
      unpack_half<kN>(residual.hi[i], x);
      if (kEpilogue == kUpdate || kPlanes == 2) {
        unpack_half<kN>(residual.lo[i], lo);
#pragma unroll
        for (int k = 0; k < kN; ++k) x[k] += lo[k];
      }
    }
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      v[k] *= kPlaneUnscale;
      if (kEpilogue == kPolynomial) v[k] = fmaf(cc, v[k], cb * x[k]);
      if (kEpilogue == kUpdate) v[k] = fmaf(ca, x[k], v[k]);
    }
    uint32_t h[kN / 2], l[kN / 2] = {};
    if (kEpilogue == kUpdate || kPlanes == 2) split_values<kN>(v, h, l);
    else pack_half<kN>(v, h);
    store_words(out, h);
    if (kEpilogue == kUpdate || kPlanes == 2) store_words(out + out_plane, l);
    if (mirrored) {  // both planes of an element in one word
      const int r = 8 * i + row;
#pragma unroll
      for (int k = 0; k < 2; ++k)
        *(uint4*)(slot + r * 32 + ((2 * c + k) ^ (r & 7)) * 4) = make_uint4(__byte_perm(h[2 * k], l[2 * k], 0x5410), __byte_perm(h[2 * k], l[2 * k], 0x7632),
                                                                           __byte_perm(h[2 * k + 1], l[2 * k + 1], 0x5410), __byte_perm(h[2 * k + 1], l[2 * k + 1], 0x7632));
    }
  }
  if (!mirrored) return;
  __syncwarp();  // rows n0 + ..., columns m0 + ...
  const int m = m0 + 8 * c, all_columns = g.N, all_rows = g.M;
  out = (__half*)g.out + t.q * g.out_batch + (int64_t)(n0 + row) * g.out_row + m;
#pragma unroll
  for (int i = 0; i < 4; ++i, out += out_step) {
    const int column = 8 * i + row;
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(slot[(8 * c + k) * 32 + ((column / 4) ^ k) * 4 + column % 4]);
    if (n0 + column >= all_columns || m >= all_rows) continue;
    *(uint4*)out = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[4], w[5], 0x5410), __byte_perm(w[6], w[7], 0x5410));
    if (kPlanes == 2)
      *(uint4*)(out + out_plane) = make_uint4(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632), __byte_perm(w[4], w[5], 0x7632), __byte_perm(w[6], w[7], 0x7632));
  }
}

// kPlanes = 2 (fp32 operands): every kPromote steps of 64 k the accumulator goes to fp32 registers and starts over.  The tensor cores drop
// what lies below the running sum's last bit at every 16 k, so the error grows with k (2-norm, K = 2048: 7.4e-6); with the sum taken over
// every 256 k it is 8.4e-7 at any K (fp32 FMAs: 4.1e-7 at K = 512, 1.1e-6 at 4096), every 128 k 3.9e-7, but then the products wait for
// accumulators (four layers of 2048 x 2048 x 2048: 183 us, 172 so, 168 without).
constexpr int kPromote = 4;
// One plane: products of up to 2^15 k stay in one accumulator.  What its 2^11 steps drop of a sum whose terms have one sign is then at most
// 2^-12 of it, a sixteenth of bfloat16's rounding (sums of 2^23 positive products came out 5 % too small without a limit).  kLong has the epilogue add up
// parts of that length, in local memory: it is touched once in 512 steps (in registers a warp has room for one chunk, and tiles of half the columns
// took 7.1 ms instead of 4.7 for the gradient of 65,536 x 4096 x 4096).  Its instances are those whose k is a batch's rows, a layer's inputs or outputs
// or a matrix's longer side; the others' k is a smaller side, at most 46,340.
constexpr int kLongPart = 512;

template <int kCtas, int kEpilogue, int kPlanes, bool kLong = false>
__global__ __launch_bounds__(kProductThreads, 1) void product_kernel(const __grid_constant__ ProductParams p) {
  static_assert(kPlanes == 1 || !kLong, "two planes have short parts anyway");
  constexpr int kLoader = kEpilogueWarps, kMultiplier = kEpilogueWarps + 1;
  extern __shared__ unsigned char raw[];
  constexpr int kAccumulators = accumulators(kPlanes), kAccumulatorColumns = 512 / kAccumulators;
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 2 * kAccumulators];
  __shared__ uint32_t tmem_at;
  __shared__ volatile uint32_t gave_up;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = kCtas == 2 ? ptx::cluster_rank() : 0;
  // (the same offset in both CTAs of a pair: dynamic shared memory starts at the same address in every CTA)
  const uint32_t base = (ptx::smem(raw) + 1023) & ~1023u;
  float* const slots = (float*)(raw + (base - ptx::smem(raw)) + (size_t)p.stages * p.stage_bytes);
  const uint32_t full = ptx::smem(bars), empty = full + 8 * kMaxStages, done = empty + 8 * kMaxStages, drained = done + 8 * kAccumulators;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      ptx::barrier_init(full + 8 * s, 1);
      ptx::barrier_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < kAccumulators; ++b) {
      ptx::barrier_init(done + 8 * b, 1);
      ptx::barrier_init(drained + 8 * b, kEpilogueWarps * kCtas);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    gave_up = 0;
  }
  if (warp == kMultiplier) ptx::tmem_alloc<kCtas>(ptx::smem(&tmem_at), 512);
  ptx::fence_before();
  __syncthreads();
  if (kCtas == 2) ptx::cluster_sync();
  ptx::fence_after();
  const uint32_t tmem = tmem_at;
  ptx::let_successor_start();
  ptx::wait_for_predecessor();
  if (p.clear_error && blockIdx.x == 0 && threadIdx.x == 0) *p.error = 0;

  const int first = blockIdx.x / kCtas, stride = gridDim.x / kCtas;
  auto failed = [&] {
    gave_up = 1;
    *(volatile unsigned int*)p.error = 1;
    __threadfence_system();
  };
  if (warp == kLoader && ptx::elect()) {  // ---- loads
    int issued = 0;  // stages filled so far
    bool ok = true;
    for (int t = first; t < p.tiles && ok; t += stride) {
      const Tile tile = find_tile(p, t);
      const ProductGroup& g = p.group[tile.g];
      const int rows_b = g.bn / kCtas;
      const int m0 = (tile.i * kCtas + (int)rank) * 128, n0 = tile.j * g.bn + (int)rank * rows_b;
      const int qa = g.a_batched ? tile.q : 0, qb = g.b_batched ? tile.q : 0;
      const int boxes_b = rows_b / kProductBox;
      const uint32_t bytes = (uint32_t)(kPlanes * (2 + boxes_b) * kBoxBytes) * kCtas;
      const int steps = steps_of(g, tile), before = first_step(g, tile);
      for (int kb = 0; kb < steps; ++kb, ++issued) {
        const int s = issued % p.stages, lap = issued / p.stages;
        if (lap > 0 && !ptx::wait(empty + 8 * s, (lap - 1) & 1)) { ok = false; break; }
        if (gave_up) { ok = false; break; }
        if (rank == 0) ptx::expect_tx(full + 8 * s, bytes);
        const uint32_t bar = kCtas == 2 ? ptx::map_to(full + 8 * s, 0) : full + 8 * s;
        const uint32_t at = base + s * p.stage_bytes;
        for (int plane = 0; plane < kPlanes; ++plane) {
          for (int b = 0; b < 2; b += g.a_box / 64)
            ptx::load_box<kCtas>(at + plane * p.a_bytes + b * kBoxBytes, &g.a, bar, g.a_mn ? m0 + 64 * b : (before + kb) * 64, g.a_mn ? (before + kb) * 64 : m0 + 64 * b, qa, plane);
          for (int b = 0; b < boxes_b; b += g.b_box / 64)
            ptx::load_box<kCtas>(at + kPlanes * p.a_bytes + plane * p.b_bytes + b * kBoxBytes, &g.b, bar, g.b_mn ? n0 + 64 * b : (before + kb) * 64,
                                 g.b_mn ? (before + kb) * 64 : n0 + 64 * b, qb, plane);
        }
      }
    }
    if (!ok) failed();
    // no CTA leaves while its own copies are under way: what is still in flight ends within the limit of these waits
    for (int back = min(issued, p.stages); back > 0; --back) {
      const int k = issued - back, s = k % p.stages, lap = k / p.stages;
      if (!ptx::wait((ok ? empty : full) + 8 * s, lap & 1) && ok) {
        ok = false;
        failed();
      }
    }
  } else if (warp == kMultiplier && rank == 0 && ptx::elect()) {  // ---- products
    int used = 0, part = 0;  // stages and accumulators so far
    bool ok = true;
    for (int t = first; t < p.tiles && ok; t += stride) {
      const Tile tile = find_tile(p, t);
      const ProductGroup& g = p.group[tile.g];
      // (in 16 bytes, all worked out here: one thread issues, and a product of 256 x 128 x 16 takes 64 cycles)
      const uint32_t step_a = (g.a_mn ? 2048 : 32) >> 4, step_b = (g.b_mn ? 2048 : 32) >> 4;  // 16 k further
      const uint32_t low_a = ptx::descriptor_low(base, g.a_mn ? kBoxBytes : 16), low_b = ptx::descriptor_low(base + kPlanes * p.a_bytes, g.b_mn ? kBoxBytes : 16);
      const uint32_t plane_a = p.a_bytes >> 4, plane_b = p.b_bytes >> 4, stage_step = p.stage_bytes >> 4, idesc = g.idesc;
      const int steps = steps_of(g, tile), per_part = kPlanes == 2 ? kPromote : kLong ? kLongPart : steps;
      for (int begin = 0; begin < steps && ok; begin += per_part, ++part) {
        const int acc = part % kAccumulators, lap = part / kAccumulators;
        if (lap > 0 && !ptx::wait(drained + 8 * acc, (lap - 1) & 1)) { ok = false; break; }
        ptx::fence_after();
        const uint32_t d = tmem + acc * kAccumulatorColumns;
        for (int kb = begin; kb < min(steps, begin + per_part); ++kb, ++used) {
          const int s = used % p.stages;
          if (!ptx::wait(full + 8 * s, (used / p.stages) & 1) || gave_up) { ok = false; break; }
          ptx::fence_after();
          const uint32_t at = s * stage_step;
#pragma unroll
          for (int term = 0; term < (kPlanes == 2 ? 3 : 1); ++term) {  // hi lo, lo hi, hi hi: the small ones first
            const uint32_t a = low_a + at + (kPlanes == 2 && term == 1 ? plane_a : 0), b = low_b + at + (kPlanes == 2 && term == 0 ? plane_b : 0);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              ptx::mma<kCtas>(d, ptx::descriptor(a + k * step_a), ptx::descriptor(b + k * step_b), idesc, kb > begin || term + k > 0);
          }
          ptx::commit<kCtas>(empty + 8 * s);
        }
        if (ok) ptx::commit<kCtas>(done + 8 * acc);
      }
    }
    if (!ok) failed();
  } else if (warp < kEpilogueWarps) {  // ---- epilogue: warp w has lanes 32 (w % 4) ... of the accumulator and every second (fourth) 32 columns from w / 4 on
    const uint32_t quadrant = warp % 4, column = warp / 4 * 32;
    float* const slot = slots + warp * (kSlotBytes / 4);
    int part = 0;
    bool ok = true;
    for (int t = first; t < p.tiles && ok; t += stride) {
      const Tile tile = find_tile(p, t);
      const ProductGroup& g = p.group[tile.g];
      const int m0 = (tile.i * kCtas + (int)rank) * 128 + (int)quadrant * 32, n0 = tile.j * g.bn;
      const int columns = m0 < g.M ? min(g.bn, g.N - n0) : 0;
      int exponent = 0;
      if (kEpilogue == kLayerF32) exponent = -((g.exp_a_rows ? 0 : g.exp_a[g.a_batched ? tile.q : 0]) + (g.exp_b_rows ? 0 : g.exp_b[g.b_batched ? tile.q : 0]));
      const int steps = steps_of(g, tile), per_part = kPlanes == 2 ? kPromote : kLong ? kLongPart : steps;
      Residual<lane_columns(kEpilogue)> residual;
      if ((int)column < columns) load_residual<kEpilogue, kPlanes>(g, tile.q, m0, n0 + column, lane, residual);
      float sum[32], before[kLong ? 2 : 1][32];  // of the warp's chunks, up to this part
      if (kPlanes == 2) {
#pragma unroll
        for (int c = 0; c < 32; ++c) sum[c] = 0.0f;
      }
      for (int begin = 0; begin < steps; begin += per_part, ++part) {
        const int acc = part % kAccumulators, lap = part / kAccumulators;
        if (!__all_sync(0xFFFFFFFFu, ptx::wait(done + 8 * acc, lap & 1))) {
          if (lane == 0) failed();
          ok = false;
          break;
        }
        ptx::fence_after();
        const uint32_t from = tmem + (quadrant * 32 << 16) + acc * kAccumulatorColumns;
        if (kPlanes == 2) {
          if ((int)column < columns) {
            float v[32];
            ptx::tmem_load32(from + column, v);
#pragma unroll
            for (int e = 0; e < 32; ++e) sum[e] += v[e];
          }
        } else {
#pragma unroll 1
          for (int c = (int)column; c < columns; c += 128) {
            if (c != (int)column) load_residual<kEpilogue, kPlanes>(g, tile.q, m0, n0 + c, lane, residual);
            ptx::tmem_load32(from + c, sum);
            if (kLong) {
              float* const so_far = before[c / 128];
              if (begin > 0) {
#pragma unroll
                for (int e = 0; e < 32; ++e) sum[e] += so_far[e];
              }
              if (begin + per_part < steps) {
#pragma unroll
                for (int e = 0; e < 32; ++e) so_far[e] = sum[e];
                continue;
              }
            }
            __syncwarp();
            stage_row(slot, sum);
            epilogue_chunk<kEpilogue, kPlanes>(p, g, tile, m0, n0 + c, exponent, slot, residual);
          }
        }
        ptx::fence_before();
        __syncwarp();
        if (lane == 0) {
          if (kCtas == 2) ptx::arrive_cluster(ptx::map_to(drained + 8 * acc, 0));
          else asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(drained + 8 * acc) : "memory");
        }
      }
      if (kPlanes == 2 && ok && (int)column < columns) {
        __syncwarp();
        stage_row(slot, sum);
        epilogue_chunk<kEpilogue, kPlanes>(p, g, tile, m0, n0 + column, exponent, slot, residual);
      }
    }
  }
  __syncwarp();
  ptx::fence_before();
  __syncthreads();
  if (kCtas == 2) ptx::cluster_sync();  // (neither CTA's shared memory goes while the other may still signal it)
  ptx::fence_after();
  if (warp == kMultiplier) ptx::tmem_free<kCtas>(tmem, 512);
}

}  // namespace netmax
