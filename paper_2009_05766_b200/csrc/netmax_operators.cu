// Host side of the operators on real weights: validation, workspaces, tensor maps, launches.
#include "../../include/netmax.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <numeric>
#include <tuple>
#include <unordered_map>
#include <vector>

#include "netmax_few_rows.cuh"
#include "netmax_operators.cuh"
#include "netmax_operators.h"
#include "netmax_policy.h"
#include "netmax_small.cuh"

using namespace netmax;

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr size_t kHeader = 256;                      // of a workspace: the error word
constexpr size_t kProductSmem = (size_t)225 * 1024;  // dynamic shared memory that a launch may take
constexpr size_t kLeastSmem = (size_t)120 * 1024;    // more than half an SM's: no two of these CTAs, which take all of TMEM, share one

int fail_op(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_global_error(buf);
  return code;
}
int fail_caught(int code, const char* what) { return fail_op(code, "%s", what); }

#define OP_CUDA(call)                                                                          \
  do {                                                                                         \
    cudaError_t e_ = (call);                                                                   \
    if (e_ != cudaSuccess)                                                                     \
      return fail_op(e_ == cudaErrorMemoryAllocation ? NETMAX_OOM : NETMAX_CUDA_ERROR, "%s: %s", #call, cudaGetErrorString(e_)); \
  } while (0)
#define OP_DO(call)          \
  do {                       \
    int rc_ = (call);        \
    if (rc_) return rc_;     \
  } while (0)

struct OnDevice {
  int prev = -1;
  bool ok = true;
  explicit OnDevice(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
    if (prev != dev) ok = cudaSetDevice(dev) == cudaSuccess;
    if (!ok) cudaGetLastError();
  }
  ~OnDevice() {
    int cur = -1;
    if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
  }
};

cudaError_t raise_smem_limit(const void* kernel, size_t bytes) {
  struct Limit {
    uint64_t context = 0;
    size_t bytes = 0;
  };
  static std::mutex mu;
  static auto* set = new std::unordered_map<uint64_t, Limit>();
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t key = (uint64_t)(uintptr_t)kernel * 64u + (uint64_t)(dev & 63), context = context_number();
  std::lock_guard<std::mutex> lock(mu);
  Limit& have = (*set)[key];
  if (have.context == context && bytes <= have.bytes) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) {
    have.context = context;
    have.bytes = bytes;
  }
  return e;
}

int sm_count() {
  static std::atomic<int> known[64];
  int dev = 0, n = 148;
  if (cudaGetDevice(&dev) != cudaSuccess) return n;
  if (const int have = known[dev & 63].load()) return have;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) known[dev & 63].store(n);
  return n;
}

size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }
int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
template <typename T>
T ceil_div(T a, T b) { return (a + b - 1) / b; }

// Carves up a workspace, or only counts.
struct Carver {
  unsigned char* base;
  size_t used = kHeader;
  explicit Carver(void* p) : base((unsigned char*)p) {}
  void* take(size_t bytes) {
    void* at = base ? base + used : nullptr;
    used += up(bytes, 256);
    return at;
  }
};

// ---- tensor maps ------------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encoder() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult status;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &status) != cudaSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return (EncodeTiled)p;
  }();
  return f;
}

// 16-bit matrices for the tensor cores: element (outer, inner) of matrix q in plane s.
struct Operand {
  const void* data = nullptr;
  bool bf16 = false;
  int64_t inner = 0, outer = 0, row = 0, batch = 0, plane = 0;
  int count = 1, planes = 1;
  // maps for boxes of 64 and 128 rows, made when a launch first asks for them
  mutable bool have[2] = {false, false};
  mutable CUtensorMap map[2];
};
int tensor_map(const Operand& o, int box_rows, CUtensorMap* out) {
  const int k = box_rows == 128;
  if (!o.have[k]) {
    const EncodeTiled f = encoder();
    if (!f) return fail_op(NETMAX_CUDA_ERROR, "the driver has no cuTensorMapEncodeTiled");
    const cuuint64_t dims[4] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)o.count, (cuuint64_t)o.planes};
    const int64_t whole = o.row * std::max<int64_t>(1, o.outer);
    const cuuint64_t strides[3] = {(cuuint64_t)o.row * 2, (cuuint64_t)(o.count > 1 ? o.batch : whole) * 2, (cuuint64_t)(o.planes > 1 ? o.plane : whole) * 2};
    const cuuint32_t box[4] = {kProductBox, (cuuint32_t)box_rows, 1, 1}, steps[4] = {1, 1, 1, 1};
    const CUresult r = f(&o.map[k], o.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(o.data), dims, strides, box,
                         steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
      return fail_op(NETMAX_CUDA_ERROR, "cuTensorMapEncodeTiled: error %d (%lld x %lld, row %lld, %d matrices %lld apart)", (int)r, (long long)o.outer,
                     (long long)o.inner, (long long)o.row, o.count, (long long)o.batch);
    o.have[k] = true;
  }
  *out = o.map[k];
  return NETMAX_OK;
}

// ---- launches -----------------------------------------------------------------------------------
struct Stream {
  cudaStream_t stream;
  unsigned int* error;
  bool clear = true;  // the next kernel resets the error word (every call's first one does)
  int64_t launches = 0;
};

template <typename... Params, typename... Args>
int launch(Stream& s, void (*kernel)(Params...), dim3 grid, int threads, size_t smem, int cluster, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s.stream;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // (every kernel here waits for its predecessor itself)
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = (unsigned)cluster;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  OP_CUDA(cudaLaunchKernelEx(&cfg, kernel, Params(args)...));
  s.launches += 1;
  return NETMAX_OK;
}

using ProductKernel = void (*)(const ProductParams);
template <int kCtas>
ProductKernel pick_product(int epilogue, int planes, bool long_sums) {
  if (long_sums)
    return epilogue == kLayerBf16 ? product_kernel<kCtas, kLayerBf16, 1, true> : epilogue == kGram ? product_kernel<kCtas, kGram, 1, true>
                                                                                                   : product_kernel<kCtas, kPartial, 1, true>;
  switch (epilogue) {
    case kLayerF32: return product_kernel<kCtas, kLayerF32, 2>;
    case kLayerBf16: return product_kernel<kCtas, kLayerBf16, 1>;
    case kGram: return planes == 2 ? product_kernel<kCtas, kGram, 2> : product_kernel<kCtas, kGram, 1>;
    case kPolynomial: return planes == 2 ? product_kernel<kCtas, kPolynomial, 2> : product_kernel<kCtas, kPolynomial, 1>;
    case kUpdate: return planes == 2 ? product_kernel<kCtas, kUpdate, 2> : product_kernel<kCtas, kUpdate, 1>;
    case kLastF32: return product_kernel<kCtas, kLastF32, 2>;
    case kLastBf16: return product_kernel<kCtas, kLastBf16, 1>;
    case kStepF32: return product_kernel<kCtas, kStepF32, 2>;
    case kPartial: return planes == 2 ? product_kernel<kCtas, kPartial, 2> : product_kernel<kCtas, kPartial, 1>;
    default: return product_kernel<kCtas, kStepBf16, 1>;
  }
}

// What a group of a launch multiplies.
struct Factors {
  const Operand *a = nullptr, *b = nullptr;
  int batch = 0;
  float* parts = nullptr;  // kGram: room for the sums over parts of k, most_splits of them
  int64_t most_splits = 1;
};

// Chooses the tile shape for all groups of a launch and runs it.
int run_products(Stream& s, ProductParams& p, const Factors* factors, int epilogue) {
  for (int k = 0; k < p.groups; ++k) {
    ProductGroup& g = p.group[k];
    const int64_t unit = epilogue == kLayerBf16 || epilogue == kLastBf16 ? 8 : 4;
    auto fits = [&](const void* at, int64_t row, int64_t batch) { return ((uintptr_t)at & 15) == 0 && row % unit == 0 && (factors[k].batch == 1 || batch % unit == 0); };
    const bool layer = epilogue == kLayerF32 || epilogue == kLayerBf16;
    g.pieces = g.N % 8 == 0 && fits(g.out, g.out_row, g.out_batch) && (!layer || ((!g.z || fits(g.z, g.z_row, g.z_batch)) &&
               (!g.residual || fits(g.residual, g.residual_row, g.residual_batch))));
  }
  const int sms = sm_count();
  auto tiles_of = [&](const ProductGroup& g, int batch, int tile_m, int bn) {
    const int64_t tm = ceil_div(g.M, tile_m), tn = ceil_div(g.N, bn);
    return (int64_t)batch * (g.symmetric ? tile_m / bn * (tm * (tm - 1) / 2) + tn : tm * tn);
  };
  bool long_sums = false;  // (see kLongPart)
  for (int k = 0; k < p.groups; ++k) long_sums = long_sums || (p.planes == 1 && (epilogue == kLayerBf16 || epilogue == kGram) && p.group[k].K > kLongPart * 64);
  // Columns of a pair's tile: 256 with one plane, 128 with two (and of narrow outputs; symmetric ones never have more columns than rows).
  auto pair_columns = [&](const ProductGroup& g) { return p.planes == 2 || (!g.symmetric && g.N <= 128) ? 128 : 256; };
  int64_t pairs = 0, wide = 0, area = 0;
  for (int k = 0; k < p.groups; ++k) {
    const ProductGroup& g = p.group[k];
    const int64_t n = tiles_of(g, factors[k].batch, 256, pair_columns(g));
    pairs += n;
    area += n * 256 * pair_columns(g);
    wide += tiles_of(g, factors[k].batch, 128, 128);
  }
  // pairs where they keep four fifths of the SMs busy and cover not much more than tiles of 128 x 128 would (32 rows of 8 workers' fp32
  // 4096 x 4096 layers: the call takes 375 us with half of every pair's tile empty, 308 so)
  int ctas = pairs * 5 >= sms / 2 * 4 && area * 2 <= wide * 128 * 128 * 3 ? 2 : 1;
  if (epilogue == kGram && p.groups == 1 && factors[0].parts && ctas == 1 && area * 2 <= wide * 128 * 128 * 3) {
    const int64_t most = std::min<int64_t>(factors[0].most_splits, ceil_div(p.group[0].K, 64) / 8);
    if (pairs * most * 5 >= sms / 2 * 4) ctas = 2;  // in parts of k: see below
  }
  int64_t tiles = 0, combine_blocks = 0;
  int most_b = 0;
  for (int k = 0; k < p.groups; ++k) {
    ProductGroup& g = p.group[k];
    if (ctas == 2) g.bn = pair_columns(g);
    else g.bn = g.symmetric ? 128 : g.N <= 64 || wide * 2 <= sms ? 64 : 128;
    g.tiles_m = ceil_div(g.M, 128 * ctas);
    g.tiles_n = ceil_div(g.N, g.bn);
    if (g.symmetric) g.symmetric = 128 * ctas / g.bn;
    g.tile_begin = (int)tiles;
    tiles += tiles_of(g, factors[k].batch, 128 * ctas, g.bn);
    // the longer a box, the fewer of them: 128 rows of a k-contiguous operand (8 x 4096^3: 950 us with boxes of 64, 880 so)
    g.a_box = g.a_mn ? 64 : 128;
    g.b_box = g.b_mn || g.bn / ctas < 128 ? 64 : 128;
    OP_DO(tensor_map(*factors[k].a, g.a_box, &g.a));
    OP_DO(tensor_map(*factors[k].b, g.b_box, &g.b));
    g.idesc = 1u << 4 | (factors[k].a->bf16 ? 1u << 7 | 1u << 10 : 0u) | (uint32_t)g.a_mn << 15 | (uint32_t)g.b_mn << 16 | (uint32_t)(g.bn / 8) << 17 |
              (uint32_t)(128 * ctas / 16) << 24;
    most_b = std::max(most_b, g.bn / ctas);
  }
  if (tiles == 0) return NETMAX_OK;
  // Few tiles with long sums: several CTAs (or pairs) add up parts of k, and a launch behind them the parts.  At least eight steps of 64 k
  // a part.
  CombineParams combine;
  if (epilogue == kGram && tiles * 2 <= sms / ctas) {
    const int64_t share = sms / ctas / tiles;
    bool split = false;
    tiles = 0;
    for (int k = 0; k < p.groups; ++k) {
      ProductGroup& g = p.group[k];
      const int64_t all = ceil_div(g.K, 64), want = factors[k].parts ? std::min({share, factors[k].most_splits, all / 8}) : 1;
      g.splits = want > 1 ? (int)ceil_div(all, ceil_div(all, want)) : 1;  // (every part has steps)
      split = split || g.splits > 1;
      g.tile_begin = (int)tiles;
      tiles += tiles_of(g, factors[k].batch * g.splits, 128 * ctas, g.bn);
    }
    int64_t blocks = 0;
    for (int k = 0; split && k < p.groups; ++k) {
      ProductGroup& g = p.group[k];
      CombineGroup& c = combine.group[k];
      c.parts = factors[k].parts;
      c.out = (__half*)g.out;
      c.row = g.out_row;
      c.part_batch = c.out_batch = g.out_batch;
      c.out_plane = g.out_plane;
      c.side = g.M;
      c.splits = g.splits;
      c.first_block = (int)blocks;
      const int64_t edge = ceil_div(g.M, 32);
      blocks += factors[k].batch * (edge * (edge + 1) / 2);
      g.out = factors[k].parts;
      combine.groups = k + 1;
    }
    if (split) epilogue = kPartial;
    combine.planes = p.planes;
    combine_blocks = blocks;
  }
  if (tiles > (int64_t)1 << 30) return fail_op(NETMAX_INVALID_ARG, "the problem has %lld tiles, more than 2^30", (long long)tiles);
  p.tiles = (int)tiles;
  p.a_bytes = 128 * 128;
  p.b_bytes = (uint32_t)most_b * 128;
  p.stage_bytes = (uint32_t)p.planes * (p.a_bytes + p.b_bytes);
  const size_t slots = (size_t)kEpilogueWarps * kSlotBytes;
  p.stages = (int)std::min<size_t>(kMaxStages, (kProductSmem - 1024 - slots) / p.stage_bytes);
  const size_t smem = std::max(kLeastSmem, (size_t)1024 + slots + (size_t)p.stages * p.stage_bytes);
  p.error = s.error;
  p.clear_error = s.clear;
  ProductKernel kernel = ctas == 2 ? pick_product<2>(epilogue, p.planes, long_sums) : pick_product<1>(epilogue, p.planes, long_sums);
  OP_CUDA(raise_smem_limit((const void*)kernel, smem));
  const int grid = (int)std::min<int64_t>(tiles, sms / ctas) * ctas;
  OP_DO(launch(s, kernel, dim3(grid), kProductThreads, smem, ctas, p));
  s.clear = false;
  if (combine_blocks > 0) OP_DO(launch(s, combine_kernel, dim3((unsigned)combine_blocks), kElementThreads, 0, 1, combine));
  return NETMAX_OK;
}

// ---- operands ---------------------------------------------------------------------------------
// Whether the tensor cores can read a view of 16-bit values in place: every row on a 16-byte boundary, matrices behind one another.
bool in_place(const netmax_view& v, int count, int64_t rows, int64_t cols) {
  if (((uintptr_t)v.data & 15) != 0 || (rows > 1 && v.row_stride % 8 != 0)) return false;
  return count == 1 || (v.worker_stride % 8 == 0 && v.worker_stride >= (rows - 1) * v.row_stride + cols);
}

struct Prepared {
  Operand operand;
  bool batched = true;
  int32_t* exponent = nullptr;  // of each matrix, or of each row
  bool by_rows = false;
};

Sweep make_sweep(int count, int64_t rows, int64_t cols) {
  Sweep s;
  s.rows = (int32_t)rows;
  s.cols = (int32_t)cols;
  s.count = count;
  while (s.shift < 5 && (8 << s.shift) < cols) ++s.shift;
  s.col_tiles = (int)ceil_div<int64_t>(cols, 8 << s.shift);
  // up to sixteen rows a thread; fewer where an SM would have less than two CTAs
  const int lanes = kElementThreads >> s.shift;
  int each = 16;
  while (each > 1 && (int64_t)count * s.col_tiles * ceil_div<int64_t>(rows, (int64_t)lanes * each) < 296) each /= 2;
  s.rows_per_block = lanes * each;
  s.row_blocks = (int)std::max<int64_t>(1, ceil_div<int64_t>(rows, s.rows_per_block));
  return s;
}
int blocks_of(const Sweep& s) { return s.col_tiles * s.row_blocks; }

// Room for an operand of `count` matrices of rows x cols that has to be laid out.
struct OperandRoom {
  void* planes = nullptr;
  float* maxima = nullptr;
  int32_t* exponent = nullptr;
};
OperandRoom take_operand(Carver& c, int count, int64_t rows, int64_t cols, int storage) {
  OperandRoom r;
  const size_t values = (size_t)count * (size_t)rows * (size_t)up8(cols);
  r.planes = c.take(values * 2 * (storage == NETMAX_STORAGE_F32 ? 2 : 1));
  if (storage == NETMAX_STORAGE_F32) {
    // (a shared matrix is swept as one, in up to as many blocks as all of them)
    r.maxima = (float*)c.take(std::max((size_t)count * blocks_of(make_sweep(count, rows, cols)), (size_t)blocks_of(make_sweep(1, rows, cols))) * sizeof(float));
    r.exponent = (int32_t*)c.take((size_t)count * (size_t)rows * sizeof(int32_t));
  }
  return r;
}

struct LayerRoom {
  OperandRoom x, weight, dz;
  float* sums = nullptr;
  size_t total = 0;
};
LayerRoom layer_room(void* workspace, int M, int64_t n, int64_t n_in, int64_t n_out, int storage) {
  LayerRoom r;
  Carver c(workspace);
  r.x = take_operand(c, M, n, n_in, storage);
  r.weight = take_operand(c, M, n_out, n_in, storage);
  r.dz = take_operand(c, M, n, n_out, storage);
  r.sums = (float*)c.take((size_t)M * (size_t)make_sweep(M, n, n_out).row_blocks * (size_t)n_out * sizeof(float));
  r.total = c.used;
  return r;
}

void fill_source(OperandJob& j, const netmax_view& v, const netmax_view* z, int activation, int count, int64_t rows, int64_t cols) {
  j.sweep = make_sweep(count, rows, cols);
  j.src = v.data;
  j.row = v.row_stride;
  j.batch = v.worker_stride;
  if (!z) return;
  j.z = z->data;
  j.z_row = z->row_stride;
  j.z_batch = z->worker_stride;
  j.activation = activation;
}

// Either the view itself, where the tensor cores can read it, or a job that lays it out.
Prepared prepare_operand(const netmax_view& v, const netmax_view* z, int activation, int count, int64_t rows, int64_t cols, int storage, const OperandRoom& room,
                         OperandParams& jobs, int& n_jobs, bool by_rows = false) {
  Prepared r;
  const bool shared = v.worker_stride == 0 && (!z || z->worker_stride == 0);
  const int matrices = shared ? 1 : count;
  r.batched = matrices > 1;
  Operand& o = r.operand;
  o.bf16 = storage == NETMAX_STORAGE_BF16;
  o.inner = cols;
  o.outer = rows;
  o.count = matrices;
  if (o.bf16 && !z && in_place(v, matrices, rows, cols)) {
    o.data = v.data;
    o.row = rows > 1 ? v.row_stride : up8(cols);
    o.batch = v.worker_stride;
    return r;
  }
  OperandJob& j = jobs.job[n_jobs++];
  fill_source(j, v, z, activation, matrices, rows, cols);
  j.dst = room.planes;
  j.dst_row = up8(cols);
  j.dst_batch = rows * j.dst_row;
  j.dst_plane = j.dst_batch * matrices;
  j.maxima = room.maxima;
  j.exponent = room.exponent;
  o.data = room.planes;
  o.row = j.dst_row;
  o.batch = j.dst_batch;
  o.plane = j.dst_plane;
  o.planes = o.bf16 ? 1 : 2;
  r.exponent = room.exponent;
  r.by_rows = by_rows && !o.bf16;
  return r;
}

// fp32 operands whose rows have exponents of their own.
int run_row_jobs(Stream& s, OperandParams& jobs, int n_jobs) {
  int count = 1, rows = 1;
  for (int k = 0; k < n_jobs; ++k) {
    count = std::max(count, jobs.job[k].sweep.count);
    rows = std::max(rows, jobs.job[k].sweep.rows);
  }
  jobs.error = s.error;
  jobs.clear_error = s.clear;
  s.clear = false;
  const int64_t cols = jobs.job[0].sweep.cols;
  const int lanes = cols <= 1024 ? 32 : cols <= 2048 ? 64 : cols <= 4096 ? 128 : 256;
  const dim3 grid((unsigned)ceil_div(rows, kElementThreads / lanes), (unsigned)std::min(count, 32768), (unsigned)n_jobs);
  return launch(s, lanes == 32 ? operand_rows_kernel<32> : lanes == 64 ? operand_rows_kernel<64> : lanes == 128 ? operand_rows_kernel<128> : operand_rows_kernel<256>,
                grid, kElementThreads, 0, 1, jobs);
}

int run_jobs(Stream& s, OperandParams& jobs, int n_jobs, int storage) {
  if (n_jobs == 0) return NETMAX_OK;
  int count = 1, blocks = 1;
  bool laid_out = storage == NETMAX_STORAGE_BF16;
  for (int k = 0; k < n_jobs; ++k) {
    count = std::max(count, jobs.job[k].sweep.count);
    blocks = std::max(blocks, blocks_of(jobs.job[k].sweep));
    laid_out = laid_out || jobs.job[k].dst;
  }
  jobs.error = s.error;
  const dim3 grid((unsigned)blocks, (unsigned)std::min(count, 32768), (unsigned)n_jobs);
  if (storage == NETMAX_STORAGE_F32) {
    jobs.clear_error = s.clear;
    s.clear = false;
    OP_DO(launch(s, operand_maxima_kernel, grid, kElementThreads, 0, 1, jobs));
  }
  if (!laid_out) return NETMAX_OK;
  jobs.clear_error = s.clear;
  s.clear = false;
  return launch(s, storage == NETMAX_STORAGE_F32 ? operand_kernel<float> : operand_kernel<__nv_bfloat16>, grid, kElementThreads, 0, 1, jobs);
}

int few_rows(Stream& s, const netmax_layer& l) {
  FewRowsParams p;
  p.x = l.x.data;
  p.x_row = l.x.row_stride;
  p.x_batch = l.x.worker_stride;
  p.weight = l.weight.data;
  p.weight_row = l.weight.row_stride;
  p.weight_batch = l.weight.worker_stride;
  p.bias = l.bias.data;
  p.bias_batch = l.bias.worker_stride;
  p.residual = l.residual.data;
  p.residual_row = l.residual.row_stride;
  p.residual_batch = l.residual.worker_stride;
  p.y = l.y.data;
  p.y_row = l.y.row_stride;
  p.y_batch = l.y.worker_stride;
  p.z = l.z.data;
  p.z_row = l.z.row_stride;
  p.z_batch = l.z.worker_stride;
  p.n = (int32_t)l.n;
  p.n_in = (int32_t)l.n_in;
  p.n_out = (int32_t)l.n_out;
  p.activation = l.activation;
  p.error = s.error;
  const bool f32 = l.storage == NETMAX_STORAGE_F32;
  const int64_t unit = f32 ? 4 : 8;
  auto fits = [&](const netmax_view& v, int64_t rows) {
    return ((uintptr_t)v.data & 15) == 0 && (rows == 1 || v.row_stride % unit == 0) && (l.M == 1 || v.worker_stride % unit == 0);
  };
  p.pieces = fits(l.x, l.n) && fits(l.weight, l.n_out);
  const int rows = l.n <= 1 ? 1 : l.n <= 2 ? 2 : l.n <= 4 ? 4 : 8;
  // several outputs a warp share the loads of x; one where that would leave SMs without work
  const int most = rows >= 4 ? 4 : 2, outputs = l.M * ceil_div<int64_t>(l.n_out, 8 * most) >= sm_count() ? most : 1;
  const dim3 grid((unsigned)ceil_div<int64_t>(l.n_out, 8 * outputs), (unsigned)l.M, (unsigned)ceil_div<int64_t>(l.n, rows));
  auto run = [&](void (*several)(const FewRowsParams), void (*one)(const FewRowsParams)) {
    return launch(s, outputs > 1 ? several : one, grid, kElementThreads, 0, 1, p);
  };
  if (f32) {
    switch (rows) {
      case 1: return run(few_rows_kernel<float, 1, 2>, few_rows_kernel<float, 1, 1>);
      case 2: return run(few_rows_kernel<float, 2, 2>, few_rows_kernel<float, 2, 1>);
      case 4: return run(few_rows_kernel<float, 4, 4>, few_rows_kernel<float, 4, 1>);
      default: return run(few_rows_kernel<float, 8, 4>, few_rows_kernel<float, 8, 1>);
    }
  }
  using B = __nv_bfloat16;
  switch (rows) {
    case 1: return run(few_rows_kernel<B, 1, 2>, few_rows_kernel<B, 1, 1>);
    case 2: return run(few_rows_kernel<B, 2, 2>, few_rows_kernel<B, 2, 1>);
    default: return run(few_rows_kernel<B, 4, 4>, few_rows_kernel<B, 4, 1>);
  }
}

template <typename T, int kRows>
int few_rows_backward(Stream& s, const netmax_layer& l, float* parts) {
  constexpr int kN = 16 / sizeof(T);
  FewRowsBackParams p;
  const bool active = l.activation != NETMAX_ACTIVATION_NONE;
  p.dy = l.dy.data;
  p.dy_row = l.dy.row_stride;
  p.dy_batch = l.dy.worker_stride;
  if (active) {
    p.z = l.z.data;
    p.z_row = l.z.row_stride;
    p.z_batch = l.z.worker_stride;
  }
  p.x = l.x.data;
  p.x_row = l.x.row_stride;
  p.x_batch = l.x.worker_stride;
  p.weight = l.weight.data;
  p.weight_row = l.weight.row_stride;
  p.weight_batch = l.weight.worker_stride;
  p.dx = l.dx.data;
  p.dx_row = l.dx.row_stride;
  p.dx_batch = l.dx.worker_stride;
  p.dweight = l.dweight.data;
  p.dweight_row = l.dweight.row_stride;
  p.dweight_batch = l.dweight.worker_stride;
  p.dbias = l.dbias.data;
  p.dbias_batch = l.dbias.worker_stride;
  p.M = l.M;
  p.n = (int32_t)l.n;
  p.n_in = (int32_t)l.n_in;
  p.n_out = (int32_t)l.n_out;
  p.activation = l.activation;
  p.error = s.error;
  while (p.shift < 8 && ((int64_t)kN << p.shift) < l.n_in) ++p.shift;
  const int64_t tiles = ceil_div<int64_t>(l.n_in, (int64_t)kN << p.shift);
  p.col_tiles = (int32_t)tiles;
  if (l.dweight.data || l.dbias.data) {
    const int64_t columns = l.dweight.data ? tiles : 1;
    p.col_tiles = (int32_t)columns;
    const int64_t blocks = columns * ceil_div<int64_t>(l.n_out, kFewOutputs);
    if (blocks >= (int64_t)1 << 31) return fail_op(NETMAX_INVALID_ARG, "the layer's gradient has too many parts");
    p.clear_error = s.clear;
    s.clear = false;
    OP_DO(launch(s, few_rows_dweight_kernel<T, kRows>, dim3((unsigned)blocks, (unsigned)l.M), kElementThreads, 0, 1, p));
    p.col_tiles = (int32_t)tiles;
  }
  if (l.dx.data) {
    // outputs are shared out until every SM has two CTAs; 64 at least, so that the parts fit in the room for the laid out weights
    int64_t per = ceil_div<int64_t>(l.n_out, kFewOutputs) * kFewOutputs;
    while (per > kFewOutputs && tiles * l.M * ceil_div(l.n_out, per) < 2 * sm_count()) per = ceil_div<int64_t>(per / 2, kFewOutputs) * kFewOutputs;
    p.outputs_per_block = (int32_t)per;
    p.chunks = (int32_t)ceil_div(l.n_out, per);
    p.parts = parts;
    if (tiles * p.chunks >= (int64_t)1 << 31) return fail_op(NETMAX_INVALID_ARG, "the layer's gradient has too many parts");
    p.clear_error = s.clear;
    s.clear = false;
    OP_DO(launch(s, few_rows_dx_kernel<T, kRows>, dim3((unsigned)(tiles * p.chunks), (unsigned)l.M), kElementThreads, 0, 1, p));
    if (p.chunks > 1) {
      const int64_t total = (int64_t)l.M * l.n * l.n_in;
      OP_DO(launch(s, few_rows_total_kernel<T>, dim3((unsigned)std::min<int64_t>(ceil_div<int64_t>(total, kElementThreads), 4096)), kElementThreads, 0, 1, p));
    }
  }
  if (s.clear) OP_CUDA(cudaMemsetAsync(l.workspace, 0, 4, s.stream));
  return NETMAX_OK;
}

// One product of a launch: D[m][n] over k.
void fill_product(ProductGroup& g, const Prepared& a, bool a_mn, const Prepared& b, bool b_mn, int64_t M, int64_t N, int64_t K) {
  g.M = (int32_t)M;
  g.N = (int32_t)N;
  g.K = (int32_t)K;
  g.a_mn = a_mn;
  g.b_mn = b_mn;
  g.a_batched = a.batched;
  g.b_batched = b.batched;
  g.exp_a = a.exponent;
  g.exp_b = b.exponent;
  g.exp_a_rows = a.by_rows ? (int32_t)M : 0;
  g.exp_b_rows = b.by_rows ? (int32_t)N : 0;
}

// ---- checks ---------------------------------------------------------------------------------------
int check_device(int device) {
  int n = 0;
  if (cudaGetDeviceCount(&n) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return fail_op(NETMAX_CUDA_ERROR, "no CUDA device is available");
  }
  if (device < 0 || device >= n) return fail_op(NETMAX_INVALID_ARG, "device = %d outside [0, %d)", device, n);
  return NETMAX_OK;
}
int check_storage(int storage) {
  if (storage != NETMAX_STORAGE_F32 && storage != NETMAX_STORAGE_BF16)
    return fail_op(NETMAX_INVALID_ARG, "storage = %d is neither NETMAX_STORAGE_F32 nor NETMAX_STORAGE_BF16", storage);
  return NETMAX_OK;
}
// The elements between a view's first and last one must be addressable; outputs must not overlap themselves.
int check_view(const char* name, const netmax_view& v, int64_t count, int64_t rows, int64_t cols, bool output, size_t element) {
  if (!v.data) return fail_op(NETMAX_INVALID_ARG, "%s is NULL", name);
  if ((uintptr_t)v.data % element) return fail_op(NETMAX_INVALID_ARG, "%s is not aligned to its elements", name);
  const int64_t limit = (int64_t)1 << 38;
  if (v.row_stride < 0 || v.worker_stride < 0 || v.row_stride > limit || v.worker_stride > limit)
    return fail_op(NETMAX_INVALID_ARG, "%s: strides %lld and %lld outside [0, 2^38]", name, (long long)v.row_stride, (long long)v.worker_stride);
  if (rows > 1 && v.row_stride < cols)
    return fail_op(NETMAX_INVALID_ARG, "%s: row stride %lld is less than its %lld columns", name, (long long)v.row_stride, (long long)cols);
  if (output && count > 1 && rows > 0) {
    const int64_t row = rows > 1 ? v.row_stride : cols;
    const bool apart = v.worker_stride >= (rows - 1) * row + cols;
    const bool woven = v.worker_stride >= cols && row >= (count - 1) * v.worker_stride + cols;
    if (!apart && !woven) return fail_op(NETMAX_INVALID_ARG, "%s: worker stride %lld lets matrices overlap", name, (long long)v.worker_stride);
  }
  return NETMAX_OK;
}
int check_workspace(const void* workspace, size_t bytes, size_t needed) {
  if (!workspace) return fail_op(NETMAX_INVALID_ARG, "workspace is NULL");
  if ((uintptr_t)workspace & 255) return fail_op(NETMAX_INVALID_ARG, "workspace is not 256-byte aligned");
  if (bytes < needed) return fail_op(NETMAX_OOM, "workspace holds %zu bytes, %zu needed", bytes, needed);
  return NETMAX_OK;
}
int check_layer_sizes(int32_t M, int64_t n, int64_t n_in, int64_t n_out, int32_t storage) {
  OP_DO(check_storage(storage));
  const int64_t limit = (int64_t)1 << 31, most = (int64_t)1 << 30;  // (indices of a row or column, with a tile's overhang, fit 32 bits)
  if (M < 1 || M > 16384) return fail_op(NETMAX_INVALID_ARG, "M = %d outside [1, 16384]", M);
  if (n < 0 || n_in < 1 || n_out < 1 || n > most || n_in > most || n_out > most || n * n_in >= limit || n * n_out >= limit || n_in * n_out >= limit)
    return fail_op(NETMAX_INVALID_ARG, "n = %lld, n_in = %lld, n_out = %lld: sizes must be positive (n may be 0), at most 2^30 each, and their products below 2^31", (long long)n,
                   (long long)n_in, (long long)n_out);
  return NETMAX_OK;
}
size_t element_size(int storage) { return storage == NETMAX_STORAGE_F32 ? 4 : 2; }

// First and last byte of what a view names; of its matrices, how long each is and how far apart they stand (0: there is one); of its rows,
// how long each is and how far apart they stand (0: there is one).
struct Span {
  uintptr_t first, last;
  size_t extent, period, width, row;
};
Span span_of(const netmax_view& v, int64_t count, int64_t rows, int64_t cols, size_t element) {
  const int64_t extent = (rows - 1) * v.row_stride + cols, end = (count - 1) * v.worker_stride + extent;
  return {(uintptr_t)v.data, (uintptr_t)v.data + (size_t)end * element - 1, (size_t)extent * element, count > 1 ? (size_t)v.worker_stride * element : 0,
          (size_t)cols * element, rows > 1 ? (size_t)v.row_stride * element : 0};
}
bool meet(const Span& a, const Span& b) {
  if (a.first > b.last || b.first > a.last) return false;
  // Every row of either starts a multiple of the strides' common divisor behind the first one: columns of one wide buffer are apart if they
  // are apart in that.
  const size_t common = std::gcd(std::gcd(a.row, b.row), std::gcd(a.period, b.period));
  if (common > 0) {
    const size_t behind = b.first >= a.first ? (size_t)(b.first - a.first) % common : (common - (size_t)(a.first - b.first) % common) % common;
    if (behind >= a.width && behind + b.width <= common) return false;
  }
  if (a.period == 0 || a.period != b.period) return true;  // (woven in some other way: taken to overlap)
  // both once in every replica, as a layer's gradients are: apart if they are apart in one period
  const size_t between = (size_t)((b.first - a.first) % a.period + a.period) % a.period;
  return b.first >= a.first ? between < a.extent || between + b.extent > a.period : meet(b, a);
}
int check_apart(const char* name, const Span& out, const char* other, const Span& in) {
  if (meet(out, in)) return fail_op(NETMAX_INVALID_ARG, "%s overlaps %s", name, other);
  return NETMAX_OK;
}

}  // namespace

extern "C" {

int netmax_layer_workspace_size(int32_t M, int64_t n, int64_t n_in, int64_t n_out, int32_t storage, size_t* bytes) try {
  OP_DO(check_layer_sizes(M, n, n_in, n_out, storage));
  if (!bytes) return fail_op(NETMAX_INVALID_ARG, "bytes is NULL");
  *bytes = layer_room(nullptr, M, n, n_in, n_out, storage).total;
  return NETMAX_OK;
} NM_CATCH(fail_caught)

int netmax_layer_forward(const netmax_layer* l) try {
  if (!l) return fail_op(NETMAX_INVALID_ARG, "layer is NULL");
  OP_DO(check_layer_sizes(l->M, l->n, l->n_in, l->n_out, l->storage));
  if (l->activation < 0 || l->activation > 3) return fail_op(NETMAX_INVALID_ARG, "activation = %d is none of NETMAX_ACTIVATION_*", l->activation);
  const size_t size = element_size(l->storage);
  const int64_t n = l->n, n_in = l->n_in, n_out = l->n_out;
  if (n > 0) {
    OP_DO(check_view("x", l->x, l->M, n, n_in, false, size));
    OP_DO(check_view("y", l->y, l->M, n, n_out, true, size));
    OP_DO(check_view("weight", l->weight, l->M, n_out, n_in, false, size));
    if (l->bias.data) OP_DO(check_view("bias", l->bias, l->M, 1, n_out, false, size));
    if (l->residual.data) OP_DO(check_view("residual", l->residual, l->M, n, n_out, false, size));
    if (l->z.data) OP_DO(check_view("z", l->z, l->M, n, n_out, true, size));
    const Span y = span_of(l->y, l->M, n, n_out, size), x = span_of(l->x, l->M, n, n_in, size), w = span_of(l->weight, l->M, n_out, n_in, size);
    OP_DO(check_apart("y", y, "x", x));
    OP_DO(check_apart("y", y, "weight", w));
    if (l->bias.data) OP_DO(check_apart("y", y, "bias", span_of(l->bias, l->M, 1, n_out, size)));
    const bool in_place = l->residual.data == l->y.data && (n == 1 || l->residual.row_stride == l->y.row_stride) &&
                          (l->M == 1 || l->residual.worker_stride == l->y.worker_stride);
    if (l->residual.data && !in_place) OP_DO(check_apart("y", y, "residual", span_of(l->residual, l->M, n, n_out, size)));
    if (l->z.data) {
      const Span z = span_of(l->z, l->M, n, n_out, size);
      OP_DO(check_apart("z", z, "x", x));
      OP_DO(check_apart("z", z, "weight", w));
      OP_DO(check_apart("z", z, "y", y));
      if (l->bias.data) OP_DO(check_apart("z", z, "bias", span_of(l->bias, l->M, 1, n_out, size)));
      if (l->residual.data) OP_DO(check_apart("z", z, "residual", span_of(l->residual, l->M, n, n_out, size)));
    }
  }
  const LayerRoom room = layer_room(l->workspace, l->M, n, n_in, n_out, l->storage);
  OP_DO(check_workspace(l->workspace, l->workspace_bytes, room.total));
  OP_DO(check_device(l->device));
  OnDevice on(l->device);
  if (!on.ok) return fail_op(NETMAX_CUDA_ERROR, "cudaSetDevice failed");
  Stream s{(cudaStream_t)l->stream, (unsigned int*)l->workspace};
  if (n == 0) {
    OP_CUDA(cudaMemsetAsync(l->workspace, 0, 4, s.stream));
    return NETMAX_OK;
  }
  const bool f32 = l->storage == NETMAX_STORAGE_F32;
  if (n <= (f32 ? kFewRowsF32 : kFewRowsBf16)) return few_rows(s, *l);
  OperandParams jobs;
  int n_jobs = 0;
  // (both factors' rows end in the output, so each row has a scale of its own and the values are read once from memory)
  const Prepared w = prepare_operand(l->weight, nullptr, 0, l->M, n_out, n_in, l->storage, room.weight, jobs, n_jobs, true);
  const Prepared x = prepare_operand(l->x, nullptr, 0, l->M, n, n_in, l->storage, room.x, jobs, n_jobs, true);
  if (f32) OP_DO(run_row_jobs(s, jobs, n_jobs));
  else OP_DO(run_jobs(s, jobs, n_jobs, l->storage));
  ProductParams p;
  p.groups = 1;
  p.planes = l->storage == NETMAX_STORAGE_F32 ? 2 : 1;
  ProductGroup& g = p.group[0];
  fill_product(g, x, false, w, false, n, n_out, n_in);
  g.out = l->y.data;
  g.out_row = l->y.row_stride;
  g.out_batch = l->y.worker_stride;
  g.z = l->z.data;
  g.z_row = l->z.row_stride;
  g.z_batch = l->z.worker_stride;
  g.bias = l->bias.data;
  g.bias_batch = l->bias.worker_stride;
  g.residual = l->residual.data;
  g.residual_row = l->residual.row_stride;
  g.residual_batch = l->residual.worker_stride;
  g.activation = l->activation;
  const Factors factors{&x.operand, &w.operand, l->M};
  return run_products(s, p, &factors, w.operand.bf16 ? kLayerBf16 : kLayerF32);
} NM_CATCH(fail_caught)

int netmax_layer_backward(const netmax_layer* l) try {
  if (!l) return fail_op(NETMAX_INVALID_ARG, "layer is NULL");
  OP_DO(check_layer_sizes(l->M, l->n, l->n_in, l->n_out, l->storage));
  if (l->activation < 0 || l->activation > 3) return fail_op(NETMAX_INVALID_ARG, "activation = %d is none of NETMAX_ACTIVATION_*", l->activation);
  const size_t size = element_size(l->storage);
  const int64_t n = l->n, n_in = l->n_in, n_out = l->n_out;
  const bool active = l->activation != NETMAX_ACTIVATION_NONE;
  struct Named {
    const char* name;
    const netmax_view* v;
    int64_t rows, cols;
  };
  std::vector<Named> in, out;
  if (n > 0) {
    in.push_back({"dy", &l->dy, n, n_out});
    if (active) in.push_back({"z", &l->z, n, n_out});
    if (l->dweight.data) in.push_back({"x", &l->x, n, n_in});
    if (l->dx.data) in.push_back({"weight", &l->weight, n_out, n_in});
    if (l->dx.data) out.push_back({"dx", &l->dx, n, n_in});
  }
  if (l->dweight.data) out.push_back({"dweight", &l->dweight, n_out, n_in});
  if (l->dbias.data) out.push_back({"dbias", &l->dbias, 1, n_out});
  for (const Named& v : in) OP_DO(check_view(v.name, *v.v, l->M, v.rows, v.cols, false, size));
  for (const Named& v : out) OP_DO(check_view(v.name, *v.v, l->M, v.rows, v.cols, true, size));
  for (size_t k = 0; k < out.size(); ++k) {
    const Span o = span_of(*out[k].v, l->M, out[k].rows, out[k].cols, size);
    for (const Named& v : in) OP_DO(check_apart(out[k].name, o, v.name, span_of(*v.v, l->M, v.rows, v.cols, size)));
    for (size_t q = 0; q < k; ++q) OP_DO(check_apart(out[k].name, o, out[q].name, span_of(*out[q].v, l->M, out[q].rows, out[q].cols, size)));
  }
  const LayerRoom room = layer_room(l->workspace, l->M, n, n_in, n_out, l->storage);
  OP_DO(check_workspace(l->workspace, l->workspace_bytes, room.total));
  OP_DO(check_device(l->device));
  OnDevice on(l->device);
  if (!on.ok) return fail_op(NETMAX_CUDA_ERROR, "cudaSetDevice failed");
  Stream s{(cudaStream_t)l->stream, (unsigned int*)l->workspace};
  if (n == 0) {  // no rows: the gradients of the parameters are zero
    OP_CUDA(cudaMemsetAsync(l->workspace, 0, 4, s.stream));
    for (int i = 0; i < l->M; ++i) {
      if (l->dweight.data)
        OP_CUDA(cudaMemset2DAsync((char*)l->dweight.data + (size_t)i * l->dweight.worker_stride * size, (size_t)std::max(l->dweight.row_stride, n_in) * size, 0,
                                  (size_t)n_in * size, (size_t)n_out, s.stream));
      if (l->dbias.data) OP_CUDA(cudaMemsetAsync((char*)l->dbias.data + (size_t)i * l->dbias.worker_stride * size, 0, (size_t)n_out * size, s.stream));
    }
    return NETMAX_OK;
  }
  const bool f32 = l->storage == NETMAX_STORAGE_F32;
  if (f32 && n <= kFewRowsF32)
    return n <= 4 ? few_rows_backward<float, 4>(s, *l, (float*)room.weight.planes) : n <= 8 ? few_rows_backward<float, 8>(s, *l, (float*)room.weight.planes)
                                                                                   : few_rows_backward<float, 16>(s, *l, (float*)room.weight.planes);
  if (!f32 && n <= kFewRowsBf16) return few_rows_backward<__nv_bfloat16, 4>(s, *l, (float*)room.weight.planes);
  OperandParams jobs;
  int n_jobs = 0;
  Prepared dz, w, x;
  if (l->dx.data || l->dweight.data)
    dz = prepare_operand(l->dy, active ? &l->z : nullptr, l->activation, l->M, n, n_out, l->storage, room.dz, jobs, n_jobs);
  const bool laid_out = n_jobs > 0 && jobs.job[0].sweep.count == l->M;  // dz, for every worker
  if (l->dx.data) w = prepare_operand(l->weight, nullptr, 0, l->M, n_out, n_in, l->storage, room.weight, jobs, n_jobs);
  if (l->dweight.data) x = prepare_operand(l->x, nullptr, 0, l->M, n, n_in, l->storage, room.x, jobs, n_jobs);
  if (l->dbias.data) {  // along with dz where that is laid out
    const int at = laid_out ? 0 : n_jobs++;
    if (!laid_out) fill_source(jobs.job[at], l->dy, active ? &l->z : nullptr, l->activation, l->M, n, n_out);
    jobs.job[at].sums = room.sums;
  }
  OP_DO(run_jobs(s, jobs, n_jobs, l->storage));
  if (l->dbias.data) {
    const int n_parts = make_sweep(l->M, n, n_out).row_blocks;
    const unsigned totals = (unsigned)std::min<int64_t>(ceil_div<int64_t>((int64_t)l->M * n_out, kElementThreads), 4096);
    if (f32)
      OP_DO(launch(s, column_totals_kernel<float>, dim3(totals), kElementThreads, 0, 1, (const float*)room.sums, n_parts, (int)n_out, (int)l->M,
                   (float*)l->dbias.data, l->dbias.worker_stride));
    else
      OP_DO(launch(s, column_totals_kernel<__nv_bfloat16>, dim3(totals), kElementThreads, 0, 1, (const float*)room.sums, n_parts, (int)n_out, (int)l->M,
                   (__nv_bfloat16*)l->dbias.data, l->dbias.worker_stride));
  }
  if (!l->dx.data && !l->dweight.data) {
    if (s.clear) OP_CUDA(cudaMemsetAsync(l->workspace, 0, 4, s.stream));
    return NETMAX_OK;
  }
  ProductParams p;
  p.planes = f32 ? 2 : 1;
  Factors factors[2];
  if (l->dx.data) {
    ProductGroup& g = p.group[p.groups];
    factors[p.groups++] = {&dz.operand, &w.operand, l->M};
    fill_product(g, dz, false, w, true, n, n_in, n_out);
    g.out = l->dx.data;
    g.out_row = l->dx.row_stride;
    g.out_batch = l->dx.worker_stride;
  }
  if (l->dweight.data) {
    ProductGroup& g = p.group[p.groups];
    factors[p.groups++] = {&dz.operand, &x.operand, l->M};
    fill_product(g, dz, true, x, true, n_out, n_in, n);
    g.out = l->dweight.data;
    g.out_row = l->dweight.row_stride;
    g.out_batch = l->dweight.worker_stride;
  }
  return run_products(s, p, factors, f32 ? kLayerF32 : kLayerBf16);
} NM_CATCH(fail_caught)

}  // extern "C"

// ---- Newton-Schulz --------------------------------------------------------------------------------
namespace {

// Equal matrices that are orthogonalised together: iterates in two buffers of two planes each, S = X X^T (or X^T X of tall ones) and
// the polynomial b S + c S^2.
struct SchulzGroup {
  int64_t rows = 0, cols = 0;
  int batch = 0;
  bool tall = false;
  int64_t side = 0;
  __half *x[2] = {nullptr, nullptr}, *gram = nullptr, *poly = nullptr;
  int64_t x_row = 0, x_batch = 0, x_plane = 0, s_row = 0, s_batch = 0, s_plane = 0;
  Operand op_x[2], op_gram, op_poly;
  void set(int64_t r, int64_t c, int n) {
    rows = r;
    cols = c;
    batch = n;
    tall = rows > cols;
    side = std::min(rows, cols);
    x_row = up8(cols);
    x_batch = rows * x_row;
    x_plane = x_batch * batch;
    s_row = up8(side);
    s_batch = side * s_row;
    s_plane = s_batch * batch;
  }
  void take(Carver& carver, int planes) {
    for (auto& v : x) v = (__half*)carver.take((size_t)x_plane * 2 * sizeof(__half));
    gram = (__half*)carver.take((size_t)s_plane * (size_t)planes * sizeof(__half));
    poly = (__half*)carver.take((size_t)s_plane * (size_t)planes * sizeof(__half));
  }
  void describe(int planes) {  // (behind take())
    for (int k = 0; k < 2; ++k) {
      Operand& o = op_x[k];
      o.data = x[k];
      o.inner = cols;
      o.outer = rows;
      o.row = x_row;
      o.batch = x_batch;
      o.plane = x_plane;
      o.count = batch;
      o.planes = 2;
    }
    for (Operand* o : {&op_gram, &op_poly}) {
      o->data = o == &op_gram ? gram : poly;
      o->inner = o->outer = side;
      o->row = s_row;
      o->batch = s_batch;
      o->plane = s_plane;
      o->count = batch;
      o->planes = planes;
    }
  }
};

int planes_of(int storage) { return storage == NETMAX_STORAGE_F32 ? 2 : 1; }

// The `steps` steps of all groups; `last` finishes the group of the last product (where its output goes).
template <typename Last>
int run_schulz(Stream& s, std::vector<SchulzGroup>& groups, int steps, int planes, int last_epilogue, ProductParams& p, const Last& last) {
  p.planes = planes;
  p.ca = kA;
  p.cb = kB;
  p.cc = kC;
  for (int step = 0; step < steps; ++step) {
    const int now = step & 1;
    for (int phase = 0; phase < 3; ++phase) {
      const bool final = phase == 2 && step + 1 == steps;
      for (size_t first = 0; first < groups.size(); first += kMaxGroups) {
        const size_t n = std::min<size_t>(kMaxGroups, groups.size() - first);
        Factors factors[kMaxGroups];
        p.groups = (int)n;
        for (size_t k = 0; k < n; ++k) {
          const SchulzGroup& q = groups[first + k];
          ProductGroup g;
          factors[k].batch = q.batch;
          if (phase < 2) {
            g.symmetric = 1;
            g.M = g.N = (int32_t)q.side;
            g.K = (int32_t)(phase == 0 && !q.tall ? q.cols : phase == 0 ? q.rows : q.side);
            g.a_mn = g.b_mn = phase == 0 && q.tall;
            factors[k].a = factors[k].b = phase == 0 ? &q.op_x[now] : &q.op_gram;
            if (phase == 0) {  // (the other iterate is written behind the polynomial only)
              factors[k].parts = (float*)q.x[now ^ 1];
              factors[k].most_splits = q.x_batch / q.s_batch;  // fp32 parts in the room of two planes
            }
            g.out = phase == 0 ? q.gram : q.poly;
            g.out_row = q.s_row;
            g.out_batch = q.s_batch;
            g.out_plane = q.s_plane;
            if (phase == 1) {
              g.residual = q.gram;
              g.residual_row = q.s_row;
              g.residual_batch = q.s_batch;
              g.residual_plane = q.s_plane;
            }
          } else {
            g.M = (int32_t)q.rows;
            g.N = (int32_t)q.cols;
            g.K = (int32_t)q.side;
            factors[k].a = q.tall ? &q.op_x[now] : &q.op_poly;
            factors[k].b = q.tall ? &q.op_poly : &q.op_x[now];
            g.b_mn = !q.tall;
            g.residual = q.x[now];
            g.residual_row = q.x_row;
            g.residual_batch = q.x_batch;
            g.residual_plane = q.x_plane;
            g.out = q.x[now ^ 1];
            g.out_row = q.x_row;
            g.out_batch = q.x_batch;
            g.out_plane = q.x_plane;
            if (final) last(first + k, g);
          }
          p.group[k] = g;
        }
        OP_DO(run_products(s, p, factors, phase == 0 ? kGram : phase == 1 ? kPolynomial : final ? last_epilogue : kUpdate));
      }
    }
  }
  return NETMAX_OK;
}

int check_orthogonal_sizes(int32_t count, int64_t rows, int64_t cols, int32_t storage) {
  OP_DO(check_storage(storage));
  const int64_t limit = (int64_t)1 << 31, most = (int64_t)1 << 30;
  if (count < 1 || count > 1 << 20) return fail_op(NETMAX_INVALID_ARG, "count = %d outside [1, 2^20]", count);
  if (rows < 1 || cols < 1 || rows > most || cols > most || rows * cols >= limit)
    return fail_op(NETMAX_INVALID_ARG, "rows = %lld, cols = %lld: both must be positive, at most 2^30, and their product below 2^31", (long long)rows, (long long)cols);
  return NETMAX_OK;
}
struct OrthogonalRoom {
  SchulzGroup group;
  double* parts;
  Sweep sweep;
  size_t total;
};
OrthogonalRoom orthogonal_room(void* workspace, int count, int64_t rows, int64_t cols, int storage) {
  OrthogonalRoom r;
  Carver c(workspace);
  r.group.set(rows, cols, count);
  r.group.take(c, planes_of(storage));
  r.sweep = make_sweep(count, rows, cols);
  r.parts = (double*)c.take((size_t)count * blocks_of(r.sweep) * sizeof(double));
  r.total = c.used;
  return r;
}
// Matrices that a CTA or a cluster each orthogonalises.
int run_small(Stream& s, SmallParams& p, unsigned clusters, size_t smem, uint32_t tmem_columns, void (*kernel)(const SmallParams)) {
  p.tmem_columns = tmem_columns;
  p.ca = kA;
  p.cb = kB;
  p.cc = kC;
  p.error = s.error;
  p.clear_error = s.clear;
  s.clear = false;
  // The CTAs of a cluster wait for one another, and a CTA for its TMEM: with one CTA per SM no two clusters hold what the other one needs.
  if (p.ctas > 1) smem = std::max(smem, kLeastSmem);
  OP_CUDA(raise_smem_limit((const void*)kernel, smem));
  if (p.ctas > 8) OP_CUDA(cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  return launch(s, kernel, dim3(clusters * (unsigned)p.ctas), kSmallThreads, smem, p.ctas, p);
}
int check_steps(int steps) {
  if (steps < 1 || steps > 20) return fail_op(NETMAX_INVALID_ARG, "steps = %d outside [1, 20]", steps);
  return NETMAX_OK;
}

}  // namespace

extern "C" {

int netmax_orthogonalise_workspace_size(int32_t count, int64_t rows, int64_t cols, int32_t storage, size_t* bytes) try {
  OP_DO(check_orthogonal_sizes(count, rows, cols, storage));
  if (!bytes) return fail_op(NETMAX_INVALID_ARG, "bytes is NULL");
  *bytes = orthogonal_room(nullptr, count, rows, cols, storage).total;
  return NETMAX_OK;
} NM_CATCH(fail_caught)

int netmax_orthogonalise(const netmax_orthogonal* o) try {
  if (!o) return fail_op(NETMAX_INVALID_ARG, "o is NULL");
  OP_DO(check_orthogonal_sizes(o->count, o->rows, o->cols, o->storage));
  OP_DO(check_steps(o->steps));
  const size_t size = element_size(o->storage);
  OP_DO(check_view("u", o->u, o->count, o->rows, o->cols, false, size));
  OP_DO(check_view("out", o->out, o->count, o->rows, o->cols, true, size));
  OP_DO(check_apart("out", span_of(o->out, o->count, o->rows, o->cols, size), "u", span_of(o->u, o->count, o->rows, o->cols, size)));
  OrthogonalRoom room = orthogonal_room(o->workspace, o->count, o->rows, o->cols, o->storage);
  OP_DO(check_workspace(o->workspace, o->workspace_bytes, room.total));
  OP_DO(check_device(o->device));
  OnDevice on(o->device);
  if (!on.ok) return fail_op(NETMAX_CUDA_ERROR, "cudaSetDevice failed");
  Stream s{(cudaStream_t)o->stream, (unsigned int*)o->workspace};
  const bool f32 = o->storage == NETMAX_STORAGE_F32;
  if (is_small(o->rows, o->cols)) {
    SmallParams sp;
    sp.u = o->u.data;
    sp.row = o->u.row_stride;
    sp.batch = o->u.worker_stride;
    sp.out = o->out.data;
    sp.out_row = o->out.row_stride;
    sp.out_batch = o->out.worker_stride;
    sp.rows = (int32_t)o->rows;
    sp.cols = (int32_t)o->cols;
    sp.steps = o->steps;
    const uint32_t rows = (uint32_t)o->rows, cols = (uint32_t)o->cols;
    sp.ctas = (int32_t)small_ctas(o->count, rows, cols, sm_count());
    return run_small(s, sp, (unsigned)o->count, small_smem(rows, cols, sp.ctas), small_tmem(rows, cols, sp.ctas),
                     f32 ? small_schulz_kernel<float, false> : small_schulz_kernel<__nv_bfloat16, false>);
  }
  SchulzGroup& q = room.group;
  NormParams np;
  np.u = o->u.data;
  np.row = o->u.row_stride;
  np.batch = o->u.worker_stride;
  np.sweep = room.sweep;
  np.parts = room.parts;
  np.planes = q.x[0];
  np.dst_row = q.x_row;
  np.dst_batch = q.x_batch;
  np.dst_plane = q.x_plane;
  np.error = s.error;
  np.clear_error = 1;
  s.clear = false;
  const dim3 grid((unsigned)blocks_of(room.sweep), (unsigned)std::min(o->count, 32768));
  OP_DO(launch(s, f32 ? norm_parts_kernel<float> : norm_parts_kernel<__nv_bfloat16>, grid, kElementThreads, 0, 1, np));
  OP_DO(launch(s, f32 ? first_iterate_kernel<float> : first_iterate_kernel<__nv_bfloat16>, grid, kElementThreads, 0, 1, np));
  q.describe(planes_of(o->storage));
  std::vector<SchulzGroup> groups(1, q);
  ProductParams p;
  return run_schulz(s, groups, o->steps, planes_of(o->storage), f32 ? kLastF32 : kLastBf16, p, [&](size_t, ProductGroup& g) {
    g.out = o->out.data;
    g.out_row = o->out.row_stride;
    g.out_batch = o->out.worker_stride;
  });
} NM_CATCH(fail_caught)

int netmax_workspace_status(const void* workspace, int32_t device, void* stream) try {
  if (!workspace) return fail_op(NETMAX_INVALID_ARG, "workspace is NULL");
  OP_DO(check_device(device));
  OnDevice on(device);
  if (!on.ok) return fail_op(NETMAX_CUDA_ERROR, "cudaSetDevice failed");
  unsigned int word = 0;
  OP_CUDA(cudaMemcpyAsync(&word, workspace, sizeof word, cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  OP_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
  if (word) return fail_op(NETMAX_CUDA_ERROR, "a bounded wait inside a kernel ran out; the outputs of the last call that used this workspace are not to be used");
  return NETMAX_OK;
} NM_CATCH(fail_caught)

}  // extern "C"

// ---- the step --------------------------------------------------------------------------------------
namespace {

struct StepPlan {
  std::vector<netmax_matrix> small;    // those that a CTA or a cluster orthogonalises
  std::vector<netmax_matrix> sorted;   // the others by shape, then by offset: the order of the tables
  std::vector<SchulzGroup> groups;     // of equal shapes
  std::vector<int> first;              // of a group, in `sorted`
  std::vector<StepSegment> segments;   // by offset
  uint32_t pieces = 0;
  double* parts = nullptr;
  size_t total = 0;
};

int plan_step(int32_t M, int64_t d, const netmax_matrix* matrices, int32_t n, int32_t storage, void* workspace, StepPlan& plan) {
  OP_DO(check_storage(storage));
  if (M < 1 || M > 16384) return fail_op(NETMAX_INVALID_ARG, "M = %d outside [1, 16384]", M);
  if (d < 1 || d >= ((int64_t)1 << 30) - 32) return fail_op(NETMAX_INVALID_ARG, "d = %lld outside [1, 2^30 - 32)", (long long)d);
  if (n < 0 || n > kMaxMatrices) return fail_op(NETMAX_INVALID_ARG, "n_matrices = %d outside [0, %d]", n, kMaxMatrices);
  if (n > 0 && !matrices) return fail_op(NETMAX_INVALID_ARG, "matrices is NULL");
  plan.sorted.assign(matrices, matrices + n);
  for (const netmax_matrix& m : plan.sorted) {
    if (m.rows < 1 || m.cols < 1 || m.offset < 0 || m.rows > d || m.cols > d || m.offset > d || m.rows * m.cols > d - m.offset)
      return fail_op(NETMAX_INVALID_ARG, "a matrix of %lld x %lld at %lld does not lie in a replica of %lld elements", (long long)m.rows, (long long)m.cols,
                     (long long)m.offset, (long long)d);
    if (!std::isfinite((float)m.scale)) return fail_op(NETMAX_INVALID_ARG, "the scale of the matrix at %lld is not finite in fp32", (long long)m.offset);
    if ((int64_t)M * m.rows * m.cols >= (int64_t)1 << 40) return fail_op(NETMAX_INVALID_ARG, "M matrices of %lld x %lld are too many", (long long)m.rows, (long long)m.cols);
  }
  const bool larger = std::any_of(plan.sorted.begin(), plan.sorted.end(), [](const netmax_matrix& m) { return !is_small(m.rows, m.cols); });
  const auto apart = std::stable_partition(plan.sorted.begin(), plan.sorted.end(), [&](const netmax_matrix& m) {
    return !is_small(m.rows, m.cols) || (larger && joins_larger(m.rows, m.cols));
  });
  plan.small.assign(apart, plan.sorted.end());
  plan.sorted.erase(apart, plan.sorted.end());
  std::sort(plan.sorted.begin(), plan.sorted.end(), [](const netmax_matrix& a, const netmax_matrix& b) {
    return std::tie(a.rows, a.cols, a.offset) < std::tie(b.rows, b.cols, b.offset);
  });
  const int others = (int)plan.sorted.size();
  auto matrix = [&](int k) -> const netmax_matrix& { return k < others ? plan.sorted[k] : plan.small[k - others]; };
  std::vector<int> by_offset((size_t)n);
  for (int k = 0; k < n; ++k) by_offset[k] = k;
  std::sort(by_offset.begin(), by_offset.end(), [&](int a, int b) { return matrix(a).offset < matrix(b).offset; });
  int64_t at = 0;
  auto add = [&](int64_t length, int matrix) {
    if (length == 0) return;
    plan.segments.push_back({plan.pieces, (uint32_t)at, (uint32_t)length, matrix});
    plan.pieces += (uint32_t)ceil_div<int64_t>((at & 7) + length, kPiece);
    at += length;
  };
  for (int k : by_offset) {
    const netmax_matrix& m = matrix(k);
    if (m.offset < at) return fail_op(NETMAX_INVALID_ARG, "the matrix at %lld overlaps the one before it", (long long)m.offset);
    add(m.offset - at, -1);
    if (k < others) add(m.rows * m.cols, k);
    else at += m.rows * m.cols;  // (its kernel takes the whole update)
  }
  add(d - at, -1);
  Carver c(workspace);
  for (size_t k = 0; k < plan.sorted.size();) {
    size_t end = k;
    while (end < plan.sorted.size() && plan.sorted[end].rows == plan.sorted[k].rows && plan.sorted[end].cols == plan.sorted[k].cols) ++end;
    SchulzGroup g;
    g.set(plan.sorted[k].rows, plan.sorted[k].cols, (int)(end - k) * M);
    g.take(c, planes_of(storage));
    plan.groups.push_back(g);
    plan.first.push_back((int)k);
    k = end;
  }
  plan.parts = (double*)c.take((size_t)M * plan.pieces * sizeof(double));
  plan.total = c.used;
  return NETMAX_OK;
}

}  // namespace

namespace netmax {

int check_step(const netmax_step& t) {
  StepPlan plan;
  OP_DO(plan_step(t.M, t.d, t.matrices, t.n_matrices, t.storage, nullptr, plan));
  OP_DO(check_workspace(t.workspace, t.workspace_bytes, plan.total));
  OP_DO(check_steps(t.steps));
  if (!std::isfinite((float)t.lr) || !std::isfinite((float)t.mu) || !std::isfinite((float)t.decay))
    return fail_op(NETMAX_INVALID_ARG, "lr, mu and decay must be finite in fp32");
  const size_t size = element_size(t.storage);
  OP_DO(check_view("x", t.x, t.M, 1, t.d, false, size));
  OP_DO(check_view("x_next", t.x_next, t.M, 1, t.d, true, size));
  OP_DO(check_view("gradient", t.gradient, t.M, 1, t.d, false, size));
  OP_DO(check_view("momentum", t.momentum, t.M, 1, t.d, false, 4));
  OP_DO(check_view("momentum_next", t.momentum_next, t.M, 1, t.d, true, 4));
  if (!t.peers || !t.weights) return fail_op(NETMAX_INVALID_ARG, "peers or weights is NULL");
  const Span x = span_of(t.x, t.M, 1, t.d, size), next = span_of(t.x_next, t.M, 1, t.d, size), g = span_of(t.gradient, t.M, 1, t.d, size),
             m = span_of(t.momentum, t.M, 1, t.d, 4), m_next = span_of(t.momentum_next, t.M, 1, t.d, 4);
  OP_DO(check_apart("x_next", next, "x", x));
  OP_DO(check_apart("x_next", next, "gradient", g));
  OP_DO(check_apart("x_next", next, "momentum", m));
  OP_DO(check_apart("momentum_next", m_next, "x_next", next));
  OP_DO(check_apart("momentum_next", m_next, "x", x));
  OP_DO(check_apart("momentum_next", m_next, "gradient", g));
  const bool in_place = t.momentum.data == t.momentum_next.data && (t.M == 1 || t.momentum.worker_stride == t.momentum_next.worker_stride);
  if (!in_place) OP_DO(check_apart("momentum_next", m_next, "momentum", m));
  return NETMAX_OK;
}

// Enqueues a step that check_step has passed, on the current device.
int enqueue_step(const netmax_step& t, int draw_stride, unsigned int* error, int64_t* launches) {
  StepPlan plan;
  OP_DO(plan_step(t.M, t.d, t.matrices, t.n_matrices, t.storage, t.workspace, plan));
  Stream s{(cudaStream_t)t.stream, error ? error : (unsigned int*)t.workspace};
  if (error) s.clear = false;  // (a context's own word, which its next synchronisation reads)
  const bool f32 = t.storage == NETMAX_STORAGE_F32;
  StepParams sp;
  std::copy(plan.segments.begin(), plan.segments.end(), sp.segment);
  sp.gradient = t.gradient.data;
  sp.gradient_row = t.gradient.worker_stride;
  sp.momentum = (const float*)t.momentum.data;
  sp.momentum_row = t.momentum.worker_stride;
  sp.momentum_next = (float*)t.momentum_next.data;
  sp.momentum_next_row = t.momentum_next.worker_stride;
  sp.mu = (float)t.mu;
  sp.nesterov = t.nesterov != 0;
  sp.segments = (int)plan.segments.size();
  sp.pieces = (int)plan.pieces;
  sp.workers = t.M;
  sp.parts = plan.parts;
  sp.pull.x = t.x.data;
  sp.pull.x_row = t.x.worker_stride;
  sp.pull.x_next = t.x_next.data;
  sp.pull.next_row = t.x_next.worker_stride;
  sp.pull.peers = t.peers;
  sp.pull.weights = t.weights;
  sp.pull.draw_stride = draw_stride;
  sp.pull.lr = (float)t.lr;
  sp.pull.decay = (float)t.decay;
  sp.pull.workers = t.M;
  sp.error = s.error;
  const dim3 grid(plan.pieces, (unsigned)t.M);
  if (plan.pieces > 0) {
    sp.clear_error = s.clear;
    s.clear = false;
    OP_DO(launch(s, f32 ? step_momentum_kernel<float> : step_momentum_kernel<__nv_bfloat16>, grid, kElementThreads, 0, 1, sp));
  }
  // The small matrices, those that need equally large clusters in one launch; only the first of these runs beside the rest.
  std::vector<uint32_t> needs(plan.small.size());
  for (size_t k = 0; k < plan.small.size(); ++k)
    needs[k] = small_ctas((int64_t)plan.small.size() * t.M, (uint32_t)plan.small[k].rows, (uint32_t)plan.small[k].cols, sm_count());
  bool beside = plan.pieces > 0;
  for (uint32_t ctas = 1; ctas <= kMostCtas; ctas *= 2) {
    SmallParams mp;
    unsigned n = 0;
    size_t smem = 0;
    uint32_t columns = 0;
    for (size_t k = 0; k < plan.small.size(); ++k) {
      if (needs[k] != ctas) continue;
      const netmax_matrix& m = plan.small[k];
      mp.matrix[n++] = {(uint32_t)m.offset, (uint32_t)m.rows, (uint32_t)m.cols, (float)m.scale};
      smem = std::max(smem, small_smem((uint32_t)m.rows, (uint32_t)m.cols, ctas));
      columns = std::max(columns, small_tmem((uint32_t)m.rows, (uint32_t)m.cols, ctas));
    }
    if (n == 0) continue;
    mp.gradient = sp.gradient;
    mp.gradient_row = sp.gradient_row;
    mp.momentum = sp.momentum;
    mp.momentum_next = sp.momentum_next;
    mp.momentum_row = sp.momentum_row;
    mp.momentum_next_row = sp.momentum_next_row;
    mp.mu = sp.mu;
    mp.nesterov = sp.nesterov;
    mp.pull = sp.pull;
    mp.steps = t.steps;
    mp.ctas = (int32_t)ctas;
    mp.behind_rest = beside;
    beside = false;
    OP_DO(run_small(s, mp, n * (unsigned)t.M, smem, columns, f32 ? small_schulz_kernel<float, true> : small_schulz_kernel<__nv_bfloat16, true>));
  }
  if (!plan.groups.empty()) {
    StepIterateParams tables;
    std::memset(&tables, 0, sizeof tables);
    ProductParams p;
    for (size_t k = 0; k < plan.groups.size(); ++k) {
      SchulzGroup& g = plan.groups[k];
      const int members = g.batch / t.M;
      for (int j = 0; j < members; ++j) {
        const int at = plan.first[k] + j;
        tables.matrix[at] = {g.x[0] + (int64_t)j * t.M * g.x_batch, g.x_row, g.x_batch, g.x_plane, (uint32_t)g.cols, 0};
        p.matrix_offset[at] = (uint32_t)plan.sorted[at].offset;
        p.matrix_scale[at] = (float)plan.sorted[at].scale;
      }
      g.describe(planes_of(t.storage));
    }
    OP_DO(launch(s, f32 ? step_first_iterate_kernel<float> : step_first_iterate_kernel<__nv_bfloat16>, grid, kElementThreads, 0, 1, sp, tables));
    p.step = sp.pull;
    OP_DO(run_schulz(s, plan.groups, t.steps, planes_of(t.storage), f32 ? kStepF32 : kStepBf16, p, [&](size_t k, ProductGroup& g) {
      g.out_row = plan.groups[k].cols;  // (rows of a replica's matrix stand without gaps)
      g.first_matrix = plan.first[k];
    }));
  }
  if (launches) *launches += s.launches;
  return NETMAX_OK;
}

}  // namespace netmax

extern "C" {

int netmax_orthogonalised_step_workspace_size(int32_t M, int64_t d, const netmax_matrix* matrices, int32_t n_matrices, int32_t storage, size_t* bytes) try {
  StepPlan plan;
  OP_DO(plan_step(M, d, matrices, n_matrices, storage, nullptr, plan));
  if (!bytes) return fail_op(NETMAX_INVALID_ARG, "bytes is NULL");
  *bytes = plan.total;
  return NETMAX_OK;
} NM_CATCH(fail_caught)

int netmax_orthogonalised_step(const netmax_step* t) try {
  if (!t) return fail_op(NETMAX_INVALID_ARG, "step is NULL");
  OP_DO(check_step(*t));
  OP_DO(check_device(t->device));
  OnDevice on(t->device);
  if (!on.ok) return fail_op(NETMAX_CUDA_ERROR, "cudaSetDevice failed");
  return enqueue_step(*t, 1, nullptr, nullptr);
} NM_CATCH(fail_caught)

}  // extern "C"
