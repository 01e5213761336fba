// C ABI of the routed products (see include/gmagnus.h): routes, products by a sparse factor whose entries pick blocks, their
// gradients, sums over entries, 8-bit forms.  Nothing here waits for the device.
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <new>

#include "gm_host.h"
#include "gm_route_plan.cuh"
#include "gm_route_product.cuh"
#include "gm_route_sum.cuh"
#include "gm_route_quantize.cuh"

using gm::i64;

struct gm_route {
  i64 n_rows = 0, nnz = 0;
  int E = 0;
  const i64* row_ptr = nullptr;
  const float* val = nullptr;
  i64* offsets = nullptr;
  int32_t* rows = nullptr;
  int32_t* order = nullptr;
  int32_t* pos = nullptr;
  gm::RouteWord word;     // whether a kernel gave up a wait
};

namespace gm {

// A launch that may begin while the kernel before it in the stream ends (see grid_wait); cluster: blocks per cluster, 0 = as the
// kernel says.
template <typename... P, typename... A>
static int launch(void (*kernel)(P...), i64 blocks, int threads, size_t smem, cudaStream_t st, unsigned cluster, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster ? 2 : 1;
  GM_CUDA(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
  return GM_OK;
}

static size_t elem_size(int dtype) {
  switch (dtype) {
    case GM_F32: return 4;
    case GM_BF16: case GM_F16: return 2;
    case GM_E4M3: return 1;
    default: return 0;
  }
}
static bool is_float_type(int dtype) { return dtype == GM_F32 || dtype == GM_BF16 || dtype == GM_F16; }

static int check_dense(const gm_dense* M, const char* name) {
  if (!M) return fail(GM_ERR_INVALID_ARG, std::string(name) + " is null");
  if (M->n_blocks < 0 || M->n_rows < 0 || M->n_cols < 0 || M->n_blocks > INT32_MAX || M->n_rows > INT32_MAX - 65536 || M->n_cols > INT32_MAX - 65536)
    return fail(GM_ERR_INVALID_ARG, std::string(name) + ": sizes out of range");
  if (elem_size(M->dtype) == 0) return fail(GM_ERR_DTYPE, std::string(name) + ": unknown dtype");
  if (M->block_stride < 0 || M->row_stride < 0 || M->col_stride < 0) return fail(GM_ERR_INVALID_ARG, std::string(name) + ": negative stride");
  if (!M->data && M->n_blocks && M->n_rows && M->n_cols) return fail(GM_ERR_INVALID_ARG, std::string(name) + ": null data");
  if (reinterpret_cast<uintptr_t>(M->data) % elem_size(M->dtype)) return fail(GM_ERR_INVALID_ARG, std::string(name) + ": data not aligned to its type");
  return GM_OK;
}
// Results: rows contiguous, apart from each other.
static int check_out(const gm_dense* M, const char* name) {
  GM_TRY(check_dense(M, name));
  if (M->n_cols > 1 && M->col_stride != 1) return fail(GM_ERR_INVALID_ARG, std::string(name) + ": rows of a result must be contiguous");
  if ((M->n_rows > 1 && M->row_stride < M->n_cols) || (M->n_blocks > 1 && M->block_stride < (M->n_rows - 1) * M->row_stride + M->n_cols))
    return fail(GM_ERR_INVALID_ARG, std::string(name) + ": rows of a result overlap");
  return GM_OK;
}
// The largest power of two, up to 32, that the addresses of a result's rows are multiples of.
static int out_align(const gm_dense& M) {
  const i64 es = static_cast<i64>(elem_size(M.dtype));
  int align = 32;
  while (align > 1 && (reinterpret_cast<uintptr_t>(M.data) % align || (M.n_rows > 1 && M.row_stride * es % align) || (M.n_blocks > 1 && M.block_stride * es % align))) align /= 2;
  return align;
}
static int check_shape(const gm_dense* M, const char* name, i64 blocks, i64 rows, i64 cols) {
  if (M->n_blocks != blocks || M->n_rows != rows || M->n_cols != cols)
    return fail(GM_ERR_DIM_MISMATCH, std::string(name) + ": " + std::to_string(M->n_blocks) + " x " + std::to_string(M->n_rows) + " x " + std::to_string(M->n_cols) +
                                         " instead of " + std::to_string(blocks) + " x " + std::to_string(rows) + " x " + std::to_string(cols));
  return GM_OK;
}

static PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
static std::mutex g_encode_mutex;

static int encoder(PFN_cuTensorMapEncodeTiled_v12000* out) {
  std::lock_guard<std::mutex> lock(g_encode_mutex);
  if (!g_encode) {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    GM_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found));
    if (!f || found != cudaDriverEntryPointSuccess) return fail(GM_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
    g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }
  *out = g_encode;
  return GM_OK;
}

// rank 2 or 3; strides of the outer dimensions in bytes; 128-byte swizzle, what lies outside reads as zero.
static int make_map(CUtensorMap* map, int dtype, int rank, const void* base, const uint64_t* dims, const uint64_t* strides, const uint32_t* box) {
  PFN_cuTensorMapEncodeTiled_v12000 encode;
  GM_TRY(encoder(&encode));
  const uint32_t ones[3] = {1, 1, 1};
  const CUtensorMapDataType type = dtype == GM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : dtype == GM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : dtype == GM_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  const CUresult rc = encode(map, type, rank, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (rc != CUDA_SUCCESS) return fail(GM_ERR_CUDA, "cuTensorMapEncodeTiled: error " + std::to_string(static_cast<int>(rc)));
  return GM_OK;
}

// Memory of one call, given back in stream order when it ends.
struct Scratch {
  cudaStream_t st;
  void* held[4] = {};
  int n = 0;
  explicit Scratch(cudaStream_t s) : st(s) {}
  ~Scratch() { for (int i = 0; i < n; ++i) dev_free(held[i], st); }
  void* get(size_t bytes) {
    void* p = dev_alloc(bytes, st);
    if (p) held[n++] = p;
    return p;
  }
};

// What a tensor map can be laid over: 16-byte aligned base and outer strides, none of them zero, the inner dimension contiguous, its runs apart.
static bool map_fits(const gm_dense& M, bool rows_inner) {
  const i64 es = static_cast<i64>(elem_size(M.dtype));
  const i64 inner = rows_inner ? M.row_stride : M.col_stride, outer = rows_inner ? M.col_stride : M.row_stride;
  const i64 n_inner = rows_inner ? M.n_rows : M.n_cols, n_outer = rows_inner ? M.n_cols : M.n_rows;
  const auto ok = [&](i64 stride, i64 n) { return n <= 1 || (stride > 0 && stride * es % 16 == 0 && stride * es < (i64{1} << 40)); };
  return reinterpret_cast<uintptr_t>(M.data) % 16 == 0 && (inner == 1 || n_inner <= 1) && ok(outer, n_outer) && (n_outer <= 1 || outer >= n_inner) &&
         ok(M.block_stride, M.n_blocks);
}

static int pack(const gm_dense& M, Scratch* mem, int num_sms, gm_dense* out) {
  const i64 es = static_cast<i64>(elem_size(M.dtype)), per = 16 / es, padded = (M.n_cols + per - 1) / per * per;
  const size_t bytes = static_cast<size_t>(M.n_blocks) * M.n_rows * padded * es;
  void* p = mem->get(bytes);
  if (!p) return fail(GM_ERR_OOM, "no room for an aligned copy of " + std::to_string(bytes) + " bytes");
  if (M.col_stride == 1 || M.n_cols <= 1) {  // rows of whole units, as large as their addresses allow
    i64 unit = 8;
    while (unit > es && (reinterpret_cast<uintptr_t>(M.data) % unit || M.n_cols * es % unit || (M.n_rows > 1 && M.row_stride * es % unit) || (M.n_blocks > 1 && M.block_stride * es % unit))) unit /= 2;
    const i64 grid = std::min<i64>((M.n_blocks * M.n_rows + 7) / 8, static_cast<i64>(num_sms) * 8);
    const auto go = [&](auto* tag) {
      using T = std::remove_pointer_t<decltype(tag)>;
      return launch(k_route_pack_rows<T>, grid, 256, 0, mem->st, 0, static_cast<const T*>(M.data), M.block_stride * es / unit, M.row_stride * es / unit, M.n_blocks, M.n_rows,
                    static_cast<int>(M.n_cols * es / unit), static_cast<int>(padded * es / unit), static_cast<T*>(p));
    };
    GM_TRY(unit == 8 ? go(static_cast<uint64_t*>(nullptr)) : unit == 4 ? go(static_cast<uint32_t*>(nullptr)) : unit == 2 ? go(static_cast<uint16_t*>(nullptr)) : go(static_cast<uint8_t*>(nullptr)));
  } else {
    const i64 grid = std::min<i64>((M.n_blocks * M.n_rows * padded + 255) / 256, static_cast<i64>(num_sms) * 16);
    const auto go = [&](auto* tag) {
      using T = std::remove_pointer_t<decltype(tag)>;
      return launch(k_route_pack<T>, grid, 256, 0, mem->st, 0, static_cast<const T*>(M.data), M.block_stride, M.row_stride, M.col_stride, M.n_blocks, M.n_rows, M.n_cols, padded, static_cast<T*>(p));
    };
    GM_TRY(es == 2 ? go(static_cast<uint16_t*>(nullptr)) : es == 4 ? go(static_cast<uint32_t*>(nullptr)) : go(static_cast<uint8_t*>(nullptr)));
  }
  *out = M;
  out->data = p;
  out->col_stride = 1;
  out->row_stride = padded;
  out->block_stride = M.n_rows * padded;
  return GM_OK;
}

// Inputs of the kernels that read with ordinary loads: any block and row strides, rows contiguous.
static int contiguous_rows(gm_dense* M, Scratch* mem) {
  if (M->n_cols <= 1 || M->col_stride == 1 || M->n_rows == 0 || M->n_blocks == 0) return GM_OK;
  int num_sms, smem_optin;
  GM_TRY(device_facts_basic(&num_sms, &smem_optin));
  return pack(gm_dense(*M), mem, num_sms, M);
}

// Rows that start on 16 bytes: as they are, or copied.
static int aligned_rows(gm_dense* M, Scratch* mem, int num_sms) {
  const i64 es = static_cast<i64>(elem_size(M->dtype));
  const bool fits = reinterpret_cast<uintptr_t>(M->data) % 16 == 0 && (M->col_stride == 1 || M->n_cols <= 1) && (M->n_rows <= 1 || M->row_stride * es % 16 == 0);
  return fits ? GM_OK : pack(gm_dense(*M), mem, num_sms, M);
}

// A map of rows, `at_a_time` of them by 128 bytes; `rows`: what it lies over.
static int map_rows(CUtensorMap* map, gm_dense* rows, uint32_t at_a_time, Scratch* mem, int num_sms) {
  if (!map_fits(*rows, false)) GM_TRY(pack(gm_dense(*rows), mem, num_sms, rows));
  const gm_dense& M = *rows;
  const i64 es = static_cast<i64>(elem_size(M.dtype));
  const uint64_t dims[2] = {static_cast<uint64_t>(M.n_cols), static_cast<uint64_t>(M.n_rows)};
  const uint64_t strides[1] = {static_cast<uint64_t>(M.n_rows > 1 ? M.row_stride * es : (M.n_cols * es + 15) / 16 * 16)};
  const uint32_t box[2] = {static_cast<uint32_t>(kRowBytes / es), at_a_time};
  return make_map(map, M.dtype, 2, M.data, dims, strides, box);
}

// A map of a result's blocks (or of one matrix), written 32 rows by 128 bytes at a time.  Only where the rows' addresses allow it (out_align).
static int map_out(CUtensorMap* map, const gm_dense& M) {
  const i64 es = static_cast<i64>(elem_size(M.dtype));
  const uint64_t row = static_cast<uint64_t>(M.n_rows > 1 ? M.row_stride * es : (M.n_cols * es + 15) / 16 * 16);
  const uint64_t dims[3] = {static_cast<uint64_t>(M.n_cols), static_cast<uint64_t>(M.n_rows), static_cast<uint64_t>(M.n_blocks)};
  const uint64_t strides[2] = {row, M.n_blocks > 1 ? static_cast<uint64_t>(M.block_stride * es) : row * M.n_rows};
  const uint32_t box[3] = {static_cast<uint32_t>(kRowBytes / es), 32, 1};
  return make_map(map, M.dtype, 3, M.data, dims, strides, box);
}

// (not destroyed at the process's end, where routes may still be given back)
static RouteWords& words() {
  static RouteWords* all = new RouteWords;
  return *all;
}

static int route_ready(const gm_route* r) {
  if (!r) return fail(GM_ERR_INVALID_ARG, "route is null");
  if (route_word_reported(r->word))
    return fail(GM_ERR_TIMEOUT, "an earlier call on this route gave up waiting on the device: its results are not valid");
  return GM_OK;
}

// The most dynamic shared memory these kernels ask for (what a block may have, less their static arrays), allowed once per device.
constexpr int kMostSmem = 232448 - 1024;
struct SmemAllowed { std::atomic<unsigned long long> devices{0}; };
template <auto kernel>
static int allow_most_smem() {
  static SmemAllowed allowed;
  int dev = 0;
  GM_CUDA(cudaGetDevice(&dev));
  const unsigned long long bit = 1ull << (dev & 63);
  if (allowed.devices.load(std::memory_order_relaxed) & bit) return GM_OK;
  GM_CUDA(cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
  allowed.devices.fetch_or(bit, std::memory_order_relaxed);
  return GM_OK;
}

template <int kN>
constexpr size_t kT5Smem = static_cast<size_t>(Shape<kN>::kStages) * Shape<kN>::kStage + 1024 + sizeof(T5Block);
template <int kN>
constexpr size_t kScaleSmem = kScaleSlots * (kN == kFewN ? kFewSlot : kScaleSlot) * 4 + sizeof(ScaleBlock);
template <int kN>
static size_t product_smem(int E, bool bits8) {
  return kT5Smem<kN> + static_cast<size_t>(E + 1) * 8 + (bits8 ? kScaleSmem<kN> : 0);
}
static_assert(std::max(kT5Smem<kTileN> + kScaleSmem<kTileN>, kT5Smem<kFewN> + kScaleSmem<kFewN>) + (kRouteMaxCols + 1) * 8 <= kMostSmem, "fits a block's shared memory");

static_assert(kRouteMaxCols == GM_ROUTE_MAX_COLS, "as the header says");

// Whether tiles of few places are the better ones: while a column has at most three quarters of such a tile's on average (64 columns of 1536 x 4096: with 8
// places each 158 us against 165 with tiles of 256, in 8 bits 98 against 125; with 48 164 : 169 and 106 : 133, with 64 180 : 171 and 135 : 133).  Measured with
// columns that are all alike: where few columns of very many hold most entries, the average is low and these, too, go in tiles of 64.
static bool few_places(const gm_route* r) { return r->nnz <= static_cast<i64>(kFewN * 3 / 4) * std::min<i64>(r->E, r->nnz); }
static i64 tile_count(const gm_route* r, i64 n_m, int n) { return ((r->nnz + n - 1) / n + std::min<i64>(r->E, r->nnz)) * ((n_m + kTileM - 1) / kTileM); }

// Whether clusters of kRouteBlocks fit the current device (more than 8 blocks are not promised), found out once.
static bool wide_clusters() {
  static std::atomic<unsigned long long> known{0}, fits{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const unsigned long long bit = 1ull << (dev & 63);
  if (!(known.load() & bit)) {
    int n = 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kRouteBlocks);
    cfg.blockDim = dim3(kRouteThreads);
    cfg.dynamicSmemBytes = kMostSmem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = kRouteBlocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(reinterpret_cast<const void*>(k_route_plan<true>), cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
        cudaOccupancyMaxActiveClusters(&n, k_route_plan<true>, &cfg) == cudaSuccess && n > 0)
      fits.fetch_or(bit);
    cudaGetLastError();
    known.fetch_or(bit);
  }
  return fits.load() & bit;
}

// A result of no terms: rows of zeros.
static int zero_out(const gm_dense& M, cudaStream_t st) {
  const size_t es = elem_size(M.dtype);
  if (M.n_cols == 0) return GM_OK;
  for (i64 b = 0; b < M.n_blocks; ++b)
    if (M.n_rows) GM_CUDA(cudaMemset2DAsync(static_cast<char*>(M.data) + static_cast<size_t>(b) * M.block_stride * es, static_cast<size_t>(M.n_rows > 1 ? M.row_stride : M.n_cols) * es, 0, M.n_cols * es, M.n_rows, st));
  return GM_OK;
}

// A pair of blocks per tile, at most one pair per two SMs.
template <auto kernel, typename... A>
static int launch_t5(i64 tiles, int num_sms, int threads, size_t smem, cudaStream_t st, const A&... args) {
  GM_TRY(allow_most_smem<kernel>());
  return launch(kernel, 2 * std::max<i64>(1, std::min<i64>(tiles, num_sms / 2)), threads, smem, st, 0, args...);
}

// out[p, m] = sum_k B[e(p)](m, k) X[x row of p, k];  w_transposed: B's rows are W's columns.
static int product(const gm_route* r, const gm_dense& X, bool by_entry, const gm_dense& W, bool w_transposed, const gm_dense& out, cudaStream_t st) {
  const i64 n_m = w_transposed ? W.n_cols : W.n_rows, n_k = w_transposed ? W.n_rows : W.n_cols;
  if (r->nnz == 0 || n_m == 0) return GM_OK;
  if (n_k == 0 || r->E == 0) return zero_out(out, st);
  int num_sms, smem_optin;
  GM_TRY(device_facts_basic(&num_sms, &smem_optin));
  Scratch mem(st);
  // the block of W as (rows m) x (sums over k): which of the two is contiguous decides the form in shared memory
  gm_dense V = W;
  if (w_transposed) {
    std::swap(V.n_rows, V.n_cols);
    std::swap(V.row_stride, V.col_stride);
  }
  bool m_inner = false;
  if (!map_fits(V, false)) {
    m_inner = map_fits(V, true);
    if (!m_inner) {
      gm_dense packed;
      GM_TRY(pack(W, &mem, num_sms, &packed));
      V = packed;
      if (w_transposed) {
        std::swap(V.n_rows, V.n_cols);
        std::swap(V.row_stride, V.col_stride);
        m_inner = true;
      }
    }
  }
  CUtensorMap map_w, map_x;
  const i64 es = 2;
  const i64 inner = m_inner ? V.n_rows : V.n_cols, outer = m_inner ? V.n_cols : V.n_rows, outer_stride = m_inner ? V.col_stride : V.row_stride;
  const uint64_t row_bytes = static_cast<uint64_t>(outer > 1 ? outer_stride * es : (inner * es + 15) / 16 * 16);
  const uint64_t dims[3] = {static_cast<uint64_t>(inner), static_cast<uint64_t>(outer), static_cast<uint64_t>(V.n_blocks)};
  const uint64_t strides[2] = {row_bytes, V.n_blocks > 1 ? static_cast<uint64_t>(V.block_stride * es) : row_bytes * outer};
  const uint32_t box[3] = {64, m_inner ? 64u : 128u, 1};
  GM_TRY(make_map(&map_w, V.dtype, 3, V.data, dims, strides, box));
  gm_dense rows = X;
  if (by_entry) {
    GM_TRY(map_rows(&map_x, &rows, 32, &mem, num_sms));
  } else {
    GM_TRY(aligned_rows(&rows, &mem, num_sms));
    map_x = map_w;  // (not used)
  }
  ProductArgs a = {};
  a.offsets = r->offsets;
  a.rows = r->rows;
  a.E = r->E;
  a.n_m = static_cast<int>(n_m);
  a.n_k = static_cast<int>(n_k);
  a.x = static_cast<const char*>(rows.data);
  a.x_stride = rows.row_stride * es;
  a.places = r->nnz;
  a.out = out.data;
  a.out_stride = out.row_stride;
  a.type = X.dtype == GM_BF16 ? 1 : 0;
  a.word = r->word;
  const auto typed = [&](auto* tag) {
    using TO = std::remove_pointer_t<decltype(tag)>;
    const auto sized = [&]<int kN>() {
      const auto go = [&]<auto kernel>() {
        return launch_t5<kernel>(tile_count(r, n_m, kN), num_sms, by_entry ? 192 : 352, product_smem<kN>(r->E, false), st, map_w, map_x, a);
      };
      if (m_inner) return by_entry ? go.template operator()<k_route_product<kN, true, false, TO>>() : go.template operator()<k_route_product<kN, true, true, TO>>();
      return by_entry ? go.template operator()<k_route_product<kN, false, false, TO>>() : go.template operator()<k_route_product<kN, false, true, TO>>();
    };
    return few_places(r) ? sized.template operator()<kFewN>() : sized.template operator()<kTileN>();
  };
  switch (out.dtype) {
    case GM_F32: return typed(static_cast<float*>(nullptr));
    case GM_BF16: return typed(static_cast<__nv_bfloat16*>(nullptr));
    default: return typed(static_cast<__half*>(nullptr));
  }
}

static int sum_grid(i64 blocks, const char* what) {
  return blocks > INT32_MAX ? fail(GM_ERR_INVALID_ARG, std::string(what) + ": too many rows and columns for one launch") : GM_OK;
}

static bool rows_aligned(const gm_dense& M) {
  return reinterpret_cast<uintptr_t>(M.data) % 16 == 0 && M.n_cols % 8 == 0 && (M.n_rows <= 1 || M.row_stride * elem_size(M.dtype) % 16 == 0);
}

static int sum_rows(const gm_route* r, const gm_dense& P, bool weighted, const gm_dense& Y, cudaStream_t st) {
  if (Y.n_rows == 0 || Y.n_cols == 0) return GM_OK;
  SumArgs a = {};
  a.row_ptr = r->row_ptr;
  a.val = weighted ? r->val : nullptr;
  a.offsets = r->offsets;
  a.rows = r->rows;
  a.pos = r->pos;
  a.E = r->E;
  a.entries = r->nnz;
  a.width = static_cast<int>(Y.n_cols);
  a.p = P.data;
  a.p_stride = P.row_stride;
  a.y = Y.data;
  a.y_stride = Y.row_stride;
  const bool vec = rows_aligned(P) && rows_aligned(Y);
  // as many threads as a row has use for
  const auto typed2 = [&](auto* ti, auto* to) {
    using TI = std::remove_pointer_t<decltype(ti)>;
    using TO = std::remove_pointer_t<decltype(to)>;
    const auto aligned = [&]<bool kVec>() -> int {
      constexpr int kUnits = kSumUnits<TI, kVec>;
      const auto go = [&]<int kThreads>() -> int {
        const i64 columns = kThreads * kUnits * (kVec ? 16 / sizeof(TI) : 1), chunks = (a.width + columns - 1) / columns;
        GM_TRY(sum_grid(chunks * r->n_rows, "sum"));
        return launch(k_route_sum<TI, TO, kVec, kUnits, kThreads>, chunks * r->n_rows, kThreads, 0, st, 0, a, static_cast<int>(chunks));
      };
      const int per = 32 * kUnits * (kVec ? 16 / static_cast<int>(sizeof(TI)) : 1);
      return a.width <= per ? go.template operator()<32>() : a.width <= 2 * per ? go.template operator()<64>() : go.template operator()<128>();
    };
    return vec ? aligned.template operator()<true>() : aligned.template operator()<false>();
  };
  const auto typed = [&](auto* ti) {
    switch (Y.dtype) {
      case GM_F32: return typed2(ti, static_cast<float*>(nullptr));
      case GM_BF16: return typed2(ti, static_cast<__nv_bfloat16*>(nullptr));
      default: return typed2(ti, static_cast<__half*>(nullptr));
    }
  };
  switch (P.dtype) {
    case GM_F32: return typed(static_cast<float*>(nullptr));
    case GM_BF16: return typed(static_cast<__nv_bfloat16*>(nullptr));
    default: return typed(static_cast<__half*>(nullptr));
  }
}

static int guarded(const auto& body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return GM_ERR_OOM;
  } catch (...) {
    return GM_ERR_INTERNAL;
  }
}

static int check_products(const gm_dense* X, const gm_dense* W, const gm_dense* out, const char* x_name, const char* out_name) {
  if (X->dtype != GM_BF16 && X->dtype != GM_F16) return fail(GM_ERR_DTYPE, std::string(x_name) + ": bf16 or f16 expected");
  if (W && W->dtype != X->dtype) return fail(GM_ERR_DTYPE, "the factors' types differ");
  if (!is_float_type(out->dtype)) return fail(GM_ERR_DTYPE, std::string(out_name) + ": f32, bf16 or f16 expected");
  return GM_OK;
}

}  // namespace gm

using namespace gm;

extern "C" {

int gm_route_plan(const gm_csr* R, int64_t* offsets, int32_t* rows, int32_t* order, int32_t* pos, void* cuda_stream, gm_route** route_out) {
  return guarded([&]() -> int {
    if (!R || !route_out) return fail(GM_ERR_INVALID_ARG, "null argument");
    *route_out = nullptr;
    if (R->n_rows < 0 || R->n_cols < 0 || R->nnz < 0 || R->n_rows > INT32_MAX - 65536 || R->nnz > INT32_MAX - 65536)
      return fail(GM_ERR_INVALID_ARG, "R: sizes out of range");
    if (R->n_cols > kRouteMaxCols) return fail(GM_ERR_CAPACITY, "R: more than " + std::to_string(kRouteMaxCols) + " columns");
    if (R->n_rows == 0 && R->nnz > 0) return fail(GM_ERR_BAD_CSR, "R: entries without rows");
    if (!R->row_ptr || (R->nnz > 0 && (!R->col_idx || !R->vals))) return fail(GM_ERR_INVALID_ARG, "R: null array");
    if (!offsets || (R->nnz > 0 && (!rows || !order || !pos))) return fail(GM_ERR_INVALID_ARG, "null array");
    if (R->dtype != GM_F32) return fail(GM_ERR_DTYPE, "R: f32 values expected");
    int num_sms, smem_optin;
    GM_TRY(device_facts_basic(&num_sms, &smem_optin));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    gm_route* r = new (std::nothrow) gm_route;
    if (!r) return fail(GM_ERR_OOM, "out of host memory");
    const auto drop = [&](int rc) { gm_route_destroy(r); return rc; };
    r->n_rows = R->n_rows;
    r->nnz = R->nnz;
    r->E = static_cast<int>(R->n_cols);
    r->row_ptr = R->row_ptr;
    r->val = static_cast<const float*>(R->vals);
    r->word = words().take(page_locked);
    if (!r->word.at) return drop(fail(GM_ERR_OOM, "no page-locked memory"));
    r->offsets = offsets;
    r->rows = rows;
    r->order = order;
    r->pos = pos;
    const int warps = route_warps(r->E), n_rows = static_cast<int>(r->n_rows);
    int rc = allow_most_smem<k_route_plan<true>>();
    if (rc != GM_OK) return drop(rc);
    if (r->nnz > kRouteWide && r->E <= kRouteWideCols) {
      rc = allow_most_smem<k_route_plan<false>>();
      if (rc != GM_OK) return drop(rc);
      Scratch mem(st);
      const int few = std::min(warps, kRouteWideThreads / 32);
      u32* sums = static_cast<u32*>(mem.get(static_cast<size_t>(kRouteWideBlocks) * (r->E + 1) * 4));
      if (!sums) return drop(fail(GM_ERR_OOM, "no room for the blocks' sums"));
      rc = launch(k_route_count, kRouteWideBlocks, few * 32, static_cast<size_t>(r->E + 1) * 4, st, 0, R->col_idx, r->nnz, r->E, sums);
      if (rc == GM_OK)
        rc = launch(k_route_plan<false>, kRouteWideBlocks, few * 32, route_smem(r->E, few), st, 0, r->row_ptr, R->col_idx, n_rows, r->nnz, r->E, sums, r->offsets,
                    r->rows, r->order, r->pos);
    } else {
      // a thread per entry while there are blocks for that (4096 entries: 6.1 us by four blocks, 12.2 by one)
      unsigned blocks = 1;
      while (blocks < kRouteBlocks && static_cast<i64>(blocks) * warps * 32 < r->nnz) blocks *= 2;
      if (blocks > 8 && !wide_clusters()) blocks = 8;
      rc = launch(k_route_plan<true>, blocks, warps * 32, route_smem(r->E, warps), st, blocks, r->row_ptr, R->col_idx, n_rows, r->nnz, r->E,
                  static_cast<const u32*>(nullptr), r->offsets, r->rows, r->order, r->pos);
    }
    if (rc != GM_OK) return drop(rc);
    *route_out = r;
    return GM_OK;
  });
}

int gm_route_status(const gm_route* route) { return guarded([&]() -> int { return route_ready(route); }); }

void gm_route_destroy(gm_route* route) {
  if (!route) return;
  guarded([&]() -> int {
    words().give(route->word);
    return GM_OK;
  });
  delete route;
}

int gm_route_product(const gm_route* route, const gm_dense* X, int by_entry, const gm_dense* W, const gm_dense* P, void* cuda_stream) {
  return guarded([&]() -> int {
    GM_TRY(route_ready(route));
    GM_TRY(check_dense(X, "X"));
    GM_TRY(check_dense(W, "W"));
    GM_TRY(check_out(P, "P"));
    GM_TRY(check_products(X, W, P, "X", "P"));
    GM_TRY(check_shape(X, "X", 1, by_entry ? route->nnz : route->n_rows, W->n_cols));
    GM_TRY(check_shape(W, "W", route->E, W->n_rows, W->n_cols));
    GM_TRY(check_shape(P, "P", 1, route->nnz, W->n_rows));
    return product(route, *X, by_entry != 0, *W, false, *P, static_cast<cudaStream_t>(cuda_stream));
  });
}

int gm_route_product_dx(const gm_route* route, const gm_dense* dP, const gm_dense* W, int by_entry, const gm_dense* dX, void* terms, void* cuda_stream) {
  return guarded([&]() -> int {
    GM_TRY(route_ready(route));
    GM_TRY(check_dense(dP, "dP"));
    GM_TRY(check_dense(W, "W"));
    GM_TRY(check_out(dX, "dX"));
    GM_TRY(check_products(dP, W, dX, "dP", "dX"));
    GM_TRY(check_shape(dP, "dP", 1, route->nnz, W->n_rows));
    GM_TRY(check_shape(W, "W", route->E, W->n_rows, W->n_cols));
    GM_TRY(check_shape(dX, "dX", 1, by_entry ? route->nnz : route->n_rows, W->n_cols));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (by_entry) return product(route, *dP, true, *W, true, *dX, st);
    if (route->nnz == 0) return zero_out(*dX, st);
    // the entries' terms in 32 bits, then one sum per row of R: each result is rounded once
    Scratch mem(st);
    gm_dense T = {};
    T.n_blocks = 1;
    T.n_rows = route->nnz;
    T.n_cols = W->n_cols;
    T.row_stride = (W->n_cols + 7) / 8 * 8;
    T.col_stride = 1;
    T.dtype = GM_F32;
    if (reinterpret_cast<uintptr_t>(terms) % 16) return fail(GM_ERR_INVALID_ARG, "terms: not aligned to 16 bytes");
    T.data = terms ? terms : mem.get(static_cast<size_t>(T.n_rows) * T.row_stride * 4);
    if (!T.data) return fail(GM_ERR_OOM, "no room for the entries' terms");
    GM_TRY(product(route, *dP, true, *W, true, T, st));
    return sum_rows(route, T, false, *dX, st);
  });
}

int gm_route_product_dw(const gm_route* route, const gm_dense* dP, const gm_dense* X, int by_entry, const gm_dense* dW, void* cuda_stream) {
  return guarded([&]() -> int {
    GM_TRY(route_ready(route));
    GM_TRY(check_dense(dP, "dP"));
    GM_TRY(check_dense(X, "X"));
    GM_TRY(check_out(dW, "dW"));
    GM_TRY(check_products(dP, X, dW, "dP", "dW"));
    GM_TRY(check_shape(dP, "dP", 1, route->nnz, dP->n_cols));
    GM_TRY(check_shape(X, "X", 1, by_entry ? route->nnz : route->n_rows, X->n_cols));
    GM_TRY(check_shape(dW, "dW", route->E, dP->n_cols, X->n_cols));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dW->n_blocks == 0 || dW->n_rows == 0 || dW->n_cols == 0) return GM_OK;
    if (route->nnz == 0) return zero_out(*dW, st);
    int num_sms, smem_optin;
    GM_TRY(device_facts_basic(&num_sms, &smem_optin));
    Scratch mem(st);
    gm_dense G = *dP, V = *X;
    CUtensorMap map_p, map_x;
    GM_TRY(map_rows(&map_p, &G, 64, &mem, num_sms));
    if (by_entry) {
      GM_TRY(map_rows(&map_x, &V, 64, &mem, num_sms));
    } else {
      GM_TRY(aligned_rows(&V, &mem, num_sms));
      map_x = map_p;  // (not used)
    }
    DwArgs a = {};
    a.offsets = route->offsets;
    a.rows = route->rows;
    a.E = route->E;
    a.n_m = static_cast<int>(dP->n_cols);
    a.n_j = static_cast<int>(X->n_cols);
    a.dp = static_cast<const char*>(G.data);
    a.dp_stride = G.row_stride * 2;
    a.x = static_cast<const char*>(V.data);
    a.x_stride = V.row_stride * 2;
    a.out = dW->data;
    a.out_block = dW->block_stride;
    a.out_stride = dW->row_stride;
    a.out_align = out_align(*dW);
    a.type = dP->dtype == GM_BF16 ? 1 : 0;
    a.word = route->word;
    const i64 tiles = static_cast<i64>(a.E) * ((a.n_m + kTileM - 1) / kTileM) * ((a.n_j + kTileN - 1) / kTileN);
    CUtensorMap out_map = map_p;  // (used where the rows of dW are aligned)
    if (a.out_align >= 16) GM_TRY(map_out(&out_map, *dW));
    const size_t smem = static_cast<size_t>(kDwStages) * kStage + 8 * kOutBytes + 1024 + sizeof(T5Block) + (a.E + 1) * 4;
    const auto go = [&]<auto kernel>() { return launch_t5<kernel>(tiles, num_sms, 480, smem, st, map_p, map_x, out_map, a); };
    switch (dW->dtype) {
      case GM_F32: return by_entry ? go.template operator()<k_route_dw<false, float>>() : go.template operator()<k_route_dw<true, float>>();
      case GM_BF16: return by_entry ? go.template operator()<k_route_dw<false, __nv_bfloat16>>() : go.template operator()<k_route_dw<true, __nv_bfloat16>>();
      default: return by_entry ? go.template operator()<k_route_dw<false, __half>>() : go.template operator()<k_route_dw<true, __half>>();
    }
  });
}

int gm_route_sum(const gm_route* route, const gm_dense* P, int weighted, const gm_dense* Y, void* cuda_stream) {
  return guarded([&]() -> int {
    GM_TRY(route_ready(route));
    GM_TRY(check_dense(P, "P"));
    GM_TRY(check_out(Y, "Y"));
    if (!is_float_type(P->dtype) || !is_float_type(Y->dtype)) return fail(GM_ERR_DTYPE, "f32, bf16 or f16 expected");
    GM_TRY(check_shape(P, "P", 1, route->nnz, P->n_cols));
    GM_TRY(check_shape(Y, "Y", 1, route->n_rows, P->n_cols));
    Scratch mem(static_cast<cudaStream_t>(cuda_stream));
    gm_dense V = *P;
    GM_TRY(contiguous_rows(&V, &mem));
    return sum_rows(route, V, weighted != 0, *Y, mem.st);
  });
}

int gm_route_sum_grads(const gm_route* route, const gm_dense* dY, const gm_dense* P, const gm_dense* dP, float* dval, void* cuda_stream) {
  return guarded([&]() -> int {
    GM_TRY(route_ready(route));
    GM_TRY(check_dense(dY, "dY"));
    GM_TRY(check_dense(P, "P"));
    GM_TRY(check_out(dP, "dP"));
    if (!is_float_type(dY->dtype) || P->dtype != dY->dtype || dP->dtype != dY->dtype) return fail(GM_ERR_DTYPE, "dY, P and dP of one type (f32, bf16 or f16) expected");
    GM_TRY(check_shape(P, "P", 1, route->nnz, P->n_cols));
    GM_TRY(check_shape(dY, "dY", 1, route->n_rows, P->n_cols));
    GM_TRY(check_shape(dP, "dP", 1, route->nnz, P->n_cols));
    if (route->nnz == 0) return GM_OK;
    if (!dval) return fail(GM_ERR_INVALID_ARG, "dval is null");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    Scratch mem(st);
    gm_dense G = *dY, V = *P;
    GM_TRY(contiguous_rows(&G, &mem));
    GM_TRY(contiguous_rows(&V, &mem));
    SumArgs a = {};
    a.row_ptr = route->row_ptr;
    a.val = route->val;
    a.offsets = route->offsets;
    a.rows = route->rows;
    a.pos = route->pos;
    a.E = route->E;
    a.entries = route->nnz;
    a.width = static_cast<int>(P->n_cols);
    a.p = V.data;
    a.p_stride = V.row_stride;
    a.y = G.data;
    a.y_stride = G.row_stride;
    const bool vec = rows_aligned(V) && rows_aligned(G) && rows_aligned(*dP);
    const auto typed = [&](auto* tag) {
      using T = std::remove_pointer_t<decltype(tag)>;
      const auto kernel = vec ? k_route_sum_grads<T, T, true> : k_route_sum_grads<T, T, false>;
      return launch(kernel, (route->nnz + 7) / 8, 256, 0, st, 0, a, static_cast<T*>(dP->data), dP->row_stride, dval);
    };
    switch (dY->dtype) {
      case GM_F32: return typed(static_cast<float*>(nullptr));
      case GM_BF16: return typed(static_cast<__nv_bfloat16*>(nullptr));
      default: return typed(static_cast<__half*>(nullptr));
    }
  });
}

int gm_block_quantize(const gm_dense* X, int block_rows, const gm_dense* Q, const gm_dense* S, void* cuda_stream) {
  return guarded([&]() -> int {
    GM_TRY(check_dense(X, "X"));
    GM_TRY(check_out(Q, "Q"));
    GM_TRY(check_out(S, "S"));
    if (block_rows != 1 && block_rows != 128) return fail(GM_ERR_INVALID_ARG, "block_rows: 1 or 128 expected");
    if (X->dtype != GM_BF16 && X->dtype != GM_F16) return fail(GM_ERR_DTYPE, "X: bf16 or f16 expected");
    if (Q->dtype != GM_E4M3 || S->dtype != GM_F32) return fail(GM_ERR_DTYPE, "Q: e4m3, S: f32 expected");
    const i64 cg = (X->n_cols + 127) / 128, rg = (X->n_rows + block_rows - 1) / block_rows;
    GM_TRY(check_shape(Q, "Q", X->n_blocks, X->n_rows, X->n_cols));
    GM_TRY(check_shape(S, "S", X->n_blocks, rg, cg));
    const auto dense = [](const gm_dense* M) {
      return (M->n_rows <= 1 || M->row_stride == M->n_cols) && (M->n_blocks <= 1 || M->block_stride == M->n_rows * M->n_cols);
    };
    if (X->n_blocks == 0 || X->n_rows == 0 || X->n_cols == 0) return GM_OK;
    if (!dense(Q) || !dense(S)) return fail(GM_ERR_INVALID_ARG, "Q and S must be contiguous");
    QuantArgs a = {};
    a.x = X->data;
    a.x_block = X->block_stride;
    a.x_row = X->row_stride;
    a.x_col = X->col_stride;
    a.n_blocks = X->n_blocks;
    a.n_rows = X->n_rows;
    a.n_cols = static_cast<int>(X->n_cols);
    a.col_groups = static_cast<int>(cg);
    a.q = static_cast<unsigned char*>(Q->data);
    a.s = static_cast<float*>(S->data);
    const bool vec = X->col_stride == 1 && rows_aligned(*X) && (X->n_blocks <= 1 || X->block_stride % 8 == 0) && reinterpret_cast<uintptr_t>(Q->data) % 8 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool flat = vec && X->n_cols % 128 == 0 && (X->n_rows <= 1 || X->row_stride == X->n_cols) && (X->n_blocks <= 1 || X->block_stride == X->n_rows * X->n_cols);
    const i64 units = X->n_blocks * rg * cg, blocks = block_rows == 1 ? (units + 16 * kQuantAhead - 1) / (16 * kQuantAhead) : units;
    GM_TRY(sum_grid(blocks, "quantize"));
    const auto typed = [&](auto* tag) {
      using T = std::remove_pointer_t<decltype(tag)>;
      if (block_rows == 1)
        return launch(flat ? k_quantize_rows<T, true, true> : vec ? k_quantize_rows<T, true, false> : k_quantize_rows<T, false, false>, blocks, 256, 0, st, 0, a);
      return launch(vec ? k_quantize_tiles<T, true> : k_quantize_tiles<T, false>, blocks, 256, 0, st, 0, a, static_cast<int>(rg));
    };
    return X->dtype == GM_BF16 ? typed(static_cast<__nv_bfloat16*>(nullptr)) : typed(static_cast<__half*>(nullptr));
  });
}

int gm_route_product_scaled(const gm_route* route, const gm_dense* Xq, const gm_dense* Xs, int by_entry, const gm_dense* Wq, const gm_dense* Ws,
                          const gm_dense* P, void* cuda_stream) {
  return guarded([&]() -> int {
    GM_TRY(route_ready(route));
    GM_TRY(check_dense(Xq, "Xq"));
    GM_TRY(check_dense(Xs, "Xs"));
    GM_TRY(check_dense(Wq, "Wq"));
    GM_TRY(check_dense(Ws, "Ws"));
    GM_TRY(check_out(P, "P"));
    if (Xq->dtype != GM_E4M3 || Wq->dtype != GM_E4M3) return fail(GM_ERR_DTYPE, "Xq and Wq: e4m3 expected");
    if (Xs->dtype != GM_F32 || Ws->dtype != GM_F32) return fail(GM_ERR_DTYPE, "Xs and Ws: f32 expected");
    if (!is_float_type(P->dtype)) return fail(GM_ERR_DTYPE, "P: f32, bf16 or f16 expected");
    const i64 cg = (Wq->n_cols + 127) / 128, x_rows = by_entry ? route->nnz : route->n_rows;
    GM_TRY(check_shape(Xq, "Xq", 1, x_rows, Wq->n_cols));
    GM_TRY(check_shape(Xs, "Xs", 1, x_rows, cg));
    GM_TRY(check_shape(Wq, "Wq", route->E, Wq->n_rows, Wq->n_cols));
    const bool row_scales = Ws->n_rows == Wq->n_rows && Wq->n_rows > 1;  // (of one row the two forms are the same)
    GM_TRY(check_shape(Ws, "Ws", route->E, row_scales ? Wq->n_rows : (Wq->n_rows + 127) / 128, cg));
    GM_TRY(check_shape(P, "P", 1, route->nnz, Wq->n_rows));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (route->nnz == 0 || Wq->n_rows == 0) return GM_OK;
    if (Wq->n_cols == 0 || route->E == 0) return zero_out(*P, st);
    int num_sms, smem_optin;
    GM_TRY(device_facts_basic(&num_sms, &smem_optin));
    Scratch mem(st);
    gm_dense V = *Wq, xs = *Xs, ws = *Ws;
    GM_TRY(contiguous_rows(&xs, &mem));
    GM_TRY(contiguous_rows(&ws, &mem));
    if (!map_fits(V, false)) GM_TRY(pack(*Wq, &mem, num_sms, &V));
    CUtensorMap map_w, map_x;
    const uint64_t row_bytes = static_cast<uint64_t>(V.n_rows > 1 ? V.row_stride : (V.n_cols + 15) / 16 * 16);
    const uint64_t dims[3] = {static_cast<uint64_t>(V.n_cols), static_cast<uint64_t>(V.n_rows), static_cast<uint64_t>(V.n_blocks)};
    const uint64_t strides[2] = {row_bytes, V.n_blocks > 1 ? static_cast<uint64_t>(V.block_stride) : row_bytes * V.n_rows};
    const uint32_t box[3] = {kRowBytes, 128, 1};
    GM_TRY(make_map(&map_w, GM_E4M3, 3, V.data, dims, strides, box));
    gm_dense rows = *Xq;
    if (by_entry) {
      GM_TRY(map_rows(&map_x, &rows, 32, &mem, num_sms));
    } else {
      GM_TRY(aligned_rows(&rows, &mem, num_sms));
      map_x = map_w;  // (not used)
    }
    ProductArgs a = {};
    a.offsets = route->offsets;
    a.rows = route->rows;
    a.E = route->E;
    a.n_m = static_cast<int>(Wq->n_rows);
    a.n_k = static_cast<int>(Wq->n_cols);
    a.x = static_cast<const char*>(rows.data);
    a.x_stride = rows.row_stride;
    a.places = route->nnz;
    a.out = P->data;
    a.out_stride = P->row_stride;
    a.out_align = out_align(*P);
    a.type = 0;
    a.xs = static_cast<const float*>(xs.data);
    a.xs_stride = xs.row_stride;
    a.ws = static_cast<const float*>(ws.data);
    a.ws_block = ws.block_stride;
    a.ws_row = ws.row_stride;
    a.word = route->word;
    const bool few = few_places(route);
    const i64 tiles = tile_count(route, a.n_m, few ? kFewN : kTileN);
    const size_t smem = few ? product_smem<kFewN>(route->E, true) : product_smem<kTileN>(route->E, true);
    const auto typed = [&](auto* tag) {
      using TO = std::remove_pointer_t<decltype(tag)>;
      const auto go = [&]<bool kGather, bool kRowScales>() {
        const auto with = [&]<auto kernel>() { return launch_t5<kernel>(tiles, num_sms, few && by_entry ? 384 : 512, smem, st, map_w, map_x, a); };
        return few ? with.template operator()<k_route_product_scaled_few<kGather, kRowScales, TO>>() : with.template operator()<k_route_product_scaled<kGather, kRowScales, TO>>();
      };
      if (row_scales) return by_entry ? go.template operator()<false, true>() : go.template operator()<true, true>();
      return by_entry ? go.template operator()<false, false>() : go.template operator()<true, false>();
    };
    switch (P->dtype) {
      case GM_F32: return typed(static_cast<float*>(nullptr));
      case GM_BF16: return typed(static_cast<__nv_bfloat16*>(nullptr));
      default: return typed(static_cast<__half*>(nullptr));
    }
  });
}

}  // extern "C"
