// embed_api.cu -- the C ABI of the embedding (declared in include/flashrec.h).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <new>

#include "../../include/flashrec.h"
#include "embed.h"
#include "host.h"
#include "kernels.h"

using namespace frk;

struct fr_embed_s {
  int device = 0;
  void* d_memory = nullptr;
  uint64_t rows = 0, dim = 0, max_tokens = 0, first = 0, device_bytes = 0;
  SortPlan sort;
  uint64_t ranges = 0;  // the most that a call has
  Met* d_sorted[2] = {};
  uint32_t* d_counts = nullptr;
  uint32_t* d_longs = nullptr;
  float* d_parts = nullptr;
  uint32_t* d_numbers = nullptr;  // found, n_long
};

namespace {

bool on(const void* p, uint64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
bool is_float(uint32_t dtype) { return dtype == FR_DT_BF16 || dtype == FR_DT_F32; }
uint32_t type_bytes(uint32_t dtype) { return dtype == FR_DT_F32 ? 4 : 2; }

// With fewer tokens than rows all rows are filled with zeros beside the sort, with more those that no token meets, once they are known: rows that
// are met are written once then.  (50,257 rows, 8,000 tokens of 768 41 us, by rows 83, 32,768 57 and 84, 131,072 122 and 117; 16,032 rows, 65,536
// tokens of 4,096 138 and 130.)
constexpr uint64_t kFillRows = 1;

constexpr uint64_t kMostRows = (1ull << 31) - 1, kMostDim = 1ull << 20, kMostElems = 1ull << 40, kMostFirst = 1ull << 62;

fr_status fill_embed(fr_embed p) {
  PlanMemory mem;
  const uint64_t n = p->max_tokens;
  if (p->dim > 0) p->ranges = std::max(ranges_of(n, p->dim, false), ranges_of(n, p->dim, true));
  mem.scratch(&p->d_sorted[0], n);
  if (p->sort.passes > 1) mem.scratch(&p->d_sorted[1], n);
  if (n > kClusterTokens) mem.scratch(&p->d_counts, static_cast<uint64_t>(kSortCtas) * p->sort.bins());
  mem.scratch(&p->d_longs, p->ranges / kSumWarps);
  mem.scratch(&p->d_parts, 2 * (p->ranges / kSumWarps) * p->dim);
  mem.scratch(&p->d_numbers, 2);
  p->device_bytes = mem.bytes();
  cudaError_t e = mem.commit(&p->d_memory);
  if (e != cudaSuccess) return report_cuda("plan device tables", e);
  e = configure_sort();
  if (e == cudaSuccess) e = configure_sum();
  return e == cudaSuccess ? FR_OK : report_cuda("shared memory of the gradient's kernels", e);
}

// What both calls ask of their arguments.
fr_status check(const char* me, fr_embed p, const void* table, uint32_t table_dtype, const void* tokens, uint32_t token_bytes, uint64_t n, float scale,
                const void* out, uint32_t out_dtype) {
  if (p == nullptr) return report_invalid(me, "plan is null");
  if (!is_float(table_dtype) || !is_float(out_dtype)) return report_invalid(me, "tables and rows are bf16 or fp32");
  if (token_bytes != 4 && token_bytes != 8) return report_invalid(me, "tokens have 4 or 8 bytes");
  if (n > p->max_tokens) return report_invalid(me, "more tokens than the plan is for");
  if (!std::isfinite(scale)) return report_invalid(me, "scale must be finite");
  if (n > 0 && tokens == nullptr) return report_invalid(me, "tokens is null");
  if (n > 0 && p->dim > 0 && out == nullptr) return report_invalid(me, "out is null");
  if (p->rows > 0 && p->dim > 0 && table == nullptr) return report_invalid(me, "the table is null");
  if (!on(table, type_bytes(table_dtype)) || !on(out, type_bytes(out_dtype)) || !on(tokens, token_bytes)) {
    report_invalid(me, "a buffer is not aligned to its element size");
    return FR_ERR_ALIGNMENT;
  }
  return FR_OK;
}

}  // namespace

extern "C" {

fr_status fr_embed_create(uint64_t rows, uint64_t dim, uint64_t max_tokens, uint64_t first, fr_embed* out) {
  CallRange nvtx("fr_embed_create");
  const char* const me = "fr_embed_create";
  if (out == nullptr) return report_invalid(me, "out is null");
  *out = nullptr;
  if (rows > kMostRows || max_tokens > kMostRows || dim > kMostDim || first > kMostFirst) return report_invalid(me, "too large");
  if (dim > 0 && (rows > kMostElems / dim || max_tokens > kMostElems / dim)) return report_invalid(me, "too many elements");

  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda("cudaGetDevice", e);

  fr_embed p = new (std::nothrow) fr_embed_s;
  if (p == nullptr) return report_invalid(me, "out of host memory");
  p->device = dev;
  p->rows = rows;
  p->dim = dim;
  p->max_tokens = max_tokens;
  p->first = first;
  p->sort = sort_plan(rows);
  fr_status st;
  try {
    st = fill_embed(p);
  } catch (const std::exception&) {
    st = report_invalid(me, "out of host memory");
  }
  if (st != FR_OK) {
    cudaFree(p->d_memory);
    delete p;
    return st;
  }
  *out = p;
  return FR_OK;
}

fr_status fr_embed_info(fr_embed p, uint64_t* rows, uint64_t* dim, uint64_t* max_tokens, uint64_t* device_bytes) {
  if (p == nullptr) return report_invalid("fr_embed_info", "plan is null");
  if (rows) *rows = p->rows;
  if (dim) *dim = p->dim;
  if (max_tokens) *max_tokens = p->max_tokens;
  if (device_bytes) *device_bytes = p->device_bytes;
  return FR_OK;
}

void fr_embed_destroy(fr_embed p) {
  CallRange nvtx("fr_embed_destroy");
  if (p == nullptr) return;
  DeviceGuard g(p->device);
  cudaDeviceSynchronize();
  cudaFree(p->d_memory);
  delete p;
}

fr_status fr_embed_lookup(fr_embed p, const void* table, uint32_t table_dtype, const void* tokens, uint32_t token_bytes, uint64_t n, float scale, void* out,
                          uint32_t out_dtype, void* stream) {
  CallRange nvtx("fr_embed_lookup");
  const fr_status st = check("fr_embed_lookup", p, table, table_dtype, tokens, token_bytes, n, scale, out, out_dtype);
  if (st != FR_OK) return st;
  if (n == 0 || p->dim == 0) return FR_OK;
  DeviceGuard g(p->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  LookupParams lp = {};
  lp.tokens = {tokens, n, p->first, p->rows, token_bytes == 8};
  lp.table = table;
  lp.out = out;
  lp.dim = p->dim;
  lp.scale = scale;
  lp.bf16_table = table_dtype == FR_DT_BF16;
  lp.bf16_out = out_dtype == FR_DT_BF16;
  const cudaError_t e = launch_lookup(lp, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FR_OK : report_cuda("lookup kernel launch", e);
}

fr_status fr_embed_grad(fr_embed p, const void* out, uint32_t out_dtype, const void* tokens, uint32_t token_bytes, uint64_t n, float scale, void* grad,
                        uint32_t grad_dtype, uint32_t accumulate, void* stream) {
  CallRange nvtx("fr_embed_grad");
  const char* const me = "fr_embed_grad";
  const fr_status st = check(me, p, grad, grad_dtype, tokens, token_bytes, n, scale, out, out_dtype);
  if (st != FR_OK) return st;
  if (accumulate > 1) return report_invalid(me, "accumulate must be 0 or 1");
  if (p->rows == 0 || p->dim == 0 || (accumulate && n == 0)) return FR_OK;
  DeviceGuard g(p->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  SortParams sp = {};
  sp.tokens = {tokens, n, p->first, p->rows, token_bytes == 8};
  sp.sorted[0] = p->d_sorted[0];
  sp.sorted[1] = p->d_sorted[1];
  sp.counts = p->d_counts;
  sp.found = p->d_numbers;
  sp.n_long = p->d_numbers + 1;
  const bool fill = !accumulate && n < kFillRows * p->rows;
  if (fill) {
    sp.fill = static_cast<uint8_t*>(grad);
    sp.fill_bytes = p->rows * p->dim * type_bytes(grad_dtype);
  }
  int last = 0;
  cudaError_t e = launch_sort(sp, p->sort, &last, s);
  if (e != cudaSuccess) return report_cuda("sort kernel launch", e);
  SumParams q = {};
  q.sorted = p->d_sorted[last];
  q.found = sp.found;
  q.n_long = sp.n_long;
  q.longs = p->d_longs;
  q.parts = p->d_parts;
  q.accumulate = accumulate;
  q.out = out;
  q.grad = grad;
  q.dim = p->dim;
  q.scale = scale;
  q.v = kind_of(p->dim, vector_elems(p->dim, out, type_bytes(out_dtype), grad, type_bytes(grad_dtype)));
  q.tiles = column_tiles(p->dim, q.v);
  q.ranges = ranges_of(n, p->dim, accumulate);
  q.ctas = q.ranges / kSumWarps * q.tiles;
  q.rows = p->rows;
  q.n = n;
  if (!accumulate && !fill) {
    // about 64 KiB per warp
    const uint64_t row_bytes = p->dim * type_bytes(grad_dtype);
    q.rows_per_zero_warp = static_cast<uint32_t>(std::min<uint64_t>(32, std::max<uint64_t>(1, (64 << 10) / row_bytes)));
    const uint32_t per_cta = q.rows_per_zero_warp * kSumWarps;
    q.zero_ctas = static_cast<uint32_t>((p->rows + per_cta - 1) / per_cta);
  }
  q.bf16_out = out_dtype == FR_DT_BF16;
  q.bf16_grad = grad_dtype == FR_DT_BF16;
  if (n > 0) e = launch_sum(q, s);
  return e == cudaSuccess ? FR_OK : report_cuda("gradient kernel launch", e);
}

}  // extern "C"
