// C-ABI entry points of the operators over a cache in pages: host checks, then the launch.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "fsx.h"
#include "kernels.h"
#include "pages.h"

namespace fsx {
void set_error_message(const char* msg);
}

namespace {

fsx_status fail(fsx_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  fsx::set_error_message(buf);
  return s;
}

fsx_status launched(cudaError_t e, const char* what) {
  return e == cudaSuccess ? FSX_OK : fail(FSX_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

constexpr long long kMaxRows = 0x7fffffffll;

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool is16(int dtype) { return dtype == FSX_BF16 || dtype == FSX_F16; }

fsx_status check_heads(int n_heads, int n_kv_heads, int head_dim) {
  if (head_dim != fsx::kHeadDim) return fail(FSX_ERR_UNSUPPORTED, "head_dim must be 128");
  if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0)
    return fail(FSX_ERR_INVALID_ARG, "n_heads must be a positive multiple of n_kv_heads");
  if (n_heads / n_kv_heads > fsx::kMaxGroup || n_heads > 4096)
    return fail(FSX_ERR_UNSUPPORTED, "at most 64 heads per kv head and 4096 heads");
  return FSX_OK;
}

fsx_status check_rows(const char* what, const void* p, long long stride, int heads) {
  if (!p) return fail(FSX_ERR_INVALID_ARG, "%s is NULL", what);
  if (stride < static_cast<long long>(heads) * fsx::kHeadDim || stride > (1ll << 32) || stride % 8 != 0)
    return fail(FSX_ERR_INVALID_ARG, "%s: the row stride must cover the heads and be a multiple of 16 bytes", what);
  if (!aligned(p, 16)) return fail(FSX_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
  return FSX_OK;
}

// log2 of the rows of a page
fsx_status check_page_rows(int page_rows, int& shift) {
  if (page_rows < 16 || page_rows > 1024 || (page_rows & (page_rows - 1)) != 0)
    return fail(FSX_ERR_UNSUPPORTED, "page_rows must be a power of two from 16 to 1024");
  shift = 0;
  while ((1 << shift) < page_rows) ++shift;
  return FSX_OK;
}

fsx_status check_pages(const int32_t* table, const int64_t* lengths, int B, int width, int page_rows, long long cache_rows,
                       fsx::PagedCache& out) {
  if (!table || !lengths) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (B < 1 || B > fsx::kMaxSequences) return fail(FSX_ERR_INVALID_ARG, "B must be in 1..1024");
  const fsx_status s = check_page_rows(page_rows, out.shift);
  if (s != FSX_OK) return s;
  if (width < 1) return fail(FSX_ERR_INVALID_ARG, "a table has one page a request or more");
  if (width > (kMaxRows >> out.shift)) return fail(FSX_ERR_UNSUPPORTED, "a request's pages must hold fewer than 2^31 rows");
  if (cache_rows < 0 || cache_rows % page_rows != 0) return fail(FSX_ERR_INVALID_ARG, "cache_rows must be whole pages");
  if (cache_rows > kMaxRows) return fail(FSX_ERR_UNSUPPORTED, "cache_rows must be below 2^31");
  out.table = table;
  out.lengths = lengths;
  out.B = B;
  out.width = width;
  out.n_pages = static_cast<int>(cache_rows >> out.shift);
  return FSX_OK;
}

// Turns a position of a pair, as 64-bit fixed point: the fraction of rate / (2 pi), rounded down. |rate| is m 2^(e - 53), m whole;
// 1 / (2 pi) to 128 bits behind the point; of the product 64 bits behind the point are kept.
uint64_t turns_of(double rate) {
  uint64_t bits;
  memcpy(&bits, &rate, sizeof(bits));
  const int biased = static_cast<int>(bits >> 52 & 0x7ff), e = biased - 1022;
  if (biased == 0) return 0;  // zero, or below 2^-1022
  const uint64_t m = (bits & ((1ull << 52) - 1)) | 1ull << 52;
  constexpr uint64_t kHi = 0x28BE60DB9391054Aull, kLo = 0x7F09D5F47D4D3770ull;  // 1 / (2 pi) = 0.28BE60DB...
  const unsigned __int128 hi = static_cast<unsigned __int128>(m) * kHi, lo = static_cast<unsigned __int128>(m) * kLo;
  // m / (2 pi) as w2.w1..., then times 2^(e - 53)
  const unsigned __int128 mid = static_cast<uint64_t>(hi) + (lo >> 64);
  const uint64_t w1 = static_cast<uint64_t>(mid), w2 = static_cast<uint64_t>(hi >> 64) + static_cast<uint64_t>(mid >> 64);
  const int right = 53 - e;  // the point moves this far to the left; 33 <= right, from |rate| <= 2^20
  uint64_t turns;
  if (right >= 128) turns = 0;
  else if (right > 64) turns = w2 >> (right - 64);
  else if (right == 64) turns = w2;
  else turns = w2 << (64 - right) | w1 >> right;
  return rate < 0 ? 0 - turns : turns;
}

fsx_status check_state(const int32_t* table, const int64_t* lengths, const int32_t* refs, int B, int width, int n_pages, int page_rows,
                       const int* d_status, int& shift) {
  if (!table || !lengths || !refs || !d_status) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (B < 1 || B > fsx::kMaxSequences) return fail(FSX_ERR_INVALID_ARG, "B must be in 1..1024");
  const fsx_status s = check_page_rows(page_rows, shift);
  if (s != FSX_OK) return s;
  if (width < 1 || n_pages < 1) return fail(FSX_ERR_INVALID_ARG, "a table has one page a request or more, a cache one page or more");
  if (width > (kMaxRows >> shift) || n_pages > (kMaxRows >> shift))
    return fail(FSX_ERR_UNSUPPORTED, "a request's and the cache's pages must hold fewer than 2^31 rows");
  return FSX_OK;
}

}  // namespace

extern "C" {

fsx_status fsx_rotary(const void* d_q, long long q_stride, const void* d_k, const void* d_v, long long kv_stride, int dtype,
                      const int64_t* d_positions, int n_axes, const int* axis, const double* rate, int layout, long long n_rows,
                      int n_heads, int n_kv_heads, int head_dim, void* d_q_out, long long q_out_stride, void* d_k_out,
                      long long k_out_stride, const int64_t* d_rows, void* d_k_cache, void* d_v_cache, float* d_k_scale,
                      float* d_v_scale, int cache_dtype, long long cache_rows, int* d_status, void* stream) {
  fsx::set_error_message("");
  if (!d_status || !axis || !rate) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (!is16(dtype)) return fail(FSX_ERR_INVALID_ARG, "dtype must be FSX_BF16 or FSX_F16");
  if (layout != FSX_ROTARY_HALVES && layout != FSX_ROTARY_ADJACENT) return fail(FSX_ERR_INVALID_ARG, "bad layout");
  if (n_axes < 1 || n_axes > fsx::kMaxAxes) return fail(FSX_ERR_INVALID_ARG, "n_axes must be in 1..4");
  if (n_rows < 0) return fail(FSX_ERR_INVALID_ARG, "n_rows must be >= 0");
  if (n_rows > kMaxRows) return fail(FSX_ERR_UNSUPPORTED, "n_rows must be below 2^31");
  fsx_status s = check_heads(n_heads, n_kv_heads, head_dim);
  if (s != FSX_OK) return s;
  fsx::RotaryArgs a{};
  for (int j = 0; j < fsx::kHeadDim / 2; ++j) {
    if (axis[j] < 0 || axis[j] >= n_axes) return fail(FSX_ERR_INVALID_ARG, "axis[%d] must be in 0..n_axes - 1", j);
    if (!(std::fabs(rate[j]) <= 1048576.0)) return fail(FSX_ERR_INVALID_ARG, "rate[%d] must be within +-2^20", j);
    a.axis[j] = static_cast<uint8_t>(axis[j]);
    a.turns[j] = turns_of(rate[j]);
  }
  const bool cached = d_k_cache || d_v_cache;
  if (n_rows == 0) return FSX_OK;
  if (!d_q && !d_k) return fail(FSX_ERR_INVALID_ARG, "neither queries nor keys");
  if (!d_positions) return fail(FSX_ERR_INVALID_ARG, "d_positions is NULL");
  if (!!d_q != !!d_q_out) return fail(FSX_ERR_INVALID_ARG, "d_q and d_q_out go together");
  if (d_q && ((s = check_rows("d_q", d_q, q_stride, n_heads)) != FSX_OK || (s = check_rows("d_q_out", d_q_out, q_out_stride, n_heads)) != FSX_OK)) return s;
  if (d_k ? !d_k_out && !cached : d_k_out || cached) return fail(FSX_ERR_INVALID_ARG, "d_k goes with d_k_out or a cache");
  if (d_k && (s = check_rows("d_k", d_k, kv_stride, n_kv_heads)) != FSX_OK) return s;
  if (d_k_out && (s = check_rows("d_k_out", d_k_out, k_out_stride, n_kv_heads)) != FSX_OK) return s;
  if (cached) {
    if (!d_k_cache || !d_v_cache) return fail(FSX_ERR_INVALID_ARG, "both caches or none");
    if ((s = check_rows("d_v", d_v, kv_stride, n_kv_heads)) != FSX_OK) return s;
    if (cache_dtype != dtype && cache_dtype != FSX_E4M3) return fail(FSX_ERR_INVALID_ARG, "cache_dtype must be dtype or FSX_E4M3");
    if (cache_dtype == FSX_E4M3 && (!d_k_scale || !d_v_scale)) return fail(FSX_ERR_INVALID_ARG, "an e4m3 cache needs its scales");
    if (cache_rows < 0) return fail(FSX_ERR_INVALID_ARG, "cache_rows must be >= 0");
    if (cache_rows > kMaxRows) return fail(FSX_ERR_UNSUPPORTED, "cache_rows must be below 2^31");
    if (!d_rows && n_rows > cache_rows) return fail(FSX_ERR_INVALID_ARG, "n_rows exceeds cache_rows");
    if (!aligned(d_k_cache, 16) || !aligned(d_v_cache, 16)) return fail(FSX_ERR_INVALID_ARG, "caches must be 16-byte aligned");
  }
  a.q = d_q;
  a.q_stride = q_stride;
  a.k = d_k;
  a.v = d_v;
  a.kv_stride = kv_stride;
  a.positions = d_positions;
  a.rows = n_rows;
  a.n_heads = n_heads;
  a.n_kv_heads = n_kv_heads;
  a.q_out = d_q_out;
  a.q_out_stride = q_out_stride;
  a.k_out = d_k_out;
  a.k_out_stride = k_out_stride;
  a.dst_rows = d_rows;
  a.k_cache = d_k_cache;
  a.v_cache = d_v_cache;
  a.k_scale = d_k_scale;
  a.v_scale = d_v_scale;
  a.cache_rows = cache_rows;
  a.status = d_status;
  return launched(fsx::launch_rotary(a, dtype, layout == FSX_ROTARY_ADJACENT, cached && cache_dtype == FSX_E4M3, static_cast<cudaStream_t>(stream)),
                  "rotary positions");
}

size_t fsx_paged_attention_workspace_bytes(int B, int n_heads, int n_kv_heads) {
  if (B < 1 || n_kv_heads < 1 || n_heads < n_kv_heads) return 0;
  return fsx::paged_attention_workspace_bytes(B, n_heads, n_kv_heads);
}

fsx_status fsx_paged_attention(const void* d_q, long long q_stride, int dtype, const void* d_k_cache, const void* d_v_cache,
                               const float* d_k_scale, const float* d_v_scale, int cache_dtype, long long cache_rows,
                               int page_rows, const int32_t* d_table, int width, const int64_t* d_lengths, int B,
                               const int32_t* d_picked, int n_picked, int n_heads, int n_kv_heads, int head_dim, void* d_out,
                               float* d_lse, void* d_workspace, size_t workspace_bytes, int* d_status, void* stream) {
  fsx::set_error_message("");
  if (!d_status || !d_q || !d_out) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (!is16(dtype)) return fail(FSX_ERR_INVALID_ARG, "dtype must be FSX_BF16 or FSX_F16");
  if (cache_dtype != dtype && cache_dtype != FSX_E4M3) return fail(FSX_ERR_INVALID_ARG, "cache_dtype must be dtype or FSX_E4M3");
  fsx::PagedArgs a{};
  fsx_status s = check_heads(n_heads, n_kv_heads, head_dim);
  if (s == FSX_OK) s = check_pages(d_table, d_lengths, B, width, page_rows, cache_rows, a.pages);
  if (s == FSX_OK) s = check_rows("d_q", d_q, q_stride, n_heads);
  if (s != FSX_OK) return s;
  if (cache_rows > 0 && (!d_k_cache || !d_v_cache)) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (cache_dtype == FSX_E4M3 && cache_rows > 0 && (!d_k_scale || !d_v_scale))
    return fail(FSX_ERR_INVALID_ARG, "an e4m3 cache needs its scales");
  if (d_picked && (n_picked < 1 || n_picked > fsx::kMaxPicked)) return fail(FSX_ERR_INVALID_ARG, "n_picked must be in 1..4096");
  if (!aligned(d_out, 16) || !aligned(d_k_cache, 16) || !aligned(d_v_cache, 16))
    return fail(FSX_ERR_INVALID_ARG, "d_out and the caches must be 16-byte aligned");
  const size_t need = fsx::paged_attention_workspace_bytes(B, n_heads, n_kv_heads);
  if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256))
    return fail(FSX_ERR_INVALID_ARG, "a 256-byte aligned workspace of %zu bytes is required", need);
  a.q = d_q;
  a.q_stride = q_stride;
  a.k_cache = d_k_cache;
  a.v_cache = d_v_cache;
  a.k_scale = d_k_scale;
  a.v_scale = d_v_scale;
  a.cache_rows = cache_rows;
  a.picked = d_picked;
  a.n_picked = n_picked;
  a.n_heads = n_heads;
  a.n_kv_heads = n_kv_heads;
  a.out = d_out;
  a.lse = d_lse;
  a.workspace = d_workspace;
  a.status = d_status;
  return launched(fsx::launch_paged_attention(a, dtype, cache_dtype == FSX_E4M3, static_cast<cudaStream_t>(stream)), "paged attention");
}

fsx_status fsx_page_bounds(const void* d_k_cache, const float* d_k_scale, int cache_dtype, long long cache_rows, int page_rows,
                           const int32_t* d_table, int width, const int64_t* d_lengths, const int64_t* d_start, int B, int n_kv_heads,
                           int head_dim, int8_t* d_bounds, float* d_bound_scale, int* d_status, void* stream) {
  fsx::set_error_message("");
  if (!d_status || !d_bounds || !d_bound_scale) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (!is16(cache_dtype) && cache_dtype != FSX_E4M3) return fail(FSX_ERR_INVALID_ARG, "cache_dtype must be FSX_BF16, FSX_F16 or FSX_E4M3");
  fsx::BoundsArgs a{};
  fsx_status s = check_heads(n_kv_heads, n_kv_heads, head_dim);
  if (s == FSX_OK) s = check_pages(d_table, d_lengths, B, width, page_rows, cache_rows, a.pages);
  if (s != FSX_OK) return s;
  if (cache_rows > 0 && !d_k_cache) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (cache_dtype == FSX_E4M3 && cache_rows > 0 && !d_k_scale) return fail(FSX_ERR_INVALID_ARG, "an e4m3 cache needs its scales");
  if (!aligned(d_k_cache, 16) || !aligned(d_bounds, 16)) return fail(FSX_ERR_INVALID_ARG, "the cache and the bounds must be 16-byte aligned");
  if (static_cast<long long>(width) * n_kv_heads > kMaxRows / 2) return fail(FSX_ERR_UNSUPPORTED, "width times n_kv_heads must be below 2^30");
  a.k_cache = d_k_cache;
  a.k_scale = d_k_scale;
  a.cache_rows = cache_rows;
  a.start = d_start;
  a.n_kv_heads = n_kv_heads;
  a.bounds = d_bounds;
  a.bound_scale = d_bound_scale;
  a.status = d_status;
  return launched(fsx::launch_page_bounds(a, cache_dtype, static_cast<cudaStream_t>(stream)), "page bounds");
}

fsx_status fsx_page_select(const void* d_q, long long q_stride, int dtype, const int8_t* d_bounds, const float* d_bound_scale,
                           long long cache_rows, int page_rows, const int32_t* d_table, int width, const int64_t* d_lengths, int B,
                           int n_heads, int n_kv_heads, int head_dim, int first, int last, int n_picked, int32_t* d_picked,
                           int* d_status, void* stream) {
  fsx::set_error_message("");
  if (!d_status || !d_picked) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (!is16(dtype)) return fail(FSX_ERR_INVALID_ARG, "dtype must be FSX_BF16 or FSX_F16");
  fsx::SelectArgs a{};
  fsx_status s = check_heads(n_heads, n_kv_heads, head_dim);
  if (s == FSX_OK) s = check_pages(d_table, d_lengths, B, width, page_rows, cache_rows, a.pages);
  if (s == FSX_OK) s = check_rows("d_q", d_q, q_stride, n_heads);
  if (s != FSX_OK) return s;
  if (width > fsx::kMaxPagesListed) return fail(FSX_ERR_UNSUPPORTED, "at most 32768 pages a request");
  if (n_picked < 1 || n_picked > fsx::kMaxPicked) return fail(FSX_ERR_INVALID_ARG, "n_picked must be in 1..4096");
  if (first < 0 || last < 0 || first > n_picked || last > n_picked - first)
    return fail(FSX_ERR_INVALID_ARG, "first and last must be >= 0 and n_picked at most together");
  if (cache_rows > 0 && (!d_bounds || !d_bound_scale)) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (!aligned(d_bounds, 16)) return fail(FSX_ERR_INVALID_ARG, "the bounds must be 16-byte aligned");
  if (cache_rows == 0) return fail(FSX_ERR_INVALID_ARG, "a cache of no pages");
  a.q = d_q;
  a.q_stride = q_stride;
  a.bounds = d_bounds;
  a.bound_scale = d_bound_scale;
  a.n_heads = n_heads;
  a.n_kv_heads = n_kv_heads;
  a.first = first;
  a.last = last;
  a.picked = d_picked;
  a.n_picked = n_picked;
  a.status = d_status;
  return launched(fsx::launch_page_select(a, dtype, static_cast<cudaStream_t>(stream)), "page selection");
}

fsx_status fsx_pages_step(const int32_t* d_table, const int64_t* d_lengths, const int32_t* d_refs, int B_in, const int32_t* d_source,
                          const int64_t* d_new_offsets, int B, long long new_rows, int width, int n_pages, int page_rows,
                          int32_t* d_table_out, int64_t* d_lengths_out, int32_t* d_refs_out, int64_t* d_rows, int32_t* d_pairs,
                          int32_t* d_n_pairs, int* d_status, void* stream) {
  fsx::set_error_message("");
  fsx::StepArgs a{};
  const fsx_status s = check_state(d_table, d_lengths, d_refs, B_in, width, n_pages, page_rows, d_status, a.shift);
  if (s != FSX_OK) return s;
  if (B < 1 || B > fsx::kMaxSequences) return fail(FSX_ERR_INVALID_ARG, "B must be in 1..1024");
  if (!d_new_offsets || !d_table_out || !d_lengths_out || !d_refs_out || !d_pairs || !d_n_pairs || (new_rows > 0 && !d_rows))
    return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (new_rows < 0 || new_rows > kMaxRows) return fail(FSX_ERR_INVALID_ARG, "new_rows must be in 0..2^31 - 1");
  if (!d_source && B != B_in) return fail(FSX_ERR_INVALID_ARG, "without d_source there are as many requests as before");
  if (d_source && (d_table_out == d_table || d_lengths_out == d_lengths))
    return fail(FSX_ERR_INVALID_ARG, "with d_source the new tables and lengths need buffers of their own");
  a.table = d_table;
  a.lengths = d_lengths;
  a.refs = d_refs;
  a.B_in = B_in;
  a.source = d_source;
  a.new_offsets = d_new_offsets;
  a.B = B;
  a.new_rows = new_rows;
  a.width = width;
  a.n_pages = n_pages;
  a.table_out = d_table_out;
  a.lengths_out = d_lengths_out;
  a.refs_out = d_refs_out;
  a.rows = d_rows;
  a.pairs = d_pairs;
  a.n_pairs = d_n_pairs;
  a.status = d_status;
  return launched(fsx::launch_pages_step(a, static_cast<cudaStream_t>(stream)), "step of page tables");
}

fsx_status fsx_pages_compact(const int32_t* d_table, const int64_t* d_lengths, const int32_t* d_refs, int B, int width, int n_pages,
                             int page_rows, int32_t* d_table_out, int32_t* d_refs_out, int32_t* d_pairs, int max_pairs,
                             int32_t* d_n_pairs, int* d_status, void* stream) {
  fsx::set_error_message("");
  fsx::CompactArgs a{};
  const fsx_status s = check_state(d_table, d_lengths, d_refs, B, width, n_pages, page_rows, d_status, a.shift);
  if (s != FSX_OK) return s;
  if (!d_table_out || !d_refs_out || !d_n_pairs || (n_pages > 1 && !d_pairs)) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (max_pairs < n_pages / 2) return fail(FSX_ERR_INVALID_ARG, "room for n_pages / 2 pairs is required");
  a.table = d_table;
  a.lengths = d_lengths;
  a.refs = d_refs;
  a.B = B;
  a.width = width;
  a.n_pages = n_pages;
  a.table_out = d_table_out;
  a.refs_out = d_refs_out;
  a.pairs = d_pairs;
  a.n_pairs = d_n_pairs;
  a.status = d_status;
  return launched(fsx::launch_pages_compact(a, static_cast<cudaStream_t>(stream)), "compaction of pages");
}

fsx_status fsx_pages_copy(const fsx_page_plane* planes, int n_planes, int n_pages, const int32_t* d_pairs, const int32_t* d_n_pairs,
                          int max_pairs, int* d_status, void* stream) {
  fsx::set_error_message("");
  if (!planes || !d_n_pairs || !d_status || (max_pairs > 0 && !d_pairs)) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (!aligned(d_pairs, 8)) return fail(FSX_ERR_INVALID_ARG, "d_pairs must be 8-byte aligned");
  if (n_planes < 1 || n_planes > fsx::kMaxPlanes) return fail(FSX_ERR_INVALID_ARG, "n_planes must be in 1..512");
  if (n_pages < 1 || max_pairs < 0) return fail(FSX_ERR_INVALID_ARG, "n_pages must be positive and max_pairs >= 0");
  for (int i = 0; i < n_planes; ++i) {
    const fsx_page_plane& p = planes[i];
    if (!p.base || !aligned(p.base, 4)) return fail(FSX_ERR_INVALID_ARG, "planes[%d]: a base aligned to 4 bytes is required", i);
    if (p.page_bytes < 4 || p.page_bytes % 4 != 0 || p.page_bytes > (1ll << 32) || p.segments < 1 || p.segments > 65536 ||
        (p.segments > 1 && (p.segment_stride % 4 != 0 || p.segment_stride < p.page_bytes * n_pages)))
      return fail(FSX_ERR_INVALID_ARG, "planes[%d]: bytes in fours, segments of at least n_pages pages", i);
  }
  if (max_pairs == 0) return FSX_OK;
  return launched(fsx::launch_pages_copy(planes, n_planes, n_pages, d_pairs, d_n_pairs, max_pairs, d_status, static_cast<cudaStream_t>(stream)),
                  "copy of pages");
}

}  // extern "C"
