// C-ABI front end of the serving operators: argument validation and dispatch.  The
// operations and every argument are documented in include/qm_attn.h.

#include "qm_attn.h"

#include <atomic>
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "checks.h"
#include "decode_rules.h"
#include "serving_launch.h"

namespace {

using qm::aligned16;
using qm::finite_bits;
using qm::overlaps;

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The bytes of a tensor argument.
struct Range {
  const void* p;
  uint64_t bytes;
};

template <int N>
bool any_overlap(const Range& out, const Range (&with)[N]) {
  for (const Range& r : with)
    if (out.p && r.p && overlaps(out.p, out.bytes, r.p, r.bytes)) return true;
  return false;
}

constexpr uint64_t kMost = 1ull << 62;   // bytes or elements of a tensor
// Tokens that a page table can hold for a sequence: 64 sequences' 32-token blocks are
// counted in 32 bits.
constexpr int64_t kMostTokens = 1ll << 29;

// a * b, or kMost where that is larger
uint64_t times(uint64_t a, uint64_t b) {
  return a && b > kMost / a ? kMost : a * b;
}

// Sizes of a cache; its strides and total bytes.
int check_cache(qm::PagedCache* c, uint64_t* bytes, int Hkv, int d, int num_pages, int page_size,
                int table_cols, int dtype, int cache_dtype, int cache_layout) {
  if (num_pages < 1 || table_cols < 1 || page_size < 16 || page_size % 16 || page_size > 65536)
    return QM_ERR_PAGE;
  if ((int64_t)table_cols * page_size > kMostTokens) return QM_ERR_PAGE;
  if (cache_dtype != dtype && cache_dtype != QM_E4M3) return QM_ERR_DTYPE;
  if (cache_layout != QM_BHND && cache_layout != QM_BNHD) return QM_ERR_LAYOUT;
  const uint64_t es = cache_dtype == QM_E4M3 ? 1 : 2;
  // 16 tokens of a page lie within the kernels' 32-bit offsets
  const uint64_t row = (uint64_t)Hkv * (uint64_t)d * es;
  if (row >= 1ull << 26) return QM_ERR_SHAPE;
  const uint64_t page = row * (uint64_t)page_size;   // below 2^42
  if (times(page, (uint64_t)num_pages) >= kMost) return QM_ERR_PAGE;
  *bytes = page * (uint64_t)num_pages;
  c->num_pages = num_pages;
  c->page_size = page_size;
  c->table_cols = table_cols;
  c->page_stride = (int64_t)page;
  c->token_stride = (int32_t)(cache_layout == QM_BNHD ? row : d * es);
  c->head_stride = (int32_t)(cache_layout == QM_BNHD ? d * es : (uint64_t)page_size * d * es);
  c->fp8 = cache_dtype == QM_E4M3;
  return QM_OK;
}

// One input's strides: checked, those of single elements dropped, NULL the contiguous
// ones; and the elements from its first to its last.
int check_strides(int64_t* s, uint64_t* span, const long long* given, int B, int N, int heads, int d,
                  int layout) {
  const int64_t size[3] = {B, N, heads};
  if (given) {
    for (int i = 0; i < 3; ++i) {
      s[i] = size[i] == 1 ? 0 : given[i];
      if (s[i] < 0 || s[i] % 8) return QM_ERR_STRIDE;
    }
  } else {
    s[0] = (int64_t)N * heads * d;
    s[1] = layout == QM_BNHD ? (int64_t)heads * d : d;
    s[2] = layout == QM_BNHD ? d : (int64_t)N * d;
  }
  *span = (uint64_t)d;
  for (int i = 0; i < 3; ++i) {
    *span += times((uint64_t)s[i], (uint64_t)(size[i] - 1));
    if (*span >= kMost / 4) return QM_ERR_SHAPE;
  }
  return QM_OK;
}

bool reciprocal(float scale, float* inv) {
  *inv = 1.0f / scale;
  return finite_bits(scale) && scale != 0.0f && finite_bits(*inv) && *inv != 0.0f;
}

// Both entry points; cached: the one that writes a cache.
int norm_rope(const void* q, const void* k, const void* v, void* q_out, void* k_out, void* k_cache,
              void* v_cache, const int* page_table, const void* q_weight, const void* k_weight,
              const float* cos, const float* sin, const int* starts, const int* counts, int B, int H,
              int Hkv, int N, int d, int rotary, int table_rows, float eps, int interleaved,
              int num_pages, int page_size, int table_cols, float k_scale, float v_scale,
              const long long* q_strides, const long long* k_strides, const long long* v_strides,
              hipStream_t stream, int dtype, int layout, int cache_dtype, int cache_layout,
              bool cached) {
  if (!q || !k || !q_out) return QM_ERR_NULL;
  if (cached ? !v || !k_cache || !v_cache || !page_table : !k_out) return QM_ERR_NULL;
  if (rotary > 0 && (!cos || !sin)) return QM_ERR_NULL;
  if (B < 1 || H < 1 || Hkv < 1 || N < 1) return QM_ERR_SHAPE;
  if (d != 64 && d != 128) return QM_ERR_HEADDIM;
  // rows in all: the launch's threads (d / 16 a row, rounded up to wavefronts) fit 31 bits
  const uint64_t heads = (uint64_t)H + 2ull * (uint64_t)Hkv;
  const uint64_t rows = times(times((uint64_t)B, (uint64_t)N), heads);
  if (rows >= (1ull << 27)) return QM_ERR_SHAPE;
  if (dtype != QM_F16 && dtype != QM_BF16) return QM_ERR_DTYPE;
  if (layout != QM_BHND && layout != QM_BNHD) return QM_ERR_LAYOUT;
  if (rotary < 0 || rotary > d || rotary % 16 || (interleaved != 0 && interleaved != 1) ||
      !finite_bits(eps) || eps < 0.0f)
    return QM_ERR_ROTARY;
  if (rotary > 0 && (table_rows < 1 || (!starts && N > table_rows))) return QM_ERR_ROTARY;

  qm::NormRopeArgs a = {};
  uint64_t cache_bytes = 0;
  if (cached) {
    const int st = check_cache(&a.cache, &cache_bytes, Hkv, d, num_pages, page_size, table_cols,
                               dtype, cache_dtype, cache_layout);
    if (st != QM_OK) return st;
    if (!reciprocal(k_scale, &a.k_inv) || !reciprocal(v_scale, &a.v_inv)) return QM_ERR_SCALE;
    a.cache.k = k_cache;
    a.cache.v = v_cache;
    a.cache.table = page_table;
  }
  uint64_t span[3] = {0, 0, 0};
  const long long* given[3] = {q_strides, k_strides, v_strides};
  for (int i = 0; i < (cached ? 3 : 2); ++i) {
    const int st = check_strides(a.stride[i], &span[i], given[i], B, N, i == 0 ? H : Hkv, d, layout);
    if (st != QM_OK) return st;
  }
  const uint64_t table = rotary > 0 ? (uint64_t)table_rows * (uint64_t)(rotary / 2) * 4 : 0;
  const Range in[] = {{q, span[0] * 2}, {k, span[1] * 2}, {cached ? v : nullptr, span[2] * 2},
                      {q_weight, (uint64_t)d * 2}, {k_weight, (uint64_t)d * 2},
                      {table ? cos : nullptr, table}, {table ? sin : nullptr, table},
                      {starts, (uint64_t)B * 4}, {counts, (uint64_t)B * 4},
                      {cached ? page_table : nullptr, (uint64_t)B * (uint64_t)(cached ? table_cols : 0) * 4}};
  const uint64_t row_bytes = (uint64_t)B * N * d * 2;
  const Range out[] = {{q_out, row_bytes * H}, {k_out, row_bytes * Hkv},
                       {cached ? k_cache : nullptr, cache_bytes}, {cached ? v_cache : nullptr, cache_bytes}};
  for (int i = 0; i < 4; ++i) {
    if (any_overlap(out[i], in)) return QM_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (out[i].p && out[j].p && overlaps(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
        return QM_ERR_ALIAS;
  }
  for (int i = 0; i < 7; ++i)
    if (in[i].p && !aligned16(in[i].p)) return QM_ERR_UNSUPPORTED;
  for (int i = 7; i < 10; ++i)
    if (in[i].p && !aligned4(in[i].p)) return QM_ERR_UNSUPPORTED;
  for (const Range& r : out)
    if (r.p && !aligned16(r.p)) return QM_ERR_UNSUPPORTED;

  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(cached ? v : nullptr);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_out = static_cast<uint16_t*>(k_out);
  a.q_weight = static_cast<const uint16_t*>(q_weight);
  a.k_weight = static_cast<const uint16_t*>(k_weight);
  a.cos = cos;
  a.sin = sin;
  a.starts = starts;
  a.counts = counts;
  a.B = B;
  a.H = H;
  a.Hkv = Hkv;
  a.N = N;
  a.d = d;
  a.rotary = rotary;
  a.table_rows = table_rows;
  a.interleaved = interleaved;
  a.dtype = dtype;
  a.layout = layout;
  a.eps = eps;
  return qm::launch_norm_rope(a, stream) == hipSuccess ? QM_OK : QM_ERR_LAUNCH;
}

// CUs of the current device (asked once for each of the first 64), or 0.
int device_cus() {
  static std::atomic<int> known[64];
  int id = 0, cus = 0;
  if (hipGetDevice(&id) != hipSuccess) return 0;
  if (id >= 0 && id < 64) cus = known[id].load(std::memory_order_relaxed);
  if (cus > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, id) != hipSuccess) return 0;
  if (id >= 0 && id < 64) known[id].store(cus, std::memory_order_relaxed);
  return cus;
}

// Checks of sizes that a decode call and its workspace share, and the call's split.
int plan(int B, int H, int Hkv, int d, int page_size, int table_cols, int max_length, int window,
         int sinks, qm::DecodePlan* p, int* limit) {
  if (B < 1 || H < 1 || Hkv < 1 || Hkv > H || H % Hkv != 0) return QM_ERR_SHAPE;
  if (d != 64 && d != 128) return QM_ERR_HEADDIM;
  if (table_cols < 1 || page_size < 16 || page_size % 16 || page_size > 65536 || max_length < 1)
    return QM_ERR_PAGE;
  const int64_t capacity = (int64_t)table_cols * page_size;
  if (capacity > kMostTokens) return QM_ERR_PAGE;
  if (window < 0 || sinks < 0) return QM_ERR_WINDOW;
  *limit = (int)(max_length < capacity ? max_length : capacity);
  const uint64_t tiles = ((uint64_t)(H / Hkv) + 15) / 16;
  const uint64_t rows = times(times((uint64_t)B, (uint64_t)Hkv), tiles);
  if (rows > INT_MAX / 512 || times((uint64_t)B, (uint64_t)H) > INT_MAX / 256) return QM_ERR_SHAPE;
  const int cus = device_cus();
  if (cus < 1) return QM_ERR_LAUNCH;
  *p = qm::plan_decode((int64_t)rows, qm::decode_blocks(*limit, window, sinks), cus);
  return QM_OK;
}

// Two partial results of 16 heads for each workgroup of a call in shares, and two
// numbers for each row.
size_t workspace_of(const qm::DecodePlan& p, int B, int H, int Hkv, int d) {
  const size_t rows = (size_t)B * Hkv * ((H / Hkv + 15) / 16);
  return p.grid ? (size_t)2 * p.grid * 16 * (d + 2) * sizeof(float) + rows * 2 * sizeof(int32_t) : 0;
}

}  // namespace

extern "C" int qm_qk_norm_rope(const void* q, const void* k, void* q_out, void* k_out,
                               const void* q_weight, const void* k_weight, const float* cos,
                               const float* sin, const int* starts, const int* counts, int B, int H,
                               int Hkv, int N, int d, int rotary, int table_rows, float eps,
                               int interleaved, const long long* q_strides,
                               const long long* k_strides, hipStream_t stream, int dtype,
                               int layout) {
  return norm_rope(q, k, nullptr, q_out, k_out, nullptr, nullptr, nullptr, q_weight, k_weight, cos,
                   sin, starts, counts, B, H, Hkv, N, d, rotary, table_rows, eps, interleaved, 0, 0,
                   0, 1.0f, 1.0f, q_strides, k_strides, nullptr, stream, dtype, layout, 0, 0, false);
}

extern "C" int qm_qk_norm_rope_append(
    const void* q, const void* k, const void* v, void* q_out, void* k_out, void* k_cache,
    void* v_cache, const int* page_table, const void* q_weight, const void* k_weight,
    const float* cos, const float* sin, const int* starts, const int* counts, int B, int H, int Hkv,
    int N, int d, int rotary, int table_rows, float eps, int interleaved, int num_pages,
    int page_size, int table_cols, float k_scale, float v_scale, const long long* q_strides,
    const long long* k_strides, const long long* v_strides, hipStream_t stream, int dtype,
    int layout, int cache_dtype, int cache_layout) {
  return norm_rope(q, k, v, q_out, k_out, k_cache, v_cache, page_table, q_weight, k_weight, cos, sin,
                   starts, counts, B, H, Hkv, N, d, rotary, table_rows, eps, interleaved, num_pages,
                   page_size, table_cols, k_scale, v_scale, q_strides, k_strides, v_strides, stream,
                   dtype, layout, cache_dtype, cache_layout, true);
}

extern "C" int qm_attn_decode_workspace(int B, int H, int Hkv, int d, int page_size, int table_cols,
                                        int max_length, int window, int sinks, size_t* bytes) {
  if (!bytes) return QM_ERR_NULL;
  qm::DecodePlan p;
  int limit;
  const int st = plan(B, H, Hkv, d, page_size, table_cols, max_length, window, sinks, &p, &limit);
  if (st == QM_OK) *bytes = workspace_of(p, B, H, Hkv, d);
  return st;
}

extern "C" int qm_attn_decode(const void* q, const void* k_cache, const void* v_cache, void* o,
                              float* lse, const int* page_table, const int* lengths, int B, int H,
                              int Hkv, int d, int num_pages, int page_size, int table_cols,
                              int max_length, float scale, float k_scale, float v_scale, int window,
                              int sinks, void* workspace, size_t workspace_bytes, hipStream_t stream,
                              int dtype, int cache_dtype, int cache_layout) {
  if (!q || !k_cache || !v_cache || !o || !lse || !page_table || !lengths) return QM_ERR_NULL;
  if (dtype != QM_F16 && dtype != QM_BF16) return QM_ERR_DTYPE;
  if (B < 1 || H < 1 || Hkv < 1 || Hkv > H || H % Hkv != 0) return QM_ERR_SHAPE;
  if (d != 64 && d != 128) return QM_ERR_HEADDIM;
  qm::DecodeArgs a = {};
  uint64_t cache_bytes = 0;
  int st = check_cache(&a.cache, &cache_bytes, Hkv, d, num_pages, page_size, table_cols, dtype,
                       cache_dtype, cache_layout);
  if (st != QM_OK) return st;
  if (max_length < 1) return QM_ERR_PAGE;
  if (window < 0 || sinks < 0) return QM_ERR_WINDOW;
  const double c = (double)scale * (double)k_scale * 1.4426950408889634074;
  if (!finite_bits(scale) || !finite_bits(k_scale) || !finite_bits(v_scale) ||
      !(fabs(c) < (double)FLT_MAX))
    return QM_ERR_SCALE;
  const uint64_t rows = times((uint64_t)B, (uint64_t)H);
  if (rows > INT_MAX / 256) return QM_ERR_SHAPE;
  const Range in[] = {{q, rows * d * 2}, {k_cache, cache_bytes}, {v_cache, cache_bytes},
                      {page_table, (uint64_t)B * (uint64_t)table_cols * 4}, {lengths, (uint64_t)B * 4}};
  const Range ro = {o, rows * d * 2}, rl = {lse, rows * 4};
  if (any_overlap(ro, in) || any_overlap(rl, in) || overlaps(o, ro.bytes, lse, rl.bytes))
    return QM_ERR_ALIAS;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o) ||
      !aligned16(lse) || !aligned4(page_table) || !aligned4(lengths))
    return QM_ERR_UNSUPPORTED;
  qm::DecodePlan p;
  st = plan(B, H, Hkv, d, page_size, table_cols, max_length, window, sinks, &p, &a.limit);
  if (st != QM_OK) return st;
  const size_t need = workspace_of(p, B, H, Hkv, d);
  if (need) {
    if (!workspace || workspace_bytes < need) return QM_ERR_WORKSPACE;
    const Range rw = {workspace, need};
    if (any_overlap(rw, in) || overlaps(workspace, need, o, ro.bytes) ||
        overlaps(workspace, need, lse, rl.bytes))
      return QM_ERR_ALIAS;
    if (!aligned16(workspace)) return QM_ERR_UNSUPPORTED;
  }
  a.q = static_cast<const uint16_t*>(q);
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  a.lengths = lengths;
  a.cache.k = const_cast<void*>(k_cache);
  a.cache.v = const_cast<void*>(v_cache);
  a.cache.table = page_table;
  a.B = B;
  a.H = H;
  a.Hkv = Hkv;
  a.d = d;
  a.dtype = dtype;
  a.window = window;
  a.sinks = sinks;
  a.c = (float)c;
  a.v_scale = v_scale;
  a.workspace = static_cast<float*>(workspace);
  return qm::launch_decode(a, p, stream) == hipSuccess ? QM_OK : QM_ERR_LAUNCH;
}
