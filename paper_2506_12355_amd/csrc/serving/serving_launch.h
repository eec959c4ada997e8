// Internal interface between the C-ABI front end (qm_serving.cpp) and the gfx950
// kernels of the operators around the attention forward.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace qm {

// A paged cache of keys or values: a page holds page_size tokens of every head.
struct PagedCache {
  void* k;                 // 16-bit elements, or E4M3 codes
  void* v;
  const int32_t* table;    // [B][table_cols]: a sequence's pages in order
  int num_pages, page_size, table_cols;
  int64_t page_stride;     // bytes from page to page, token to token, head to head
  int32_t token_stride, head_stride;
  int fp8;
};

struct NormRopeArgs {
  const uint16_t *q, *k, *v;             // v: NULL unless a cache is written
  uint16_t *q_out, *k_out;               // k_out may be NULL where a cache is written
  const uint16_t *q_weight, *k_weight;   // [d], or NULL: that tensor is not normalised
  const float *cos, *sin;                // [table_rows][rotary / 2]
  const int32_t *starts, *counts;        // [B], or NULL: 0 and N
  int64_t stride[3][3];                  // q, k, v: elements from batch to batch, token, head
  int B, H, Hkv, N, d, rotary, table_rows, interleaved, dtype, layout;
  float eps;
  float k_inv, v_inv;                    // what cached keys and values are multiplied by
  PagedCache cache;                      // cache.k NULL: none
};

hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream);

struct DecodeArgs {
  const uint16_t* q;       // [B][H][d]
  uint16_t* o;             // [B][H][d]
  float* lse;              // [B][H]
  const int32_t* lengths;  // [B]
  PagedCache cache;
  int B, H, Hkv, d, dtype;
  int limit;               // lengths past this are an error
  int window, sinks;       // window 0: every cached token is visible
  float c;                 // scale * k_scale * log2 e
  float v_scale;
  float* workspace;
};

// How a decode call is divided: a workgroup for each row (grid 0), or equal shares of
// all rows' blocks for `grid` workgroups, then joined.
struct DecodePlan {
  int grid;
};

hipError_t launch_decode(const DecodeArgs& a, const DecodePlan& plan, hipStream_t stream);

}  // namespace qm
