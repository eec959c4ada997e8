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
  const int32_t* positions;              // [axes][B][N], or NULL: starts + t
  int used_axes;                         // bit a set where a pair has axis a
  uint64_t pair_axis[2];                 // the axis of pair j: bits 2 (j % 32) .. of word j / 32
  float k_inv, v_inv;                    // what cached keys and values are multiplied by
  PagedCache cache;                      // cache.k NULL: none
};

hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream);

struct RmsNormArgs {
  const uint16_t *x, *residual, *weight;   // residual and weight may be NULL
  uint16_t* sum;                           // x + residual, or NULL
  void* out;                               // [rows][width], 16 bits or E4M3
  float* scales;                           // [rows][width / group], or [rows]; NULL: `inv` for all
  int64_t x_stride, residual_stride, sum_stride;   // elements from row to row
  int rows, width, group, fp8, dtype;      // group 0: a scale a row
  float eps, inv;
};

hipError_t launch_rms_norm(const RmsNormArgs& a, hipStream_t stream);

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

struct SharedArgs {
  DecodeArgs decode;            // window and sinks 0
  const int32_t* prefix_table;  // pages of the first `prefix` tokens, for all sequences
  int prefix;
};

// How a call behind a shared prefix is divided: the prefix into `splits` parts for each
// tile of 16 rt queries of a key/value head, and equal shares of the sequences' own blocks for
// own_grid workgroups (0: there can be none), in one launch of prefix_grid + own_grid; then
// join_threads threads for each head.
struct SharedPlan {
  int rt, tiles, splits, prefix_grid, own_grid, join_threads;
};

hipError_t launch_shared(const SharedArgs& a, const SharedPlan& plan, hipStream_t stream);

}  // namespace qm
