// Internal declarations of the experts' operators (routing, 8-bit
// quantisation, products, combination): argument structs and launchers.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "ciera.h"

namespace ciera {

constexpr uint32_t kBlock8 = 128;  // values that share a scale of the 8-bit format

struct RouteArgs {
  const void *logits;
  uint32_t dtype;
  uint32_t n_tokens;
  uint32_t n_experts;
  uint64_t row_stride;
  const float *bias;
  uint32_t n_groups;
  uint32_t top_groups;
  uint32_t top_k;
  uint32_t flags;
  float scale;
  int32_t *ids;
  float *weights;
};

struct RouteBackArgs {
  const void *logits;
  uint32_t dtype;
  uint32_t n_tokens;
  uint32_t n_experts;
  uint64_t row_stride;
  uint32_t top_k;
  uint32_t flags;
  float scale;
  const int32_t *ids;
  const float *d_weights;
  void *d_logits;
  uint64_t d_row_stride;
};

// Plan: tiles of pairs that a workgroup sorts, and their counts in the workspace:
// one word per expert and tile, expert by expert, then one per expert. Tiles of 1024
// occupy the card with fewer pairs, tiles of 2048 have fewer counts: 32,768 pairs 8.8
// and 9.9 us, 262,168 of 256 experts 11.2 and 12.5, 1,048,576 20.3 and 17.6.
constexpr uint32_t kPlanOne = 2048;  // in one launch
constexpr uint64_t kPlanSmall = uint64_t(1) << 19;  // the most in tiles of 1024
inline uint32_t plan_tile(uint64_t pairs) {
  return pairs <= kPlanOne || pairs > kPlanSmall ? 2048 : 1024;
}
struct PlanArgs {
  const int32_t *ids;
  uint32_t n_pairs;
  uint32_t first_expert;
  uint32_t n_experts;
  int32_t *offsets;
  int32_t *source;
  int32_t *position;
  uint32_t *counts;
};
inline uint64_t plan_tiles(uint64_t pairs) {
  return (pairs + plan_tile(pairs) - 1) / plan_tile(pairs);
}

struct QuantRowsArgs {
  const void *x;
  uint32_t dtype;
  uint64_t n_rows;
  uint64_t n_cols;
  uint64_t row_stride;
  const int32_t *position;
  uint32_t top_k;
  uint64_t q_rows;
  uint8_t *q;
  uint64_t q_stride;
  uint8_t *scales;
  uint64_t scale_stride;
};

struct QuantBlocksArgs {
  const void *w;
  uint32_t dtype;
  uint64_t batch;
  uint64_t n_rows;
  uint64_t n_cols;
  uint8_t *q;
  uint64_t q_stride;
  uint8_t *scales;
  uint64_t scale_stride;
  uint8_t *q_t;
  uint64_t qt_stride;
  uint8_t *scales_t;
  uint64_t scale_t_stride;
};

struct QuantColumnsArgs {
  const void *x;
  uint32_t dtype;
  uint64_t n_x;
  uint64_t n_rows;
  uint64_t n_cols;
  uint64_t row_stride;
  const int32_t *source;
  uint32_t top_k;
  const int32_t *offsets;
  uint32_t n_experts;
  uint8_t *q_t;
  uint64_t length;
  uint8_t *scales;
  uint64_t scale_stride;
};

struct MatmulArgs {
  const uint8_t *a;
  uint64_t a_stride;
  const uint8_t *a_scales;
  uint64_t a_scale_stride;
  uint64_t n_rows;
  const uint8_t *b;
  uint64_t b_stride;
  const uint8_t *b_scales;
  uint64_t b_scale_stride;
  uint32_t n_experts;
  uint64_t n_out;
  uint64_t depth;
  const int32_t *offsets;
  void *out;
  uint32_t out_dtype;
  uint64_t out_stride;
};

struct WeightGradArgs {
  const uint8_t *dy_t;
  const uint8_t *dy_scales;
  uint64_t dy_scale_stride;
  const uint8_t *x_t;
  const uint8_t *x_scales;
  uint64_t x_scale_stride;
  uint64_t length;
  uint32_t n_experts;
  uint64_t n_out;
  uint64_t n_cols;
  const int32_t *offsets;
  void *d_w;
  uint32_t out_dtype;
};

struct CombineArgs {
  const void *rows;
  uint32_t dtype;
  uint64_t n_rows;
  uint64_t n_cols;
  uint64_t row_stride;
  const float *weights;
  const int32_t *position;
  uint64_t n_tokens;
  uint32_t top_k;
  void *out;
  uint64_t out_stride;
};

struct CombineBackArgs {
  const void *d_out;
  uint64_t d_out_stride;
  const void *rows;
  uint32_t dtype;
  uint64_t n_rows;
  uint64_t n_cols;
  uint64_t row_stride;
  const float *weights;
  const int32_t *position;
  uint64_t n_tokens;
  uint32_t top_k;
  void *d_rows;
  uint64_t d_row_stride;
  float *d_weights;
};

hipError_t launch_route(const RouteArgs &a, hipStream_t s);
hipError_t launch_route_backward(const RouteBackArgs &a, hipStream_t s);
hipError_t launch_route_plan(const PlanArgs &a, hipStream_t s);
hipError_t launch_quantize_rows(const QuantRowsArgs &a, hipStream_t s);
hipError_t launch_quantize_blocks(const QuantBlocksArgs &a, hipStream_t s);
hipError_t launch_quantize_columns(const QuantColumnsArgs &a, hipStream_t s);
hipError_t launch_expert_matmul(const MatmulArgs &a, hipStream_t s);
hipError_t launch_weight_grad(const WeightGradArgs &a, hipStream_t s);
hipError_t launch_combine(const CombineArgs &a, hipStream_t s);
hipError_t launch_combine_backward(const CombineBackArgs &a, hipStream_t s);

}  // namespace ciera
