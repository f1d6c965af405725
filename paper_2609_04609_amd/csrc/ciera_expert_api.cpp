// C ABI of the experts' operators: host-side argument checks and launches.
// Declarations and the contract of every entry point are in include/ciera.h.
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "ciera.h"
#include "ciera_expert.h"

namespace {

using namespace ciera;

// On entry, a HIP error that earlier work left pending on this thread is
// cleared, so that a launch's status is the call's own.
struct CallScope {
  CallScope() { (void)hipGetLastError(); }
  CallScope(const CallScope &) = delete;
};

bool aligned(const void *p, uintptr_t a) {
  return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}
uint32_t value_bytes(uint32_t dtype) { return dtype == CIERA_DT_FP32 ? 4 : 2; }
// a wide matrix: its type, pointer and row stride
bool wide_ok(const void *p, uint32_t dtype, uint64_t cols, uint64_t stride) {
  return dtype <= CIERA_DT_FP32 && p && aligned(p, value_bytes(dtype)) &&
         stride >= cols;
}
uint64_t up128(uint64_t n) { return (n + 127) & ~uint64_t(127); }
// an 8-bit matrix with `filled` bytes a row and its scales, one a 128
bool narrow_ok(const void *q, uint64_t stride, const uint8_t *scales,
               uint64_t scale_stride, uint64_t filled) {
  return q && scales && aligned(q, 16) && aligned(scales, 4) &&
         stride % 16 == 0 && stride >= filled && scale_stride % 4 == 0 &&
         scale_stride >= filled / 128;
}
// 32-bit quantities inside the kernels: rows, columns and grid sizes
constexpr uint64_t kMost = uint64_t(1) << 31;
constexpr uint64_t kMostCols = uint64_t(1) << 30;
// a launch has fewer than 2^32 threads: workgroups of 256, and their waves
constexpr uint64_t kMostGroups = uint64_t(1) << 24;
constexpr uint64_t kMostWaves = 4 * kMostGroups;
bool ints_ok(const void *p) { return p && aligned(p, 4); }
// sizes whose tiles one launch does not hold are the launchers' to find
int status(hipError_t e) {
  return e == hipSuccess                      ? CIERA_OK
         : e == hipErrorInvalidConfiguration ? CIERA_EINVAL
                                              : CIERA_EHIP;
}

}  // namespace

extern "C" {

int ciera_route(const void *logits, uint32_t dtype, uint64_t n_tokens,
                uint32_t n_experts, uint64_t row_stride, const float *bias,
                uint32_t n_groups, uint32_t top_groups, uint32_t top_k,
                uint32_t flags, float scale, int32_t *expert_ids,
                float *weights, hipStream_t stream) {
  CallScope scope;
  if (flags & ~(CIERA_ROUTE_SIGMOID | CIERA_ROUTE_NORMALIZE |
                CIERA_ROUTE_GROUP_TOP_TWO))
    return CIERA_EINVAL;
  if (n_experts == 0 || n_experts > CIERA_MAX_EXPERTS || n_groups == 0 ||
      n_groups > CIERA_MAX_GROUPS || n_experts % n_groups != 0 ||
      top_groups == 0 || top_groups > n_groups || top_k == 0 ||
      top_k > CIERA_MAX_TOP_K || top_k > n_experts / n_groups * top_groups)
    return CIERA_EINVAL;
  if (dtype > CIERA_DT_FP32 || n_tokens >= kMostWaves ||
      n_tokens * top_k >= kMost)
    return CIERA_EINVAL;
  if (n_tokens == 0) return CIERA_OK;
  if (!wide_ok(logits, dtype, n_experts, row_stride) || !aligned(bias, 4) ||
      !ints_ok(expert_ids) || !ints_ok(weights))
    return CIERA_EINVAL;
  const RouteArgs a{logits,     dtype,    uint32_t(n_tokens), n_experts,
                    row_stride, bias,     n_groups,           top_groups,
                    top_k,      flags,    scale,              expert_ids,
                    weights};
  return status(launch_route(a, stream));
}

int ciera_route_backward(const void *logits, uint32_t dtype,
                         uint64_t n_tokens, uint32_t n_experts,
                         uint64_t row_stride, uint32_t top_k, uint32_t flags,
                         float scale, const int32_t *expert_ids,
                         const float *d_weights, void *d_logits,
                         uint64_t d_row_stride, hipStream_t stream) {
  CallScope scope;
  if (flags & ~(CIERA_ROUTE_SIGMOID | CIERA_ROUTE_NORMALIZE))
    return CIERA_EINVAL;
  if (n_experts == 0 || n_experts > CIERA_MAX_EXPERTS || top_k == 0 ||
      top_k > CIERA_MAX_TOP_K || dtype > CIERA_DT_FP32 ||
      n_tokens >= kMostWaves || n_tokens * top_k >= kMost)
    return CIERA_EINVAL;
  if (n_tokens == 0) return CIERA_OK;
  if (!wide_ok(logits, dtype, n_experts, row_stride) ||
      !wide_ok(d_logits, dtype, n_experts, d_row_stride) ||
      !ints_ok(expert_ids) || !ints_ok(d_weights))
    return CIERA_EINVAL;
  const RouteBackArgs a{logits, dtype,      uint32_t(n_tokens), n_experts,
                        row_stride, top_k,  flags,              scale,
                        expert_ids, d_weights, d_logits,        d_row_stride};
  return status(launch_route_backward(a, stream));
}

uint64_t ciera_plan_workspace_bytes(uint64_t n_tokens, uint32_t top_k,
                                    uint32_t n_experts) {
  if (n_experts == 0 || n_experts > CIERA_MAX_EXPERTS || top_k == 0 ||
      top_k > CIERA_MAX_TOP_K || n_tokens >= kMost || n_tokens * top_k >= kMost)
    return 0;
  // enough for fewer pairs too, which smaller tiles may take
  uint64_t tiles = plan_tiles(n_tokens * top_k);
  if (n_tokens * top_k > kPlanSmall && tiles < plan_tiles(kPlanSmall))
    tiles = plan_tiles(kPlanSmall);
  return ((tiles + 1) * n_experts * 4 + 255) & ~uint64_t(255);
}

int ciera_route_plan(const int32_t *expert_ids, uint64_t n_tokens,
                     uint32_t top_k, uint32_t first_expert,
                     uint32_t n_experts, int32_t *offsets, int32_t *source,
                     int32_t *position, void *workspace,
                     uint64_t workspace_bytes, hipStream_t stream) {
  CallScope scope;
  const uint64_t need = ciera_plan_workspace_bytes(n_tokens, top_k, n_experts);
  // the last expert is an int32 too: differences of negative ids stay outside
  if (need == 0 || first_expert > kMost - n_experts || !ints_ok(offsets))
    return CIERA_EINVAL;
  if (n_tokens > 0 && (!ints_ok(expert_ids) || !ints_ok(source) ||
                       !ints_ok(position) || !ints_ok(workspace)))
    return CIERA_EINVAL;
  if (n_tokens > 0 && workspace_bytes < need) return CIERA_ENOSPC;
  const PlanArgs a{expert_ids, uint32_t(n_tokens * top_k),
                   first_expert, n_experts, offsets, source, position,
                   static_cast<uint32_t *>(workspace)};
  return status(launch_route_plan(a, stream));
}

int ciera_quantize_rows(const void *x, uint32_t dtype, uint64_t n_rows,
                        uint64_t n_cols, uint64_t row_stride,
                        const int32_t *position, uint32_t top_k,
                        uint64_t q_rows, void *q, uint64_t q_stride,
                        uint8_t *scales, uint64_t scale_stride,
                        hipStream_t stream) {
  CallScope scope;
  if (dtype > CIERA_DT_FP32 || n_rows >= kMostWaves || n_cols >= kMostCols ||
      q_rows >= kMost || top_k == 0 || top_k > CIERA_MAX_TOP_K ||
      (!position && (top_k != 1 || q_rows < n_rows)))
    return CIERA_EINVAL;
  if (n_rows == 0 || n_cols == 0 || q_rows == 0) return CIERA_OK;
  if (!wide_ok(x, dtype, n_cols, row_stride) || !aligned(position, 4) ||
      !narrow_ok(q, q_stride, scales, scale_stride, up128(n_cols)))
    return CIERA_EINVAL;
  const QuantRowsArgs a{x,      dtype,    n_rows,
                        n_cols, row_stride, position,
                        top_k,  q_rows,   static_cast<uint8_t *>(q),
                        q_stride, scales, scale_stride};
  return status(launch_quantize_rows(a, stream));
}

int ciera_quantize_blocks(const void *w, uint32_t dtype, uint64_t batch,
                          uint64_t n_rows, uint64_t n_cols, void *q,
                          uint64_t q_stride, uint8_t *scales,
                          uint64_t scale_stride, void *q_t,
                          uint64_t qt_stride, uint8_t *scales_t,
                          uint64_t scale_t_stride, hipStream_t stream) {
  CallScope scope;
  if (dtype > CIERA_DT_FP32 || n_rows >= kMostCols || n_cols >= kMostCols ||
      batch >= kMost || (!q_t) != (!scales_t))
    return CIERA_EINVAL;
  if (batch == 0 || n_rows == 0 || n_cols == 0) return CIERA_OK;
  const uint64_t rb = (n_rows + 127) / 128, cb = (n_cols + 127) / 128;
  if (rb * cb >= kMostGroups || batch * rb * cb >= kMostGroups) return CIERA_EINVAL;
  if (!wide_ok(w, dtype, n_cols, n_cols) ||
      !narrow_ok(q, q_stride, scales, scale_stride, up128(n_cols)) ||
      (q_t &&
       !narrow_ok(q_t, qt_stride, scales_t, scale_t_stride, up128(n_rows))))
    return CIERA_EINVAL;
  const QuantBlocksArgs a{w, dtype, batch, n_rows, n_cols,
                          static_cast<uint8_t *>(q), q_stride, scales,
                          scale_stride, static_cast<uint8_t *>(q_t), qt_stride,
                          scales_t, scale_t_stride};
  return status(launch_quantize_blocks(a, stream));
}

uint64_t ciera_columns_length(uint64_t n_rows, uint32_t n_experts) {
  const uint64_t some = n_rows < n_experts ? n_rows : n_experts;
  return (n_rows + 127 * some) / 128 * 128;
}

int ciera_quantize_columns(const void *x, uint32_t dtype, uint64_t n_x,
                           uint64_t n_rows, uint64_t n_cols,
                           uint64_t row_stride, const int32_t *source,
                           uint32_t top_k, const int32_t *offsets,
                           uint32_t n_experts, void *q_t, uint64_t length,
                           uint8_t *scales, uint64_t scale_stride,
                           hipStream_t stream) {
  CallScope scope;
  if (dtype > CIERA_DT_FP32 || n_x >= kMost || n_rows >= kMost ||
      n_cols >= kMostCols || n_experts == 0 || n_experts > CIERA_MAX_EXPERTS ||
      top_k == 0 || top_k > CIERA_MAX_TOP_K || (!source && n_x != n_rows) ||
      length % 128 != 0 || length >= kMost)
    return CIERA_EINVAL;
  const uint64_t need = ciera_columns_length(n_rows, n_experts);
  if (length < need) return CIERA_ENOSPC;
  if (n_rows == 0 || n_cols == 0) return CIERA_OK;
  if (need / 128 * ((n_cols + 127) / 128) >= kMostGroups) return CIERA_EINVAL;
  if (!wide_ok(x, dtype, n_cols, row_stride) || !aligned(source, 4) ||
      !ints_ok(offsets) || !narrow_ok(q_t, length, scales, scale_stride, length))
    return CIERA_EINVAL;
  const QuantColumnsArgs a{x,       dtype,     n_x,
                           n_rows,  n_cols,    row_stride,
                           source,  top_k,     offsets,
                           n_experts, static_cast<uint8_t *>(q_t), length,
                           scales,  scale_stride};
  return status(launch_quantize_columns(a, stream));
}

int ciera_expert_matmul(const void *a, uint64_t a_stride,
                        const uint8_t *a_scales, uint64_t a_scale_stride,
                        uint64_t n_rows, const void *b, uint64_t b_stride,
                        const uint8_t *b_scales, uint64_t b_scale_stride,
                        uint32_t n_experts, uint64_t n_out, uint64_t depth,
                        const int32_t *offsets, void *out,
                        uint32_t out_dtype, uint64_t out_stride,
                        hipStream_t stream) {
  CallScope scope;
  if (out_dtype > CIERA_DT_FP32 || n_rows >= kMost || n_out >= kMostCols ||
      n_experts == 0 || n_experts > CIERA_MAX_EXPERTS || depth == 0 ||
      depth % 128 != 0 || depth > (uint64_t(1) << 23) ||
      (!offsets && n_experts != 1))
    return CIERA_EINVAL;
  if (n_rows == 0 || n_out == 0) return CIERA_OK;
  // tiles of 128 x 128, before they are paired
  if (((n_rows + 127) / 128 + n_experts) * ((n_out + 127) / 128) >= kMostGroups)
    return CIERA_EINVAL;
  if (!narrow_ok(a, a_stride, a_scales, a_scale_stride, depth) ||
      !narrow_ok(b, b_stride, b_scales, b_scale_stride, depth) ||
      !wide_ok(out, out_dtype, n_out, out_stride) || !aligned(offsets, 4))
    return CIERA_EINVAL;
  const MatmulArgs m{static_cast<const uint8_t *>(a), a_stride, a_scales,
                     a_scale_stride, n_rows, static_cast<const uint8_t *>(b),
                     b_stride, b_scales, b_scale_stride, n_experts, n_out,
                     depth, offsets, out, out_dtype, out_stride};
  return status(launch_expert_matmul(m, stream));
}

int ciera_expert_weight_grad(const void *dy_t, const uint8_t *dy_scales,
                             uint64_t dy_scale_stride, const void *x_t,
                             const uint8_t *x_scales,
                             uint64_t x_scale_stride, uint64_t length,
                             uint32_t n_experts, uint64_t n_out,
                             uint64_t n_cols, const int32_t *offsets,
                             void *d_w, uint32_t out_dtype,
                             hipStream_t stream) {
  CallScope scope;
  if (out_dtype > CIERA_DT_FP32 || n_out >= kMostCols ||
      n_cols >= kMostCols || n_experts == 0 || n_experts > CIERA_MAX_EXPERTS ||
      length % 128 != 0 || length >= kMost)
    return CIERA_EINVAL;
  if (n_out == 0 || n_cols == 0) return CIERA_OK;
  if ((n_out + 127) / 128 * ((n_cols + 127) / 128) >= kMostGroups / n_experts)
    return CIERA_EINVAL;
  // without columns nothing is read from the operands, which may be null
  if (length > 0 &&
      (!narrow_ok(dy_t, length, dy_scales, dy_scale_stride, length) ||
       !narrow_ok(x_t, length, x_scales, x_scale_stride, length)))
    return CIERA_EINVAL;
  if (!wide_ok(d_w, out_dtype, n_cols, n_cols) || !ints_ok(offsets))
    return CIERA_EINVAL;
  const WeightGradArgs a{static_cast<const uint8_t *>(dy_t), dy_scales,
                         dy_scale_stride, static_cast<const uint8_t *>(x_t),
                         x_scales, x_scale_stride, length, n_experts,
                         n_out, n_cols, offsets, d_w, out_dtype};
  return status(launch_weight_grad(a, stream));
}

int ciera_combine(const void *rows, uint32_t dtype, uint64_t n_rows,
                  uint64_t n_cols, uint64_t row_stride, const float *weights,
                  const int32_t *position, uint64_t n_tokens, uint32_t top_k,
                  void *out, uint64_t out_stride, hipStream_t stream) {
  CallScope scope;
  if (dtype > CIERA_DT_FP32 || n_rows >= kMost || n_cols >= kMostCols ||
      top_k == 0 || top_k > CIERA_MAX_TOP_K || n_tokens >= kMost ||
      n_tokens * top_k >= kMost)
    return CIERA_EINVAL;
  if (n_tokens == 0 || n_cols == 0) return CIERA_OK;
  if (n_tokens * ((n_cols + 511) / 512) >= kMostWaves) return CIERA_EINVAL;
  if ((n_rows > 0 && !wide_ok(rows, dtype, n_cols, row_stride)) ||
      !wide_ok(out, dtype, n_cols, out_stride) || !aligned(weights, 4) ||
      !ints_ok(position))
    return CIERA_EINVAL;
  const CombineArgs a{rows,    dtype,    n_rows,   n_cols, row_stride, weights,
                      position, n_tokens, top_k,   out,    out_stride};
  return status(launch_combine(a, stream));
}

int ciera_combine_backward(const void *d_out, uint64_t d_out_stride,
                           const void *rows, uint32_t dtype, uint64_t n_rows,
                           uint64_t n_cols, uint64_t row_stride,
                           const float *weights, const int32_t *position,
                           uint64_t n_tokens, uint32_t top_k, void *d_rows,
                           uint64_t d_row_stride, float *d_weights,
                           hipStream_t stream) {
  CallScope scope;
  if (dtype > CIERA_DT_FP32 || n_rows >= kMost || n_cols >= kMostCols ||
      top_k == 0 || top_k > CIERA_MAX_TOP_K || n_tokens >= kMost ||
      n_tokens * top_k >= kMostWaves)
    return CIERA_EINVAL;
  if (n_tokens == 0) return CIERA_OK;
  if (!ints_ok(weights) || !ints_ok(position) || !ints_ok(d_weights))
    return CIERA_EINVAL;
  if (n_cols > 0 &&
      (!wide_ok(d_out, dtype, n_cols, d_out_stride) ||
       (n_rows > 0 && (!wide_ok(rows, dtype, n_cols, row_stride) ||
                       !wide_ok(d_rows, dtype, n_cols, d_row_stride)))))
    return CIERA_EINVAL;
  const CombineBackArgs a{d_out,   d_out_stride, rows,     dtype,
                          n_rows,  n_cols,       row_stride, weights,
                          position, n_tokens,    top_k,    d_rows,
                          d_row_stride, d_weights};
  return status(launch_combine_backward(a, stream));
}

}  // extern "C"
