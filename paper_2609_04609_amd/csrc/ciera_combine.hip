// Combination of a token's expert rows and its gradients for CDNA4 (gfx950).
// Both are bound by memory: a row's value costs its read (and write) and one
// fp32 multiply-add.
#include "ciera_expert.h"
#include "ciera_expert_dev.h"

namespace ciera {

namespace {

template <typename T>
__device__ __forceinline__ void load_octet(Octet<T> &o, const uint8_t *row,
                                           uint64_t at, uint64_t n) {
  if (at + 8 <= n)
    o.load(row + at * T::kBytes);
  else
    o.load_some(row + at * T::kBytes, at < n ? uint32_t(n - at) : 0u);
}
template <typename T>
__device__ __forceinline__ void store_octet(const Octet<T> &o, uint8_t *row,
                                            uint64_t at, uint64_t n) {
  if (at + 8 <= n)
    o.store(row + at * T::kBytes);
  else if (at < n)
    o.store_some(row + at * T::kBytes, uint32_t(n - at));
}

// A wave takes 512 columns of a token, 8 a lane.
template <typename T>
__global__ void __launch_bounds__(256)
    combine_kernel(CombineArgs a, uint32_t chunks) {
  const uint32_t lane = threadIdx.x & 63;
  const uint64_t unit = uint64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const uint64_t token = unit / chunks;
  if (token >= a.n_tokens) return;
  const uint64_t at = (unit % chunks) * 512 + lane * 8;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  // four slots' rows are asked for before the first is used: 16384 tokens of 8 rows of
  // 2048 bf16 values 118 us (5.1 TB/s), 128 one by one
  for (uint32_t from = 0; from < a.top_k; from += 4) {
    const uint8_t *row[4];
    float w[4];
    bool held[4];
    Octet<T> o[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      const bool slot = from + j < a.top_k;
      const uint64_t pair = token * a.top_k + (slot ? from + j : from);
      const int32_t p = a.position[pair];
      held[j] = slot && p >= 0 && uint64_t(p) < a.n_rows;
      w[j] = !slot ? 0.0f : a.weights ? a.weights[pair] : 1.0f;
      row[j] = static_cast<const uint8_t *>(a.rows) +
               (held[j] ? uint64_t(p) : 0) * a.row_stride * T::kBytes;
      o[j].clear();
    }
    if (at + 8 <= a.n_cols) {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        if (held[j]) o[j].load(row[j] + at * T::kBytes);
    } else if (at < a.n_cols) {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        if (held[j])
          o[j].load_some(row[j] + at * T::kBytes, uint32_t(a.n_cols - at));
    }
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      if (held[j]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += w[j] * o[j].get(i);
      } else if (w[j] != w[j]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = w[j];
      }
    }
  }
  Octet<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.set(i, sum[i]);
  store_octet(r, static_cast<uint8_t *>(a.out) +
                     token * a.out_stride * T::kBytes, at, a.n_cols);
}

// A wave takes a (token, slot): it writes the row's gradient and adds up its
// product with the row. The slots of a token are neighbours and share its
// gradient in the cache.
template <typename T>
__global__ void __launch_bounds__(256)
    combine_backward_kernel(CombineBackArgs a) {
  const uint32_t lane = threadIdx.x & 63;
  const uint64_t pair = uint64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (pair >= a.n_tokens * a.top_k) return;
  const uint64_t token = pair / a.top_k;
  const int32_t p = a.position[pair];
  if (p < 0 || uint64_t(p) >= a.n_rows) {
    if (lane == 0) a.d_weights[pair] = 0.0f;
    return;
  }
  const float w = a.weights[pair];
  const uint8_t *g = static_cast<const uint8_t *>(a.d_out) +
                     token * a.d_out_stride * T::kBytes;
  const uint8_t *row = static_cast<const uint8_t *>(a.rows) +
                       uint64_t(p) * a.row_stride * T::kBytes;
  uint8_t *d_row = static_cast<uint8_t *>(a.d_rows) +
                   uint64_t(p) * a.d_row_stride * T::kBytes;
  float dot = 0;
  for (uint64_t from = 0; from < a.n_cols; from += 512) {
    const uint64_t at = from + lane * 8;
    Octet<T> go, ro, d;
    load_octet(go, g, at, a.n_cols);
    load_octet(ro, row, at, a.n_cols);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dot += go.get(i) * ro.get(i);
      d.set(i, w * go.get(i));
    }
    store_octet(d, d_row, at, a.n_cols);
  }
  dot = wave_sum(dot);
  if (lane == 0) a.d_weights[pair] = dot;
}

template <typename T>
hipError_t combine_typed(const CombineArgs &a, hipStream_t s) {
  const uint32_t chunks = uint32_t((a.n_cols + 511) / 512);
  combine_kernel<T><<<dim3(uint32_t((a.n_tokens * chunks + 3) / 4)), dim3(256),
                      0, s>>>(a, chunks);
  return hipGetLastError();
}
template <typename T>
hipError_t combine_back_typed(const CombineBackArgs &a, hipStream_t s) {
  combine_backward_kernel<T>
      <<<dim3(uint32_t((a.n_tokens * a.top_k + 3) / 4)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_combine(const CombineArgs &a, hipStream_t s) {
  return a.dtype == CIERA_DT_BF16   ? combine_typed<Bf16>(a, s)
         : a.dtype == CIERA_DT_FP16 ? combine_typed<Fp16>(a, s)
                                    : combine_typed<Fp32>(a, s);
}
hipError_t launch_combine_backward(const CombineBackArgs &a, hipStream_t s) {
  return a.dtype == CIERA_DT_BF16   ? combine_back_typed<Bf16>(a, s)
         : a.dtype == CIERA_DT_FP16 ? combine_back_typed<Fp16>(a, s)
                                    : combine_back_typed<Fp32>(a, s);
}

}  // namespace ciera
