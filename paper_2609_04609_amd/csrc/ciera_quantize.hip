// Quantisation into the 8-bit format for CDNA4 (gfx950): e4m3 values with a
// power-of-two scale per 128 values. All three forms are bound by memory: a
// value costs its read, one multiply and half a conversion instruction.
#include "ciera_expert.h"
#include "ciera_expert_dev.h"

namespace ciera {

namespace {

// Eight values as e4m3, in two dwords.
template <typename T>
__device__ __forceinline__ u32x2 octet_e4m3(const Octet<T> &o, float inv) {
  u32x2 r;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    r[h] = pack_e4m3(times(o.get(4 * h), inv), times(o.get(4 * h + 1), inv),
                     times(o.get(4 * h + 2), inv), times(o.get(4 * h + 3), inv));
  return r;
}
template <typename T>
__device__ __forceinline__ uint32_t octet_amax(const Octet<T> &o) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t v = finite_abs(o.get(i));
    m = v > m ? v : m;
  }
  return m;
}

// ----------------------------------------------------------------- rows ----
// A wave reads a row of x once and writes it to every row that `position`
// names. 16 lanes hold a block (8 values each), so its maximum is four DPP
// steps.
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantRowsArgs a) {
  const uint32_t lane = threadIdx.x & 63;
  const uint64_t row = uint64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= a.n_rows) return;
  const uint8_t *x =
      static_cast<const uint8_t *>(a.x) + row * a.row_stride * T::kBytes;
  const uint64_t filled = (a.n_cols + 127) & ~uint64_t(127);
  const uint64_t blocks = filled / 128;
  const uint64_t scales = (blocks + 3) & ~uint64_t(3);
  for (uint64_t from = 0; from < filled; from += 512) {
    const uint64_t at = from + lane * 8;
    Octet<T> o;
    if (at + 8 <= a.n_cols)
      o.load(x + at * T::kBytes);
    else
      o.load_some(x + at * T::kBytes,
                  at < a.n_cols ? uint32_t(a.n_cols - at) : 0u);
    const uint32_t byte = scale_byte(row_max_bits(octet_amax(o)));
    const u32x2 q = octet_e4m3(o, inverse_scale(byte));
    const uint64_t block = at / 128;
    for (uint32_t s = 0; s < a.top_k; ++s) {
      uint64_t to = row;
      if (a.position) {
        const int32_t p = a.position[row * a.top_k + s];
        to = p < 0 ? ~uint64_t(0) : uint64_t(p);
      }
      if (to >= a.q_rows) continue;
      if (at < filled) __builtin_memcpy(a.q + to * a.q_stride + at, &q, 8);
      if ((lane & 15) == 0 && block < scales)
        a.scales[to * a.scale_stride + block] =
            uint8_t(block < blocks ? byte : 127u);
    }
  }
}

// --------------------------------------------------------------- blocks ----
// A workgroup takes a 128 x 128 block: 16 lanes a row, 8 values each, 16 rows
// at a time. The transposed bytes go through LDS.
template <typename T>
__global__ void __launch_bounds__(256)
    quantize_blocks_kernel(QuantBlocksArgs a, uint32_t row_blocks,
                           uint32_t col_blocks) {
  __shared__ uint32_t top[4];
  __shared__ uint8_t tile[128][132];
  const uint32_t t = threadIdx.x, lane = t & 63;
  const uint64_t per = uint64_t(row_blocks) * col_blocks;
  const uint64_t batch = blockIdx.x / per, in = blockIdx.x % per;
  const uint32_t rb = uint32_t(in / col_blocks), cb = uint32_t(in % col_blocks);
  const uint32_t r0 = rb * 128 + t / 16, c0 = cb * 128 + (t % 16) * 8;
  const uint8_t *w =
      static_cast<const uint8_t *>(a.w) + batch * a.n_rows * a.n_cols * T::kBytes;
  Octet<T> o[8];
  uint32_t m = 0;
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    const uint64_t r = r0 + 16 * i;
    const uint8_t *p = w + (r * a.n_cols + c0) * T::kBytes;
    if (r < a.n_rows && c0 + 8 <= a.n_cols)
      o[i].load(p);
    else
      o[i].load_some(p, r < a.n_rows && c0 < a.n_cols
                            ? uint32_t(a.n_cols - c0) : 0u);
    const uint32_t v = octet_amax(o[i]);
    m = v > m ? v : m;
  }
  m = row_max_bits(m);
#pragma unroll
  for (int d = 16; d < 64; d <<= 1) {
    const uint32_t v = __shfl_xor(m, d, 64);
    m = v > m ? v : m;
  }
  if (lane == 0) top[t >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) m = top[i] > m ? top[i] : m;
  const uint32_t byte = scale_byte(m);
  const float inv = inverse_scale(byte);
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    const uint64_t r = r0 + 16 * i;
    const u32x2 q = octet_e4m3(o[i], inv);
    if (r < a.n_rows)
      __builtin_memcpy(a.q + (batch * a.n_rows + r) * a.q_stride + c0, &q, 8);
    if (a.q_t) __builtin_memcpy(&tile[t / 16 + 16 * i][(t % 16) * 8], &q, 8);
  }
  if (t < 4) {
    // a scale, and the filling of its row's last dword
    const uint64_t at = batch * row_blocks + rb;
    if (t == 0) a.scales[at * a.scale_stride + cb] = uint8_t(byte);
    else if (cb == col_blocks - 1 && (cb & 3) + t < 4)
      a.scales[at * a.scale_stride + cb + t] = 127;
  }
  if (!a.q_t) return;
  if (t < 4) {
    const uint64_t at = batch * col_blocks + cb;
    if (t == 0) a.scales_t[at * a.scale_t_stride + rb] = uint8_t(byte);
    else if (rb == row_blocks - 1 && (rb & 3) + t < 4)
      a.scales_t[at * a.scale_t_stride + rb + t] = 127;
  }
  __syncthreads();
  // column c of the block is a row of the transpose: 16 bytes a thread
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t c = t / 8 + 32 * i, r = (t % 8) * 16;
    if (cb * 128 + c >= a.n_cols) continue;
    u32x4 q;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      q[k] = uint32_t(tile[r + 4 * k][c]) | uint32_t(tile[r + 4 * k + 1][c]) << 8 |
             uint32_t(tile[r + 4 * k + 2][c]) << 16 |
             uint32_t(tile[r + 4 * k + 3][c]) << 24;
    __builtin_memcpy(a.q_t + (batch * a.n_cols + cb * 128 + c) * a.qt_stride +
                         rb * 128 + r, &q, 16);
  }
}

// -------------------------------------------------------------- columns ----
// A workgroup takes 128 rows of one expert and 128 columns. Block t of the
// columns belongs to the expert that the running sum of rounded-up row counts
// puts it in, which every wave finds for itself.
template <typename T>
__global__ void __launch_bounds__(256)
    quantize_columns_kernel(QuantColumnsArgs a, uint32_t col_tiles) {
  __shared__ uint32_t top[16][128];
  __shared__ uint8_t tile[128][132];
  const uint32_t t = threadIdx.x, lane = t & 63;
  const uint32_t block = blockIdx.x / col_tiles;
  const uint32_t c0 = (blockIdx.x % col_tiles) * 128 + (t % 16) * 8;
  const ExpertTile where = find_tile(a.offsets, a.n_experts,
                                     uint32_t(a.n_rows), block, 7, lane);
  if (where.expert == kNoExpert) return;
  Octet<T> o[8];
  uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    const uint32_t p = where.first + t / 16 + 16 * i;
    uint64_t r = p;
    bool held = p < where.end;
    if (held && a.source) {
      const int32_t pair = a.source[p];
      r = uint32_t(pair) / a.top_k;
      held = pair >= 0;
    }
    held = held && r < a.n_x;
    const uint8_t *x = static_cast<const uint8_t *>(a.x) +
                       (r * a.row_stride + c0) * T::kBytes;
    if (held && c0 + 8 <= a.n_cols)
      o[i].load(x);
    else
      o[i].load_some(x, held && c0 < a.n_cols ? uint32_t(a.n_cols - c0) : 0u);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t v = finite_abs(o[i].get(k));
      m[k] = v > m[k] ? v : m[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) top[t / 16][(t % 16) * 8 + k] = m[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t v = top[r][(t % 16) * 8 + k];
      m[k] = v > m[k] ? v : m[k];
    }
  }
  float inv[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t byte = scale_byte(m[k]);
    inv[k] = inverse_scale(byte);
    if (t < 16 && c0 + k < a.n_cols)
      a.scales[(uint64_t(c0) + k) * a.scale_stride + block] = uint8_t(byte);
  }
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    u32x2 q;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      q[h] = pack_e4m3(times(o[i].get(4 * h), inv[4 * h]),
                       times(o[i].get(4 * h + 1), inv[4 * h + 1]),
                       times(o[i].get(4 * h + 2), inv[4 * h + 2]),
                       times(o[i].get(4 * h + 3), inv[4 * h + 3]));
    __builtin_memcpy(&tile[t / 16 + 16 * i][(t % 16) * 8], &q, 8);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t c = t / 8 + 32 * i, r = (t % 8) * 16;
    const uint64_t col = (blockIdx.x % col_tiles) * 128 + c;
    if (col >= a.n_cols) continue;
    u32x4 q;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      q[k] = uint32_t(tile[r + 4 * k][c]) | uint32_t(tile[r + 4 * k + 1][c]) << 8 |
             uint32_t(tile[r + 4 * k + 2][c]) << 16 |
             uint32_t(tile[r + 4 * k + 3][c]) << 24;
    __builtin_memcpy(a.q_t + col * a.length + uint64_t(block) * 128 + r, &q, 16);
  }
}

template <typename T>
hipError_t rows_typed(const QuantRowsArgs &a, hipStream_t s) {
  quantize_rows_kernel<T>
      <<<dim3(uint32_t((a.n_rows + 3) / 4)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}
template <typename T>
hipError_t blocks_typed(const QuantBlocksArgs &a, hipStream_t s) {
  const uint32_t rb = uint32_t((a.n_rows + 127) / 128);
  const uint32_t cb = uint32_t((a.n_cols + 127) / 128);
  quantize_blocks_kernel<T>
      <<<dim3(uint32_t(a.batch * rb * cb)), dim3(256), 0, s>>>(a, rb, cb);
  return hipGetLastError();
}
template <typename T>
hipError_t columns_typed(const QuantColumnsArgs &a, hipStream_t s) {
  const uint32_t ct = uint32_t((a.n_cols + 127) / 128);
  const uint32_t blocks = uint32_t(
      ciera_columns_length(a.n_rows, a.n_experts) / 128);
  quantize_columns_kernel<T>
      <<<dim3(blocks * ct), dim3(256), 0, s>>>(a, ct);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const QuantRowsArgs &a, hipStream_t s) {
  return a.dtype == CIERA_DT_BF16   ? rows_typed<Bf16>(a, s)
         : a.dtype == CIERA_DT_FP16 ? rows_typed<Fp16>(a, s)
                                    : rows_typed<Fp32>(a, s);
}
hipError_t launch_quantize_blocks(const QuantBlocksArgs &a, hipStream_t s) {
  return a.dtype == CIERA_DT_BF16   ? blocks_typed<Bf16>(a, s)
         : a.dtype == CIERA_DT_FP16 ? blocks_typed<Fp16>(a, s)
                                    : blocks_typed<Fp32>(a, s);
}
hipError_t launch_quantize_columns(const QuantColumnsArgs &a, hipStream_t s) {
  return a.dtype == CIERA_DT_BF16   ? columns_typed<Bf16>(a, s)
         : a.dtype == CIERA_DT_FP16 ? columns_typed<Fp16>(a, s)
                                    : columns_typed<Fp32>(a, s);
}

}  // namespace ciera
