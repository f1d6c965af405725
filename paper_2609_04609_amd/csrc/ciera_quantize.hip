// Quantisation into the 8-bit format for CDNA4 (gfx950): e4m3 values with a
// power-of-two scale per 128 values. All three forms are bound by memory: a value
// costs its read, half an instruction for the maximum and half a conversion, which
// scales too. 16384 tokens of 2048 bf16 values to 8 rows each: 69 us for 340 MB; a
// layer of 64 x 1024 x 2048 both ways round: 102 us for 540 MB; 40024 rows gathered
// from 5003 tokens, by columns: 26 us for 82 MB written and 164 MB read, of which 51 MB
// from memory (counted; tokens are 20 MB, met by several XCDs) and the rest from the L2s.
#include <type_traits>

#include "ciera_expert.h"
#include "ciera_expert_dev.h"

namespace ciera {

namespace {

// The bits of |x|, 16-bit types by pairs: largest values and the values that are not
// finite, which lie at kInfinite and above, are found on the bits themselves, two
// values an instruction. Only a wave that meets one that is not finite takes them one
// by one.
template <typename T>
struct Magnitude {
  static constexpr uint32_t kWords = T::kBytes * 2;  // of eight values
  static constexpr uint32_t kInfinite =
      T::kBytes == 4 ? 0x7F800000u : std::is_same_v<T, Bf16> ? 0x7F80u : 0x7C00u;
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    if constexpr (T::kBytes == 4) return a > b ? a : b;
    else {
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      return __builtin_bit_cast(
          uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                              __builtin_bit_cast(u16x2, b)));
    }
  }
  // word i of an octet, without signs
  static __device__ __forceinline__ uint32_t word(const Octet<T> &o, uint32_t i) {
    return o.w[i / 4][i % 4] & (T::kBytes == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu);
  }
  static __device__ __forceinline__ uint32_t finite(uint32_t w) {
    if constexpr (T::kBytes == 4) return w < kInfinite ? w : 0u;
    else
      return ((w & 0xFFFFu) < kInfinite ? w & 0xFFFFu : 0u) |
             (w >> 16 < kInfinite ? w & 0xFFFF0000u : 0u);
  }
  static __device__ __forceinline__ bool infinite(uint32_t w) {
    if constexpr (T::kBytes == 4) return w >= kInfinite;
    else
      return w >= kInfinite << 16 || (w & 0xFFFFu) >= kInfinite;
  }
  // NaN for infinities
  static __device__ __forceinline__ void without_infinities(Octet<T> &o) {
#pragma unroll
    for (uint32_t i = 0; i < kWords; ++i) {
      const uint32_t w = o.w[i / 4][i % 4];
      o.w[i / 4][i % 4] =
          T::kBytes == 4
              ? ((w & 0x7FFFFFFFu) < kInfinite ? w : 0x7FFFFFFFu)
              : ((w & 0x7FFFu) < kInfinite ? w & 0xFFFFu : 0x7FFFu) |
                    ((w >> 16 & 0x7FFFu) < kInfinite ? w & 0xFFFF0000u
                                                     : 0x7FFF0000u);
    }
  }
  // the bits of the fp32 value of half h of a word (fp32: of the word)
  static __device__ __forceinline__ uint32_t wide(uint32_t w, uint32_t h) {
    if constexpr (T::kBytes == 4) return w;
    else
      return __float_as_uint(T::to_float(h ? w >> 16 : w & 0xFFFFu));
  }
  // the larger half of a word
  static __device__ __forceinline__ uint32_t one(uint32_t w) {
    if constexpr (T::kBytes == 4) return w;
    else
      return (w >> 16) > (w & 0xFFFFu) ? w >> 16 : w & 0xFFFFu;
  }
};

// Two values, the halves of a word or `x` and `y`, divided by the scale 2^e (its
// exponent alone is read) and rounded to nearest even, as two e4m3 bytes in the
// upper (HIGH) or lower half of `old`, in one instruction. Values are within 448
// scales, or NaN.
typedef short s16x2 __attribute__((ext_vector_type(2)));
template <typename T, bool HIGH>
__device__ __forceinline__ uint32_t pack_word(uint32_t w, float scale,
                                              uint32_t old) {
  const s16x2 o = __builtin_bit_cast(s16x2, old);
  s16x2 r;
  if constexpr (std::is_same_v<T, Bf16>) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
        o, __builtin_bit_cast(bf16x2, w), scale, HIGH);
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(
        o, __builtin_bit_cast(f16x2, w), scale, HIGH);
  }
  return __builtin_bit_cast(uint32_t, r);
}
template <bool HIGH>
__device__ __forceinline__ uint32_t pack_two(float x, float y, float scale,
                                             uint32_t old) {
  return __builtin_bit_cast(
      uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(
                    __builtin_bit_cast(s16x2, old), x, y, scale, HIGH));
}
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte << 23);
}
// an octet's eight bytes
template <typename T>
__device__ __forceinline__ u32x2 pack_row(const Octet<T> &o, float scale) {
  u32x2 r;
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h) {
    if constexpr (T::kBytes == 4)
      r[h] = pack_two<true>(
          o.get(4 * h + 2), o.get(4 * h + 3), scale,
          pack_two<false>(o.get(4 * h), o.get(4 * h + 1), scale, 0));
    else
      r[h] = pack_word<T, true>(o.w[0][2 * h + 1], scale,
                                pack_word<T, false>(o.w[0][2 * h], scale, 0));
  }
  return r;
}
// value k of two rows, side by side
template <bool HIGH, typename T>
__device__ __forceinline__ uint32_t pack_pair(const Octet<T> &a,
                                              const Octet<T> &b, uint32_t k,
                                              float scale, uint32_t old) {
  if constexpr (T::kBytes == 4)
    return pack_two<HIGH>(a.get(k), b.get(k), scale, old);
  else
    return pack_word<T, HIGH>(
        __builtin_amdgcn_perm(b.w[0][k / 2], a.w[0][k / 2],
                              k % 2 ? 0x07060302u : 0x05040100u),
        scale, old);
}
// value k of eight rows
template <typename T>
__device__ __forceinline__ u32x2 pack_column(const Octet<T> (&o)[8], uint32_t k,
                                             float scale) {
  u32x2 r;
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h)
    r[h] = pack_pair<true>(
        o[4 * h + 2], o[4 * h + 3], k, scale,
        pack_pair<false>(o[4 * h], o[4 * h + 1], k, scale, 0));
  return r;
}
// Largest finite |x| of N octets of this lane, as one value's bits; infinities of a
// wave that has values that are not finite become NaN.
template <typename T, int N>
__device__ __forceinline__ uint32_t octets_amax(Octet<T> (&o)[N]) {
  using M = Magnitude<T>;
  uint32_t m = 0;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (uint32_t i = 0; i < M::kWords; ++i) m = M::larger(m, M::word(o[n], i));
  if (__ballot(M::infinite(m)) != 0) {
    m = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (uint32_t i = 0; i < M::kWords; ++i)
        m = M::larger(m, M::finite(M::word(o[n], i)));
      M::without_infinities(o[n]);
    }
  }
  return M::wide(M::one(m), 0);
}

// ----------------------------------------------------------------- rows ----
// A wave reads a row of x once and writes it to every row that `position`
// names: 1024 columns at a time, 16 a lane, so that every store is 16 bytes a lane.
// Eight lanes hold a block; its maximum is three DPP steps.
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantRowsArgs a) {
  const uint32_t lane = threadIdx.x & 63;
  const uint64_t row = uint64_t(blockIdx.x) * 4 +
                       __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.n_rows) return;
  const uint8_t *x =
      static_cast<const uint8_t *>(a.x) + row * a.row_stride * T::kBytes;
  const uint64_t filled = (a.n_cols + 127) & ~uint64_t(127);
  const uint64_t scale_bytes = (filled / 128 + 3) & ~uint64_t(3);
  // lane s: the row of slot s
  int32_t named = -1;
  if (!a.position)
    named = int32_t(row);
  else if (lane < a.top_k)
    named = a.position[row * a.top_k + lane];
  for (uint64_t from = 0; from < filled; from += 1024) {
    const uint64_t at = from + lane * 16;
    Octet<T> o[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t c = at + 8 * h;
      if (c + 8 <= a.n_cols)
        o[h].load(x + c * T::kBytes);
      else
        o[h].load_some(x + c * T::kBytes,
                       c < a.n_cols ? uint32_t(a.n_cols - c) : 0u);
    }
    const uint32_t byte = scale_byte(eight_max(octets_amax(o)));
    const float scale = scale_of(byte);
    const u32x2 lo = pack_row(o[0], scale), hi = pack_row(o[1], scale);
    const u32x4 q = {lo[0], lo[1], hi[0], hi[1]};
    // the scales of the eight blocks, those past the row's end 127
    uint32_t s[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t b = __builtin_amdgcn_readlane(byte, 8 * k);
      s[k / 4] |= (from + 128 * k < filled ? b : 127u) << (8 * (k % 4));
    }
    const bool two = from / 128 + 8 <= scale_bytes;
    for (uint32_t k = 0; k < a.top_k; ++k) {
      const int32_t to = __builtin_amdgcn_readlane(named, int(k));
      if (to < 0 || uint64_t(to) >= a.q_rows) continue;
      if (at < filled)
        *reinterpret_cast<u32x4 *>(a.q + uint64_t(to) * a.q_stride + at) = q;
      if (lane < (two ? 2u : 1u))
        *reinterpret_cast<uint32_t *>(a.scales + uint64_t(to) * a.scale_stride +
                                      from / 128 + 4 * lane) =
            lane == 0 ? s[0] : s[1];
    }
  }
}

// --------------------------------------------------------------- blocks ----
// 128 columns' pieces of eight rows each, column c's piece of rows 8 g on at place
// g ^ (c / 8 % 16): a thread writes eight columns of one g, and 8 threads read a
// column's 128 bytes.
struct Columns {
  u32x2 tile[128][16];
  __device__ __forceinline__ void put(uint32_t c, uint32_t g, u32x2 v) {
    tile[c][g ^ (c / 8)] = v;
  }
  // rows 16 i to 16 i + 15 of column c
  __device__ __forceinline__ u32x4 get(uint32_t c, uint32_t i) const {
    const u32x2 lo = tile[c][(2 * i) ^ (c / 8)], hi = tile[c][(2 * i + 1) ^ (c / 8)];
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
};

// A workgroup takes a 128 x 128 block, a thread 8 x 8 values of it: 16 lanes read
// 256 bytes (16-bit types) of a row.
template <typename T>
__global__ void __launch_bounds__(256)
    quantize_blocks_kernel(QuantBlocksArgs a, uint32_t row_blocks,
                           uint32_t col_blocks) {
  __shared__ uint32_t top[4];
  __shared__ Columns columns;
  const uint32_t t = threadIdx.x, lane = t & 63;
  const uint64_t per = uint64_t(row_blocks) * col_blocks;
  const uint64_t batch = blockIdx.x / per, in = blockIdx.x % per;
  const uint32_t rb = uint32_t(in / col_blocks), cb = uint32_t(in % col_blocks);
  const uint32_t r0 = rb * 128 + t / 16 * 8, c0 = cb * 128 + (t % 16) * 8;
  const uint8_t *w =
      static_cast<const uint8_t *>(a.w) + batch * a.n_rows * a.n_cols * T::kBytes;
  Octet<T> o[8];
  if (rb * 128 + 128 <= a.n_rows && cb * 128 + 128 <= a.n_cols) {
    // without a branch between them, so that all are in flight at once
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      o[i].load(w + (uint64_t(r0 + i) * a.n_cols + c0) * T::kBytes);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const uint64_t r = r0 + i;
      const uint8_t *p = w + (r * a.n_cols + c0) * T::kBytes;
      if (r < a.n_rows && c0 + 8 <= a.n_cols)
        o[i].load(p);
      else
        o[i].load_some(p, r < a.n_rows && c0 < a.n_cols
                              ? uint32_t(a.n_cols - c0) : 0u);
    }
  }
  uint32_t m = row_max(octets_amax(o));
#pragma unroll
  for (int d = 16; d < 64; d <<= 1) m = larger(m, uint32_t(__shfl_xor(m, d, 64)));
  if (lane == 0) top[t >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) m = larger(m, top[i]);
  const uint32_t byte = scale_byte(m);
  const float scale = scale_of(byte);
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    const uint64_t r = r0 + i;
    const u32x2 q = pack_row(o[i], scale);
    if (r < a.n_rows)
      __builtin_memcpy(a.q + (batch * a.n_rows + r) * a.q_stride + c0, &q, 8);
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
#pragma unroll
  for (uint32_t k = 0; k < 8; ++k)
    columns.put((t % 16) * 8 + k, t / 16, pack_column(o, k, scale));
  __syncthreads();
  // column c of the block is a row of the transpose: 16 bytes a thread
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t c = t / 8 + 32 * i;
    if (cb * 128 + c >= a.n_cols) continue;
    const u32x4 q = columns.get(c, t % 8);
    __builtin_memcpy(a.q_t + (batch * a.n_cols + cb * 128 + c) * a.qt_stride +
                         rb * 128 + (t % 8) * 16, &q, 16);
  }
}

// -------------------------------------------------------------- columns ----
// A workgroup takes 128 rows of one expert and 128 columns, a thread 8 x 8 of
// them, which the conversion takes by pairs of rows; LDS puts the columns' pieces of
// eight bytes together. Block t of the columns belongs to the expert that the running sum
// of rounded-up row counts puts it in, which every wave finds for itself.
template <typename T>
__global__ void __launch_bounds__(256)
    quantize_columns_kernel(QuantColumnsArgs a, uint32_t col_tiles) {
  __shared__ uint32_t top[4][128];
  __shared__ float scales[128];
  __shared__ uint32_t row_of[128];
  __shared__ Columns columns;
  const uint32_t t = threadIdx.x, lane = t & 63;
  const uint32_t block = blockIdx.x / col_tiles;
  const uint32_t tile_col = (blockIdx.x % col_tiles) * 128;
  const uint32_t c0 = tile_col + (t % 16) * 8;
  const ExpertTile where = find_tile(a.offsets, a.n_experts,
                                     uint32_t(a.n_rows), block, 7, lane);
  if (where.expert == kNoExpert) return;
  // the rows' places in x, once for all columns; none: zeros
  constexpr uint32_t kNone = ~0u;
  if (t < 128) {
    const uint32_t p = where.first + t;
    uint32_t r = p < where.end ? p : kNone;
    if (r != kNone && a.source) {
      const int32_t pair = a.source[p];
      r = pair < 0 ? kNone : uint32_t(pair) / a.top_k;
    }
    row_of[t] = r < a.n_x ? r : kNone;
  }
  __syncthreads();
  Octet<T> o[8];
  const uint8_t *const x = static_cast<const uint8_t *>(a.x);
  if (tile_col + 128 <= a.n_cols && a.n_x > 0) {
    // without a branch between them, so that all are in flight at once
    uint32_t r[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      r[i] = row_of[t / 16 * 8 + i];
      o[i].load(x + (uint64_t(r[i] == kNone ? 0 : r[i]) * a.row_stride + c0) *
                        T::kBytes);
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (r[i] == kNone) o[i].clear();
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const uint32_t r = row_of[t / 16 * 8 + i];
      const uint8_t *at = x + (uint64_t(r) * a.row_stride + c0) * T::kBytes;
      if (r != kNone && c0 + 8 <= a.n_cols)
        o[i].load(at);
      else
        o[i].load_some(at, r != kNone && c0 < a.n_cols
                               ? uint32_t(a.n_cols - c0) : 0u);
    }
  }
  using M = Magnitude<T>;
  uint32_t m[M::kWords];
#pragma unroll
  for (uint32_t w = 0; w < M::kWords; ++w) m[w] = 0;
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i)
#pragma unroll
    for (uint32_t w = 0; w < M::kWords; ++w)
      m[w] = M::larger(m[w], M::word(o[i], w));
  bool any = false;
#pragma unroll
  for (uint32_t w = 0; w < M::kWords; ++w) any = any || M::infinite(m[w]);
  if (__ballot(any) != 0) {
#pragma unroll
    for (uint32_t w = 0; w < M::kWords; ++w) m[w] = 0;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
#pragma unroll
      for (uint32_t w = 0; w < M::kWords; ++w)
        m[w] = M::larger(m[w], M::finite(M::word(o[i], w)));
      M::without_infinities(o[i]);
    }
  }
  // over the wave's four groups of rows, then over the waves
#pragma unroll
  for (uint32_t w = 0; w < M::kWords; ++w) {
#pragma unroll
    for (int d = 16; d < 64; d <<= 1)
      m[w] = M::larger(m[w], __shfl_xor(m[w], d, 64));
    if (lane < 16) top[t >> 6][lane * M::kWords + w] = m[w];
  }
  __syncthreads();
  // a thread a column
  if (t < 128) {
    constexpr uint32_t kHalves = T::kBytes == 4 ? 1 : 2;
    uint32_t word = top[0][t / kHalves];
#pragma unroll
    for (int w = 1; w < 4; ++w) word = M::larger(word, top[w][t / kHalves]);
    const uint32_t byte = scale_byte(M::wide(word, t % kHalves));
    scales[t] = scale_of(byte);
    if (tile_col + t < a.n_cols)
      a.scales[uint64_t(tile_col + t) * a.scale_stride + block] = uint8_t(byte);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < 8; ++k) {
    const uint32_t c = (t % 16) * 8 + k;
    columns.put(c, t / 16, pack_column(o, k, scales[c]));
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t c = t / 8 + 32 * i;
    const uint64_t col = tile_col + c;
    if (col < a.n_cols)
      *reinterpret_cast<u32x4 *>(a.q_t + col * a.length + uint64_t(block) * 128 +
                                 (t % 8) * 16) = columns.get(c, t % 8);
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
