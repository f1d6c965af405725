// Products of 8-bit matrices with block scales for CDNA4 (gfx950): rows of
// experts times their weights, and the weights' gradients.
//
// One matrix instruction, v_mfma_scale_f32_16x16x128_f8f6f4, covers exactly
// one block of 128 of the contracted dimension and takes a power-of-two
// scale for each of its 16 rows and 16 columns, so no vector work is left in the
// loop. It adds eight neighbouring products to one number with 14 bits, counted
// from the largest of the eight, before fp32 takes over: a result is off by
// 1.5e-5 of the root of its products' squares, whatever the depth (the
// 16x16x32 8-bit instruction does the same). That is a hundredth of what
// rounding to bf16 costs (1.7e-3), a tenth for fp16, and results of these types
// take it. Results in fp32 do not: there the bytes are converted to bf16,
// which holds e4m3 times a power of two exactly, in registers and multiplied by
// v_mfma_f32_16x16x32_bf16 at half the rate; its sums are fp32's (4e-8 at a
// depth of 1024).
//
// Both products contract the dimension that both operands hold contiguous. The
// "rows" operand gives the rows of the result (tokens; outputs n of the weight
// gradient), the "columns" operand its contiguous dimension (outputs n; inputs c).
// The columns operand is the instruction's first: a lane's four results are
// then consecutive in memory.
#include "ciera_expert.h"
#include "ciera_expert_dev.h"

namespace ciera {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 16 bytes a lane from global memory into LDS at `to` + 16 * lane; `to` is the
// same for the whole wave.
__device__ __forceinline__ void load_to_lds(const uint8_t *from, uint8_t *to) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) void *)from,
      (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// Tiles in LDS: rows of 128 bytes in eight 16-byte chunks, chunk c of row r at
// place c ^ ((r >> 1) & 7), so that the 16 rows that a fragment reads at one
// chunk cover all 64 banks. A load instruction fills eight rows: lane i has
// place i & 7 of row i >> 3.
__device__ __forceinline__ uint32_t place_of(uint32_t row, uint32_t chunk) {
  return row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4);
}

// Fragment of 16 rows: lane l has row l % 16 and 32 of its 128 bytes, chunks l
// / 16 and l / 16 + 4. The instruction sums over all of them, so any order
// does that both operands share.
__device__ __forceinline__ i32x8 fragment(const uint8_t *tile, uint32_t row,
                                          uint32_t quarter) {
  const i32x4 lo =
      *reinterpret_cast<const i32x4 *>(tile + place_of(row, quarter));
  const i32x4 hi =
      *reinterpret_cast<const i32x4 *>(tile + place_of(row, quarter + 4));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The same fragment as bf16, scaled: eight values a lane for each of four
// instructions.
struct Wide {
  bf16x8 k[4];
};
__device__ __forceinline__ Wide widen(const i32x8 &f, int scale_byte) {
  const float scale = __uint_as_float(uint32_t(scale_byte) << 23);
  Wide r;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(
          uint32_t(f[2 * k + h]), scale, false);
      const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(
          uint32_t(f[2 * k + h]), scale, true);
      r.k[k][4 * h] = lo[0];
      r.k[k][4 * h + 1] = lo[1];
      r.k[k][4 * h + 2] = hi[0];
      r.k[k][4 * h + 3] = hi[1];
    }
  }
  return r;
}

// What a workgroup multiplies: `steps` blocks of 128.
struct Operand {
  const uint8_t *data;  // block 0 of row 0
  uint64_t stride;      // bytes a row
  uint32_t rows;        // rows there are; later ones repeat the last
};

template <typename T>
__device__ __forceinline__ void store_four(void *out, uint64_t at, uint32_t n,
                                           bool whole, f32x4 v) {
  typename T::Raw *p = static_cast<typename T::Raw *>(out) + at;
  if (whole && n >= 4) {
    typename T::Raw r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = T::from_float(v[i]);
    __builtin_memcpy(__builtin_assume_aligned(p, 4 * T::kBytes), r,
                     4 * T::kBytes);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (uint32_t(i) < n) p[i] = T::from_float(v[i]);
  }
}

// A TR x TC tile by four waves, 2 x 2. Two stages in LDS: the loads of a block
// are in flight while the one before is multiplied. row_scale(f, kb) and
// col_scale(g, kb): the scale bytes of this lane's row in fragments f, g.
template <bool EXACT, int TR, int TC, typename RS, typename CS>
__device__ __forceinline__ void multiply(
    const Operand &rows, const Operand &cols, uint32_t steps, uint8_t *lds,
    RS row_scale, CS col_scale, f32x4 (&acc)[TR / 32][TC / 32]) {
  constexpr int FR = TR / 32, FC = TC / 32;  // fragments of a wave
  constexpr int LR = TR / 32, LC = TC / 32;  // load instructions of a wave
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint8_t *from_r[LR], *from_c[LC];
#pragma unroll
  for (int i = 0; i < LR; ++i) {
    const uint32_t r = (wave * LR + i) * 8 + (lane >> 3);
    const uint32_t held = r < rows.rows ? r : rows.rows - 1;
    from_r[i] = rows.data + held * rows.stride +
                (((lane & 7) ^ ((r >> 1) & 7)) << 4);
  }
#pragma unroll
  for (int i = 0; i < LC; ++i) {
    const uint32_t r = (wave * LC + i) * 8 + (lane >> 3);
    const uint32_t held = r < cols.rows ? r : cols.rows - 1;
    from_c[i] = cols.data + held * cols.stride +
                (((lane & 7) ^ ((r >> 1) & 7)) << 4);
  }
  const auto fetch = [&](uint32_t kb, uint32_t stage) {
    uint8_t *to = lds + stage * (TR + TC) * 128;
#pragma unroll
    for (int i = 0; i < LR; ++i)
      load_to_lds(from_r[i] + uint64_t(kb) * 128, to + (wave * LR + i) * 1024);
    to += TR * 128;
#pragma unroll
    for (int i = 0; i < LC; ++i)
      load_to_lds(from_c[i] + uint64_t(kb) * 128, to + (wave * LC + i) * 1024);
  };
  int sr[FR], sc[FC], next_r[FR], next_c[FC];
#pragma unroll
  for (int f = 0; f < FR; ++f) sr[f] = row_scale(f, 0);
#pragma unroll
  for (int g = 0; g < FC; ++g) sc[g] = col_scale(g, 0);
  fetch(0, 0);
  __syncthreads();
  const uint32_t row0 = (wave >> 1) * (TR / 2) + (lane & 15);
  const uint32_t col0 = (wave & 1) * (TC / 2) + (lane & 15);
  const uint32_t quarter = lane >> 4;
  for (uint32_t kb = 0; kb < steps; ++kb) {
    if (kb + 1 < steps) {
#pragma unroll
      for (int f = 0; f < FR; ++f) next_r[f] = row_scale(f, kb + 1);
#pragma unroll
      for (int g = 0; g < FC; ++g) next_c[g] = col_scale(g, kb + 1);
      fetch(kb + 1, (kb + 1) & 1);
    }
    const uint8_t *tr = lds + (kb & 1) * (TR + TC) * 128;
    const uint8_t *tc = tr + TR * 128;
    if constexpr (EXACT) {
      Wide fr[FR];
#pragma unroll
      for (int f = 0; f < FR; ++f)
        fr[f] = widen(fragment(tr, row0 + 16 * f, quarter), sr[f]);
#pragma unroll
      for (int g = 0; g < FC; ++g) {
        const Wide fc = widen(fragment(tc, col0 + 16 * g, quarter), sc[g]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int f = 0; f < FR; ++f)
            acc[f][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                fc.k[k], fr[f].k[k], acc[f][g], 0, 0, 0);
      }
    } else {
      i32x8 fr[FR];
#pragma unroll
      for (int f = 0; f < FR; ++f) fr[f] = fragment(tr, row0 + 16 * f, quarter);
#pragma unroll
      for (int g = 0; g < FC; ++g) {
        const i32x8 fc = fragment(tc, col0 + 16 * g, quarter);
#pragma unroll
        for (int f = 0; f < FR; ++f)
          acc[f][g] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              fc, fr[f], acc[f][g], 0, 0, 0, sc[g], 0, sr[f]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FR; ++f) sr[f] = next_r[f];
#pragma unroll
    for (int g = 0; g < FC; ++g) sc[g] = next_c[g];
  }
}

// Rows r0 ... of a tile's result, columns c0 ...
template <int TR, int TC, typename T>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[TR / 32][TC / 32],
                                           void *out, uint64_t stride,
                                           uint64_t row, uint32_t rows,
                                           uint32_t col, uint32_t n_cols,
                                           bool whole) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int f = 0; f < TR / 32; ++f) {
    const uint32_t r = (wave >> 1) * (TR / 2) + 16 * f + (lane & 15);
    if (r >= rows) continue;
#pragma unroll
    for (int g = 0; g < TC / 32; ++g) {
      const uint32_t c =
          col + (wave & 1) * (TC / 2) + 16 * g + (lane >> 4) * 4;
      if (c < n_cols)
        store_four<T>(out, (row + r) * stride + c, n_cols - c, whole,
                      acc[f][g]);
    }
  }
}

constexpr int kTile = 128;

// Grid: tiles of the result's columns, then of the experts' rows.
template <typename T>
__global__ void __launch_bounds__(256)
    expert_matmul_kernel(MatmulArgs a, uint32_t col_tiles, bool whole) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * kTile * 128];
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t tile = blockIdx.x / col_tiles;
  const uint32_t col = (blockIdx.x % col_tiles) * kTile;
  ExpertTile where{0, tile * kTile, uint32_t(a.n_rows)};
  if (a.offsets)
    where = find_tile(a.offsets, a.n_experts, uint32_t(a.n_rows), tile, 7, lane);
  if (where.expert == kNoExpert) return;
  const uint32_t held = where.end - where.first;
  const Operand rows{a.a + uint64_t(where.first) * a.a_stride, a.a_stride,
                     held < kTile ? held : kTile};
  const uint32_t n = uint32_t(a.n_out);
  const Operand cols{a.b + (uint64_t(where.expert) * n + col) * a.b_stride,
                     a.b_stride, n - col < kTile ? n - col : kTile};
  const uint32_t first = (threadIdx.x >> 7) * (kTile / 2) + (lane & 15);
  const auto row_scale = [&](int f, uint32_t kb) -> int {
    const uint32_t r = first + 16 * f;
    const uint32_t p = where.first + (r < rows.rows ? r : rows.rows - 1);
    return a.a_scales[p * a.a_scale_stride + kb];
  };
  const uint8_t *b_scale =
      a.b_scales +
      (uint64_t(where.expert) * ((n + 127) / 128) + col / 128) * a.b_scale_stride;
  const auto col_scale = [&](int, uint32_t kb) -> int { return b_scale[kb]; };
  f32x4 acc[kTile / 32][kTile / 32] = {};
  multiply<T::kBytes == 4, kTile, kTile>(rows, cols, uint32_t(a.depth / 128),
                                         lds, row_scale, col_scale, acc);
  store_tile<kTile, kTile, T>(acc, a.out, a.out_stride, where.first, rows.rows,
                              col, n, whole);
}

// Where an expert's columns start and how many there are, in blocks of 128
// rows.
__device__ __forceinline__ void blocks_of_expert(const int32_t *offsets,
                                                 uint32_t expert, uint32_t lane,
                                                 uint32_t &start,
                                                 uint32_t &blocks) {
  uint32_t sum = 0;
  for (uint32_t e = lane; e < expert; e += 64) {
    const uint32_t lo = offset_of(offsets, e, ~0u);
    const uint32_t hi = offset_of(offsets, e + 1, ~0u);
    sum += hi > lo ? (hi - lo + 127) / 128 : 0;
  }
  uint32_t total;
  wave_prefix(sum, lane, total);
  start = total;
  const uint32_t lo = offset_of(offsets, expert, ~0u);
  const uint32_t hi = offset_of(offsets, expert + 1, ~0u);
  blocks = hi > lo ? (hi - lo + 127) / 128 : 0;
}

template <typename T>
__global__ void __launch_bounds__(256)
    weight_grad_kernel(WeightGradArgs a, uint32_t row_tiles, uint32_t col_tiles,
                       bool whole) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * kTile * 128];
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t col = (blockIdx.x % col_tiles) * kTile;
  const uint32_t row = (blockIdx.x / col_tiles % row_tiles) * kTile;
  const uint32_t expert = blockIdx.x / col_tiles / row_tiles;
  uint32_t start, blocks;
  blocks_of_expert(a.offsets, expert, lane, start, blocks);
  const uint32_t most = uint32_t(a.length / 128);
  if (start > most) start = most;
  if (blocks > most - start) blocks = most - start;
  const uint32_t n = uint32_t(a.n_out), c = uint32_t(a.n_cols);
  const Operand rows{a.dy_t + row * a.length + uint64_t(start) * 128, a.length,
                     n - row < kTile ? n - row : kTile};
  const Operand cols{a.x_t + col * a.length + uint64_t(start) * 128, a.length,
                     c - col < kTile ? c - col : kTile};
  const uint32_t row0 = (threadIdx.x >> 7) * (kTile / 2) + (lane & 15);
  const uint32_t col0 = ((threadIdx.x >> 6) & 1) * (kTile / 2) + (lane & 15);
  const auto row_scale = [&](int f, uint32_t kb) -> int {
    const uint32_t r = row0 + 16 * f;
    return a.dy_scales[(row + (r < rows.rows ? r : rows.rows - 1)) *
                           a.dy_scale_stride + start + kb];
  };
  const auto col_scale = [&](int g, uint32_t kb) -> int {
    const uint32_t r = col0 + 16 * g;
    return a.x_scales[(col + (r < cols.rows ? r : cols.rows - 1)) *
                          a.x_scale_stride + start + kb];
  };
  f32x4 acc[kTile / 32][kTile / 32] = {};
  if (blocks > 0)
    multiply<T::kBytes == 4, kTile, kTile>(rows, cols, blocks, lds, row_scale,
                                           col_scale, acc);
  store_tile<kTile, kTile, T>(acc, a.d_w, c, uint64_t(expert) * n + row,
                              rows.rows, col, c, whole);
}

// Whether four consecutive results at columns that are multiples of 4 may be
// stored at once.
bool aligned_fours(const void *out, uint64_t stride, uint32_t bytes) {
  return stride % 4 == 0 &&
         (reinterpret_cast<uintptr_t>(out) & (4 * bytes - 1)) == 0;
}

template <typename T>
hipError_t matmul_typed(const MatmulArgs &a, uint32_t row_tiles,
                        uint32_t col_tiles, hipStream_t s) {
  expert_matmul_kernel<T><<<dim3(row_tiles * col_tiles), dim3(256), 0, s>>>(
      a, col_tiles, aligned_fours(a.out, a.out_stride, T::kBytes));
  return hipGetLastError();
}

template <typename T>
hipError_t grad_typed(const WeightGradArgs &a, hipStream_t s) {
  const uint32_t rt = uint32_t((a.n_out + kTile - 1) / kTile);
  const uint32_t ct = uint32_t((a.n_cols + kTile - 1) / kTile);
  weight_grad_kernel<T><<<dim3(a.n_experts * rt * ct), dim3(256), 0, s>>>(
      a, rt, ct, aligned_fours(a.d_w, a.n_cols, T::kBytes));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_matmul(const MatmulArgs &a, hipStream_t s) {
  const uint64_t some =
      !a.offsets ? 1 : a.n_rows < a.n_experts ? a.n_rows : a.n_experts;
  const uint32_t rt = uint32_t((a.n_rows + (kTile - 1) * some) / kTile);
  const uint32_t ct = uint32_t((a.n_out + kTile - 1) / kTile);
  return a.out_dtype == CIERA_DT_BF16   ? matmul_typed<Bf16>(a, rt, ct, s)
         : a.out_dtype == CIERA_DT_FP16 ? matmul_typed<Fp16>(a, rt, ct, s)
                                        : matmul_typed<Fp32>(a, rt, ct, s);
}

hipError_t launch_weight_grad(const WeightGradArgs &a, hipStream_t s) {
  return a.out_dtype == CIERA_DT_BF16   ? grad_typed<Bf16>(a, s)
         : a.out_dtype == CIERA_DT_FP16 ? grad_typed<Fp16>(a, s)
                                        : grad_typed<Fp32>(a, s);
}

}  // namespace ciera
