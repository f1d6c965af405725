// Device helpers of the experts' operators.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ciera {

// A wide type by its storage: bf16 and fp16 values are read and written as
// 16-bit patterns.
struct Bf16 {
  using Raw = uint16_t;
  static constexpr uint32_t kBytes = 2;
  static __device__ __forceinline__ float to_float(uint32_t bits) {
    return __uint_as_float(bits << 16);
  }
  // one rounding, to nearest even (v_cvt_pk_bf16_f32)
  static __device__ __forceinline__ Raw from_float(float x) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
  }
};
struct Fp16 {
  using Raw = uint16_t;
  static constexpr uint32_t kBytes = 2;
  static __device__ __forceinline__ float to_float(uint32_t bits) {
    return static_cast<float>(
        __builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
  }
  static __device__ __forceinline__ Raw from_float(float x) {
    return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
  }
};
struct Fp32 {
  using Raw = uint32_t;
  static constexpr uint32_t kBytes = 4;
  static __device__ __forceinline__ float to_float(uint32_t bits) {
    return __uint_as_float(bits);
  }
  static __device__ __forceinline__ Raw from_float(float x) {
    return __float_as_uint(x);
  }
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive values in registers: 16 bytes of bf16 or fp16, 32 of fp32.
// The device takes 16-byte accesses at any address.
template <typename T>
struct Octet {
  u32x4 w[T::kBytes / 2];
  __device__ __forceinline__ void load(const void *p) {
    const u32x4 *q = static_cast<const u32x4 *>(p);
#pragma unroll
    for (uint32_t i = 0; i < T::kBytes / 2; ++i)
      __builtin_memcpy(&w[i], q + i, 16);
  }
  __device__ __forceinline__ void store(void *p) const {
    u32x4 *q = static_cast<u32x4 *>(p);
#pragma unroll
    for (uint32_t i = 0; i < T::kBytes / 2; ++i)
      __builtin_memcpy(q + i, &w[i], 16);
  }
  __device__ __forceinline__ void load_some(const void *p, uint32_t n) {
    const typename T::Raw *q = static_cast<const typename T::Raw *>(p);
    typename T::Raw v[8];
    clear();
    if (n == 0) return;
    // the first again for those that are not there: all reads are under way at once (56,718
    // tokens of 6 rows of 391 bf16 values each combined: 98 us instead of 129)
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) v[i] = q[i < n ? i : 0];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) set_raw(i, i < n ? v[i] : 0);
  }
  __device__ __forceinline__ void store_some(void *p, uint32_t n) const {
    typename T::Raw *q = static_cast<typename T::Raw *>(p);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < n) q[i] = raw(i);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint32_t i = 0; i < T::kBytes / 2; ++i) w[i] = u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ typename T::Raw raw(uint32_t i) const {
    if constexpr (T::kBytes == 4) return w[i / 4][i % 4];
    else
      return static_cast<typename T::Raw>(w[0][i / 2] >> (16 * (i % 2)));
  }
  __device__ __forceinline__ void set_raw(uint32_t i, typename T::Raw v) {
    if constexpr (T::kBytes == 4) w[i / 4][i % 4] = v;
    else
      w[0][i / 2] = i % 2 ? (w[0][i / 2] & 0xFFFFu) | uint32_t(v) << 16
                          : (w[0][i / 2] & 0xFFFF0000u) | v;
  }
  __device__ __forceinline__ float get(uint32_t i) const {
    if constexpr (T::kBytes == 4) return __uint_as_float(w[i / 4][i % 4]);
    else
      return T::to_float(i % 2 ? w[0][i / 2] >> 16 : w[0][i / 2] & 0xFFFFu);
  }
  __device__ __forceinline__ void set(uint32_t i, float x) {
    set_raw(i, T::from_float(x));
  }
};

// ---------------------------------------------------- the 8-bit format ----
// The scale byte of a block whose largest finite |x| has the bits `amax`: e +
// 127 for the smallest e with amax <= 448 * 2^e, 448 = 1.75 * 2^8. A normal
// amax is m 2^a with 1 <= m < 2, so e is a - 8, or a - 7 where m > 1.75. Below
// 448 * 2^-127 (subnormals among it) e is -127, the smallest there is.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  if (amax == 0) return 127;
  const int e = int(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e > 0 ? uint32_t(e) : 0u;
}

// ------------------------------------------------------ across a wave ----
// DPP controls: the other lane of a pair or of a pair of pairs, the mirrored
// lane of 8 or 16, lane 15 (31) to the row (the half) behind it, and within a
// row the lane n below (kDppUp + n).
constexpr int kDppPair = 0xB1, kDppQuad = 0x4E, kDppHalfMirror = 0x141,
              kDppMirror = 0x140, kDppBcast15 = 0x142, kDppBcast31 = 0x143,
              kDppUp = 0x110;

// x of the lane that CTRL names; `old` where there is none
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float dpp(float old, float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(
      __float_as_int(old), __float_as_int(x), CTRL, ROWS, 0xF, false));
}
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double dpp(double old, double x) {
  const long long o = __double_as_longlong(old), v = __double_as_longlong(x);
  const uint32_t lo = uint32_t(__builtin_amdgcn_update_dpp(
      int(o), int(v), CTRL, ROWS, 0xF, false));
  const uint32_t hi = uint32_t(__builtin_amdgcn_update_dpp(
      int(o >> 32), int(v >> 32), CTRL, ROWS, 0xF, false));
  return __longlong_as_double((long long)(uint64_t(hi) << 32 | lo));
}
__device__ __forceinline__ float lane_of(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  const long long v = __double_as_longlong(x);
  const uint32_t lo = uint32_t(__builtin_amdgcn_readlane(int(v), lane));
  const uint32_t hi = uint32_t(__builtin_amdgcn_readlane(int(v >> 32), lane));
  return __longlong_as_double((long long)(uint64_t(hi) << 32 | lo));
}

// Whole numbers of 32 and 64 bits. 0, or a lane without a source, is the least:
// a maximum takes the other lane's value in one instruction.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t x) {
  return uint32_t(
      __builtin_amdgcn_update_dpp(0, int(x), CTRL, ROWS, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ uint64_t dpp_or_zero(uint64_t x) {
  return uint64_t(dpp_or_zero<CTRL>(uint32_t(x >> 32))) << 32 |
         dpp_or_zero<CTRL>(uint32_t(x));
}
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int lane) {
  return uint32_t(__builtin_amdgcn_readlane(int(x), lane));
}
__device__ __forceinline__ uint64_t lane_of(uint64_t x, int lane) {
  return uint64_t(lane_of(uint32_t(x >> 32), lane)) << 32 |
         lane_of(uint32_t(x), lane);
}
template <typename K>
__device__ __forceinline__ K larger(K a, K b) {
  return a > b ? a : b;
}
// over 8 lanes, over the 16 of a row, in every lane; and over the wave
template <typename O>
__device__ __forceinline__ O eight_max(O x) {
  x = larger(x, dpp_or_zero<kDppPair>(x));
  x = larger(x, dpp_or_zero<kDppQuad>(x));
  return larger(x, dpp_or_zero<kDppHalfMirror>(x));
}
template <typename O>
__device__ __forceinline__ O row_max(O x) {
  x = eight_max(x);
  return larger(x, dpp_or_zero<kDppMirror>(x));
}
template <typename O>
__device__ __forceinline__ O wave_max(O x) {
  x = row_max(x);
  x = larger(x, dpp_or_zero<kDppBcast15>(x));
  x = larger(x, dpp_or_zero<kDppBcast31>(x));
  return lane_of(x, 63);
}
// Floats as whole numbers of the same order (no NaN; -0 as 0), and back.
__device__ __forceinline__ uint32_t to_order(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ (uint32_t(int(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t to_order(double x) {
  const uint64_t b = uint64_t(__double_as_longlong(x + 0.0));
  return b ^ (uint64_t((long long)(b) >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ float from_order(uint32_t o) {
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ double from_order(uint64_t o) {
  return __longlong_as_double((long long)(
      o ^ (o >> 63 ? 0x8000000000000000ull : 0xFFFFFFFFFFFFFFFFull)));
}
template <typename K>
__device__ __forceinline__ K row_sum(K x) {  // in every lane of the row
  x += dpp<kDppPair>(K(0), x);
  x += dpp<kDppQuad>(K(0), x);
  x += dpp<kDppHalfMirror>(K(0), x);
  return x + dpp<kDppMirror>(K(0), x);
}
template <typename K>
__device__ __forceinline__ K wave_sum(K x) {
  x = row_sum(x);
  x += dpp<kDppBcast15, 0xA>(K(0), x);
  x += dpp<kDppBcast31, 0xC>(K(0), x);
  return lane_of(x, 63);
}

// LDS that a wave alone uses: what its lanes wrote before is there for what they
// read after
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// sum of x over the lanes below this one, and over the wave
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x, uint32_t &total) {
  uint32_t s = x;
  s += dpp_or_zero<kDppUp + 1>(s);
  s += dpp_or_zero<kDppUp + 2>(s);
  s += dpp_or_zero<kDppUp + 4>(s);
  s += dpp_or_zero<kDppUp + 8>(s);
  s += dpp_or_zero<kDppBcast15, 0xA>(s);
  s += dpp_or_zero<kDppBcast31, 0xC>(s);
  total = __builtin_amdgcn_readlane(s, 63);
  return s - x;
}

// ------------------------------------------------- rows of the experts ----
constexpr uint32_t kNoExpert = ~0u;
// Tile `tile` of all experts' rows, each expert's rows in tiles of 2^log2_tile:
// from row `first` of `expert`, whose rows end before `end`.
struct ExpertTile {
  uint32_t expert, first, end;
};
// Row `e` of offsets as a row number that every access may use: within
// [0, n_rows] whatever the caller's array holds.
__device__ __forceinline__ uint32_t offset_of(const int32_t *offsets,
                                              uint32_t e, uint32_t n_rows) {
  const int32_t v = offsets[e];
  return v < 0 ? 0u : uint32_t(v) > n_rows ? n_rows : uint32_t(v);
}
// The same for all lanes: 64 experts at a time, by a prefix sum of their tiles.
__device__ __forceinline__ ExpertTile find_tile(const int32_t *offsets,
                                                uint32_t n_experts,
                                                uint32_t n_rows, uint32_t tile,
                                                uint32_t log2_tile,
                                                uint32_t lane) {
  uint32_t before = 0;
  for (uint32_t from = 0; from < n_experts; from += 64) {
    const uint32_t e = from + lane;
    uint32_t lo = 0, hi = 0;
    if (e < n_experts) {
      lo = offset_of(offsets, e, n_rows);
      hi = offset_of(offsets, e + 1, n_rows);
      if (hi < lo) hi = lo;
    }
    const uint32_t tiles = (hi - lo + (1u << log2_tile) - 1) >> log2_tile;
    uint32_t total;
    const uint32_t start = before + wave_prefix(tiles, total);
    const uint64_t here = __ballot(tile >= start && tile < start + tiles);
    if (here) {
      const int l = __builtin_ctzll(here);
      ExpertTile r;
      r.expert = from + uint32_t(l);
      r.end = __builtin_amdgcn_readlane(hi, l);
      r.first = __builtin_amdgcn_readlane(lo, l) +
                ((tile - __builtin_amdgcn_readlane(start, l)) << log2_tile);
      return r;
    }
    before += total;
  }
  return ExpertTile{kNoExpert, 0, 0};
}

}  // namespace ciera
