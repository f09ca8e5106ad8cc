// wc_mx.h -- device helpers of the microscaled 4-bit layers: MXFP4 blocks (32 e2m1 codes, two
// to a byte, the even one low, and an e8m0 scale) and their products on
// v_mfma_scale_f32_16x16x128_f8f6f4.
//
// A product of two codes is a multiple of 1/4 up to 36, so a block's sum is exact in fp32, and so
// is the sum over blocks as long as their scales keep it within 24 bits.
#pragma once

#include <type_traits>

#include "wc_i8.h"

namespace wc_mx {

using namespace wc_i8;

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Blocks of 512 of k: four products of 128 of k, whose lane groups of sixteen take a block each.
constexpr uint32_t kSuper = 16;

inline uint32_t blocks_of(uint32_t k) { return uint32_t(WC_MX_BLOCKS(k)); }

// The scale byte of a block from the bits of its largest magnitude as a float: two below its
// exponent, so that the magnitude lies from 4 to 8 (e2m1's largest are 4 and 6). 255, a NaN,
// where the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t max_bits) {
  const uint32_t field = max_bits >> 23;
  return field == 255 ? 255u : max(field, 2u) - 2u;
}
// 2^(byte - 127) as the conversions take it.
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte ? byte << 23 : 1u << 22);
}

// Eight elements in registers: four words of a 16-bit type, or eight floats.
template <int kType>
struct Eight {
  static constexpr int kWords = kType == WC_FP32 ? 8 : 4;
  uint32_t v[kWords];
  // the largest magnitude, as bits that order like it: of the element's type
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (kType == WC_FP32) {
      uint32_t t = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) t = max(t, v[i] & 0x7FFFFFFFu);
      return t;
    } else {
      u16x2 t = {0, 0};
#pragma unroll
      for (int i = 0; i < 4; i++)
        t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, v[i] & 0x7FFF7FFFu));
      return max(uint32_t(t[0]), uint32_t(t[1]));
    }
  }
  // its codes: to nearest, ties to the even code, at most 6
  __device__ __forceinline__ uint32_t codes(float scale) const {
    uint32_t c = 0;
    if constexpr (kType == WC_FP32) {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(v[0]), __uint_as_float(v[1]), scale, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(v[2]), __uint_as_float(v[3]), scale, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(v[4]), __uint_as_float(v[5]), scale, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(v[6]), __uint_as_float(v[7]), scale, 3);
    } else if constexpr (kType == WC_BF16) {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[0]), scale, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[1]), scale, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[2]), scale, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[3]), scale, 3);
    } else {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v[0]), scale, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v[1]), scale, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v[2]), scale, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v[3]), scale, 3);
    }
    return c;
  }
};
// A largest magnitude of kType as a float's bits.
template <int kType>
__device__ __forceinline__ uint32_t float_bits(uint32_t top) {
  if constexpr (kType == WC_FP32) return top;
  return kType == WC_BF16 ? top << 16 : __float_as_uint(fp16_to_float(top));
}
// Eight elements at address p (aligned to the element), of which `left` are the row's; the
// others are zeros and not read.
template <int kType>
__device__ __forceinline__ Eight<kType> load_eight(uint64_t p, int32_t left) {
  Eight<kType> e;
  if (left >= 8) {
    const auto from = global<const u32x4u>(p);
#pragma unroll
    for (int i = 0; i < Eight<kType>::kWords / 4; i++) {
      const u32x4 w = from[i];
#pragma unroll
      for (int j = 0; j < 4; j++) e.v[4 * i + j] = w[j];
    }
    return e;
  }
#pragma unroll
  for (int i = 0; i < Eight<kType>::kWords; i++) e.v[i] = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    if (i >= left) continue;
    if constexpr (kType == WC_FP32) e.v[i] = global<const uint32_t>(p)[i];
    else e.v[i / 2] |= uint32_t(global<const uint16_t>(p)[i]) << (16 * (i % 2));
  }
  return e;
}

// A lane's four blocks of 512 of k of one row: step s has block 4 s + lane / 16, and byte s of
// `scales` is its scale.
struct Part {
  u32x4 codes[4];
  uint32_t scales;
};

// Scales in groups of 16, those of 512 of k: rows of them `pitch` bytes apart, a row's groups `step`.
// The public layout has step 16; x and h of a call have theirs group by group (pitch 16), so that a
// tile's rows of a group are next to each other.
struct Scales {
  uint64_t at;
  uint32_t pitch, step;
};
inline uint64_t groups_of(uint64_t k) { return (WC_MX_BLOCKS(k) + 15) / 16; }
inline uint64_t own_scales_bytes(uint64_t rows, uint64_t k) { return rows * groups_of(k) * 16; }
inline Scales own_scales(uint64_t at, uint64_t rows, uint64_t k) {
  // offsets in a tile are 32-bit
  if (own_scales_bytes(rows, k) >> 30) return {at, uint32_t(groups_of(k) * 16), 16};
  return {at, 16, uint32_t(rows * 16)};
}

// The row of an MXFP4 matrix that a lane multiplies: `off` and `scale_off` bytes from `codes` and
// `scales` (where those are the same for all lanes, addresses take one register a lane).
struct Row {
  uint64_t codes, scales;
  uint32_t step, off, scale_off;
};
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
  return uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(v >> 32)))) << 32 |
         uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(v)));
}
// Row min(first + r, n - 1) of a matrix; `first` the same for all lanes, rows at most 2^27 bytes apart.
__device__ __forceinline__ Row row_at(uint64_t codes, uint64_t pitch, const Scales& s, uint32_t first, uint32_t r,
                                      uint32_t n) {
  const uint32_t from = min(first, n - 1), in = min(r, n - 1 - from);
  return {uniform(codes + from * pitch), uniform(s.at + from * uint64_t(s.pitch)), s.step, in * uint32_t(pitch),
          in * s.pitch};
}
// The scales of 512 of k as they lie, and the lane's of them.
__device__ __forceinline__ u32x4 load_scales(const Row& r, uint32_t super, uint32_t blocks) {
  const uint64_t at = r.scales + uint64_t(super) * r.step;
  if (super * kSuper + kSuper <= blocks) return *global<const u32x4u>(at + r.scale_off);
  u32x4 s = {0, 0, 0, 0};
#pragma unroll
  for (uint32_t i = 0; i < 4; i++) {
    const uint32_t g = threadIdx.x % 64 / 16;
    s[i] = uint32_t(*global<const uint8_t>(at + (r.scale_off + min(4 * i + g, blocks - 1 - super * kSuper)))) << (8 * g);
  }
  return s;
}
__device__ __forceinline__ uint32_t lane_scales(u32x4 s) {
  const uint32_t g = threadIdx.x % 64 / 16, pick = g | (g + 4) << 8;  // byte g of the second, then of the first
  const uint32_t low = __builtin_amdgcn_perm(s[1], s[0], pick), high = __builtin_amdgcn_perm(s[3], s[2], pick);
  return __builtin_amdgcn_perm(high, low, 0x05040100u);
}
// Blocks past the row's are its last one again; kZero: their codes are zeros, so that a product
// with anything but a NaN scale, which the row then has in its last block too, adds nothing.
struct RawPart {
  u32x4 codes[4], scales;
  __device__ __forceinline__ Part part() const { return {{codes[0], codes[1], codes[2], codes[3]}, lane_scales(scales)}; }
};
template <bool kZero>
__device__ __forceinline__ RawPart load_raw(const Row& r, uint32_t super, uint32_t blocks) {
  const uint32_t g = threadIdx.x % 64 / 16;
  RawPart p;
#pragma unroll
  for (uint32_t i = 0; i < 4; i++) {
    const uint32_t b = super * kSuper + 4 * i + g;
    p.codes[i] = *global<const u32x4>(r.codes + (r.off + min(b, blocks - 1) * 16));
    if (kZero && b >= blocks) p.codes[i] = u32x4{0, 0, 0, 0};
  }
  p.scales = load_scales(r, super, blocks);
  return p;
}
template <bool kZero>
__device__ __forceinline__ Part load_part(const Row& r, uint32_t super, uint32_t blocks) {
  return load_raw<kZero>(r, super, blocks).part();
}
// The same of a row of k elements, quantised in registers; zeros where the lane has no row.
template <int kType>
__device__ __forceinline__ Part quantize_part(uint64_t row, bool live, uint32_t super, uint32_t k) {
  constexpr uint32_t kSize = kType == WC_FP32 ? 4 : 2;
  const uint32_t first = super * (kSuper * 32) + threadIdx.x % 64 / 16 * 32;  // of step 0
  Part p = {};
  if (!live) return p;
  const auto block = [&](const Eight<kType>(&e)[4], u32x4& codes, uint32_t step) {
    const uint32_t top = max(max(e[0].top(), e[1].top()), max(e[2].top(), e[3].top()));
    const uint32_t byte = scale_byte(float_bits<kType>(top));
    const float scale = scale_value(byte);
#pragma unroll
    for (int j = 0; j < 4; j++) codes[j] = byte == 255 ? 0u : e[j].codes(scale);
    p.scales |= byte << (8 * step);
  };
  if (super * (kSuper * 32) + kSuper * 32 <= k) {
    constexpr uint32_t kOnce = kType == WC_FP32 ? 1 : 4;  // blocks in registers at once
#pragma unroll
    for (uint32_t i0 = 0; i0 < 4; i0 += kOnce) {
      Eight<kType> e[kOnce][4];
#pragma unroll
      for (uint32_t i = 0; i < kOnce; i++)
#pragma unroll
        for (uint32_t j = 0; j < 4; j++)
          e[i][j] = load_eight<kType>(row + uint64_t(first + 128 * (i0 + i) + 8 * j) * kSize, 8);
#pragma unroll
      for (uint32_t i = 0; i < kOnce; i++) block(e[i], p.codes[i0 + i], i0 + i);
      if (kOnce < 4) __builtin_amdgcn_sched_barrier(0);
    }
    return p;
  }
  // the row's last part: one block after another, to be short
#pragma unroll 1
  for (uint32_t i = 0; i < 4; i++) {
    const uint32_t at = first + 128 * i;
    Eight<kType> e[4];
    u32x4 codes;
#pragma unroll
    for (uint32_t j = 0; j < 4; j++)
      e[j] = load_eight<kType>(row + uint64_t(at + 8 * j) * kSize, int32_t(k) - int32_t(at + 8 * j));
    block(e, codes, i);
#pragma unroll
    for (uint32_t j = 0; j < 4; j++)
      if (i == j) p.codes[j] = codes;
  }
  return p;
}

__device__ __forceinline__ i32x8 operand(u32x4 c) {
  return __builtin_bit_cast(i32x8, __builtin_shufflevector(c, c, 0, 1, 2, 3, -1, -1, -1, -1));
}
// acc += 16 rows of W times 16 rows of x over 512 of k: lane l gets W rows 4 (l / 16) .. + 3 of
// x row l mod 16.
__device__ __forceinline__ void multiply(const Part& w, const Part& x, f32x4& acc) {
  const auto step = [&]<int kStep>(std::integral_constant<int, kStep>) {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w.codes[kStep]), operand(x.codes[kStep]), acc, 4, 4,
                                                           kStep, int(w.scales), kStep, int(x.scales));
  };
  step(std::integral_constant<int, 0>{});
  step(std::integral_constant<int, 1>{});
  step(std::integral_constant<int, 2>{});
  step(std::integral_constant<int, 3>{});
}

// kN blocks of 16 rows of W by kM blocks of 16 rows of x, k split over the waves of a workgroup
// in parts of 512: straight from memory to registers.  `load_x(m, super)` gives block m's Part.
template <int kN, int kM, int kWaves>
struct Slim {
  static constexpr uint32_t kThreads = 64 * kWaves;
  static constexpr uint32_t kPart = kN * kM * 64;  // groups of four sums to a wave
  struct Shared {
    f32x4 part[kWaves][kPart];
  };
  template <class LoadX>
  static __device__ __forceinline__ void product(Shared& sh, const Row (&w)[kN], uint32_t blocks,
                                                 LoadX load_x) {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const uint32_t supers = (blocks + kSuper - 1) / kSuper;
    f32x4 acc[kN][kM];
#pragma unroll
    for (int n = 0; n < kN; n++)
#pragma unroll
      for (int m = 0; m < kM; m++) acc[n][m] = f32x4{0, 0, 0, 0};
    for (uint32_t s = wave; s < supers; s += kWaves) {
      Part wp[kN];
#pragma unroll
      for (int n = 0; n < kN; n++) wp[n] = load_part<false>(w[n], s, blocks);
#pragma unroll
      for (int m = 0; m < kM; m++) {
        const Part xp = load_x(m, s);
#pragma unroll
        for (int n = 0; n < kN; n++) multiply(wp[n], xp, acc[n][m]);
      }
    }
#pragma unroll
    for (int n = 0; n < kN; n++)
#pragma unroll
      for (int m = 0; m < kM; m++) sh.part[wave][(n * kM + m) * 64 + lane] = acc[n][m];
    __syncthreads();
  }
  // group i of the sums: block i / 64 (n kM + m), lane i mod 64 of it
  static __device__ __forceinline__ f32x4 sum(const Shared& sh, uint32_t i) {
    f32x4 v = sh.part[0][i];
#pragma unroll
    for (int w = 1; w < kWaves; w++)
#pragma unroll
      for (int j = 0; j < 4; j++) v[j] += sh.part[w][i][j];
    return v;
  }
};

// 16 kN rows of W at a time by 16 rows of x, tile after tile: a workgroup's waves take parts of 512
// of k in turn, and the rows of the next part of W are on their way while one is multiplied, across
// tiles too, so that reading W does not pause.
template <int kN, int kWaves>
struct Stream {
  static constexpr uint32_t kThreads = 64 * kWaves, kPart = kN * 64;
  struct Shared {
    f32x4 part[2][kWaves][kPart];
  };
  // Tiles first, first + step, ... below `tiles`: `rows_at(tile, w)` sets the lane's rows, `load_x(super)`
  // gives a part of x, `finish(tile, sum)` is called by all threads, sum(i) for group i of the sums.
  template <class RowsAt, class LoadX, class Finish>
  static __device__ __forceinline__ void run(Shared& sh, uint32_t first, uint32_t tiles, uint32_t step,
                                             uint32_t blocks, RowsAt rows_at, LoadX load_x, Finish finish) {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const uint32_t supers = (blocks + kSuper - 1) / kSuper;
    Row w[kN];
    RawPart next[kN];
    const auto load = [&](uint32_t super) {
#pragma unroll
      for (int n = 0; n < kN; n++) next[n] = load_raw<false>(w[n], super, blocks);
    };
    rows_at(first, w);
    if (wave < supers) load(wave);
    uint32_t turn = 0;
    for (uint32_t tile = first; tile < tiles; tile += step, turn ^= 1) {
      f32x4 acc[kN];
#pragma unroll
      for (int n = 0; n < kN; n++) acc[n] = f32x4{0, 0, 0, 0};
      for (uint32_t super = wave; super < supers; super += kWaves) {
        const Part x = load_x(super);
        Part now[kN];
#pragma unroll
        for (int n = 0; n < kN; n++) now[n] = next[n].part();
        // one copy of the loads
        const bool over = super + kWaves >= supers;
        if (over && tile + step < tiles) rows_at(tile + step, w);
        if (!over || tile + step < tiles) load(over ? wave : super + kWaves);
#pragma unroll
        for (int n = 0; n < kN; n++) multiply(now[n], x, acc[n]);
      }
#pragma unroll
      for (int n = 0; n < kN; n++) sh.part[turn][wave][n * 64 + lane] = acc[n];
      // loads of the next tile stay on their way
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      finish(tile, [&](uint32_t i) {
        f32x4 v = sh.part[turn][0][i];
#pragma unroll
        for (int u = 1; u < kWaves; u++)
#pragma unroll
          for (int j = 0; j < 4; j++) v[j] += sh.part[turn][u][i][j];
        return v;
      });
    }
  }
};

// Parts of x in LDS, by part of k: codes by step and lane, then scales.
constexpr uint32_t kHeldPart = 64 * 5 * 16;
__device__ __forceinline__ void hold_part(u32x4* held, uint32_t super, const Part& p) {
  const uint32_t lane = threadIdx.x % 64;
  u32x4* const to = held + super * (kHeldPart / 16);
#pragma unroll
  for (int i = 0; i < 4; i++) to[i * 64 + lane] = p.codes[i];
  reinterpret_cast<uint32_t*>(to + 4 * 64)[lane] = p.scales;
}
__device__ __forceinline__ Part held_part(const u32x4* held, uint32_t super) {
  const uint32_t lane = threadIdx.x % 64;
  const u32x4* const from = held + super * (kHeldPart / 16);
  return {{from[lane], from[64 + lane], from[128 + lane], from[192 + lane]},
          reinterpret_cast<const uint32_t*>(from + 4 * 64)[lane]};
}

// Four neighbouring elements of type dt from element i on at address p (any element's), of which
// `left` are in the row.
__device__ __forceinline__ void store_four(uint64_t p, int32_t dt, uint64_t i, f32x4 v, uint32_t left) {
  const uint64_t at = p + i * (dt == WC_FP32 ? 4 : 2);
  if (left >= 4 && dt == WC_FP32) {
    *global<u32x4u>(at) = __builtin_bit_cast(u32x4, v);
  } else if (left >= 4) {
    u32x2 h;
    if (dt == WC_BF16)
      h = {floats_to_bf16(v[0], v[1]), floats_to_bf16(v[2], v[3])};
    else
      h = {float_to_fp16(v[0]) | float_to_fp16(v[1]) << 16, float_to_fp16(v[2]) | float_to_fp16(v[3]) << 16};
    *global<u32x2u>(at) = h;
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4; j++)
      if (j < left) store_float(p, dt, i + j, v[j]);
  }
}

// Eight neighbouring elements of type dt from element i on at address p, of which `left` are in the row.
__device__ __forceinline__ void store_eight(uint64_t p, int32_t dt, uint64_t i, f32x4 low, f32x4 high, uint32_t left) {
  const uint64_t at = p + i * 2;
  if (left >= 8 && dt != WC_FP32) {
    u32x4 h;
    if (dt == WC_BF16)
      h = {floats_to_bf16(low[0], low[1]), floats_to_bf16(low[2], low[3]), floats_to_bf16(high[0], high[1]),
           floats_to_bf16(high[2], high[3])};
    else
      h = {float_to_fp16(low[0]) | float_to_fp16(low[1]) << 16, float_to_fp16(low[2]) | float_to_fp16(low[3]) << 16,
           float_to_fp16(high[0]) | float_to_fp16(high[1]) << 16, float_to_fp16(high[2]) | float_to_fp16(high[3]) << 16};
    *global<u32x4u>(at) = h;
    return;
  }
  store_four(p, dt, i, low, left);
  if (left > 4) store_four(p, dt, i + 4, high, left - 4);
}

// Tiles load scales as whole words: others are copied, to own_scales of all `rows`, zeros past a
// row's blocks; row r of them lies at `from` + r / per * stride + r mod per * pitch.
inline bool whole_words(const void* scale, uint64_t pitch, uint32_t k) {
  return reinterpret_cast<uintptr_t>(scale) % 4 == 0 && pitch % 4 == 0 && blocks_of(k) % 4 == 0;
}
struct ScaleCopy {
  uint64_t from, pitch, per, stride;
  Scales to;
  uint64_t rows;
  uint32_t blocks, first;  // first: its first workgroup
};
struct ScaleCopies {
  uint32_t n, groups;  // groups: workgroups of them all
  ScaleCopy copy[kMaxJobs];
  void add(uint64_t from, uint64_t pitch, uint64_t per, uint64_t stride, uint64_t rows, uint32_t k, const Scales& to);
};

// Quantise m rows of k elements of type dt to rows of `ldq` bytes of codes and to scales, of which
// each row has `scale_blocks` written, zeros past its blocks (wc_mx.hip).  In the same launch, with
// `blocks`, one more workgroup writes its table, and with `copies` some copy scales.  False on a
// launch error.
bool launch_quantize(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ldx, void* q, uint64_t ldq,
                     const Scales& scales, uint32_t scale_blocks, hipStream_t stream, const Blocks* blocks = nullptr,
                     const ScaleCopies* copies = nullptr);

inline bool off(const void* p, uint32_t to) { return !p || reinterpret_cast<uintptr_t>(p) % to != 0; }

}  // namespace wc_mx
