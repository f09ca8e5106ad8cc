// wc_i8.h -- device helpers of the 8-bit integer layers: element types, the
// int8 rows' loads and the quantisation of one row.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "wc_internal.h"

namespace wc_i8 {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Pointers into global memory: said so, since an address from a table of
// arguments is a generic one to the compiler, and a flat access waits for LDS too.
template <class T>
using global_ptr = T __attribute__((address_space(1)))*;
template <class T>
__device__ __forceinline__ global_ptr<T> global(uint64_t address) {
  return reinterpret_cast<global_ptr<T>>(address);
}

constexpr uint32_t kMaxK = 65536;     // |x w| <= 2^14: no int32 sum overflows
constexpr uint32_t kMaxExperts = 512;
constexpr uint32_t kMaxJobs = 32;
constexpr float kTinyRow = 1e-30f;    // rows below it count as zeros

inline bool float_ok(int32_t dt) { return dt == WC_BF16 || dt == WC_FP16 || dt == WC_FP32; }
inline uint32_t size_of(int32_t dt) { return dt == WC_FP32 ? 4u : 2u; }
inline uint64_t pad256(uint64_t x) { return (x + 255) & ~uint64_t(255); }

__device__ __forceinline__ float bf16_to_float(uint32_t h) { return __uint_as_float(h << 16); }
__device__ __forceinline__ float fp16_to_float(uint32_t h) {
  return float(__builtin_bit_cast(_Float16, uint16_t(h)));
}
// to nearest, ties to even; a NaN stays one
__device__ __forceinline__ uint32_t float_to_bf16(float f) {
  return __builtin_bit_cast(uint16_t, __bf16(f));
}
__device__ __forceinline__ uint32_t float_to_fp16(float f) {
  return __builtin_bit_cast(uint16_t, _Float16(f));
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t floats_to_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// element i of the elements of type dt at address p
__device__ __forceinline__ float load_float(uint64_t p, int32_t dt, uint64_t i) {
  if (dt == WC_FP32) return global<const float>(p)[i];
  const uint32_t h = global<const uint16_t>(p)[i];
  return dt == WC_BF16 ? bf16_to_float(h) : fp16_to_float(h);
}
__device__ __forceinline__ void store_float(uint64_t p, int32_t dt, uint64_t i, float v) {
  if (dt == WC_FP32)
    global<float>(p)[i] = v;
  else
    global<uint16_t>(p)[i] = uint16_t(dt == WC_BF16 ? float_to_bf16(v) : float_to_fp16(v));
}

// 16 bytes of an int8 row, of which `valid` are inside it (the others come back
// as zeros and are not read); any alignment.
__device__ __forceinline__ i32x4 load_codes(global_ptr<const uint8_t> p, int32_t valid) {
  if (valid >= 16) return __builtin_bit_cast(i32x4, *reinterpret_cast<global_ptr<const u32x4u>>(p));
  i32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; i++)
    if (i < valid) v[i / 4] |= int32_t(uint32_t(p[i]) << (8 * (i % 4)));
  return v;
}

// The scale of a row and the factor to its codes, from the bits of its largest
// magnitude (a NaN's are above an infinity's, which are above any number's).
struct RowScale {
  float scale, inverse;
};
__device__ __forceinline__ RowScale row_scale(uint32_t max_bits) {
  const float top = __uint_as_float(max_bits);
  if (top < kTinyRow) return {0.0f, 0.0f};
  return {top / 127.0f, 127.0f / top};
}
// rint(x * inverse), half to even, as a byte; NaN gives 0
__device__ __forceinline__ uint32_t code_of(float x, float inverse) {
  const float r = __builtin_rintf(x * inverse);
  return r == r ? uint32_t(int32_t(fminf(fmaxf(r, -127.0f), 127.0f))) & 0xFFu : 0u;
}

// The value of the lane a data-parallel move takes it from, 0 where there is none: within
// sixteen lanes from kCtrl - 0x110 lanes below, or (0x142, 0x143) the last lane of the
// sixteen or thirty-two below.
template <int kCtrl, int kRows = 0xF>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), kCtrl, kRows, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, moved<0x111>(v));
  v = max(v, moved<0x112>(v));
  v = max(v, moved<0x114>(v));
  v = max(v, moved<0x118>(v));
  v = max(v, moved<0x142, 0xA>(v));
  v = max(v, moved<0x143, 0xC>(v));
  return uint32_t(__builtin_amdgcn_readlane(int(v), 63));
}

// Rows of intermediate results: n columns in `step` (1, 2 or 4) classes n mod step, one
// class after another and each in whole groups of four, so that a tile, whose columns are
// of one class, stores whole groups.
__host__ __device__ constexpr uint32_t class_pitch(uint32_t n, uint32_t step) {
  return ((n + step - 1) / step + 3) & ~3u;
}
__host__ __device__ constexpr uint32_t row_pitch(uint32_t n, uint32_t step) {
  return step * class_pitch(n, step);
}
__device__ __forceinline__ uint32_t column_at(uint32_t column, uint32_t step, uint32_t each) {
  return (column & (step - 1)) * each + column / step;
}

// Which places of the experts' order a workgroup multiplies: blocks of `rows` places,
// counted expert by expert.  Entry 0 of the table holds the number of blocks, entry b + 1
// block b's {expert, first place, past the last place, 0}.
struct Blocks {
  uint64_t table, offsets;
  uint32_t experts, slots, rows, most;
};

// Quantise m rows of k elements of type dt to rows of WC_I8_ROW_BYTES(k) bytes
// (wc_i8.hip), or as many of them as the device int `limit` says; with `blocks`, one more
// workgroup writes its table; with `copies`, their shifted copies (wc_i8_tile.h) too.
// `step`: the columns' classes, fp32 rows only.  False on a launch error.
bool launch_quantize(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ldx, void* q,
                     float* scale, hipStream_t stream, const int32_t* limit = nullptr,
                     const Blocks* blocks = nullptr, void* copies = nullptr, uint32_t step = 1);

}  // namespace wc_i8
