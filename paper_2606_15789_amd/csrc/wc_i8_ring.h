// wc_i8_ring.h -- the int8 product of a few rows of x with 16-row blocks of W, k
// split over the waves of a workgroup: bound by reading W, so what counts is that
// reads are whole lines and that enough of them are on their way.
//
// Each wave streams its own blocks of 128 bytes of k through a ring of its own in LDS
// (buffer_load ... lds, eight rows of a whole line each to a load), with no barrier:
// it waits for its own loads only.  v_mfma_i32_16x16x64_i8 takes its operands row by
// lane, sixteen rows apart in memory; read that way from memory a load would touch 64
// lines for 16 bytes of each, which the L1 cache answers one at a time (3.2 TB/s).
#pragma once

#include "wc_i8_tile.h"

namespace wc_i8 {

// 16 rows of W, kX (8 or 16) rows of x, kW waves, kS stages to a ring.
// kX = 0: x is held in LDS, quantised there by the workgroup itself (hold_rows).
template <int kX, int kW, int kS>
struct Ring {
  static constexpr int kThreads = 64 * kW;
  static constexpr int kStageBytes = (16 + kX) * kStage;
  static constexpr int kWave = kS * kStageBytes, kLds = kW * kWave;
  static constexpr int kLoads = 2 + kX / 8;  // of a wave to a stage
  static_assert(kW * 1024 <= kLds && kLds <= 160 * 1024);

  // Row of its eight and byte of its line that this lane brings in load i of W, or of x.
  static __device__ __forceinline__ uint32_t row_of() { return threadIdx.x % 64 / 8; }
  static __device__ __forceinline__ uint32_t turn(uint32_t row) { return (row >> 1) & 7; }
  static __device__ __forceinline__ uint32_t byte_of(int i) {
    return ((threadIdx.x % 8) ^ turn(8 * i + row_of())) * 16;
  }

  template <int N>
  static __device__ __forceinline__ void wait_for(uint32_t later) {
    // `later` stages started after the one needed, at most N
    if constexpr (N > 0) {
      if (later < N) return wait_for<N - 1>(later);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N * kLoads) : "memory");
  }

  // acc = the products of this wave's blocks wave, wave + kW, ... of `blocks`;
  // `load_w(i, offset, lds)` starts W's rows 8 i .. 8 i + 7, `load_x(i, offset, lds)`
  // x's, at byte `offset` of their rows.
  // Once the first loads are on their way `ready()` is called; it gives the rows of x
  // held in LDS (kX = 0), `pitch` apart and `rows` of them.
  struct Held {
    const uint8_t* x;
    uint32_t pitch, rows;
  };
  template <class LoadX, class LoadW, class Ready>
  static __device__ __forceinline__ void product(uint8_t* lds, uint32_t blocks, LoadX load_x,
                                                 LoadW load_w, i32x4& acc, Ready ready) {
    const uint32_t lane = threadIdx.x % 64;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    uint8_t* mine = lds + wave * kWave;
    const uint32_t base = __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>(
        (__attribute__((address_space(3))) uint8_t*)mine)));
    acc = {0, 0, 0, 0};
    const uint32_t count = blocks > wave ? (blocks - wave + kW - 1) / kW : 0;
    const auto start = [&](uint32_t j, uint32_t slot) {
      const uint32_t to = base + slot * kStageBytes, at = (wave + j * kW) * kStage;
#pragma unroll
      for (int i = 0; i < 2; i++) load_w(i, at, to + i * 1024);
#pragma unroll
      for (int i = 0; i < kX / 8; i++) load_x(i, at, to + (2 + i) * 1024);
    };
#pragma unroll
    for (uint32_t j = 0; j < kS - 1; j++)
      if (j < count) start(j, j);
    const Held held = ready();
    // chunk lane / 16 (and four on) of row lane mod 16; of kX rows of x, mod kX
    const uint32_t r = lane % 16, c0 = (lane / 16) ^ turn(r), c1 = (lane / 16 + 4) ^ turn(r);
    const uint32_t w0 = r * kStage + c0 * 16, w1 = r * kStage + c1 * 16;
    uint32_t x0, x1;
    if constexpr (kX > 0) {
      const uint32_t row = r % kX, xr = 16 * kStage + row * kStage;
      x0 = xr + ((lane / 16) ^ turn(row)) * 16, x1 = xr + ((lane / 16 + 4) ^ turn(row)) * 16;
    } else {
      const uint32_t row = min(r, held.rows - 1), at = row * held.pitch + wave * kStage;
      x0 = at + ((lane / 16) ^ (row % 8)) * 16, x1 = at + ((lane / 16 + 4) ^ (row % 8)) * 16;
    }
    uint32_t slot = 0;
    for (uint32_t j = 0; j < count; j++) {
      // the ring's oldest stage was read before this one's products were started
      if (j + kS - 1 < count) start(j + kS - 1, slot ? slot - 1 : kS - 1);
      const uint32_t left = count - 1 - j;
      wait_for<kS - 1>(left < kS - 1 ? left : kS - 1);
      const uint8_t* s = mine + slot * kStageBytes;
      const uint8_t* x = kX > 0 ? s : held.x + j * (kW * kStage);
      const i32x4 a0 = *reinterpret_cast<const i32x4*>(x + x0);
      const i32x4 a1 = *reinterpret_cast<const i32x4*>(x + x1);
      const i32x4 b0 = *reinterpret_cast<const i32x4*>(s + w0);
      const i32x4 b1 = *reinterpret_cast<const i32x4*>(s + w1);
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b0, a0, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b1, a1, acc, 0, 0, 0);
      // the reads are done before the next stage's loads can reach their place
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      slot = slot + 1 < kS ? slot + 1 : 0;
    }
    __syncthreads();  // the rings are free for the sums
  }

  // The sums of all waves, for the caller's threads: sum(W row, x row).
  static __device__ __forceinline__ void gather(uint8_t* lds, const i32x4& acc) {
    int32_t* part = reinterpret_cast<int32_t*>(lds) + threadIdx.x / 64 * 256;
#pragma unroll
    for (int i = 0; i < 4; i++) part[i * 64 + threadIdx.x % 64] = acc[i];
    __syncthreads();
  }
  // lane l holds W rows 4 (l div 16) + i of x row l mod 16
  static __device__ __forceinline__ int32_t sum(const uint8_t* lds, uint32_t w_row, uint32_t x_row) {
    const int32_t* part = reinterpret_cast<const int32_t*>(lds);
    const uint32_t at = w_row % 4 * 64 + w_row / 4 * 16 + x_row;
    int32_t v = 0;
#pragma unroll
    for (int w = 0; w < kW; w++) v += part[w * 256 + at];
    return v;
  }
};

// A place among the blocks of a token's slots that have an expert, `blocks` to each, counted
// one such slot after another: block `block` from the start of the lowest slot of `left`, the
// set of those from there on.  settle_block moves it to the slot that block lies in (none
// left: past the last).  Slots without an expert are in no set and have no blocks, so waves
// stay as many blocks apart wherever a token's empty slots lie.
struct SlotBlock {
  uint32_t left, block;
  __host__ __device__ __forceinline__ uint32_t slot() const { return uint32_t(__builtin_ctz(left)); }
};
__host__ __device__ __forceinline__ void settle_block(SlotBlock& at, uint32_t blocks) {
  while (at.left && at.block >= blocks) at = {at.left & (at.left - 1), at.block - blocks};
}

// Quantise `rows` rows of x into LDS, chunk c of each 128-byte block of row r at chunk
// c ^ (r mod 8); `row_at(r)` is a row's address, at any element, k elements (a multiple
// of 8) of type kType.  A thread's first kKeep units of eight elements are on their way
// at once and stay in registers; any more are read again, from the caches.  scales, tops:
// LDS, one a row.
template <int kThreads, int kType, int kKeep, class RowAt>
__device__ __forceinline__ void hold_rows(uint32_t rows, uint32_t k, RowAt row_at, uint8_t* to,
                                          float* scales, uint32_t* tops) {
  constexpr int kWords = kType == WC_FP32 ? 8 : 4;
  const uint32_t pitch = uint32_t(WC_I8_ROW_BYTES(k)), units = pitch / 8, all = rows * units;
  if (threadIdx.x < rows) tops[threadIdx.x] = 0;
  const auto load = [&](uint32_t unit, uint32_t (&v)[kWords]) {
    const uint32_t u = min(unit, all - 1), row = rows == 1 ? 0 : u / units;
    const uint32_t at = (u - row * units) * 8;
    const auto p = global<const u32x4u>(row_at(row) + min(at, k - 8) * uint64_t(kType == WC_FP32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < kWords / 4; i++) {
      const u32x4 a = p[i];
#pragma unroll
      for (int j = 0; j < 4; j++) v[4 * i + j] = at < k ? a[j] : 0u;
    }
  };
  const auto value = [&](const uint32_t (&v)[kWords], int i) {
    if constexpr (kType == WC_FP32) return __uint_as_float(v[i]);
    const uint32_t h = i % 2 ? v[i / 2] >> 16 : v[i / 2] & 0xFFFFu;
    return kType == WC_BF16 ? bf16_to_float(h) : fp16_to_float(h);
  };
  const auto measure = [&](uint32_t unit, const uint32_t (&v)[kWords]) {
    const uint32_t row = rows == 1 ? 0 : min(unit, all - 1) / units;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(value(v, i)) & 0x7FFFFFFFu);
    // a wave's units are of one row, or of two where it passes a row's end
    const uint32_t lowest = __builtin_amdgcn_readfirstlane(row);
    const uint32_t here = wave_max(row == lowest ? top : 0u);
    if (threadIdx.x % 64 == 0) atomicMax(&tops[lowest], here);
    if (row != lowest) atomicMax(&tops[row], top);
  };
  const auto store = [&](uint32_t unit, const uint32_t (&v)[kWords]) {
    if (unit >= all) return;
    const uint32_t row = rows == 1 ? 0 : unit / units, at = (unit - row * units) * 8;
    const float inverse = row_scale(tops[row]).inverse;
    u32x2 c = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; i++) c[i / 4] |= code_of(value(v, i), inverse) << (8 * (i % 4));
    *reinterpret_cast<u32x2*>(to + row * pitch + at / 128 * 128 + ((at / 16 % 8) ^ (row % 8)) * 16 +
                              at % 16) = c;
  };
  uint32_t v[kKeep][kWords];
#pragma unroll
  for (int u = 0; u < kKeep; u++) load(threadIdx.x + u * kThreads, v[u]);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kKeep; u++) measure(threadIdx.x + u * kThreads, v[u]);
  for (uint32_t unit = threadIdx.x + kKeep * kThreads; unit - threadIdx.x < all; unit += kThreads) {
    uint32_t w[kWords];
    load(unit, w);
    measure(unit, w);
  }
  __syncthreads();
  if (threadIdx.x < rows) scales[threadIdx.x] = row_scale(tops[threadIdx.x]).scale;
#pragma unroll
  for (int u = 0; u < kKeep; u++) store(threadIdx.x + u * kThreads, v[u]);
  for (uint32_t unit = threadIdx.x + kKeep * kThreads; unit < all; unit += kThreads) {
    uint32_t w[kWords];
    load(unit, w);
    store(unit, w);
  }
  __syncthreads();
}

}  // namespace wc_i8
