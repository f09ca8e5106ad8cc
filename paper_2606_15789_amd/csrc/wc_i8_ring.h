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

// kNT blocks of 16 rows of W, kX (8 or 16) rows of x, kW waves, kS stages to a ring.
template <int kNT, int kX, int kW, int kS>
struct Ring {
  static constexpr int kThreads = 64 * kW;
  static constexpr int kStageBytes = (16 * kNT + kX) * kStage;
  static constexpr int kWave = kS * kStageBytes, kLds = kW * kWave;
  static constexpr int kLoads = 2 * kNT + kX / 8;  // of a wave to a stage
  static_assert(kW * kNT * 1024 <= kLds && kLds <= 160 * 1024);

  // Row of its eight and byte of its line that this lane brings.
  static __device__ __forceinline__ uint32_t row_of() { return threadIdx.x % 64 / 8; }
  static __device__ __forceinline__ uint32_t byte_of() {
    return ((threadIdx.x % 8) ^ (threadIdx.x % 64 / 8)) * 16;
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
  template <class LoadX, class LoadW>
  static __device__ __forceinline__ void product(uint8_t* lds, uint32_t blocks, LoadX load_x,
                                                 LoadW load_w, i32x4 (&acc)[kNT]) {
    const uint32_t lane = threadIdx.x % 64;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    uint8_t* mine = lds + wave * kWave;
    const uint32_t base = __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>(
        (__attribute__((address_space(3))) uint8_t*)mine)));
#pragma unroll
    for (int n = 0; n < kNT; n++) acc[n] = {0, 0, 0, 0};
    const uint32_t count = blocks > wave ? (blocks - wave + kW - 1) / kW : 0;
    const auto start = [&](uint32_t j, uint32_t slot) {
      const uint32_t to = base + slot * kStageBytes, at = (wave + j * kW) * kStage;
#pragma unroll
      for (int i = 0; i < 2 * kNT; i++) load_w(i, at, to + i * 1024);
#pragma unroll
      for (int i = 0; i < kX / 8; i++) load_x(i, at, to + (2 * kNT + i) * 1024);
    };
    // chunk lane / 16 (and four on) of row lane mod 16; of eight rows of x, mod 8
    const uint32_t r = lane % 16, c0 = (lane / 16) ^ (r % 8), c1 = (lane / 16 + 4) ^ (r % 8);
    const uint32_t w0 = r * kStage + c0 * 16, w1 = r * kStage + c1 * 16;
    const uint32_t xr = 16 * kNT * kStage + r % kX * kStage;
    const uint32_t x0 = xr + c0 * 16, x1 = xr + c1 * 16;
#pragma unroll
    for (uint32_t j = 0; j < kS - 1; j++)
      if (j < count) start(j, j);
    uint32_t slot = 0;
    for (uint32_t j = 0; j < count; j++) {
      // the ring's oldest stage was read before this one's products were started
      if (j + kS - 1 < count) start(j + kS - 1, slot ? slot - 1 : kS - 1);
      const uint32_t left = count - 1 - j;
      wait_for<kS - 1>(left < kS - 1 ? left : kS - 1);
      const uint8_t* s = mine + slot * kStageBytes;
      const i32x4 a0 = *reinterpret_cast<const i32x4*>(s + x0);
      const i32x4 a1 = *reinterpret_cast<const i32x4*>(s + x1);
#pragma unroll
      for (int n = 0; n < kNT; n++) {
        const i32x4 b0 = *reinterpret_cast<const i32x4*>(s + w0 + n * 16 * kStage);
        const i32x4 b1 = *reinterpret_cast<const i32x4*>(s + w1 + n * 16 * kStage);
        acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b0, a0, acc[n], 0, 0, 0);
        acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b1, a1, acc[n], 0, 0, 0);
      }
      // the reads are done before the next stage's loads can reach their place
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      slot = slot + 1 < kS ? slot + 1 : 0;
    }
    __syncthreads();  // the rings are free for the sums
  }

  // The sums of all waves: result (block n, W row, x row) for the caller's threads.
  static __device__ __forceinline__ void gather(uint8_t* lds, const i32x4 (&acc)[kNT]) {
    int32_t* part = reinterpret_cast<int32_t*>(lds) + threadIdx.x / 64 * (kNT * 256);
#pragma unroll
    for (int n = 0; n < kNT; n++)
#pragma unroll
      for (int i = 0; i < 4; i++) part[n * 256 + i * 64 + threadIdx.x % 64] = acc[n][i];
    __syncthreads();
  }
  // lane l holds W rows 4 (l div 16) + i of x row l mod 16
  static __device__ __forceinline__ int32_t sum(const uint8_t* lds, uint32_t w_row, uint32_t x_row) {
    const int32_t* part = reinterpret_cast<const int32_t*>(lds);
    const uint32_t at = w_row / 16 * 256 + w_row % 4 * 64 + w_row % 16 / 4 * 16 + x_row;
    int32_t v = 0;
#pragma unroll
    for (int w = 0; w < kW; w++) v += part[w * (kNT * 256) + at];
    return v;
  }
};

}  // namespace wc_i8
