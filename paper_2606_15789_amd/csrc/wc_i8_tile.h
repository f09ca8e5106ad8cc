// wc_i8_tile.h -- the int8 matrix product of one tile by one workgroup, operands
// through LDS: C[n][m] = sum_k W[n][k] x[m][k] on v_mfma_i32_32x32x32_i8.
//
// A stage is 128 bytes of k of every row of the tile.  Both operands go from
// memory to LDS without passing through registers (buffer_load ... lds), kDepth - 1
// stages ahead of the products.  A row's eight 16-byte chunks are stored in the order
// chunk ^ (row mod 8): the eight lanes that read LDS together, the same chunk of
// eight rows next to each other, then touch all banks once.
#pragma once

#include "wc_i8.h"

namespace wc_i8 {

typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int kStage = 128;  // bytes of k to a stage

// A raw buffer of `bytes` bytes: reads past them give zeros.
__device__ __forceinline__ u32x4 rows_rsrc(uint64_t base, uint32_t bytes) {
  return {uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(base))),
          uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(base >> 32) & 0xFFFFu)),
          uint32_t(__builtin_amdgcn_readfirstlane(bytes)), 0x00020000u};
}

// 64 lanes x 16 bytes from rs + offset to LDS at lds, lane after lane.  The load has no
// destination register; the wave waits on vmcnt before LDS is read.
__device__ __forceinline__ void load_lds(u32x4 rs, uint32_t lds, uint32_t offset) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(lds), "v"(offset), "s"(rs)
               : "memory");
}

// kBM rows of x by kBN rows of W, kWM x kWN waves, kDepth stages in LDS.
template <int kBM, int kBN, int kWM, int kWN, int kDepth = 2>
struct Tile {
  static constexpr int kWM_ = kWM, kWN_ = kWN, kWaves = kWM * kWN, kThreads = 64 * kWaves;
  static constexpr int kMT = kBM / kWM / 32, kNT = kBN / kWN / 32;  // 32 x 32 blocks to a wave
  static constexpr int kXLoads = kBM / 8 / kWaves, kWLoads = kBN / 8 / kWaves;
  static constexpr int kBuffer = (kBM + kBN) * kStage;
  static constexpr int kLds = kDepth * kBuffer, kRows = kBM, kCols = kBN;
  static_assert(kBM % (8 * kWaves) == 0 && kBN % (8 * kWaves) == 0);

  // Row of the tile and byte of its stage that load i of this lane brings: each
  // load of a wave is 8 rows.
  static __device__ __forceinline__ uint32_t row_of(int i) {
    return 8 * (threadIdx.x / 64 + kWaves * i) + threadIdx.x % 64 / 8;
  }
  static __device__ __forceinline__ uint32_t byte_of() {
    return ((threadIdx.x % 8) ^ (threadIdx.x % 64 / 8)) * 16;
  }

  // Waits for all but the loads of the newest `later` stages (kN at most), then for the
  // other waves.
  template <int kN>
  static __device__ __forceinline__ void arrive(uint32_t later) {
    if constexpr (kN > 0) {
      if (later < kN) return arrive<kN - 1>(later);
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kN * (kXLoads + kWLoads)) : "memory");
  }

  // `load_x(i, stage, lds)` and `load_w(i, stage, lds)` start load i of a stage's rows
  // of x and W.  A W whose rows cannot go to LDS as they are comes through registers:
  // load_w then gives load i's 16 bytes, which are stored after the products.
  template <class LoadX, class LoadW>
  static __device__ __forceinline__ void product(uint8_t* lds, uint32_t stages, LoadX load_x,
                                                 LoadW load_w, i32x16 (&acc)[kMT][kNT]) {
    constexpr bool kDirect = __is_same(decltype(load_w(0, 0u, 0u)), void);
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t wm = wave / kWN, wn = wave % kWN;
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>(
        (__attribute__((address_space(3))) uint8_t*)lds));
#pragma unroll
    for (int m = 0; m < kMT; m++)
#pragma unroll
      for (int n = 0; n < kNT; n++)
#pragma unroll
        for (int i = 0; i < 16; i++) acc[m][n][i] = 0;
    i32x4 held[kDirect ? 1 : kWLoads];
    const auto start = [&](uint32_t s, uint32_t slot) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(base + slot * kBuffer + wave * 1024);
#pragma unroll
      for (int i = 0; i < kXLoads; i++) load_x(i, s, to + uint32_t(i) * kThreads * 16);
#pragma unroll
      for (int i = 0; i < kWLoads; i++) {
        const uint32_t there = to + kBM * kStage + uint32_t(i) * kThreads * 16;
        if constexpr (kDirect) load_w(i, s, there);
        else held[i] = load_w(i, s, there);
      }
    };
    const auto keep = [&](uint32_t slot) {
      if constexpr (!kDirect) {
        uint8_t* to = lds + slot * kBuffer + kBM * kStage + threadIdx.x * 16;
#pragma unroll
        for (int i = 0; i < kWLoads; i++)
          *reinterpret_cast<i32x4*>(to + i * kThreads * 16) = held[i];
      }
    };
    // stages ahead: one where W comes through registers
    constexpr uint32_t kAhead = kDirect ? kDepth - 1 : 1;
    uint32_t at[4];
#pragma unroll
    for (int k = 0; k < 4; k++)
      at[k] = lane % 32 * kStage + ((2 * k + lane / 32) ^ (lane & 7)) * 16;
    const uint32_t xrow = wm * (kBM / kWM) * kStage, wrow = (kBM + wn * (kBN / kWN)) * kStage;
#pragma unroll
    for (uint32_t s = 0; s < kAhead; s++)
      if (s < stages) {
        start(s, s);
        keep(s);
      }
    uint32_t slot = 0, next = kAhead;
    for (uint32_t s = 0; s < stages; s++) {
      // this wave's loads of stage s are in LDS and its reads of the stage that the next
      // loads replace are done, and so with the other waves behind the barrier
      arrive<kDirect ? int(kAhead) - 1 : 0>(stages - 1 - s);
      const bool more = s + kAhead < stages;
      if (more) start(s + kAhead, next);
      const uint8_t* b = lds + slot * kBuffer;
#pragma unroll
      for (int k = 0; k < 4; k++) {
        i32x4 x[kMT], w[kNT];
#pragma unroll
        for (int m = 0; m < kMT; m++)
          x[m] = *reinterpret_cast<const i32x4*>(b + xrow + at[k] + m * 32 * kStage);
#pragma unroll
        for (int n = 0; n < kNT; n++)
          w[n] = *reinterpret_cast<const i32x4*>(b + wrow + at[k] + n * 32 * kStage);
#pragma unroll
        for (int m = 0; m < kMT; m++)
#pragma unroll
          for (int n = 0; n < kNT; n++)
            acc[m][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[n], x[m], acc[m][n], 0, 0, 0);
      }
      if (more) keep(next);
      slot = slot + 1 < kDepth ? slot + 1 : 0;
      next = next + 1 < kDepth ? next + 1 : 0;
    }
    // the waves leave together: LDS is free for the results
    __syncthreads();
  }

  // The results of one 32-row block of x through the wave's own part of LDS, so that
  // rows are written whole: `value(block, i)` is this lane's result i of the given 32
  // columns (W row 8 (i / 4) + 4 (lane / 32) + i mod 4 of x row lane mod 32);
  // `store(row, column, get)` writes four neighbouring columns of the first kOut, where
  // get(first) are the four values from column first + column on.
  template <int kOut, class Value, class Store>
  static __device__ __forceinline__ void rows_out(uint8_t* lds, Value value, Store store) {
    constexpr int kRow = kNT * 32 + 4;  // floats: rows a bank apart
    static_assert(kWaves * 32 * kRow * 4 <= kLds);
    const uint32_t lane = threadIdx.x % 64;
    float* t = reinterpret_cast<float*>(lds) + threadIdx.x / 64 * (32 * kRow);
#pragma unroll
    for (int c = 0; c < kNT; c++)
#pragma unroll
      for (int g = 0; g < 4; g++) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = value(c, 4 * g + i);
        *reinterpret_cast<f32x4*>(t + lane % 32 * kRow + c * 32 + g * 8 + lane / 32 * 4) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    constexpr int kLanes = kOut / 4;  // lanes to a row
#pragma unroll
    for (int r = 0; r < 32; r += 64 / kLanes) {
      const uint32_t row = r + lane / kLanes, col = lane % kLanes * 4;
      store(row, col, [&](int first) {
        return *reinterpret_cast<const f32x4*>(t + row * kRow + first + col);
      });
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
};

// Which tile a workgroup takes, so that those that run at once on one of the eight
// dies (workgroup i goes to die i mod 8, each with its own L2) share rows: each die
// takes a run of the tiles, ordered in bands of kBand tiles of x rows, W tile by W
// tile within a band.
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t m_tiles, uint32_t n_tiles,
                                        uint32_t& m, uint32_t& n) {
  constexpr uint32_t kDies = 8, kBand = 8;
  const uint32_t all = m_tiles * n_tiles, each = all / kDies, rest = all % kDies;
  const uint32_t die = id % kDies;
  const uint32_t t = die * each + min(die, rest) + id / kDies;
  const uint32_t band = t / (kBand * n_tiles), first = band * kBand;
  const uint32_t high = min(kBand, m_tiles - first), in = t - first * n_tiles;
  m = first + in % high;
  n = in / high;
}

}  // namespace wc_i8
