// wc_mx_tile.h -- the product of one tile of MXFP4 matrices by one workgroup, operands through
// LDS: C[n][m] = sum_k W[n][k] x[m][k] on v_mfma_scale_f32_32x32x64_f8f6f4.
//
// A stage is 256 of k: 128 bytes of codes and 8 scales of every row of the tile.  All of it goes
// from memory to LDS without passing through registers (buffer_load ... lds), kDepth - 1 stages
// ahead of the products.  Product q (of four) of a stage takes block q from its lanes 0 .. 31 and
// block 4 + q from the others, so that a lane's scales of a stage are one word, byte after byte.  A
// row's 16-byte chunks are stored in the order chunk ^ turn(row): the sixteen lanes that read LDS
// together, the same chunk of sixteen rows, then touch all 64 banks once.
#pragma once

#include <utility>

#include "wc_i8_tile.h"
#include "wc_mx.h"

namespace wc_mx {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kStageBlocks = 8;  // of 32 of k

// 64 lanes x 4 bytes from rs + offset to LDS at lds, lane after lane; waited for as load_lds.
__device__ __forceinline__ void load_lds_words(u32x4 rs, uint32_t lds, uint32_t offset) {
  asm volatile("s_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"{m0}"(lds), "v"(offset), "s"(rs) : "memory");
}

// kBM rows of x by kBN rows of W, kWM x kWN waves, kDepth stages in LDS.
template <int kBM, int kBN, int kWM, int kWN, int kDepth = 2>
struct MxTile {
  static constexpr int kWM_ = kWM, kWN_ = kWN, kWaves = kWM * kWN, kThreads = 64 * kWaves;
  static constexpr int kMT = kBM / kWM / 32, kNT = kBN / kWN / 32;  // 32 x 32 blocks to a wave
  static constexpr int kRows = kBM, kCols = kBN, kAll = kBM + kBN;
  static constexpr int kXLoads = kBM / 8 / kWaves, kWLoads = kBN / 8 / kWaves;  // eight rows each
  static constexpr int kSLoads = kAll / 32 / kWaves;                            // scales of 32 rows
  static constexpr int kLoads = kXLoads + kWLoads + kSLoads;
  static constexpr int kScales = kAll * kStage;  // where a stage's scales start
  static constexpr int kBuffer = kAll * (kStage + 8);
  static constexpr int kLds = kDepth * kBuffer;
  static_assert(kBM % (8 * kWaves) == 0 && kBN % (8 * kWaves) == 0 && kAll % (32 * kWaves) == 0 &&
                kBM % (32 * kWaves) == 0 && kLds <= 160 * 1024);

  // Row of x (or W) and 16-byte chunk of its stage that load 0 of this lane brings; load i: the
  // same chunk of a row kStep i further on.
  static constexpr uint32_t kStep = 8 * kWaves;
  static __device__ __forceinline__ uint32_t row_of(int i) {
    return 8 * __builtin_amdgcn_readfirstlane(threadIdx.x / 64) + threadIdx.x % 64 / 8 + kStep * i;
  }
  static __device__ __forceinline__ uint32_t turn(uint32_t row) { return (row >> 1) & 7; }
  static __device__ __forceinline__ uint32_t chunk_of() {
    static_assert(kWaves % 2 == 0);  // rows kStep apart turn alike
    return (threadIdx.x % 8) ^ turn(row_of(0));
  }
  // The same of scales: two words a row, the first kXScales loads of x's rows, the others of W's.
  static constexpr int kXScales = kBM / 32 / kWaves;
  static constexpr uint32_t kScaleStep = 32 * kWaves;
  static __device__ __forceinline__ uint32_t scale_row() {
    return 32 * __builtin_amdgcn_readfirstlane(threadIdx.x / 64) + threadIdx.x % 64 / 2;
  }

  // Waits for all but the loads of the newest kLater stages, then for the other waves.
  template <int kLater>
  static __device__ __forceinline__ void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater * kLoads) : "memory");
  }

  // `load_x(i, stage, lds)`, `load_w` and `load_s` start load i of a stage's rows of x, of W, and of
  // the scales.  Of a wave's blocks of 32 rows of x, those past the first `rows` are not
  // multiplied; a wave without any only loads.
  template <class LoadX, class LoadW, class LoadS>
  static __device__ __forceinline__ void product(uint8_t* lds, uint32_t stages, uint32_t rows, LoadX load_x,
                                                 LoadW load_w, LoadS load_s, f32x16 (&acc)[kMT][kNT]) {
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t wm = wave / kWN, wn = wave % kWN;
    const uint32_t base =
        uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
#pragma unroll
    for (int m = 0; m < kMT; m++)
#pragma unroll
      for (int n = 0; n < kNT; n++)
#pragma unroll
        for (int i = 0; i < 16; i++) acc[m][n][i] = 0;
    constexpr uint32_t kAhead = kDepth - 1;
    // Load i of a stage.  Stages past the last are loaded too: the buffers' ends bound them,
    // nothing reads them, and the loop has no branches.
    const auto start = [&](int i, uint32_t s, uint32_t slot) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(base + slot * kBuffer + wave * 1024);
      if (i < kXLoads) load_x(i, s, to + uint32_t(i) * kThreads * 16);
      else if (i < kXLoads + kWLoads) load_w(i - kXLoads, s, to + kBM * kStage + uint32_t(i - kXLoads) * kThreads * 16);
      else
        load_s(i - kXLoads - kWLoads, s,
               __builtin_amdgcn_readfirstlane(base + slot * kBuffer + kScales + wave * 256) +
                   uint32_t(i - kXLoads - kWLoads) * kThreads * 4);
    };
    uint32_t at[4];
#pragma unroll
    for (uint32_t q = 0; q < 4; q++) at[q] = lane % 32 * kStage + ((lane / 32 * 4 + q) ^ turn(lane % 32)) * 16;
    const uint32_t xrow = wm * (kBM / kWM), wrow = kBM + wn * (kBN / kWN);
    const uint32_t scale_at = kScales + lane % 32 * 8 + lane / 32 * 4;
    u32x4 x[2][kMT], w[2][kNT];  // operands of two products' steps
    uint32_t xs[kMT], ws[kNT], xs_next[kMT], ws_next[kNT];
    const auto read = [&](int set, const uint8_t* b, int q, int i) {
      if (i < kNT) w[set][i] = *reinterpret_cast<const u32x4*>(b + wrow * kStage + at[q] + i * 32 * kStage);
      else x[set][i - kNT] = *reinterpret_cast<const u32x4*>(b + xrow * kStage + at[q] + (i - kNT) * 32 * kStage);
    };
    const auto read_scale = [&](const uint8_t* b, int i) {
      if (i < kNT) ws_next[i] = *reinterpret_cast<const uint32_t*>(b + scale_at + wrow * 8 + i * 256);
      else xs_next[i - kNT] = *reinterpret_cast<const uint32_t*>(b + scale_at + xrow * 8 + (i - kNT) * 256);
    };
    // Step q of a stage.  Between its products, in the order written: the reads of the next step
    // (the last one's: of the stage in `slot`, with its scales), and loads kFrom .. kTo - 1 of
    // stage `s`, so that the matrix unit never waits for a queue of either to drain.
    const auto step = [&]<int kQ, int kLive, int kFrom, int kTo>(std::integer_sequence<int, kQ, kLive, kFrom, kTo>,
                                                                uint32_t slot, uint32_t s, uint32_t to) {
      const uint8_t* b = lds + slot * kBuffer;
      constexpr int kProducts = kLive * kNT, kReads = kLive + kNT, kSet = kQ % 2, kNew = kTo - kFrom;
#pragma unroll
      for (int p = 0; p < kProducts; p++) {
        const int m = p / kNT, n = p % kNT;
        acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(w[kSet][n]), operand(x[kSet][m]), acc[m][n],
                                                                    4, 4, kQ, int(ws[n]), kQ, int(xs[m]));
#pragma unroll
        for (int i = 0; i < kReads; i++)
          if (i * kProducts / kReads == p) {
            read(kSet ^ 1, b, (kQ + 1) % 4, i);
            if (kQ == 3) read_scale(b, i);
          }
#pragma unroll
        for (int i = kFrom; i < kTo; i++)
          if ((i - kFrom) * kProducts / (kNew ? kNew : 1) == p) start(i, s, to);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    constexpr int kHalf = kDepth == 2 ? kLoads : kLoads / 2;
#pragma unroll
    for (uint32_t s = 0; s < kAhead; s++)
#pragma unroll
      for (int i = 0; i < kLoads; i++) start(i, s, s);
    arrive<int(kAhead) - 1>();
#pragma unroll
    for (int i = 0; i < kHalf; i++) start(i, kAhead, kAhead);
    uint32_t slot = 0, fill = kAhead;  // the stage's place, and that of the one it loads
    const uint32_t row0 = __builtin_amdgcn_readfirstlane(wm) * (kBM / kWM);
    const uint32_t live = rows > row0 ? (rows - row0 + 31) / 32 : 0;
    if (live == 0) {
      for (uint32_t s = 0; s < stages; s++) {
#pragma unroll
        for (int i = kHalf; i < kLoads; i++) start(i, s + kAhead, fill);
        arrive<int(kAhead) - 1>();
        fill = slot;
        slot = slot + 1 < kDepth ? slot + 1 : 0;
#pragma unroll
        for (int i = 0; i < kHalf; i++) start(i, s + 1 + kAhead, fill);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      return;
    }
    const auto run = [&]<int kLive>(std::integer_sequence<int, kLive>) {
#pragma unroll
      for (int i = 0; i < kLive + kNT; i++) {
        read(0, lds, 0, i);
        read_scale(lds, i);
      }
      for (uint32_t s = 0; s < stages; s++) {
#pragma unroll
        for (int i = 0; i < kNT; i++) ws[i] = ws_next[i];
#pragma unroll
        for (int i = 0; i < kLive; i++) xs[i] = xs_next[i];
        step(std::integer_sequence<int, 0, kLive, kHalf, kLoads>{}, slot, s + kAhead, fill);
        step(std::integer_sequence<int, 1, kLive, 0, 0>{}, slot, 0, 0);
        step(std::integer_sequence<int, 2, kLive, 0, 0>{}, slot, 0, 0);
        // Before the last step's products: the next stage's loads of this wave are in LDS and its
        // reads of this stage done, and so with the other waves behind the barrier.  The
        // stage after those in flight then replaces this one.
        // lgkmcnt(0) as the compiler knows it: no waits for these operands further on
        __builtin_amdgcn_s_waitcnt(0xC07F);
        arrive<int(kAhead) - 1>();
        fill = slot;
        slot = slot + 1 < kDepth ? slot + 1 : 0;
        step(std::integer_sequence<int, 3, kLive, 0, kHalf>{}, slot, s + 1 + kAhead, fill);
      }
    };
    if (live >= kMT) run(std::integer_sequence<int, kMT>{});
    else if (kMT > 3 && live == 3) run(std::integer_sequence<int, (kMT > 3 ? 3 : 1)>{});
    else if (kMT > 2 && live == 2) run(std::integer_sequence<int, (kMT > 2 ? 2 : 1)>{});
    else run(std::integer_sequence<int, 1>{});
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // the waves leave together: LDS is free for the results
    __syncthreads();
  }

  // The results of one 32-row block of x through the wave's own part of LDS, so that rows are
  // written whole: `value(block, i)` is this lane's result i of the given 32 columns (W row 8
  // (i / 4) + 4 (lane / 32) + i mod 4 of x row lane mod 32); `store(row, column, v)` writes four
  // neighbouring columns.
  template <class Value, class Store>
  static __device__ __forceinline__ void rows_out(uint8_t* lds, Value value, Store store) {
    constexpr int kRow = kNT * 32 + 4;  // floats: rows four banks apart
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
    constexpr int kLanes = kNT * 8;  // lanes to a row
#pragma unroll
    for (int r = 0; r < 32; r += 64 / kLanes) {
      const uint32_t row = r + lane / kLanes, col = lane % kLanes * 4;
      store(row, col, *reinterpret_cast<const f32x4*>(t + row * kRow + col));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
};

// The loads of a tile: rows of codes and scales of x and W, by buffers that start at the tile's
// first rows.  `codes` and `words`: bytes of a row's codes, words of its scales (whole rows of
// words).  Chunks of x past its row are zeros (any of W times them are nothing), and so
// are words of scales past either's (another row's could be NaN).
struct RowsOf {
  u32x4 codes, scales;
};
__device__ __forceinline__ RowsOf rows_of(uint64_t codes, uint32_t pitch, uint64_t scales, uint32_t scale_pitch,
                                          uint32_t rows, uint32_t blocks) {
  return {rows_rsrc(codes, (rows - 1) * pitch + blocks * 16),
          rows_rsrc(scales, (rows - 1) * scale_pitch + (blocks + 3) / 4 * 4)};
}

}  // namespace wc_mx
