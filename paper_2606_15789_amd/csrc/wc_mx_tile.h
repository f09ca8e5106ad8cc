// wc_mx_tile.h -- the product of one tile of MXFP4 matrices by one workgroup, operands through
// LDS: C[n][m] = sum_k W[n][k] x[m][k] on v_mfma_scale_f32_32x32x64_f8f6f4.
//
// A stage is 128 bytes of codes of every row of the tile, 256 of k.  They go from
// memory to LDS without passing through registers (buffer_load ... lds), kDepth - 1 stages ahead of
// the products, and so do the scales, of 512 of k at a time: a line of memory for 16 bytes of a row.
// Product q of a stage's four takes block q from its lanes 0 .. 31 and block 4 + q
// from the others, so that a lane's scales of a stage are neighbouring bytes of a word.  A row's
// 16-byte chunks are stored in the order chunk ^ turn(row): the sixteen lanes that read LDS
// together, the same chunk of sixteen rows, then touch all 64 banks once.
#pragma once

#include <utility>

#include "wc_i8_tile.h"
#include "wc_mx.h"

namespace wc_mx {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// kBM rows of x by kBN rows of W, kWM x kWN waves, kDepth stages in LDS.  kPaired: W's rows are kBN / 2 of
// one matrix and the same of another, and a wave's blocks of W the same of either.
template <int kBM, int kBN, int kWM, int kWN, int kDepth, bool kPaired = false>
struct MxTile {
  static constexpr int kWM_ = kWM, kWN_ = kWN, kWaves = kWM * kWN, kThreads = 64 * kWaves;
  static constexpr int kMT = kBM / kWM / 32, kNT = kBN / kWN / 32;  // 32 x 32 blocks to a wave
  static constexpr int kRows = kBM, kCols = kBN, kAll = kBM + kBN, kBytes = 128;
  static constexpr int kSteps = kBytes / 32;           // products of a block by a block to a stage
  static constexpr uint32_t kBlocks = 2 * kSteps;      // MXFP4 blocks of a row in a stage
  static constexpr int kGroup = 16 / int(kBlocks);     // stages that share a load of scales
  static constexpr uint32_t kChunks = kBytes / 16;     // lanes to a row of a load
  static constexpr uint32_t kEach = 64 / kChunks;      // rows to a load of a wave
  static constexpr int kXLoads = kBM / kEach / kWaves, kWLoads = kBN / kEach / kWaves;
  static constexpr int kLoads = kXLoads + kWLoads;     // and those of scales at a group's first stage
  static constexpr int kSLoads = (kAll / 64 + kWaves - 1) / kWaves;  // 64 rows each; not all waves have the last
  static constexpr int kAhead = kDepth - 1;
  static constexpr int kBuffer = kAll * kBytes, kScaleBuffer = kAll * 16;
  static constexpr int kScaleBuffers = kAhead < kGroup ? 2 : 4;
  static constexpr int kScales = kDepth * kBuffer;     // where the scales start
  static constexpr int kLds = kScales + kScaleBuffers * kScaleBuffer;
  static_assert(kBM % (int(kEach) * kWaves) == 0 && kBN % (int(kEach) * kWaves) == 0 &&
                kBM % 64 == 0 && kBN % 64 == 0 && kLds <= 160 * 1024);
  static_assert(kAhead < kGroup + (kScaleBuffers > 2 ? 2 * kGroup : 0));

  // Row of x (or W) and 16-byte chunk of its stage that load 0 of this lane brings; load i: the
  // same chunk of a row kStep i further on.
  static constexpr uint32_t kStep = kEach * kWaves;
  static __device__ __forceinline__ uint32_t row_of(int i) {
    return kEach * __builtin_amdgcn_readfirstlane(threadIdx.x / 64) + threadIdx.x % 64 / kChunks + kStep * i;
  }
  static __device__ __forceinline__ uint32_t turn(uint32_t row) {
    return (row >> 1) & 7;
  }
  static __device__ __forceinline__ uint32_t chunk_of() {
    static_assert(kStep % 16 == 0);  // rows kStep apart turn alike
    return (threadIdx.x % kChunks) ^ turn(row_of(0));
  }
  // Row of the tile (x's, then W's) of which load j of this lane brings scales: of x for a whole wave,
  // or of W; none past kAll.
  static __device__ __forceinline__ uint32_t scale_row(int j) { return threadIdx.x + kThreads * j; }
  static __device__ __forceinline__ uint32_t first_scale_row(int j) {
    return 64 * __builtin_amdgcn_readfirstlane(threadIdx.x / 64) + kThreads * j;
  }
  // Stages of k: whole groups.
  static __host__ __device__ constexpr uint32_t stages_of(uint32_t blocks) { return (blocks + 15) / 16 * kGroup; }

  // Waits for all but the loads of the newest kLater stages (loads of scales among them count as
  // ones of codes before them), then for the other waves.
  template <int kLater>
  static __device__ __forceinline__ void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater * kLoads) : "memory");
  }

  template <int kValue>
  using Int = std::integral_constant<int, kValue>;

  // `load_x(i, stage, lds)` and `load_w` start load i of a stage's rows of x and of W, `load_s(j,
  // stage, lds)` load j of the scales of a group of stages, of which a row has `words` in all.  `stages`
  // are whole groups (stages_of); x is zeros past its row.  Of a wave's blocks of 32 rows
  // of x, those past the first `rows` are not multiplied; a wave without any only loads.
  template <class LoadX, class LoadW, class LoadS>
  static __device__ __forceinline__ void product(uint8_t* lds, uint32_t stages, uint32_t rows, uint32_t words,
                                                 LoadX load_x, LoadW load_w, LoadS load_s,
                                                 f32x16 (&acc)[kMT][kNT]) {
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
    // Load i of stage s, the kPhase-th of its group.  Stages past the last are loaded too: the
    // buffers' ends bound them, nothing reads them, and the loop has no branches.
    const auto start = [&]<int kPhase>(Int<kPhase>, int i, uint32_t s, uint32_t slot) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(base + slot * kBuffer + wave * 1024);
      if (i < kXLoads) load_x(i, s, to + uint32_t(i) * kThreads * 16);
      else load_w(i - kXLoads, s, to + kBM * kBytes + uint32_t(i - kXLoads) * kThreads * 16);
      if (i == kLoads - 1 && kPhase == 0)
#pragma unroll
        for (int j = 0; j < kSLoads; j++)
          if (kAll % kThreads == 0 || j < kSLoads - 1 || first_scale_row(j) < kAll)
            load_s(j, s, __builtin_amdgcn_readfirstlane(base + kScales + s / kGroup % kScaleBuffers * kScaleBuffer +
                                                        wave * 1024) + j * kThreads * 16);
    };
    uint32_t at[kSteps];
#pragma unroll
    for (uint32_t q = 0; q < kSteps; q++)
      at[q] = lane % 32 * kBytes + ((lane / 32 * kSteps + q) ^ turn(lane % 32)) * 16;
    const uint32_t xrow = wm * (kBM / kWM), wrow = kBM + wn * (kBN / kWN / (kPaired ? 2 : 1));
    // block n of W, from row wrow on
    const auto w_at = [](int n) { return kPaired && n >= kNT / 2 ? kBN / 2 + (n - kNT / 2) * 32 : n * 32; };
    u32x4 x[2][kMT], w[2][kNT];  // operands of two steps
    uint32_t xs[kMT], ws[kNT], xs_next[kMT], ws_next[kNT];
    const auto read = [&](int set, const uint8_t* b, int q, int i) {
      if (i < kNT) w[set][i] = *reinterpret_cast<const u32x4*>(b + wrow * kBytes + at[q] + w_at(i) * kBytes);
      else x[set][i - kNT] = *reinterpret_cast<const u32x4*>(b + xrow * kBytes + at[q] + (i - kNT) * 32 * kBytes);
    };
    // the scales of stage s, the `phase`-th of its group: from byte 0 of their words on
    const auto read_scale = [&](uint32_t s, int phase, int i) {
      const uint8_t* b = lds + kScales + s / kGroup % kScaleBuffers * kScaleBuffer + lane % 32 * 16;
      const uint32_t word = uint32_t(phase) * 2 + lane / 32;
      const uint32_t row = i < kNT ? wrow + w_at(i) : xrow + (i - kNT) * 32;
      uint32_t v = *reinterpret_cast<const uint32_t*>(b + row * 16 + word * 4);
      if (s / kGroup * 4 + word >= words) v = 0;  // past a row's end could be another's NaN
      (i < kNT ? ws_next[i < kNT ? i : 0] : xs_next[i < kNT ? 0 : i - kNT]) = v;
    };
    // Step q of a stage.  Between its products, in the order written: the reads of the next step
    // (the last one's: of stage `next`, the kNext-th of its group, with its scales), and loads kFrom ..
    // kTo - 1 of stage `s`, so that the matrix unit never waits for a queue of either to drain.
    const auto step = [&]<int kQ, int kLive, int kFrom, int kTo, int kPhase, int kNext>(
                          std::integer_sequence<int, kQ, kLive, kFrom, kTo, kPhase, kNext>, uint32_t slot, uint32_t s,
                          uint32_t to, uint32_t next) {
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
            read(kSet ^ 1, b, (kQ + 1) % kSteps, i);
            if (kQ == kSteps - 1) read_scale(next, kNext, i);
          }
#pragma unroll
        for (int i = kFrom; i < kTo; i++)
          if ((i - kFrom) * kProducts / (kNew ? kNew : 1) == p) start(Int<kPhase>{}, i, s, to);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // a stage's loads: the first half in the last step of the stage before, the others in the next
    constexpr int kHalf = kLoads / 2;
    const auto begin = [&]<int... kS>(std::integer_sequence<int, kS...>) {
      ([&] {
#pragma unroll
        for (int i = 0; i < kLoads; i++) start(Int<kS % kGroup>{}, i, kS, kS);
      }(), ...);
    };
    begin(std::make_integer_sequence<int, kAhead>{});
    arrive<kAhead - 1>();
#pragma unroll
    for (int i = 0; i < kHalf; i++) start(Int<kAhead % kGroup>{}, i, kAhead, kAhead);
    uint32_t slot = 0, fill = kAhead;  // the stage's place, and that of the one it loads
    const auto turn_over = [&] {
      fill = slot;
      slot = slot + 1 < kDepth ? slot + 1 : 0;
    };
    // all stages, a group at a time
    const auto all = [&](auto stage) {
      for (uint32_t s = 0; s < stages; s += kGroup)
        [&]<int... kS>(std::integer_sequence<int, kS...>) {
          (stage(Int<kS>{}, s + kS), ...);
        }(std::make_integer_sequence<int, kGroup>{});
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      // the waves leave together: LDS is free for what comes
      __syncthreads();
    };
    const uint32_t row0 = __builtin_amdgcn_readfirstlane(wm) * (kBM / kWM);
    const uint32_t live = rows > row0 ? (rows - row0 + 31) / 32 : 0;
    if (live == 0) {
      all([&]<int kPhase>(Int<kPhase>, uint32_t s) {
#pragma unroll
        for (int i = kHalf; i < kLoads; i++) start(Int<(kPhase + kAhead) % kGroup>{}, i, s + kAhead, fill);
        arrive<kAhead - 1>();
        turn_over();
#pragma unroll
        for (int i = 0; i < kHalf; i++) start(Int<(kPhase + 1 + kAhead) % kGroup>{}, i, s + 1 + kAhead, fill);
      });
      return;
    }
    const auto run = [&]<int kLive>(Int<kLive>) {
#pragma unroll
      for (int i = 0; i < kLive + kNT; i++) {
        read(0, lds, 0, i);
        read_scale(0, 0, i);
      }
      all([&]<int kPhase>(Int<kPhase>, uint32_t s) {
        constexpr int kLoad = (kPhase + kAhead) % kGroup, kNext = (kPhase + 1) % kGroup;
#pragma unroll
        for (int i = 0; i < kNT; i++) ws[i] = ws_next[i];
#pragma unroll
        for (int i = 0; i < kLive; i++) xs[i] = xs_next[i];
        step(std::integer_sequence<int, 0, kLive, kHalf, kLoads, kLoad, 0>{}, slot, s + kAhead, fill, 0);
        step(std::integer_sequence<int, 1, kLive, 0, 0, 0, 0>{}, slot, 0, 0, 0);
        step(std::integer_sequence<int, 2, kLive, 0, 0, 0, 0>{}, slot, 0, 0, 0);
        // Before the last step's products: the next stage's loads of this wave are in LDS and its
        // reads of this stage done, and so with the other waves behind the barrier.  The
        // stage after those in flight then replaces this one.
        // lgkmcnt(0) as the compiler knows it: no waits for these operands further on
        __builtin_amdgcn_s_waitcnt(0xC07F);
        arrive<kAhead - 1>();
        turn_over();
        step(std::integer_sequence<int, kSteps - 1, kLive, 0, kHalf, (kLoad + 1) % kGroup, kNext>{}, slot, s + 1 + kAhead,
             fill, s + 1);
      });
    };
    if (live >= kMT) run(Int<kMT>{});
    else if (kMT > 3 && live == 3) run(Int<(kMT > 3 ? 3 : 1)>{});
    else if (kMT > 2 && live == 2) run(Int<(kMT > 2 ? 2 : 1)>{});
    else run(Int<1>{});
  }
};

// The results of a 32 x 32 block, acc[i] the sum of W row 8 (i / 4) + 4 (lane / 32) + i mod 4 and x row
// lane mod 32: `store(column, low, high)` gets eight neighbouring columns of row lane mod 32, those
// from `column` on, twice.  The lanes of a row trade the halves of eight columns that they lack.
template <class Store>
__device__ __forceinline__ void rows_out(const f32x16& acc, Store store) {
#pragma unroll
  for (int p = 0; p < 2; p++) {
    f32x4 low, high;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * p + j]), __float_as_uint(acc[8 * p + 4 + j]),
                                                      false, false);
      low[j] = __uint_as_float(v[0]);
      high[j] = __uint_as_float(v[1]);
    }
    store(p * 16 + threadIdx.x % 64 / 32 * 8, low, high);
  }
}

// The buffers of a tile's rows of codes and of scales (whole words).
struct RowsOf {
  u32x4 codes, scales;
  uint32_t pitch, step;  // of the scales
};
__device__ __forceinline__ RowsOf rows_of(uint64_t codes, uint32_t pitch, const Scales& s, uint32_t first,
                                          uint32_t rows, uint32_t blocks) {
  const uint32_t groups = (blocks + 15) / 16, words = (blocks + 3) / 4;
  return {rows_rsrc(codes + first * uint64_t(pitch), (rows - 1) * pitch + blocks * 16),
          rows_rsrc(s.at + first * uint64_t(s.pitch),
                    (rows - 1) * s.pitch + (groups - 1) * s.step + words * 4 - (groups - 1) * 16),
          s.pitch, s.step};
}
// A wave's loads of scales: row `row` of `from`, groups from the `first`-th on.
struct ScaleLoad {
  u32x4 rsrc;
  uint32_t offset, step;
  __device__ __forceinline__ void set(const RowsOf& from, uint32_t row) {
    rsrc = from.scales;
    step = from.step;
    offset = row * from.pitch;
  }
  __device__ __forceinline__ void operator()(uint32_t group, uint32_t lds) const {
    load_lds(rsrc, lds, offset + group * step);
  }
};

}  // namespace wc_mx
