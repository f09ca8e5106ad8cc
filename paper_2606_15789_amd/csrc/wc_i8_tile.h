// wc_i8_tile.h -- the int8 matrix product of one tile by one workgroup, operands
// through LDS: C[n][m] = sum_k W[n][k] x[m][k] on v_mfma_i32_32x32x32_i8.
//
// A stage is 128 bytes of k of every row of the tile.  Both operands go from
// memory to LDS without passing through registers (buffer_load ... lds), kDepth - 1
// stages ahead of the products.  A row's 16-byte chunks are stored in the order
// chunk ^ turn(row): the sixteen lanes that read LDS together, the same chunk of sixteen
// rows next to each other, then touch all 64 banks once (chunk ^ (row mod 8), which is
// enough for eight lanes, took twice the cycles).
#pragma once

#include <utility>

#include "wc_i8.h"

namespace wc_i8 {

typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int kStage = 128;  // bytes of k to a block of a row

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

// Values to rs + offset; nothing where that is past the buffer's end.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t as_rsrc(u32x4 rs) {
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(uint64_t(rs[1]) << 32 | rs[0]),
                                           (short)0, (int)rs[2], (int)rs[3]);
}
__device__ __forceinline__ void store_rows(u32x4 rs, uint32_t offset, uint16_t v) {
  __builtin_amdgcn_raw_buffer_store_b16(v, as_rsrc(rs), offset, 0, 0);
}
__device__ __forceinline__ void store_rows(u32x4 rs, uint32_t offset, uint32_t v) {
  __builtin_amdgcn_raw_buffer_store_b32(v, as_rsrc(rs), offset, 0, 0);
}
__device__ __forceinline__ void store_rows(u32x4 rs, uint32_t offset, u32x2 v) {
  __builtin_amdgcn_raw_buffer_store_b64(v, as_rsrc(rs), offset, 0, 0);
}
__device__ __forceinline__ void store_rows(u32x4 rs, uint32_t offset, u32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(v, as_rsrc(rs), offset, 0, 0);
}
constexpr uint32_t kNowhere = 0x80000000u;  // an offset past the end of every buffer here

// kBM rows of x by kBN rows of W, kWM x kWN waves, kDepth stages in LDS.
template <int kBM, int kBN, int kWM, int kWN, int kDepth = 2>
struct Tile {
  static constexpr int kWM_ = kWM, kWN_ = kWN, kWaves = kWM * kWN, kThreads = 64 * kWaves;
  static constexpr int kMT = kBM / kWM / 32, kNT = kBN / kWN / 32;  // 32 x 32 blocks to a wave
  static constexpr int kEach = 1024 / kStage;  // rows to a load of a wave
  static constexpr int kXLoads = kBM / kEach / kWaves, kWLoads = kBN / kEach / kWaves;
  static constexpr int kBuffer = (kBM + kBN) * kStage;
  static constexpr int kLds = kDepth * kBuffer, kRows = kBM, kCols = kBN;
  static_assert(kBM % (kEach * kWaves) == 0 && kBN % (kEach * kWaves) == 0 && kLds <= 160 * 1024);

  // Row of the tile and byte of its stage that load i of this lane brings.
  static __device__ __forceinline__ uint32_t first_row(int i) {
    return kEach * (__builtin_amdgcn_readfirstlane(threadIdx.x / 64) + kWaves * i);
  }
  static __device__ __forceinline__ uint32_t row_of(int i) {
    return first_row(i) + threadIdx.x % 64 / (kStage / 16);
  }
  static __device__ __forceinline__ uint32_t turn(uint32_t row) { return (row >> 1) & 7; }
  static __device__ __forceinline__ uint32_t byte_of() {
    // the same for every load: rows kWaves loads apart turn alike
    static_assert(kWaves % 2 == 0);
    return ((threadIdx.x % (kStage / 16)) ^ turn(row_of(0))) * 16;
  }

  // Waits for all but the loads of the newest kLater stages, then for the other waves.
  template <int kLater>
  static __device__ __forceinline__ void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater * (kXLoads + kWLoads)) : "memory");
  }

  // `load_x(i, stage, lds)` and `load_w(i, stage, lds)` start load i of a stage's rows
  // of x and W.
  // Of a wave's blocks of 32 rows of x, those past the first `rows` are not multiplied; a wave
  // without any only loads.  A block then takes the matrix unit, and the power, of its rows.
  template <class LoadX, class LoadW>
  static __device__ __forceinline__ void product(uint8_t* lds, uint32_t stages, uint32_t rows,
                                                 LoadX load_x, LoadW load_w,
                                                 i32x16 (&acc)[kMT][kNT]) {
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
    constexpr uint32_t kAhead = kDepth - 1;
    constexpr int kAll = kXLoads + kWLoads;
    // Load i of a stage.  Stages past the last are loaded too: the buffers' ends bound
    // them, nothing reads them, and the loop has no branches.
    const auto start = [&](int i, uint32_t s, uint32_t slot) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(base + slot * kBuffer + wave * 1024);
      if (i < kXLoads) load_x(i, s, to + uint32_t(i) * kThreads * 16);
      else load_w(i - kXLoads, s, to + kBM * kStage + uint32_t(i - kXLoads) * kThreads * 16);
    };
    constexpr int kQuarters = kStage / 32;
    uint32_t at[kQuarters];
#pragma unroll
    for (int k = 0; k < kQuarters; k++)
      at[k] = lane % 32 * kStage + ((2 * k + lane / 32) ^ turn(lane % 32)) * 16;
    const uint32_t xrow = wm * (kBM / kWM) * kStage, wrow = (kBM + wn * (kBN / kWN)) * kStage;
    i32x4 x[2][kMT], w[2][kNT];  // operands of two 32-byte quarters of a block
    const auto read = [&](int set, const uint8_t* b, int k, int i) {
      if (i < kNT) w[set][i] = *reinterpret_cast<const i32x4*>(b + wrow + at[k] + i * 32 * kStage);
      else x[set][i - kNT] = *reinterpret_cast<const i32x4*>(b + xrow + at[k] + (i - kNT) * 32 * kStage);
    };
    // The products of one quarter, operand set `set`.  Between them, in the order written:
    // the reads of the next quarter k of the stage in `slot`, and loads kFrom .. kTo - 1 of
    // stage `s`, so that the matrix unit never waits for a queue of either to drain.
    const auto quarter = [&]<int kLive, int kFrom, int kTo>(
                             int set, uint32_t slot, int k, uint32_t s, uint32_t to,
                             std::integer_sequence<int, kLive, kFrom, kTo>) {
      const uint8_t* b = lds + slot * kBuffer;
      constexpr int kProducts = kLive * kNT, kReads = kLive + kNT;
#pragma unroll
      for (int p = 0; p < kProducts; p++) {
        const int m = p / kNT, n = p % kNT;
        acc[m][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[set][n], x[set][m], acc[m][n], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kReads; i++)
          if (i * kProducts / kReads == p) read(set ^ 1, b, k, i);
#pragma unroll
        for (int i = kFrom; i < kTo; i++)
          if ((i - kFrom) * kProducts / (kTo - kFrom) == p) start(i, s, to);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // two stages: all loads as early as they can be (1546 us against 1583 at m = 8192, k = 8192,
    // n = 28672); more are spread over two quarters
    constexpr int kHalf = kDepth == 2 ? kAll : kAll / 2;
#pragma unroll
    for (uint32_t s = 0; s < kAhead; s++)
#pragma unroll
      for (int i = 0; i < kAll; i++) start(i, s, s);
    arrive<int(kAhead) - 1>();
#pragma unroll
    for (int i = 0; i < kHalf; i++) start(i, kAhead, kAhead);
    uint32_t slot = 0, fill = kAhead;  // the stage's place, and that of the one it loads
    const uint32_t row0 = __builtin_amdgcn_readfirstlane(wm) * (kBM / kWM);
    const uint32_t live = rows > row0 ? (rows - row0 + 31) / 32 : 0;
    if (live == 0) {
      for (uint32_t s = 0; s < stages; s++) {
#pragma unroll
        for (int i = kHalf; i < kAll; i++) start(i, s + kAhead, fill);
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
      using First = std::integer_sequence<int, kLive, 0, kHalf>;
      using Second = std::integer_sequence<int, kLive, kHalf, kAll>;
      using None = std::integer_sequence<int, kLive, 0, 0>;
#pragma unroll
      for (int i = 0; i < kLive + kNT; i++) read(0, lds, 0, i);
      for (uint32_t s = 0; s < stages; s++) {
        quarter(0, slot, 1, s + kAhead, fill, Second{});
#pragma unroll
        for (int k = 1; k < kQuarters - 1; k++) quarter(k & 1, slot, k + 1, 0, 0, None{});
        // Before the last quarter's products: the next stage's loads of this wave are in LDS
        // and its reads of this stage done, and so with the other waves behind the barrier.
        // The stage after those in flight then replaces this one.
        // lgkmcnt(0) as the compiler knows it: no waits for these operands further on
        __builtin_amdgcn_s_waitcnt(0xC07F);
        arrive<int(kAhead) - 1>();
        fill = slot;
        slot = slot + 1 < kDepth ? slot + 1 : 0;
        quarter(1, slot, 0, s + 1 + kAhead, fill, First{});
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

// Rows of an int8 matrix that start at the same byte of a dword: rows first, first +
// step, ... of n rows `ld` bytes apart, step 1, 2 or 4.  Loads to LDS take whole dwords, so
// such a row is read from the dword it starts in, and multiplied by x shifted as far.
__host__ __device__ constexpr uint32_t steps_of(uint64_t ld) { return ld % 4 == 0 ? 1 : ld % 2 == 0 ? 2 : 4; }
struct ClassRows {
  uint64_t base;                      // of the dword that row `first` starts in
  uint32_t pitch, rows, shift, bytes;  // bytes: of a row and its shift, whole dwords
};
__device__ __forceinline__ ClassRows class_rows(uint64_t w, uint64_t ld, uint32_t n, uint32_t k,
                                                uint32_t step, uint32_t first) {
  const uint64_t at = w + first * ld;
  const uint32_t shift = uint32_t(at & 3);
  return {at - shift, uint32_t(ld) * step, (n - first + step - 1) / step, shift, (k + shift + 3) & ~3u};
}
// Quantised activations: rows of WC_I8_ROW_BYTES(k) bytes, and where a matrix needs them
// three copies of WC_I8_ROW_BYTES(k + 3), shifted by one to three bytes.
struct Shifted {
  uint64_t base;
  uint32_t pitch;
};
__device__ __forceinline__ Shifted shifted(uint64_t q, uint64_t copies, uint64_t rows, uint32_t k,
                                           uint32_t shift) {
  if (!shift) return {q, uint32_t(WC_I8_ROW_BYTES(k))};
  const uint32_t pitch = uint32_t(WC_I8_ROW_BYTES(k + 3));
  return {copies + (shift - 1) * (rows * pitch), pitch};
}
inline uint64_t copies_bytes(uint64_t rows, uint64_t k) {
  return pad256(3 * rows * WC_I8_ROW_BYTES(k + 3) + 16);
}

// Which tile a workgroup takes, so that those that run at once on one of the eight
// dies (workgroup i goes to die i mod 8, each with its own L2) share rows: each die
// takes a run of the tiles, ordered in bands of kBand tiles of x rows, W tile by W
// tile within a band.  The tiles may be fewer than the workgroups (false for those
// without one): the dies' shares are still even.
__device__ __forceinline__ bool tile_at(uint32_t id, uint32_t m_tiles, uint32_t n_tiles,
                                        uint32_t& m, uint32_t& n) {
  constexpr uint32_t kDies = 8, kBand = 4;
  const uint32_t all = m_tiles * n_tiles, each = all / kDies, rest = all % kDies;
  const uint32_t die = id % kDies;
  if (id / kDies >= each + (die < rest)) return false;
  const uint32_t t = die * each + min(die, rest) + id / kDies;
  const uint32_t band = t / (kBand * n_tiles), first = band * kBand;
  const uint32_t high = min(kBand, m_tiles - first), in = t - first * n_tiles;
  m = first + in % high;
  n = in / high;
  return true;
}

}  // namespace wc_i8
