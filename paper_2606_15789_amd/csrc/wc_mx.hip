// wc_mx.hip -- microscaled 4-bit (MXFP4) linear layers: wc_quantize_mx, wc_dequantize_mx,
// wc_matmul_mx, wc_linear_mx.
#include <algorithm>
#include <cmath>

#include "wc_mx_tile.h"

namespace {

using namespace wc_mx;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kLaunchRows = 1u << 23;  // a grid's axis has less than 2^32 threads

struct QuantArgs {
  uint64_t x, ldx, q, ldq, scale, lds;
  uint32_t m, k, scale_blocks, scale_step, each, groups;  // rows to a workgroup; workgroups of rows
  Blocks blocks;
};

// A workgroup's rows of one copy, four words a thread: neighbouring threads have neighbouring rows.
__device__ __forceinline__ void copy_scales(const ScaleCopies& all, uint32_t group) {
  uint32_t c = 0;
  for (uint32_t i = 1; i < all.n; i++)
    if (group >= all.copy[i].first) c = i;
  const ScaleCopy& C = all.copy[c];
  const uint32_t groups = (C.blocks + 15) / 16, each = kThreads / groups;
  const uint64_t row = uint64_t(group - C.first) * each + threadIdx.x % each;
  const uint32_t at = threadIdx.x / each;
  if (at >= groups || row >= C.rows) return;
  const auto from = global<const uint8_t>(C.from + row / C.per * C.stride + row % C.per * C.pitch + at * 16);
  u32x4 v = {0, 0, 0, 0};
  if (at * 16 + 16 <= C.blocks)
    v = *reinterpret_cast<global_ptr<const u32x4u>>(from);
  else
#pragma unroll
    for (uint32_t i = 0; i < 16; i++)
      if (at * 16 + i < C.blocks) v[i / 4] |= uint32_t(from[i]) << (8 * (i % 4));
  *global<u32x4>(C.to.at + row * C.to.pitch + uint64_t(at) * C.to.step) = v;
}

__global__ __launch_bounds__(kThreads) void wc_copy_scales_mx_kernel(ScaleCopies copies) {
  copy_scales(copies, blockIdx.x);
}
bool launch_copies(const ScaleCopies& copies, hipStream_t stream) {
  hipLaunchKernelGGL(wc_copy_scales_mx_kernel, dim3(copies.groups), dim3(kThreads), 0, stream, copies);
  return hipGetLastError() == hipSuccess;
}

// Four lanes to a block of 32, eight elements each: loads and stores of neighbouring lanes are
// next to each other.  Long rows have kUnits units of eight to a thread, all on their way at once;
// rows of less than a workgroup's elements share one.  After the rows' workgroups one that writes the
// table of blocks of places, if there is one, then those that copy scales.  Bound by memory:
// 28672 x 8192 bf16 133 us, 4.5 TB/s (a large copy 4.8); 333 x 5461 fp32 3.6.
struct NoCopies {};
template <int kType, int kUnits, class Copies>
__global__ __launch_bounds__(kThreads) void wc_quantize_mx_kernel(QuantArgs a, Copies copies) {
  if (blockIdx.x >= a.groups) {
    if (blockIdx.y) return;
    const uint32_t extra = blockIdx.x - a.groups, table = a.blocks.table != 0;
    if (extra < table) {
      __shared__ uint32_t starts[kMaxExperts + 1];
      write_blocks<kThreads>(a.blocks, starts);
    } else if constexpr (std::is_same_v<Copies, ScaleCopies>) {
      copy_scales(copies, extra - table);
    }
    return;
  }
  const uint32_t units = a.scale_blocks * 4;
  uint64_t row = blockIdx.x;
  uint32_t first = blockIdx.y * (kThreads * kUnits) + threadIdx.x;
  if (a.each > 1) {
    row = uint64_t(blockIdx.x) * a.each + threadIdx.x / units;
    first = threadIdx.x / units < a.each ? threadIdx.x % units : units;
  }
  Eight<kType> e[kUnits];
#pragma unroll
  for (uint32_t i = 0; i < kUnits; i++) {
    const uint32_t unit = first + i * kThreads;
    e[i] = load_eight<kType>(a.x + (row * a.ldx + unit * 8) * (kType == WC_FP32 ? 4 : 2),
                             row < a.m && unit < units ? int32_t(a.k) - int32_t(unit * 8) : 0);
  }
#pragma unroll
  for (uint32_t i = 0; i < kUnits; i++) {
    const uint32_t unit = first + i * kThreads;
    uint32_t top = float_bits<kType>(e[i].top());
    top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0xB1, 0xF, 0xF, false)));  // lane ^ 1
    top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0x4E, 0xF, 0xF, false)));  // lane ^ 2
    if (row >= a.m || unit >= units) continue;
    const uint32_t byte = scale_byte(top);
    if (unit < (a.k + 31) / 32 * 4)
      global<uint32_t>(a.q + row * a.ldq)[unit] = byte == 255 ? 0u : e[i].codes(scale_value(byte));
    if (unit % 4 == 0)
      *global<uint8_t>(a.scale + row * a.lds + uint64_t(unit / 64) * a.scale_step + unit / 4 % 16) = uint8_t(byte);
  }
}

struct DequantArgs {
  uint64_t q, ldq, scale, lds, y, ldy;
  uint32_t m, k, each;
};

// The same the other way: eight codes a lane.  Values are exact in fp32, and rounded once to
// y's type.  28672 x 8192 to bf16 88 us, 6.7 TB/s, the codes just written.
template <int kType, int kUnits>
__global__ __launch_bounds__(kThreads) void wc_dequantize_mx_kernel(DequantArgs a) {
  const uint32_t units = (a.k + 7) / 8;
  uint64_t row = blockIdx.x;
  uint32_t first = blockIdx.y * (kThreads * kUnits) + threadIdx.x;
  if (a.each > 1) {
    row = uint64_t(blockIdx.x) * a.each + threadIdx.x / units;
    first = threadIdx.x / units < a.each ? threadIdx.x % units : units;
  }
  if (row >= a.m) return;
  uint32_t codes[kUnits], bytes[kUnits];
#pragma unroll
  for (uint32_t i = 0; i < kUnits; i++) {
    const uint32_t unit = min(first + i * kThreads, units - 1);
    codes[i] = global<const uint32_t>(a.q + row * a.ldq)[unit];
    bytes[i] = global<const uint8_t>(a.scale + row * a.lds)[unit / 4];
  }
#pragma unroll
  for (uint32_t i = 0; i < kUnits; i++) {
    const uint32_t unit = first + i * kThreads;
    if (unit >= units) return;
    const float scale = bytes[i] == 255 ? __builtin_nanf("") : scale_value(bytes[i]);
    f32x4 v[2];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const f32x2 p = j == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], 1.0f, 0)
                      : j == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], 1.0f, 1)
                      : j == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], 1.0f, 2)
                               : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], 1.0f, 3);
      v[j / 2][j % 2 * 2] = p[0] * scale;
      v[j / 2][j % 2 * 2 + 1] = p[1] * scale;
    }
    store_eight(a.y, kType, row * a.ldy + unit * 8, v[0], v[1], a.k - unit * 8);
  }
}

struct MatJob {
  uint64_t w, bias, y, ldw, ldy;
  Scales scales;
  uint64_t part;  // sums of the parts of k, in fp32: parts x m x n (to whole eights)
  uint32_t n, first;  // its first tile
  int32_t bias_dtype, y_dtype;
};
template <uint32_t kJobs>
struct MatArgsOf {
  uint64_t x, ldx;  // rows of codes, or of elements (ldx in bytes)
  Scales xs;
  uint32_t m, k, n_jobs;
  uint32_t splits;  // parts of k
  MatJob job[kJobs];
};
using MatArgs = MatArgsOf<kMaxJobs>;
constexpr uint32_t kFewJobs = 4;  // 2.5 KB less of arguments, which the host takes 0.8 us for
template <uint32_t kJobs>
__device__ __forceinline__ uint32_t job_of(const MatArgsOf<kJobs>& a, uint32_t tile) {
  uint32_t j = 0;
  for (uint32_t i = 1; i < a.n_jobs; i++)
    if (tile >= a.job[i].first) j = i;
  return j;
}

// 16 kN rows of W by 16 kM rows of quantised x, for what is too small for a tile, or rows too far
// apart: each load touches sixteen rows.  100 x 512 -> 512 6.0 us with the quantisation, on tiles
// 6.6; 512 x 28672 -> 8192 360, on tiles 91.
template <int kN, int kM, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void wc_matmul_mx_slim_kernel(MatArgs a) {
  using S = Slim<kN, kM, kWaves>;
  __shared__ typename S::Shared sh;
  const MatJob& J = a.job[job_of(a, blockIdx.x)];
  const uint32_t n0 = (blockIdx.x - J.first) * (16 * kN), m0 = blockIdx.y * (16 * kM);
  const uint32_t r = threadIdx.x % 16;
  Row w[kN];
#pragma unroll
  for (uint32_t n = 0; n < kN; n++) {
    const uint64_t row = min(n0 + 16 * n + r, J.n - 1);
    w[n] = {J.w + row * J.ldw, J.scales.at + row * J.scales.pitch, J.scales.step, 0, 0};
  }
  const uint32_t blocks = (a.k + 31) / 32;
  S::product(sh, w, blocks, [&](int m, uint32_t super) {
    const uint64_t row = m0 + 16 * uint32_t(m) + r;
    const uint64_t at = min(row, uint64_t(a.m - 1));
    return load_part<true>(Row{a.x + at * a.ldx, a.xs.at + at * a.xs.pitch, a.xs.step, 0, 0}, super, blocks);
  });
  for (uint32_t i = threadIdx.x; i < S::kPart; i += S::kThreads) {
    const uint32_t tile = i / 64, lane = i % 64;
    const uint32_t n = n0 + tile / kM * 16 + lane / 16 * 4, m = m0 + tile % kM * 16 + lane % 16;
    if (m >= a.m || n >= J.n) continue;
    f32x4 v = S::sum(sh, i);
    if (J.bias)
#pragma unroll
      for (uint32_t j = 0; j < 4; j++) v[j] += load_float(J.bias, J.bias_dtype, min(n + j, J.n - 1));
    store_four(J.y, J.y_dtype, m * J.ldy + n, v, J.n - n);
  }
}

// Up to 16 rows of x, 16 kN rows of W at a time.  kType: the elements of x, which the workgroup
// quantises to LDS, or 0: quantised rows in memory.  Bound by reading W: 13 x 8192 -> 28672 30 us
// (125 MB of W, 4.1 TB/s from the launch on; a large copy 4.8); one row of 4096 -> 6144 7.2, a
// chain of latencies.  With a launch for the quantisation and a workgroup for every tile, which
// waits for its first rows of W, 13 x 8192 -> 28672 took 58.
template <int kN, int kType, uint32_t kJobs>
__global__ __launch_bounds__(512) void wc_matmul_mx_stream_kernel(MatArgsOf<kJobs> a, uint32_t tiles) {
  using S = Stream<kN, 8>;
  __shared__ typename S::Shared sh;
  extern __shared__ u32x4 held[];  // only its own wave reads a part
  const uint32_t lane = threadIdx.x % 64, r = lane % 16, blocks = (a.k + 31) / 32;
  if constexpr (kType != 0)
    for (uint32_t super = threadIdx.x / 64; super < (blocks + kSuper - 1) / kSuper; super += 8)
      hold_part(held, super, quantize_part<kType>(a.x + r * a.ldx, r < a.m, super, a.k));
  S::run(
      sh, blockIdx.x, tiles, gridDim.x, blocks,
      [&](uint32_t tile, Row(&w)[kN]) {
        const MatJob& J = a.job[job_of(a, tile)];
#pragma unroll
        for (uint32_t n = 0; n < kN; n++) w[n] = row_at(J.w, J.ldw, J.scales, (tile - J.first) * (16 * kN) + 16 * n, r, J.n);
      },
      [&](uint32_t super) {
        if constexpr (kType != 0) return held_part(held, super);
        const uint64_t row = min(r, a.m - 1);
        return load_part<true>(Row{a.x + row * a.ldx, a.xs.at + row * a.xs.pitch, a.xs.step, 0, 0}, super, blocks);
      },
      [&](uint32_t tile, auto sum) {
        const MatJob& J = a.job[job_of(a, tile)];
        const uint32_t n = (tile - J.first) * (16 * kN) + threadIdx.x / 64 * 16 + lane / 16 * 4;
        if (threadIdx.x >= S::kPart || r >= a.m || n >= J.n) return;
        f32x4 v = sum(threadIdx.x);
        if (J.bias)
#pragma unroll
          for (uint32_t j = 0; j < 4; j++) v[j] += load_float(J.bias, J.bias_dtype, min(n + j, J.n - 1));
        store_four(J.y, J.y_dtype, r * J.ldy + n, v, J.n - n);
      });
}

// A tile of y, or of its sums over one part of k (blockIdx.y).  Tiles of 256: 8192 x 8192 -> 28672
// 933 to 966 us, 4.0 PFLOP/s, the matrix units busy 58 % of the cycles.  What bounds them is the
// loads first (without any, an earlier state of the kernel took 663 us of 1012), then the card's
// power: on zeros the call takes 829 us instead of 976, and the units alone, a loop of their
// instruction on registers, reach 9.5 PFLOP/s on zeros and 6.4 on random codes.  Tiles of 128 wait for their stages: 512 x 28672 -> 8192 75 us,
// 0.67 a stage, the matrix units busy 33 % of the cycles.  Four
// waves of 128 x 128 to a tile of 256 took 1.6 times as long, stages of 64 bytes with four of them
// in LDS 8 % longer, operands read from LDS two steps ahead the same.
template <class T>
__global__ __launch_bounds__(T::kThreads) void wc_matmul_mx_tile_kernel(MatArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
  constexpr uint32_t kBM = T::kRows, kBN = T::kCols;
  const MatJob& J = a.job[job_of(a, blockIdx.x)];
  uint32_t mt, nt;
  if (!tile_at(blockIdx.x - J.first, (a.m + kBM - 1) / kBM, (J.n + kBN - 1) / kBN, mt, nt)) return;
  const uint32_t m0 = mt * kBM, n0 = nt * kBN, m_rows = min(kBM, a.m - m0), n_rows = min(kBN, J.n - n0);
  const uint32_t blocks = (a.k + 31) / 32, words = (blocks + 3) / 4;
  // whole groups of stages to a part
  const uint32_t groups = (blocks + 15) / 16, each = (groups + a.splits - 1) / a.splits * T::kGroup;
  const uint32_t first = blockIdx.y * each, all = groups * T::kGroup, stages = first < all ? min(each, all - first) : 0;
  const uint32_t ldx = uint32_t(a.ldx), ldw = uint32_t(J.ldw);
  const RowsOf X = rows_of(a.x, ldx, a.xs, m0, m_rows, blocks), W = rows_of(J.w, ldw, J.scales, n0, n_rows, blocks);
  const uint32_t chunk = T::chunk_of();
  const uint32_t xoff = T::row_of(0) * ldx + chunk * 16, woff = T::row_of(0) * ldw + chunk * 16;
  ScaleLoad scales[T::kSLoads];
#pragma unroll
  for (int j = 0; j < T::kSLoads; j++)
    if (T::first_scale_row(j) < kBM) scales[j].set(X, T::scale_row(j));
    else scales[j].set(W, T::scale_row(j) - kBM);
  f32x16 acc[T::kMT][T::kNT];
  // rows past the tile's last are past the buffers' ends; chunks of x past its row are zeros
  T::product(
      lds, stages, m_rows, words - min(words, first / T::kGroup * 4),
      [&](int i, uint32_t s, uint32_t to) {
        s += first;
        load_lds(X.codes, to, (s * T::kBlocks + chunk < blocks ? xoff : kNowhere) + (i * T::kStep * ldx + s * T::kBytes));
      },
      [&](int i, uint32_t s, uint32_t to) { load_lds(W.codes, to, woff + (i * T::kStep * ldw + (s + first) * T::kBytes)); },
      [&](int j, uint32_t s, uint32_t to) { scales[j]((s + first) / T::kGroup, to); },
      acc);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t wm0 = wave / T::kWN_ * (T::kMT * 32), wn0 = wave % T::kWN_ * (T::kNT * 32);
  const uint32_t pitch = (J.n + 7) & ~7u, lane = threadIdx.x % 64;
#pragma unroll
  for (int nb = 0; nb < T::kNT; nb++) {
    const uint32_t c0 = n0 + wn0 + nb * 32;
    f32x4 bias[2][2] = {};
    if (J.bias && a.splits == 1)
#pragma unroll
      for (uint32_t j = 0; j < 16; j++)
        bias[j / 8][j / 4 % 2][j % 4] =
            load_float(J.bias, J.bias_dtype, min(c0 + j / 8 * 16 + lane / 32 * 8 + j % 8, J.n - 1));
#pragma unroll
    for (int mb = 0; mb < T::kMT; mb++) {
      const uint32_t m = m0 + wm0 + mb * 32 + lane % 32;
      if (m0 + wm0 + mb * 32 >= a.m) break;
      rows_out(acc[mb][nb], [&](uint32_t column, f32x4 low, f32x4 high) {
        const uint32_t n = c0 + column;
        if (m >= a.m || n >= J.n) return;
        if (a.splits > 1) {
          const auto to = global<f32x4>(J.part + ((uint64_t(blockIdx.y) * a.m + m) * pitch + n) * 4);
          to[0] = low;
          to[1] = high;
          return;
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
          low[j] += bias[column / 16][0][j];
          high[j] += bias[column / 16][1][j];
        }
        store_eight(J.y, J.y_dtype, m * J.ldy + n, low, high, J.n - n);
      });
    }
  }
}

// y from the sums of the parts of k, in their order.
__global__ __launch_bounds__(256) void wc_matmul_mx_join_kernel(MatArgs a) {
  const MatJob& J = a.job[blockIdx.z];
  const uint32_t n = (blockIdx.y * 256 + threadIdx.x) * 4, pitch = (J.n + 7) & ~7u;
  if (n >= J.n) return;
  f32x4 bias = {0, 0, 0, 0};
  if (J.bias)
#pragma unroll
    for (uint32_t j = 0; j < 4; j++) bias[j] = load_float(J.bias, J.bias_dtype, min(n + j, J.n - 1));
  for (uint64_t m = blockIdx.x; m < a.m; m += gridDim.x) {
    f32x4 v = *global<f32x4>(J.part + (m * pitch + n) * 4);
    for (uint32_t s = 1; s < a.splits; s++) {
      const f32x4 p = *global<f32x4>(J.part + ((uint64_t(s) * a.m + m) * pitch + n) * 4);
#pragma unroll
      for (int j = 0; j < 4; j++) v[j] += p[j];
    }
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] += bias[j];
    store_four(J.y, J.y_dtype, m * J.ldy + n, v, J.n - n);
  }
}

bool rows_ok(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ld) {
  return float_ok(dt) && k >= 1 && k <= kMaxK && !(m >> 31) && ld >= k && !(ld >> 31) &&
         (m == 0 || !off(x, size_of(dt)));
}
// rows of codes and scales
bool coded_ok(const void* q, uint64_t ldq, const void* scale, uint64_t lds, uint32_t k) {
  return !off(q, 16) && scale && ldq >= WC_MX_ROW_BYTES(k) && ldq % 16 == 0 && !(ldq >> 31) &&
         lds >= WC_MX_BLOCKS(k) && !(lds >> 31);
}
bool jobs_ok(uint32_t m, uint32_t k, uint32_t n_jobs, const wc_mx_job* jobs) {
  if (!jobs || n_jobs < 1 || n_jobs > kMaxJobs || k < 1 || k > kMaxK || m >> 31) return false;
  uint64_t rows = 0;
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_mx_job& J = jobs[i];
    if (!coded_ok(J.w, J.ldw, J.scale, J.lds, k) || J.n < 1 || J.n >> 27 || !float_ok(J.y_dtype) ||
        J.ldy < J.n || J.ldy >> 31 || (m && off(J.y, size_of(J.y_dtype))) ||
        (J.bias && (!float_ok(J.bias_dtype) || off(J.bias, size_of(J.bias_dtype)))))
      return false;
    rows += J.n;
  }
  return !(rows >> 27);
}

// k up to which a workgroup holds 16 rows of x in LDS
constexpr uint32_t kHeldK = 12288;
enum class Kernel { kStream16, kStream32, kStream64, kSlim, kTile64, kTile128, kTile128Deep, kTile256 };
constexpr bool streams(Kernel k) { return k <= Kernel::kStream64; }
using Tile64 = MxTile<64, 64, 2, 2, 4>;
using Tile128 = MxTile<128, 128, 2, 2, 2>;
using Tile128Deep = MxTile<128, 128, 2, 2, 4>;
using Tile256 = MxTile<256, 256, 2, 4, 2>;
template <class F>
void with_tile(Kernel k, F f) {
  switch (k) {
    case Kernel::kTile64: return f(Tile64{});
    case Kernel::kTile128: return f(Tile128{});
    case Kernel::kTile128Deep: return f(Tile128Deep{});
    case Kernel::kTile256: return f(Tile256{});
    default: return;
  }
}
uint32_t tiles_of(Kernel k, uint32_t m, uint32_t n) {
  if (streams(k)) return (n + (16u << int(k)) - 1) / (16u << int(k));
  uint32_t tiles = (n + 31) / 32;
  with_tile(k, [&](auto t) { tiles = (m + t.kRows - 1) / t.kRows * ((n + t.kCols - 1) / t.kCols); });
  return tiles;
}

// What a tile's kernel takes, in us: a stage of 256 of k, one workgroup's and two's where two fit a
// compute unit, and all else of a round of workgroups.  Taken so that the least sum is the fastest
// kernel, or within 5 % of it, at each of these (m, k, n; in us on tiles of 64, of 128 with two and
// with four stages in LDS, and of 256, in the best of 1, 2 and 4 parts of k; with the quantisation):
//   32, 4096, 14336 13.2, 19.6, 16.9, 19.9; 64, 8192, 8192 19.2, 28.9, 21.4, 27.0; 100, 14336,
//   4096 21.9, 39.4, 24.8, 37.6; 128, 8192, 28672 53.7, 45.0, 39.3, 51.4; 333, 5461, 2047 16.7,
//   23.9, 22.3, 33.2; 512, 28672, 8192 133, 100, 88, 93; 1024, 4096, 4096 25.5, 22.9, 21.3,
//   31.9; 1024, 8192, 28672 256, 173, 180, 135; 2000, 2048, 2048 17.8, 15.8, 15.4, 22.1; 4096, 4096,
//   14336 285, 176, 225, 153; 8192, 8192, 28672 1872, 1240, 1392, 992.
struct TileCost {
  Kernel kernel;
  double stage, stage_of_two, round;
};
constexpr TileCost kCosts[] = {{Kernel::kTile64, 0.37, 0.65, 3},
                               {Kernel::kTile128, 1.05, 1.2, 4},
                               {Kernel::kTile128Deep, 0.75, 0, 4},
                               {Kernel::kTile256, 1.85, 0, 6}};
constexpr double kUnits = 256, kJoin = 4.0, kBytesPerUs = 4e6, kReadPerUs = 5e6;

// What a call does, by the sizes and alignments alone.
struct Plan {
  Kernel kernel;
  bool inside;        // the product's kernel quantises x itself
  uint32_t splits;    // parts of k
  uint64_t parts;     // bytes of their sums
  uint64_t scales;    // bytes of copies of scales
  uint32_t m;
  // Whether a tile's kernel gets a copy of a matrix's scales, with the rows of a group next to each
  // other: where it cannot load them as they are, and where enough rows of x make up for it.  us
  // without and with: 512 x 28672 -> 8192 93.5 and 88.6, 512 x 8192 -> 8192 35.1 and 32.0, 8192 x
  // 8192 -> 28672 992 and 970; 256 x 4096 -> 14336 21.5 and 21.3, 48 x 8192 -> 28672 34.8 and 38.2.
  bool copies(const void* scale, uint64_t pitch, uint32_t k) const {
    return kernel >= Kernel::kTile64 && (m >= 256 || !whole_words(scale, pitch, k));
  }
};
Plan plan_of(uint32_t m, uint32_t k, uint32_t n_jobs, const wc_mx_job* jobs) {
  Plan p{Kernel::kSlim, false, 1, 0, 0, m};
  bool near = true, narrow = m < (1u << 24);
  uint64_t n = 0, sums = 0;
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_mx_job& J = jobs[i];
    n += J.n;
    sums += uint64_t(m) * ((J.n + 7) & ~7u) * 4;
    // offsets within a row of tiles are 32-bit
    near = near && J.ldw <= (1u << 27) && J.lds <= (1u << 27);
    narrow = narrow && J.ldw <= (1u << 22) && J.lds <= (1u << 22);
  }
  if (m <= 16 && near) {
    // by the rows of W to a tile, 16, 32 and 64: 2 x 2048 -> 4096 5.0, 6.1, 7.5 us; 16 x 14336 -> 4096
    // 13.3, 16.7, 24.5; 1 x 4096 -> 6144 8.3, 7.6, 9.6; 13 x 8192 -> 28672 36.8, 35.8, 34.1; 13 x
    // 28672 -> 8192 36.2, 31.6, 46.8
    p.kernel = n <= 4096 ? Kernel::kStream16 : n >= 16384 && k <= 8192 ? Kernel::kStream64 : Kernel::kStream32;
    p.inside = k <= kHeldK;
    return p;
  }
  // small products: 20 x 4096 -> 4096 9.2 us, on tiles of 64 10.2; 100 x 512 -> 512 6.0 and 6.6
  if (!narrow || (m <= 32 && n * k <= (1u << 24)) || uint64_t(m) * n * k <= (1u << 25)) return p;
  const uint32_t stages = (k + 255) / 256;
  double best = 0;
  for (const TileCost& c : kCosts) {
    uint64_t tiles = 0, threads = 0;
    with_tile(c.kernel, [&](auto t) { threads = t.kThreads; });
    for (uint32_t i = 0; i < n_jobs; i++) tiles += tiles_of(c.kernel, m, jobs[i].n);
    if (tiles * threads >> 32) continue;  // a grid's axis has less than 2^32 threads
    for (uint32_t splits : {1u, 2u, 4u, 8u}) {
      if (splits > 1 && stages < 4 * splits) break;
      const double groups = double(tiles * splits);
      const bool two = c.stage_of_two > 0 && groups > kUnits;
      const double rounds = std::ceil(groups / (two ? 2 * kUnits : kUnits));
      double us = rounds * (c.round + (stages + splits - 1) / splits * (two ? c.stage_of_two : c.stage));
      us = std::max(us, double(n) * k * 17 / 32 / kReadPerUs);
      if (splits > 1) us += kJoin + 2.0 * double(sums) * splits / kBytesPerUs;
      if (best == 0 || us < best) {
        best = us;
        p.kernel = c.kernel;
        p.splits = splits;
      }
    }
  }
  if (p.kernel == Kernel::kSlim) return p;
  for (uint32_t i = 0; i < n_jobs; i++) {
    if (p.copies(jobs[i].scale, jobs[i].lds, k)) p.scales += pad256(own_scales_bytes(jobs[i].n, k));
    if (p.splits > 1) p.parts += pad256(uint64_t(m) * ((jobs[i].n + 7) & ~7u) * 4 * p.splits);
  }
  return p;
}
uint64_t workspace_of(const Plan& p) { return p.parts + p.scales; }
// x in MXFP4, its scales in groups
uint64_t codes_bytes(uint32_t m, uint32_t k) { return pad256(uint64_t(m) * WC_MX_ROW_BYTES(k)); }
uint64_t quantized_bytes(uint32_t m, uint32_t k) {
  return codes_bytes(m, k) + pad256(own_scales_bytes(m, k));
}
bool workspace_ok(const void* p, uint64_t bytes, uint64_t need) {
  return need == 0 || (!off(p, 256) && bytes >= need);
}

template <int kM>
void start_slim(uint32_t tiles, const MatArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((wc_matmul_mx_slim_kernel<2, kM, 8>), dim3(tiles, (a.m + 16 * kM - 1) / (16 * kM)), dim3(512), 0,
                     st, a);
}
template <int kN, uint32_t kJobs>
void start_stream(const MatArgsOf<kJobs>& a, uint32_t tiles, int32_t x_dtype, hipStream_t st) {
  // as many tiles to every workgroup, one to a compute unit
  const uint32_t held = x_dtype ? uint32_t(groups_of(a.k)) * kHeldPart : 0;
  const uint32_t rounds = (tiles + 255) / 256;
  const dim3 grid((tiles + rounds - 1) / rounds), block(512);
  const auto start = [&]<int kType>(std::integral_constant<int, kType>) {
    hipLaunchKernelGGL((wc_matmul_mx_stream_kernel<kN, kType, kJobs>), grid, block, held, st, a, tiles);
  };
  if (x_dtype == WC_BF16) start(std::integral_constant<int, WC_BF16>{});
  else if (x_dtype == WC_FP16) start(std::integral_constant<int, WC_FP16>{});
  else if (x_dtype == WC_FP32) start(std::integral_constant<int, WC_FP32>{});
  else start(std::integral_constant<int, 0>{});
}
template <int kN>
void start_stream(const MatArgs& a, uint32_t tiles, int32_t x_dtype, hipStream_t st) {
  if (a.n_jobs > kFewJobs) return start_stream<kN, kMaxJobs>(a, tiles, x_dtype, st);
  MatArgsOf<kFewJobs> f{a.x, a.ldx, a.xs, a.m, a.k, a.n_jobs, a.splits, {}};
  for (uint32_t i = 0; i < a.n_jobs; i++) f.job[i] = a.job[i];
  start_stream<kN, kFewJobs>(f, tiles, x_dtype, st);
}

// The copies of scales of a plan.
ScaleCopies copies_of(const Plan& p, uint32_t k, uint32_t n_jobs, const wc_mx_job* jobs, const void* workspace) {
  ScaleCopies c;
  c.n = c.groups = 0;
  uint64_t to = reinterpret_cast<uint64_t>(workspace) + p.parts;
  for (uint32_t i = 0; p.scales && i < n_jobs; i++) {
    const wc_mx_job& J = jobs[i];
    if (!p.copies(J.scale, J.lds, k)) continue;
    c.add(reinterpret_cast<uint64_t>(J.scale), J.lds, J.n, 0, J.n, k, own_scales(to, J.n, k));
    to += pad256(own_scales_bytes(J.n, k));
  }
  return c;
}

// The products of x: rows of codes and scales, or (x_dtype) of elements; ldx in bytes.
// Copies of scales that the plan has are written by the caller (copies_of).
wc_status matmul(const void* x, uint64_t ldx, const Scales& xs, int32_t x_dtype, uint32_t m, uint32_t k,
                 uint32_t n_jobs, const wc_mx_job* jobs, const Plan& p, void* workspace, hipStream_t st) {
  MatArgs a{};
  a.x = reinterpret_cast<uint64_t>(x);
  a.ldx = ldx;
  a.xs = xs;
  a.k = k;
  a.n_jobs = n_jobs;
  a.splits = p.splits;
  uint32_t tiles = 0, widest = 0;
  uint64_t part = reinterpret_cast<uint64_t>(workspace), copy = part + p.parts;
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_mx_job& J = jobs[i];
    a.job[i] = {reinterpret_cast<uint64_t>(J.w), reinterpret_cast<uint64_t>(J.bias),
                reinterpret_cast<uint64_t>(J.y), J.ldw, J.ldy,
                {reinterpret_cast<uint64_t>(J.scale), uint32_t(J.lds), 16}, part, J.n, tiles, J.bias_dtype, J.y_dtype};
    tiles += tiles_of(p.kernel, m, J.n);
    widest = std::max(widest, J.n);
    if (p.splits > 1) part += pad256(uint64_t(m) * ((J.n + 7) & ~7u) * 4 * p.splits);
    if (p.copies(J.scale, J.lds, k)) {
      a.job[i].scales = own_scales(copy, J.n, k);
      copy += pad256(own_scales_bytes(J.n, k));
    }
  }
  if (streams(p.kernel)) {
    a.m = m;
    if (p.kernel == Kernel::kStream16) start_stream<1>(a, tiles, x_dtype, st);
    else if (p.kernel == Kernel::kStream32) start_stream<2>(a, tiles, x_dtype, st);
    else start_stream<4>(a, tiles, x_dtype, st);
    return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
  }
  if (p.kernel >= Kernel::kTile64) {
    a.m = m;
    with_tile(p.kernel, [&](auto t) {
      using T = decltype(t);
      hipLaunchKernelGGL(wc_matmul_mx_tile_kernel<T>, dim3(tiles, p.splits), dim3(T::kThreads), 0, st, a);
    });
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
    if (p.splits > 1)
      hipLaunchKernelGGL(wc_matmul_mx_join_kernel, dim3(std::min(m, 65536u), (widest + 1023) / 1024, n_jobs),
                         dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
  }
  // a grid's second axis holds 65535 blocks of 64 rows
  constexpr uint32_t kSlice = 65535u * 64;
  for (uint32_t m0 = 0; m0 < m; m0 += kSlice) {
    a.m = std::min(m - m0, kSlice);
    if (a.m <= 16) start_slim<1>(tiles, a, st);
    else if (a.m <= 32) start_slim<2>(tiles, a, st);
    else start_slim<4>(tiles, a, st);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
    a.x += uint64_t(a.m) * ldx;
    a.xs.at += uint64_t(a.m) * a.xs.pitch;
    for (uint32_t i = 0; i < n_jobs; i++)
      a.job[i].y += uint64_t(a.m) * a.job[i].ldy * size_of(a.job[i].y_dtype);
  }
  return WC_OK;
}

}  // namespace

namespace wc_mx {

void ScaleCopies::add(uint64_t from, uint64_t pitch, uint64_t per, uint64_t stride, uint64_t rows, uint32_t k,
                      const Scales& to) {
  copy[n++] = {from, pitch, per, stride, to, rows, blocks_of(k), groups};
  const uint32_t each = kThreads / uint32_t(groups_of(k));
  groups += uint32_t((rows + each - 1) / each);
}

template <int kType, int kUnits>
void start_quantize(const dim3& grid, const QuantArgs& a, const ScaleCopies* copies, hipStream_t stream) {
  if (copies)
    hipLaunchKernelGGL((wc_quantize_mx_kernel<kType, kUnits, ScaleCopies>), grid, dim3(kThreads), 0, stream, a, *copies);
  else
    hipLaunchKernelGGL((wc_quantize_mx_kernel<kType, kUnits, NoCopies>), grid, dim3(kThreads), 0, stream, a, NoCopies{});
}

bool launch_quantize(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ldx, void* q, uint64_t ldq,
                     const Scales& scales, uint32_t scale_blocks, hipStream_t stream, const Blocks* blocks,
                     const ScaleCopies* copies) {
  const uint32_t units = scale_blocks * 4, each = units < kThreads ? kThreads / units : 1;
  const bool wide = units > kThreads && m >= 64;
  const uint32_t span = kThreads * (wide ? 4 : 1);
  for (uint32_t first = 0; first == 0 || first < m; first += kLaunchRows) {
    const uint32_t rows = std::min(m - first, kLaunchRows), groups = (rows + each - 1) / each;
    const bool more = first == 0, copying = more && copies && copies->n;
    const QuantArgs a = {reinterpret_cast<uint64_t>(x) + first * ldx * size_of(dt), ldx,
                         reinterpret_cast<uint64_t>(q) + first * ldq, ldq,
                         scales.at + uint64_t(first) * scales.pitch, scales.pitch, rows, k, scale_blocks, scales.step,
                         each, groups, blocks && more ? *blocks : Blocks{}};
    const dim3 grid(groups + (blocks && more) + (copying ? copies->groups : 0), (units + span - 1) / span);
    const ScaleCopies* const some = copying ? copies : nullptr;
    if (dt == WC_BF16) wide ? start_quantize<WC_BF16, 4>(grid, a, some, stream) : start_quantize<WC_BF16, 1>(grid, a, some, stream);
    else if (dt == WC_FP16) wide ? start_quantize<WC_FP16, 4>(grid, a, some, stream) : start_quantize<WC_FP16, 1>(grid, a, some, stream);
    else wide ? start_quantize<WC_FP32, 4>(grid, a, some, stream) : start_quantize<WC_FP32, 1>(grid, a, some, stream);
    if (hipGetLastError() != hipSuccess) return false;
  }
  return true;
}

}  // namespace wc_mx

extern "C" wc_status wc_quantize_mx(const void* dev_x, int32_t x_dtype, uint32_t m, uint32_t k, uint64_t ldx,
                                    uint8_t* dev_q, uint64_t ldq, uint8_t* dev_scale, uint64_t lds,
                                    void* stream) {
  if (!rows_ok(dev_x, x_dtype, m, k, ldx)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!coded_ok(dev_q, ldq, dev_scale, lds, k)) return WC_EINVAL;
  return launch_quantize(dev_x, x_dtype, m, k, ldx, dev_q, ldq,
                         {reinterpret_cast<uint64_t>(dev_scale), uint32_t(lds), 16}, blocks_of(k),
                         reinterpret_cast<hipStream_t>(stream))
             ? WC_OK
             : WC_EHIP;
}

extern "C" wc_status wc_dequantize_mx(const uint8_t* dev_q, uint64_t ldq, const uint8_t* dev_scale,
                                      uint64_t lds, uint32_t m, uint32_t k, void* dev_y, int32_t y_dtype,
                                      uint64_t ldy, void* stream) {
  if (!rows_ok(dev_y, y_dtype, m, k, ldy)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!coded_ok(dev_q, ldq, dev_scale, lds, k)) return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const uint32_t units = (k + 7) / 8, each = units < kThreads ? kThreads / units : 1;
  const bool wide = units > kThreads && m >= 64;
  const uint32_t span = kThreads * (wide ? 4 : 1);
  for (uint32_t first = 0; first < m; first += kLaunchRows) {
    const uint32_t rows = std::min(m - first, kLaunchRows);
    const DequantArgs a = {reinterpret_cast<uint64_t>(dev_q) + first * ldq, ldq,
                           reinterpret_cast<uint64_t>(dev_scale) + first * lds, lds,
                           reinterpret_cast<uint64_t>(dev_y) + first * ldy * size_of(y_dtype), ldy, rows, k, each};
    const dim3 grid((rows + each - 1) / each, (units + span - 1) / span);
    const auto start = [&]<int kType>(std::integral_constant<int, kType>) {
      if (wide) hipLaunchKernelGGL((wc_dequantize_mx_kernel<kType, 4>), grid, dim3(kThreads), 0, st, a);
      else hipLaunchKernelGGL((wc_dequantize_mx_kernel<kType, 1>), grid, dim3(kThreads), 0, st, a);
    };
    if (y_dtype == WC_BF16) start(std::integral_constant<int, WC_BF16>{});
    else if (y_dtype == WC_FP16) start(std::integral_constant<int, WC_FP16>{});
    else start(std::integral_constant<int, WC_FP32>{});
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
  }
  return WC_OK;
}

// Workspace: the sums of the parts of k, copies of the matrices' scales, and then of x's, or x in
// MXFP4.  Rows of x of matmul's own may need copies of their scales too: room for them always.
namespace {
uint64_t x_scales_bytes(const Plan& p, uint32_t m, uint32_t k) {
  return p.kernel < Kernel::kTile64 ? 0 : pad256(own_scales_bytes(m, k));
}
}  // namespace

extern "C" wc_status wc_matmul_mx_workspace_bytes(uint32_t m, uint32_t k, uint32_t n_jobs,
                                                  const wc_mx_job* jobs, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  const Plan p = plan_of(m, k, n_jobs, jobs);
  *bytes = workspace_of(p) + x_scales_bytes(p, m, k);
  return WC_OK;
}

extern "C" wc_status wc_matmul_mx(const uint8_t* dev_q, uint64_t ldq, const uint8_t* dev_scale, uint64_t lds,
                                  uint32_t m, uint32_t k, uint32_t n_jobs, const wc_mx_job* jobs,
                                  void* dev_workspace, uint64_t workspace_bytes, void* stream) {
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!coded_ok(dev_q, ldq, dev_scale, lds, k)) return WC_EINVAL;
  Plan p = plan_of(m, k, n_jobs, jobs);
  p.inside = false;
  if (!workspace_ok(dev_workspace, workspace_bytes, workspace_of(p) + x_scales_bytes(p, m, k))) return WC_EINVAL;
  if (p.kernel >= Kernel::kTile64 && (ldq > (1u << 22) || lds > (1u << 22))) p = Plan{Kernel::kSlim, false, 1, 0, 0, m};  // 32-bit offsets in a tile
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  Scales xs = {reinterpret_cast<uint64_t>(dev_scale), uint32_t(lds), 16};
  if (p.kernel >= Kernel::kTile64) {
    ScaleCopies copies = copies_of(p, k, n_jobs, jobs, dev_workspace);
    if (copies.n && !launch_copies(copies, st)) return WC_EHIP;
    if (!whole_words(dev_scale, lds, k)) {
      xs = own_scales(reinterpret_cast<uint64_t>(dev_workspace) + workspace_of(p), m, k);
      copies.n = copies.groups = 0;
      copies.add(reinterpret_cast<uint64_t>(dev_scale), lds, m, 0, m, k, xs);
      if (!launch_copies(copies, st)) return WC_EHIP;
    }
  }
  return matmul(dev_q, ldq, xs, 0, m, k, n_jobs, jobs, p, dev_workspace, st);
}

extern "C" wc_status wc_linear_mx_workspace_bytes(uint32_t m, uint32_t k, uint32_t n_jobs,
                                                  const wc_mx_job* jobs, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  const Plan p = plan_of(m, k, n_jobs, jobs);
  *bytes = workspace_of(p) + (p.inside ? 0 : quantized_bytes(m, k));
  return WC_OK;
}

extern "C" wc_status wc_linear_mx(const void* dev_x, int32_t x_dtype, uint32_t m, uint32_t k, uint64_t ldx,
                                  uint32_t n_jobs, const wc_mx_job* jobs, void* dev_workspace,
                                  uint64_t workspace_bytes, void* stream) {
  if (!rows_ok(dev_x, x_dtype, m, k, ldx) || !jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  const Plan p = plan_of(m, k, n_jobs, jobs);
  if (!workspace_ok(dev_workspace, workspace_bytes, workspace_of(p) + (p.inside ? 0 : quantized_bytes(m, k))))
    return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (p.inside)
    return matmul(dev_x, ldx * size_of(x_dtype), Scales{}, x_dtype, m, k, n_jobs, jobs, p, nullptr, st);
  uint8_t* q = static_cast<uint8_t*>(dev_workspace) + workspace_of(p);
  const Scales scales = own_scales(reinterpret_cast<uint64_t>(q) + codes_bytes(m, k), m, k);
  const ScaleCopies copies = copies_of(p, k, n_jobs, jobs, dev_workspace);
  if (!launch_quantize(dev_x, x_dtype, m, k, ldx, q, WC_MX_ROW_BYTES(k), scales, uint32_t(groups_of(k)) * 16, st,
                       nullptr, &copies))
    return WC_EHIP;
  return matmul(q, WC_MX_ROW_BYTES(k), scales, 0, m, k, n_jobs, jobs, p, dev_workspace, st);
}
