// wc_i8.hip -- int8 linear layers: wc_quantize_i8, wc_matmul_i8, wc_linear_i8.
#include <algorithm>
#include <cmath>

#include "wc_i8_ring.h"

namespace {

using namespace wc_i8;

struct QuantArgs {
  uint64_t x, ldx, q, scale, limit;
  uint64_t copies;  // three shifted copies of q (Shifted), or none
  uint32_t m, k, step, first;  // first: this launch's
  Blocks blocks;
};

// The table of `Blocks`, by one workgroup.
template <int kThreads>
__device__ __forceinline__ void write_blocks(const Blocks& b, uint32_t (&starts)[kMaxExperts + 1]) {
  const auto offset = [&](uint32_t e) -> uint32_t {
    const int32_t at = global<const int32_t>(b.offsets)[e];
    return at < 0 ? 0u : uint32_t(at) < b.slots ? uint32_t(at) : b.slots;
  };
  for (uint32_t e = threadIdx.x; e < b.experts; e += kThreads) {
    const uint32_t from = offset(e), to = offset(e + 1);
    starts[e + 1] = to > from ? (to - from + b.rows - 1) / b.rows : 0;
  }
  if (threadIdx.x == 0) starts[0] = 0;
  __syncthreads();
  // the blocks before each expert
  if (threadIdx.x < 64) {
    uint32_t before = 0;
    for (uint32_t e0 = 1; e0 <= b.experts; e0 += 64) {
      const uint32_t e = e0 + threadIdx.x;
      uint32_t sum = e <= b.experts ? starts[e] : 0;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const uint32_t v = uint32_t(__shfl_up(int(sum), d));
        if (threadIdx.x >= uint32_t(d)) sum += v;
      }
      if (e <= b.experts) starts[e] = before + sum;
      before += uint32_t(__shfl(int(sum), 63));
    }
  }
  __syncthreads();
  const uint32_t all = min(starts[b.experts], b.most);
  if (threadIdx.x == 0) *global<u32x4>(b.table) = u32x4{all, 0, 0, 0};
  for (uint32_t t = threadIdx.x; t < all; t += kThreads) {
    uint32_t low = 0, high = b.experts;  // starts[low] <= t < starts[high]
    while (high - low > 1) {
      const uint32_t middle = (low + high) / 2;
      (starts[middle] <= t ? low : high) = middle;
    }
    const uint32_t first = offset(low) + (t - starts[low]) * b.rows, end = offset(low + 1);
    global<u32x4>(b.table)[t + 1] = u32x4{low, first, end < first + b.rows ? end : first + b.rows, 0u};
  }
}

// One workgroup a row, which its threads hold in registers in units of eight elements
// (thread t has units t, t + kThreads, ...): read once, its largest magnitude found,
// written as codes: scale = max |x| / 127, code = rint(x * 127 / max |x|).  The bits of |x|
// order as the numbers do, so the maximum is an integer one, which keeps a NaN and does not
// depend on the order.  Bound by memory: 8192 rows of 8192 bf16 43 us, 4.7 TB/s (a large
// copy 4.9); 512 of 28672 fp16 12 us.
template <int kThreads, int kUnits, int kType>
__global__ __launch_bounds__(kThreads) void wc_quantize_i8_kernel(QuantArgs a) {
  constexpr int kWords = kType == WC_FP32 ? 8 : 4;  // to a unit
  __shared__ uint32_t tops[kThreads / 64];
  const uint64_t row = a.first + blockIdx.x;
  if (row == a.m) {
    __shared__ uint32_t starts[kMaxExperts + 1];
    return write_blocks<kThreads>(a.blocks, starts);
  }
  if (a.limit && int32_t(row) >= *global<const int32_t>(a.limit)) return;
  const uint64_t first = a.x + row * a.ldx * (kType == WC_FP32 ? 4 : 2);
  const uint32_t units = uint32_t(WC_I8_ROW_BYTES(a.k)) / 8;
  uint32_t v[kUnits][kWords];
#pragma unroll
  for (int u = 0; u < kUnits; u++) {
    const uint32_t at = (threadIdx.x + u * kThreads) * 8;
    if (kType == WC_FP32 && a.step > 1) {
      const uint32_t each = class_pitch(a.k, a.step);
#pragma unroll
      for (uint32_t i = 0; i < kWords; i++) {
        const uint32_t n = min(at + i, a.k - 1);
        const uint32_t w = global<const uint32_t>(first)[column_at(n, a.step, each)];
        v[u][i] = at + i < a.k ? w : 0u;
      }
    } else if (at + 8 <= a.k) {
      // rows at any element: as the codes of W, loads of any alignment
      const auto p = global<const u32x4u>(first + at * (kType == WC_FP32 ? 4 : 2));
#pragma unroll
      for (int i = 0; i < kWords / 4; i++) {
        const u32x4 w = p[i];
#pragma unroll
        for (int j = 0; j < 4; j++) v[u][4 * i + j] = w[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kWords; i++) v[u][i] = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        if (at + i >= a.k) continue;
        if constexpr (kType == WC_FP32)
          v[u][i] = global<const uint32_t>(first)[at + i];
        else
          v[u][i / 2] |= uint32_t(global<const uint16_t>(first)[at + i]) << (16 * (i % 2));
      }
    }
  }
  const auto value = [&](int u, int i) {
    if constexpr (kType == WC_FP32) return __uint_as_float(v[u][i]);
    const uint32_t h = i % 2 ? v[u][i / 2] >> 16 : v[u][i / 2] & 0xFFFFu;
    return kType == WC_BF16 ? bf16_to_float(h) : fp16_to_float(h);
  };
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < kUnits; u++)
#pragma unroll
    for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(value(u, i)) & 0x7FFFFFFFu);
  top = wave_max(top);
  if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; w++) top = max(top, tops[w]);
  const RowScale s = row_scale(top);
  const auto out = global<u32x2>(a.q + row * units * 8);
  u32x2 codes[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; u++) {
    const uint32_t unit = threadIdx.x + u * kThreads;
    u32x2 c = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; i++) c[i / 4] |= code_of(value(u, i), s.inverse) << (8 * (i % 4));
    codes[u] = c;
    if (unit < units) out[unit] = c;
  }
  if (threadIdx.x == 0) global<float>(a.scale)[row] = s.scale;
  if (!a.copies) return;
  // The shifted copies: every unit at its place and one to three bytes, then zeros to the
  // row's end and before its start.  What passes a row's end are zeros of padding, at the
  // zeros before the next row (the last row's: in the workspace's padding).
  const uint32_t wide = uint32_t(WC_I8_ROW_BYTES(a.k + 3)) / 8;
#pragma unroll
  for (uint32_t by = 1; by <= 3; by++) {
    const uint64_t to = a.copies + ((by - 1) * uint64_t(a.m) + row) * wide * 8 + by;
#pragma unroll
    for (int u = 0; u < kUnits; u++) {
      const uint32_t unit = threadIdx.x + u * kThreads;
      if (unit < units) *global<u32x2u>(to + unit * 8) = codes[u];
    }
    for (uint32_t unit = units + threadIdx.x; unit < wide; unit += kThreads)
      *global<u32x2u>(to + unit * 8) = u32x2{0, 0};
    if (threadIdx.x < by) *global<uint8_t>(to - by + threadIdx.x) = 0;
  }
}

// Rows to a launch: a grid's axis has less than 2^32 threads.
constexpr uint32_t kLaunchRows = 1u << 21;

template <int kThreads, int kUnits>
void start_quantize(int32_t dt, QuantArgs a, hipStream_t stream) {
  const uint32_t rows = a.m + (a.blocks.table != 0);
  for (; a.first < rows; a.first += kLaunchRows) {
    const dim3 grid(std::min(rows - a.first, kLaunchRows)), block(kThreads);
    if (dt == WC_BF16)
      hipLaunchKernelGGL((wc_quantize_i8_kernel<kThreads, kUnits, WC_BF16>), grid, block, 0, stream, a);
    else if (dt == WC_FP16)
      hipLaunchKernelGGL((wc_quantize_i8_kernel<kThreads, kUnits, WC_FP16>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((wc_quantize_i8_kernel<kThreads, kUnits, WC_FP32>), grid, block, 0, stream, a);
  }
}

// Word i of three copies of a row of q, shifted by one, two and three bytes, for codes that
// were quantised by a call of their own.  Bound by memory: 4096 rows of 8191 22 us, 6 TB/s
// read and written; 333 of 5461 6.3, a launch.
__global__ __launch_bounds__(256) void wc_shift_i8_kernel(uint64_t q, uint64_t copies, uint32_t m,
                                                          uint32_t k, uint32_t first) {
  const uint64_t row = first + blockIdx.x;
  const uint32_t words = uint32_t(WC_I8_ROW_BYTES(k)) / 4, wide = uint32_t(WC_I8_ROW_BYTES(k + 3)) / 4;
  const auto from = global<const uint32_t>(q) + row * words;
  for (uint32_t i = threadIdx.x; i < wide; i += 256) {
    const uint32_t low = i && i <= words ? from[i - 1] : 0u, high = i < words ? from[i] : 0u;
    const uint64_t both = uint64_t(high) << 32 | low;
#pragma unroll
    for (uint32_t s = 1; s <= 3; s++)
      global<uint32_t>(copies)[((s - 1) * uint64_t(m) + row) * wide + i] = uint32_t(both >> (32 - 8 * s));
  }
}

struct MatJob {
  uint64_t w, scale, bias, y, ldw, ldy;
  uint64_t part;      // where k is split: its int32 sums, split by split
  uint32_t n, tile0;  // tile0: its first workgroup
  int32_t scale_dtype, bias_dtype, y_dtype;
  uint32_t step;      // classes of rows (class_rows)
};
struct MatArgs {
  uint64_t q, qscale;
  uint64_t copies;  // of q, shifted
  uint64_t x, ldx;  // not quantised yet, where the kernel does that itself
  uint32_t m, k, n_jobs, splits;
  uint32_t sums, reserved;  // sums: results are int32 sums for the join
  MatJob job[kMaxJobs];
};

constexpr int kRowWaves = 8;

// 16 rows of W times 16 kMT rows of x a workgroup, k split over its waves in
// blocks of 128 bytes.  A lane reads 32 bytes in a row of W and of x and feeds
// two v_mfma_i32_16x16x64_i8: the sum runs over k in any order as long as both
// operands agree.  For matrices past the other kernels' 32-bit offsets: each load touches
// sixteen rows, which the L1 cache answers one line at a time (3.2 TB/s of W at best; k =
// 8192, n = 3584, rows 2^20 + 5 bytes apart: 15.6 us up to 16 rows of x, 162 at 512).
template <int kMT>
__global__ __launch_bounds__(64 * kRowWaves) void wc_matmul_i8_rows_kernel(MatArgs a) {
  __shared__ int32_t part[kRowWaves][kMT * 256];
  uint32_t j = 0;
  while (j + 1 < a.n_jobs && blockIdx.x >= a.job[j + 1].tile0) j++;
  const MatJob J = a.job[j];
  const uint32_t n0 = (blockIdx.x - J.tile0) * 16, m0 = blockIdx.y * (16 * kMT);
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t r = lane & 15, g = lane >> 4;
  const uint64_t row_bytes = WC_I8_ROW_BYTES(a.k);
  const auto w = global<const uint8_t>(J.w) + min(n0 + r, J.n - 1) * J.ldw + g * 32;
  global_ptr<const uint8_t> x[kMT];
#pragma unroll
  for (int t = 0; t < kMT; t++)
    x[t] = global<const uint8_t>(a.q) + min(m0 + 16 * t + r, a.m - 1) * row_bytes + g * 32;
  i32x4 acc[kMT];
#pragma unroll
  for (int t = 0; t < kMT; t++) acc[t] = {0, 0, 0, 0};
  const uint32_t whole = a.k / 128, blocks = (a.k + 127) / 128;
  const auto step = [&](uint32_t b, i32x4 w0, i32x4 w1) {
#pragma unroll
    for (int t = 0; t < kMT; t++) {
      const auto p = reinterpret_cast<global_ptr<const i32x4>>(x[t] + uint64_t(b) * 128);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w0, p[0], acc[t], 0, 0, 0);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w1, p[1], acc[t], 0, 0, 0);
    }
  };
  uint32_t b = wave;
  for (; b < whole; b += kRowWaves)
    step(b, load_codes(w + uint64_t(b) * 128, 16), load_codes(w + uint64_t(b) * 128 + 16, 16));
  if (b < blocks) {
    const int32_t left = int32_t(a.k - b * 128) - int32_t(g * 32);
    step(b, load_codes(w + uint64_t(b) * 128, left), load_codes(w + uint64_t(b) * 128 + 16, left - 16));
  }
#pragma unroll
  for (int t = 0; t < kMT; t++)
#pragma unroll
    for (int i = 0; i < 4; i++) part[wave][t * 256 + i * 64 + lane] = acc[t][i];
  __syncthreads();
  // lane l of tile t holds W rows 4 (l div 16) + i of x row l mod 16
  for (uint32_t o = threadIdx.x; o < kMT * 256; o += 64 * kRowWaves) {
    const uint32_t n = n0 + o % 16, m = m0 + o / 16;
    if (n >= J.n || m >= a.m) continue;
    const uint32_t at = o / 256 * 256 + (o % 4) * 64 + (o % 16) / 4 * 16 + o / 16 % 16;
    int32_t sum = 0;
#pragma unroll
    for (int v = 0; v < kRowWaves; v++) sum += part[v][at];
    float y = float(sum) * global<const float>(a.qscale)[m] * load_float(J.scale, J.scale_dtype, n);
    if (J.bias) y += load_float(J.bias, J.bias_dtype, n);
    store_float(J.y, J.y_dtype, m * J.ldy + n, y);
  }
}

// A few rows of x: 16 rows of W a workgroup, bound by reading W.  m = 13, k = 8192, n =
// 28672: 4 waves of 4 stages 43.9 us (5.4 TB/s); 2 waves of 8 stages 52.0, 8 of 4 48.9, 4 of
// 6 50.1; 32 rows of W, 4 waves of 3 stages 56.4; 64 rows 49.4.  At m = 1 40.9 us, 5.75
// TB/s, what a plain streaming kernel reaches.
// kX = 0: x comes as it is, and every workgroup quantises it for itself while its first
// rows of W are on their way.
template <int kX>
using MatRing = Ring<kX, 4, 4>;

template <int kX, int kType>
__global__ __launch_bounds__(MatRing<kX>::kThreads) void wc_matmul_i8_ring_kernel(MatArgs a) {
  using R = MatRing<kX>;
  constexpr uint32_t kRows = kX ? kX : 16;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  __shared__ float scales[16];
  __shared__ uint32_t tops[16];
  uint32_t j = 0;
  while (j + 1 < a.n_jobs && blockIdx.x >= a.job[j + 1].tile0) j++;
  const MatJob J = a.job[j];
  const uint32_t blocks = ((J.n + J.step - 1) / J.step + 15) / 16;  // to a class of rows
  const uint32_t tile = blockIdx.x - J.tile0, first = tile / blocks, r0 = tile % blocks * 16;
  const ClassRows C = class_rows(J.w, J.ldw, J.n, a.k, J.step, first);
  if (r0 >= C.rows) return;
  const uint32_t n_rows = min(16u, C.rows - r0);
  const Shifted X = shifted(a.q, a.copies, a.m, a.k, C.shift);
  const u32x4 wr = rows_rsrc(C.base + r0 * uint64_t(C.pitch), (n_rows - 1) * C.pitch + C.bytes);
  const u32x4 xr = rows_rsrc(X.base, kX ? a.m * X.pitch : 0u);
  uint32_t woff[2], xoff[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    woff[i] = min(8 * i + R::row_of(), n_rows - 1) * C.pitch + R::byte_of(i);
    xoff[i] = min(8 * i + R::row_of(), a.m - 1) * X.pitch + R::byte_of(i);
  }
  i32x4 acc;
  R::product(lds, (C.bytes + kStage - 1) / kStage,
             [&](int i, uint32_t at, uint32_t to) { load_lds(xr, to, xoff[i] + at); },
             [&](int i, uint32_t at, uint32_t to) { load_lds(wr, to, woff[i] + at); }, acc, [&] {
               if constexpr (kX == 0)
                 hold_rows<R::kThreads, kType, 2>(
                     a.m, a.k, [&](uint32_t r) { return a.x + r * a.ldx * (kType == WC_FP32 ? 4 : 2); },
                     lds + R::kLds, scales, tops);
               return typename R::Held{lds + R::kLds, X.pitch, a.m};
             });
  R::gather(lds, acc);
  for (uint32_t o = threadIdx.x; o < 16 * kRows; o += R::kThreads) {
    const uint32_t r = o % 16, m = o / 16, n = first + (r0 + r) * J.step;
    if (r >= n_rows || m >= a.m) continue;
    const float xs = kX ? global<const float>(a.qscale)[m] : scales[m];
    float y = float(R::sum(lds, r, m)) * xs * load_float(J.scale, J.scale_dtype, n);
    if (J.bias) y += load_float(J.bias, J.bias_dtype, n);
    store_float(J.y, J.y_dtype, m * J.ldy + n, y);
  }
}

// y of four neighbouring columns from their sums.
__device__ __forceinline__ void finish(const MatJob& J, uint32_t m, uint32_t n, f32x4 sum, float xs,
                                       const float (&scale)[4], const float (&bias)[4]) {
  const uint64_t at = m * J.ldy + n;
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; i++) v[i] = sum[i] * xs * scale[i] + bias[i];
  if (n + 4 <= J.n) {
    if (J.y_dtype == WC_FP32) {
      *reinterpret_cast<global_ptr<u32x4u>>(global<float>(J.y) + at) = __builtin_bit_cast(u32x4, v);
    } else {
      u32x2 h;
      if (J.y_dtype == WC_BF16)
        h = {floats_to_bf16(v[0], v[1]), floats_to_bf16(v[2], v[3])};
      else
        h = {float_to_fp16(v[0]) | float_to_fp16(v[1]) << 16, float_to_fp16(v[2]) | float_to_fp16(v[3]) << 16};
      *reinterpret_cast<global_ptr<u32x2u>>(global<uint16_t>(J.y) + at) = h;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (n + i < J.n) store_float(J.y, J.y_dtype, at + i, v[i]);
  }
}
// Scales and biases of columns n, n + step, ..
__device__ __forceinline__ void column_scales(const MatJob& J, uint32_t n, uint32_t step,
                                              float (&scale)[4], float (&bias)[4]) {
#pragma unroll
  for (uint32_t i = 0; i < 4; i++) {
    const uint32_t c = min(n + i * step, J.n - 1);
    scale[i] = load_float(J.scale, J.scale_dtype, c);
    bias[i] = J.bias ? load_float(J.bias, J.bias_dtype, c) : 0.0f;
  }
}

// A wave's results to rows of type kType (0: the int32 sums), four neighbours at once
// (kQuads) or each at its own offset `lane`.  Without a branch, so that the reads from LDS
// and the stores of all rows overlap: what is past the last row or column goes nowhere.
template <class T, int kType, bool kQuads>
__device__ __forceinline__ void tile_out(uint8_t* lds, const i32x16 (&acc)[T::kMT][T::kNT], u32x4 to,
                                         uint32_t pitch, uint32_t row0, const uint32_t (&lane)[4],
                                         const float* scales, const float (&scale)[4],
                                         const float (&bias)[4]) {
#pragma unroll
  for (int b = 0; b < T::kMT; b++)
    T::template rows_out<T::kNT * 32>(
        lds,
        [&](int c, int i) { return kType ? float(acc[b][c][i]) : __int_as_float(acc[b][c][i]); },
        [&](uint32_t r, uint32_t, auto get) {
          const uint32_t row = row0 + b * 32 + r;
          f32x4 v = get(0);
          if constexpr (kType != 0) {
            const float xs = scales[row];
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = v[i] * xs * scale[i] + bias[i];
          }
          if constexpr (kType == 0 || kType == WC_FP32) {
            if constexpr (kQuads) {
              store_rows(to, lane[0] + row * pitch, __builtin_bit_cast(u32x4, v));
            } else {
#pragma unroll
              for (int i = 0; i < 4; i++)
                store_rows(to, lane[i] + row * pitch, __float_as_uint(v[i]));
            }
          } else {
            const u32x2 h = kType == WC_BF16
                                ? u32x2{floats_to_bf16(v[0], v[1]), floats_to_bf16(v[2], v[3])}
                                : u32x2{float_to_fp16(v[0]) | float_to_fp16(v[1]) << 16,
                                        float_to_fp16(v[2]) | float_to_fp16(v[3]) << 16};
            if constexpr (kQuads) {
              store_rows(to, lane[0] + row * pitch, h);
            } else {
#pragma unroll
              for (int i = 0; i < 4; i++)
                store_rows(to, lane[i] + row * pitch, uint16_t(h[i / 2] >> (16 * (i % 2))));
            }
          }
          // row after row: all of them at once are more than the registers hold
          if constexpr (!kQuads) __builtin_amdgcn_sched_barrier(0);
        });
}

// y[m][n] = (sum_k x[m][k] W[n][k]) xs[m] ws[n] + b[n], one tile of a job (and one part of
// k) a workgroup; the sums are exact, each result is rounded once to fp32 a factor, and once
// to y's type.
// Bound by the matrix units, and they by the card's power: m = 8192, k = 8192, n = 28672 on
// 256 x 256 1500 us, 2.56 POP/s, the units busy 71 % of the cycles at 1.7 GHz; m = 512, k =
// 28672, n = 8192 on 256 x 128, two parts of k, 108 us, 2.23 POP/s.  The
// larger the tile, the fewer bytes of L2 and LDS a product needs: as large as still leaves
// tiles for all compute units (plan_of).
template <class T>
__global__ __launch_bounds__(T::kThreads) void wc_matmul_i8_tile_kernel(MatArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
  __shared__ float scales[T::kRows];  // of the tile's rows of x
  constexpr uint32_t kBM = T::kRows, kBN = T::kCols;
  uint32_t j = 0;
  while (j + 1 < a.n_jobs && blockIdx.x >= a.job[j + 1].tile0) j++;
  const MatJob J = a.job[j];
  // Classes of the same columns one after another, so that their stores meet in a cache;
  // sums are stored class by class, and class after class their tiles share a copy of x
  // (m = 4096, k = n = 8191: 352 us against 358).
  const uint32_t blocks = ((J.n + J.step - 1) / J.step + kBN - 1) / kBN;
  uint32_t mt, nt;
  if (!tile_at(blockIdx.x - J.tile0, (a.m + kBM - 1) / kBM, blocks * J.step, mt, nt)) return;
  const uint32_t m0 = mt * kBM, m_rows = min(kBM, a.m - m0);
  const uint32_t first = a.sums ? nt / blocks : nt % J.step;
  const uint32_t r0 = (a.sums ? nt % blocks : nt / J.step) * kBN;
  const ClassRows C = class_rows(J.w, J.ldw, J.n, a.k, J.step, first);
  if (r0 >= C.rows) return;
  const uint32_t n_rows = min(kBN, C.rows - r0);
  const Shifted X = shifted(a.q, a.copies, a.m, a.k, C.shift);
  // this workgroup's part of the stages
  const uint32_t all = (C.bytes + kStage - 1) / kStage;
  const uint32_t each = all / a.splits, rest = all % a.splits, part = blockIdx.y;
  const uint32_t s0 = part * each + min(part, rest), stages = each + (part < rest);
  const uint32_t k0 = s0 * kStage;
  const u32x4 xr = rows_rsrc(X.base + m0 * uint64_t(X.pitch) + k0, m_rows * X.pitch - k0);
  const u32x4 wr = rows_rsrc(C.base + r0 * uint64_t(C.pitch) + k0, (n_rows - 1) * C.pitch + C.bytes - k0);
  uint32_t xoff[T::kXLoads], woff[T::kWLoads];
#pragma unroll
  for (int i = 0; i < T::kXLoads; i++) xoff[i] = min(T::row_of(i), m_rows - 1) * X.pitch + T::byte_of();
#pragma unroll
  for (int i = 0; i < T::kWLoads; i++) woff[i] = min(T::row_of(i), n_rows - 1) * C.pitch + T::byte_of();
  // a load among the stores at the end would wait for all stores before it
  const float row_scale = global<const float>(a.qscale)[m0 + min(threadIdx.x, m_rows - 1)];
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  constexpr int kCols = T::kNT * 32;
  const uint32_t column = wave % T::kWN_ * kCols + lane % (kCols / 4) * 4;
  i32x16 acc[T::kMT][T::kNT];
  T::product(lds, stages, m_rows,
             [&](int i, uint32_t s, uint32_t to) { load_lds(xr, to, xoff[i] + s * kStage); },
             [&](int i, uint32_t s, uint32_t to) { load_lds(wr, to, woff[i] + s * kStage); }, acc);
  float scale[4] = {}, bias[4] = {};
  if (!a.sums) column_scales(J, first + (r0 + column) * J.step, J.step, scale, bias);
  if (threadIdx.x < kBM) scales[threadIdx.x] = row_scale;
  __syncthreads();
  const uint32_t row0 = wave / T::kWN_ * (T::kMT * 32);
  // Results that are neighbours in y are stored in groups of four, at any element; class by
  // class, and in the last tile of a row that ends within a group, one by one.  Sums are
  // stored class by class, in whole groups.
  const bool groups = J.step == 1 && n_rows % 4 == 0;
  const auto out = [&]<int kType, int kGroups>(std::integer_sequence<int, kType, kGroups>) {
    constexpr uint32_t kSize = kType == 0 || kType == WC_FP32 ? 4 : 2;
    const uint32_t step = kGroups ? 1 : J.step, sums = row_pitch(J.n, J.step) * 4;
    const uint32_t pitch = kType ? uint32_t(J.ldy) * kSize : sums;
    const uint64_t row = kType ? J.y + m0 * uint64_t(pitch) : J.part + (uint64_t(part) * a.m + m0) * pitch;
    const uint32_t column0 =
        (kType ? first + r0 * J.step : first * class_pitch(J.n, J.step) + r0) * kSize;
    // to the last column of the last row, or of its group of four
    const uint32_t end = ((n_rows - 1) * step + 1) * kSize, group = kGroups ? 4 * kSize : kSize;
    const u32x4 to = rows_rsrc(row + column0, (m_rows - 1) * pitch + (end + group - 1) / group * group);
    uint32_t at[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; i++)
      at[i] = column + (kGroups ? 0 : i) < n_rows ? (column + i) * step * kSize : kNowhere;
    tile_out<T, kType, kGroups>(lds, acc, to, pitch, row0, at, scales, scale, bias);
  };
  const auto of_type = [&]<int kType>(std::integer_sequence<int, kType>) {
    if (groups) out(std::integer_sequence<int, kType, 1>{});
    else out(std::integer_sequence<int, kType, 0>{});
  };
  if (a.sums) out(std::integer_sequence<int, 0, 1>{});
  else if (J.y_dtype == WC_BF16) of_type(std::integer_sequence<int, WC_BF16>{});
  else if (J.y_dtype == WC_FP16) of_type(std::integer_sequence<int, WC_FP16>{});
  else of_type(std::integer_sequence<int, WC_FP32>{});
}

// y from the sums of the parts of k, or, where W's rows are in classes, from one: each sum
// read once, four columns a thread (four of each class a thread, with loads of four, took a
// third longer for want of threads).  512 x 8192 of two parts 11.9 us (3.5 TB/s).
__global__ __launch_bounds__(256) void wc_matmul_i8_join_kernel(MatArgs a) {
  const uint32_t j = blockIdx.z;
  const MatJob J = a.job[j];
  const uint32_t n = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (n >= J.n) return;
  const uint32_t each = class_pitch(J.n, J.step), pitch = J.step * each;
  uint32_t at[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; i++) at[i] = column_at(min(n + i, J.n - 1), J.step, each);
  float scale[4], bias[4];
  column_scales(J, n, 1, scale, bias);
  for (uint32_t m = blockIdx.x; m < a.m; m += gridDim.x) {
    i32x4 sum = {0, 0, 0, 0};
    for (uint32_t p = 0; p < a.splits; p++) {
      const auto row = global<const int32_t>(J.part) + (uint64_t(p) * a.m + m) * pitch;
      if (J.step == 1) {
        sum += *reinterpret_cast<global_ptr<const i32x4>>(row + n);
      } else {
#pragma unroll
        for (int i = 0; i < 4; i++) sum[i] += row[at[i]];
      }
    }
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = float(sum[i]);
    finish(J, m, n, v, global<const float>(a.qscale)[m], scale, bias);
  }
}

bool jobs_ok(uint32_t m, uint32_t k, uint32_t n_jobs, const wc_i8_job* jobs) {
  if (!jobs || n_jobs < 1 || n_jobs > kMaxJobs || k < 1 || k > kMaxK || m > 0x7FFFFFFFu)
    return false;
  uint64_t tiles = 0;
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_i8_job& J = jobs[i];
    if (!J.w || !J.scale || (m && !J.y) || J.n < 1 || J.n > 0x7FFFFFFFu || J.ldw < k || J.ldy < J.n ||
        !float_ok(J.scale_dtype) || !float_ok(J.y_dtype) || (J.bias && !float_ok(J.bias_dtype)))
      return false;
    // nothing an address is worked out from passes 2^62
    if (J.ldw >> 31 || J.ldy >> 31) return false;
    const auto aligned = [](const void* p, uint32_t to) {
      return reinterpret_cast<uintptr_t>(p) % to == 0;
    };
    if (!aligned(J.scale, size_of(J.scale_dtype)) || !aligned(J.y, size_of(J.y_dtype)) ||
        (J.bias && !aligned(J.bias, size_of(J.bias_dtype))))
      return false;
    tiles += (uint64_t(J.n) + 15) / 16;
  }
  return tiles < (1u << 23);  // workgroups of 512 threads: less than 2^32 of them
}

bool rows_ok(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ldx) {
  return float_ok(dt) && k >= 1 && k <= kMaxK && m <= 0x7FFFFFFFu && ldx >= k && !(ldx >> 31) &&
         (m == 0 || (x && reinterpret_cast<uintptr_t>(x) % size_of(dt) == 0));
}

using Tile64 = Tile<64, 64, 1, 2, 4>;
using Tile64Wide = Tile<64, 128, 1, 4, 4>;
using Tile128 = Tile<128, 128, 2, 2, 3>;
using Tile256Half = Tile<256, 128, 4, 2, 3>;
using Tile256 = Tile<256, 256, 2, 4>;

// Quantising in the product's own launch saves a launch (2 us, 4 on the host) and costs
// every workgroup the row: linear at m = 1, k = 4096, n = 6144 9.7 us against 11.2,
// n = 14336 15.4 and 17.0, but k = 8192, n = 28672 45.3 and 43.7; m = 2, k = 4096, n =
// 6144 12.0 and 11.1 (less than the host's time for the launch), k = 8192, n = 8192 20.0
// and 17.4.
constexpr uint64_t kHoldAlways = 4096, kHoldSmall = 8192, kHoldSmallWeights = 32u << 20;

// Which kernel multiplies m rows, and in how many parts of k.
enum class Kernel { kRows, kRing, kTile64, kTile64Wide, kTile128, kTile256Half, kTile256 };
struct Plan {
  Kernel kernel;
  bool hold;        // the kernel can quantise x itself
  bool copies;      // some rows of W do not start with a dword
  uint32_t splits;
  bool sums;        // int32 sums go to the workspace, and are joined
  uint64_t part_bytes;
};
// f(Tile) for the kernel's tile.
template <class F>
void with_tile(Kernel kernel, F f) {
  switch (kernel) {
    case Kernel::kTile64: return f(Tile64{});
    case Kernel::kTile64Wide: return f(Tile64Wide{});
    case Kernel::kTile128: return f(Tile128{});
    case Kernel::kTile256Half: return f(Tile256Half{});
    case Kernel::kTile256: return f(Tile256{});
    default: return;
  }
}
// Workgroups for m rows of x and a matrix of n rows in `step` classes.
uint64_t tiles_of(Kernel kernel, uint32_t m, uint32_t n, uint32_t step) {
  const uint32_t each = (n + step - 1) / step;
  uint64_t tiles = step * ((each + 15) / 16);
  with_tile(kernel, [&](auto t) {
    tiles = uint64_t((m + t.kRows - 1) / t.kRows) * (step * ((each + t.kCols - 1) / t.kCols));
  });
  return tiles;
}

// What a tile's kernel takes, in us, as measured on whole rounds of workgroups (256 of
// them, or 512 where two fit a compute unit): a stage of 128 bytes of k, one workgroup's
// and two's, and all else of a round.  m = 1000, k = n = 8192 (256 tiles of 256 x 128)
// comes to 64.5 and measured 64.5, on 512 tiles of 128 x 128 86 and 83, 128 of 256 x 256
// 109 and 96; m = 512, k = 28672, n = 8192 in two parts of 256 x 128 128 and 124, four of
// 256 x 256 134 and 132; m = 333, k = n = 8192 on 128 x 128 43 and 39; m = 32, k = n =
// 4096 on 64 x 64 13.3 and 13.2, in four parts 12.1 and 12.2.
struct TileCost {
  Kernel kernel;
  double stage, stage_of_two, round;
};
constexpr TileCost kCosts[] = {{Kernel::kTile64, 0.26, 0.34, 5.0},
                               {Kernel::kTile64Wide, 0.36, 0.0, 4.8},
                               {Kernel::kTile128, 0.60, 0.0, 4.5},
                               {Kernel::kTile256Half, 0.90, 0.0, 6.9},
                               {Kernel::kTile256, 1.55, 0.0, 10.2}};
constexpr double kUnits = 256, kJoin = 4.0, kBytesPerUs = 4e6, kReadPerUs = 5e6;
// results of a class of rows, stored two or four apart (1000 x 8191: 30 us more)
constexpr double kStridedPerUs = 2.7e5;

Plan plan_of(uint32_t m, uint32_t k, uint32_t n_jobs, const wc_i8_job* jobs) {
  Plan p{Kernel::kRows, false, false, 1, false, 0};
  // offsets within a tile are 32-bit; the kernel for more reads W at any byte, without copies
  for (uint32_t i = 0; i < n_jobs; i++)
    if (jobs[i].ldw > (1u << 20)) return p;
  uint64_t sums = 0, strided = 0, weights = 0;
  bool narrow = true;
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_i8_job& J = jobs[i];
    weights += uint64_t(J.n) * k;
    narrow = narrow && J.n < (1u << 20) && J.ldy < (1u << 20);
    p.copies = p.copies || J.ldw % 4 || reinterpret_cast<uintptr_t>(J.w) % 4;
    sums += uint64_t(m) * row_pitch(J.n, steps_of(J.ldw)) * 4;
    if (steps_of(J.ldw) > 1) strided += uint64_t(m) * J.n;
  }
  if (m <= 16) {
    p.kernel = Kernel::kRing;
    const uint64_t held = m * WC_I8_ROW_BYTES(k);
    p.hold = !p.copies && k % 8 == 0 &&
             (held <= kHoldAlways || (held <= kHoldSmall && weights <= kHoldSmallWeights));
    return p;
  }
  const uint32_t stages = (k + kStage - 1) / kStage;
  double best = 0;
  for (const TileCost& c : kCosts) {
    uint64_t tiles = 0, threads = 0;
    with_tile(c.kernel, [&](auto t) { threads = t.kThreads; });
    for (uint32_t i = 0; i < n_jobs; i++) tiles += tiles_of(c.kernel, m, jobs[i].n, steps_of(jobs[i].ldw));
    // a grid's axis has less than 2^32 threads
    if (!narrow || tiles * threads >> 32) continue;
    for (uint32_t splits : {1u, 2u, 3u, 4u, 6u, 8u}) {
      if (splits > 1 && stages < 4 * splits) break;
      const double groups = double(tiles * splits);
      const bool two = c.stage_of_two > 0 && groups > kUnits;
      const double rounds = std::ceil(groups / (two ? 2 * kUnits : kUnits));
      double us = rounds * (c.round + (stages + splits - 1) / splits * (two ? c.stage_of_two : c.stage));
      us = std::max(us, double(weights) / kReadPerUs);
      const double join = kJoin + 2.0 * double(sums) * splits / kBytesPerUs;
      const double apart = double(strided) / kStridedPerUs;
      const bool joined = splits > 1 || join < apart;
      us += joined ? join : apart;
      if (best == 0 || us < best) {
        best = us;
        p.kernel = c.kernel;
        p.splits = splits;
        p.sums = joined;
      }
    }
  }
  p.copies = p.copies && p.kernel != Kernel::kRows;
  if (p.sums) p.part_bytes = sums * p.splits;
  return p;
}

// The copies of q, then the sums of the parts of k.
uint64_t workspace_of(const Plan& p, uint32_t m, uint32_t k) {
  return (p.copies ? copies_bytes(m, k) : 0) + p.part_bytes;
}

template <int kX, int kType = 0>
void start_ring(uint32_t tiles, const MatArgs& a, hipStream_t stream) {
  const uint32_t held = kX ? 0 : a.m * uint32_t(WC_I8_ROW_BYTES(a.k));
  hipLaunchKernelGGL((wc_matmul_i8_ring_kernel<kX, kType>), dim3(tiles), dim3(MatRing<kX>::kThreads),
                     MatRing<kX>::kLds + held, stream, a);
}

wc_status matmul(const int8_t* q, const float* scale, uint32_t m, uint32_t k, uint32_t n_jobs,
                 const wc_i8_job* jobs, const Plan& p, void* workspace, hipStream_t stream,
                 const void* x = nullptr, int32_t x_dtype = 0, uint64_t ldx = 0) {
  MatArgs a{};
  if (p.copies) a.copies = reinterpret_cast<uint64_t>(workspace);
  a.x = reinterpret_cast<uint64_t>(x);
  a.ldx = ldx;
  a.q = reinterpret_cast<uint64_t>(q);
  a.qscale = reinterpret_cast<uint64_t>(scale);
  a.k = k;
  a.n_jobs = n_jobs;
  a.splits = p.splits;
  a.sums = p.sums;
  uint32_t tiles = 0, widest = 0;
  uint64_t part = reinterpret_cast<uint64_t>(workspace) + (p.copies ? copies_bytes(m, k) : 0);
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_i8_job& J = jobs[i];
    a.job[i] = {reinterpret_cast<uint64_t>(J.w),    reinterpret_cast<uint64_t>(J.scale),
                reinterpret_cast<uint64_t>(J.bias), reinterpret_cast<uint64_t>(J.y),
                J.ldw, J.ldy, part, J.n, tiles, J.scale_dtype, J.bias_dtype, J.y_dtype,
                p.kernel == Kernel::kRows ? 1u : steps_of(J.ldw)};
    if (p.sums) part += uint64_t(m) * row_pitch(J.n, a.job[i].step) * 4 * p.splits;
    widest = J.n > widest ? J.n : widest;
    tiles += uint32_t(tiles_of(p.kernel, m, J.n, a.job[i].step));
  }
  if (p.kernel == Kernel::kRing) {
    a.m = m;
    if (p.hold && x_dtype == WC_BF16) start_ring<0, WC_BF16>(tiles, a, stream);
    else if (p.hold && x_dtype == WC_FP16) start_ring<0, WC_FP16>(tiles, a, stream);
    else if (p.hold) start_ring<0, WC_FP32>(tiles, a, stream);
    else if (m <= 8) start_ring<8>(tiles, a, stream);
    else start_ring<16>(tiles, a, stream);
    return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
  }
  if (p.kernel != Kernel::kRows) {
    a.m = m;
    const dim3 grid(tiles, p.splits);
    with_tile(p.kernel, [&](auto t) {
      using T = decltype(t);
      hipLaunchKernelGGL(wc_matmul_i8_tile_kernel<T>, grid, dim3(T::kThreads), 0, stream, a);
    });
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
    if (p.sums) {
      const uint32_t rows = m < 65536 ? m : 65536;
      hipLaunchKernelGGL(wc_matmul_i8_join_kernel, dim3(rows, (widest + 1023) / 1024, n_jobs), dim3(256),
                         0, stream, a);
      if (hipGetLastError() != hipSuccess) return WC_EHIP;
    }
    return WC_OK;
  }
  // a grid's second axis holds 65535 blocks of 64 rows
  constexpr uint32_t kSlice = 65535u * 64;
  for (uint32_t m0 = 0; m0 < m; m0 += kSlice) {
    a.m = m - m0 < kSlice ? m - m0 : kSlice;
    if (a.m <= 16)
      hipLaunchKernelGGL((wc_matmul_i8_rows_kernel<1>), dim3(tiles), dim3(64 * kRowWaves), 0, stream, a);
    else
      hipLaunchKernelGGL((wc_matmul_i8_rows_kernel<4>), dim3(tiles, (a.m + 63) / 64),
                         dim3(64 * kRowWaves), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
    a.q += uint64_t(a.m) * WC_I8_ROW_BYTES(k);
    a.qscale += uint64_t(a.m) * 4;
    for (uint32_t i = 0; i < n_jobs; i++)
      a.job[i].y += uint64_t(a.m) * a.job[i].ldy * size_of(a.job[i].y_dtype);
  }
  return WC_OK;
}

}  // namespace

namespace wc_i8 {

bool launch_quantize(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ldx, void* q,
                     float* scale, hipStream_t stream, const int32_t* limit, const Blocks* blocks,
                     void* copies, uint32_t step) {
  const QuantArgs a = {reinterpret_cast<uint64_t>(x), ldx, reinterpret_cast<uint64_t>(q),
                       reinterpret_cast<uint64_t>(scale), reinterpret_cast<uint64_t>(limit),
                       reinterpret_cast<uint64_t>(copies), m, k, step, 0, blocks ? *blocks : Blocks{}};
  // Units of eight elements to a thread: as few threads as hold a row in eight units, but four
  // times as many for few rows of more than 4096, which are latency.  us with 256 threads to a
  // row and with 1024: 16 rows of 4096 bf16 2.26 and 2.64, 256 rows 2.68 and 2.97; 16 of 5000
  // 3.06 and 2.71, 512 4.76 and 4.34, 1024 6.53 and 6.65; 16 of 8192 fp32 2.85 and 2.63, 512
  // 6.08 and 5.61, 700 7.66 and 7.88; 16 of 16384 bf16 3.72 and 3.15, 512 7.98 and 7.45.
  const bool few = m <= 512 && k > 4096;
  if (few && k <= 8192) start_quantize<1024, 1>(dt, a, stream);
  else if (few && k <= 16384) start_quantize<1024, 2>(dt, a, stream);
  else if (k <= 2048) start_quantize<256, 1>(dt, a, stream);
  else if (k <= 4096) start_quantize<256, 2>(dt, a, stream);
  else if (k <= 8192) start_quantize<256, 4>(dt, a, stream);
  else if (k <= 16384) start_quantize<256, 8>(dt, a, stream);
  else if (k <= 32768) start_quantize<1024, 4>(dt, a, stream);
  else start_quantize<1024, 8>(dt, a, stream);
  return hipGetLastError() == hipSuccess;
}

}  // namespace wc_i8

extern "C" wc_status wc_quantize_i8(const void* dev_x, int32_t x_dtype, uint32_t m, uint32_t k,
                                    uint64_t ldx, int8_t* dev_q, float* dev_scale, void* stream) {
  if (!rows_ok(dev_x, x_dtype, m, k, ldx)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!dev_q || !dev_scale || reinterpret_cast<uintptr_t>(dev_q) % 16 ||
      reinterpret_cast<uintptr_t>(dev_scale) % 4)
    return WC_EINVAL;
  return launch_quantize(dev_x, x_dtype, m, k, ldx, dev_q, dev_scale,
                         reinterpret_cast<hipStream_t>(stream))
             ? WC_OK
             : WC_EHIP;
}

extern "C" wc_status wc_matmul_i8_workspace_bytes(uint32_t m, uint32_t k, uint32_t n_jobs,
                                                  const wc_i8_job* jobs, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  *bytes = workspace_of(plan_of(m, k, n_jobs, jobs), m, k);
  return WC_OK;
}

namespace {
bool workspace_ok(const void* p, uint64_t bytes, uint64_t need) {
  return need == 0 || (p && reinterpret_cast<uintptr_t>(p) % 256 == 0 && bytes >= need);
}
}  // namespace

extern "C" wc_status wc_matmul_i8(const int8_t* dev_q, const float* dev_scale, uint32_t m,
                                  uint32_t k, uint32_t n_jobs, const wc_i8_job* jobs,
                                  void* dev_workspace, uint64_t workspace_bytes, void* stream) {
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!dev_q || !dev_scale || reinterpret_cast<uintptr_t>(dev_q) % 16 ||
      reinterpret_cast<uintptr_t>(dev_scale) % 4)
    return WC_EINVAL;
  Plan p = plan_of(m, k, n_jobs, jobs);
  p.hold = false;
  if (!workspace_ok(dev_workspace, workspace_bytes, workspace_of(p, m, k))) return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  for (uint32_t first = 0; p.copies && first < m; first += kLaunchRows) {
    hipLaunchKernelGGL(wc_shift_i8_kernel, dim3(std::min(m - first, kLaunchRows)), dim3(256), 0, st,
                       reinterpret_cast<uint64_t>(dev_q), reinterpret_cast<uint64_t>(dev_workspace), m, k,
                       first);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
  }
  return matmul(dev_q, dev_scale, m, k, n_jobs, jobs, p, dev_workspace, st);
}

extern "C" wc_status wc_linear_i8_workspace_bytes(uint32_t m, uint32_t k, uint32_t n_jobs,
                                                  const wc_i8_job* jobs, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  const Plan p = plan_of(m, k, n_jobs, jobs);
  // nothing where the product's kernel quantises x itself
  if (!p.hold)
    *bytes = pad256(uint64_t(m) * WC_I8_ROW_BYTES(k)) + pad256(uint64_t(m) * 4) + workspace_of(p, m, k);
  return WC_OK;
}

extern "C" wc_status wc_linear_i8(const void* dev_x, int32_t x_dtype, uint32_t m, uint32_t k,
                                  uint64_t ldx, uint32_t n_jobs, const wc_i8_job* jobs,
                                  void* dev_workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (!rows_ok(dev_x, x_dtype, m, k, ldx) ||
      wc_linear_i8_workspace_bytes(m, k, n_jobs, jobs, &need) != WC_OK)
    return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!workspace_ok(dev_workspace, workspace_bytes, need)) return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  int8_t* q = static_cast<int8_t*>(dev_workspace);
  float* scale = reinterpret_cast<float*>(q + pad256(uint64_t(m) * WC_I8_ROW_BYTES(k)));
  void* parts = reinterpret_cast<uint8_t*>(scale) + pad256(uint64_t(m) * 4);
  const Plan p = plan_of(m, k, n_jobs, jobs);
  if (!p.hold && !launch_quantize(dev_x, x_dtype, m, k, ldx, q, scale, st, nullptr, nullptr,
                                  p.copies ? parts : nullptr))
    return WC_EHIP;
  return matmul(q, scale, m, k, n_jobs, jobs, p, parts, st, dev_x, x_dtype, ldx);
}
