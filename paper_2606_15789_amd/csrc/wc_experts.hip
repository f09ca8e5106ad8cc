// wc_experts.hip -- the feed-forward of a mixture layer with int8 experts:
// wc_experts_i8.
//
// For a token t with experts e_j of weights g_j:
//   h_j = silu(G_ej x_t) * (U_ej x_t),  y_t = sum_j g_j D_ej h_j,
// each product of int8 codes: x_t and every h_j quantised by row, sums exact in int32, then
// times the row's and the column's scale in fp32.  The places of the router's order are cut
// into blocks of one expert's places; a workgroup multiplies one block by some of the
// expert's rows.  Two products with a quantisation of h between them (its scale needs all of
// a row), each expert's result stored by slot, and a token's slots added in their order, so
// a result does not depend on which workgroups ran first.
#include "wc_i8_ring.h"

namespace {

using namespace wc_i8;

constexpr int kRowWaves = 8;

struct Bank {
  uint64_t w, scale, stride;
  int32_t scale_dtype;
};
struct ExpertArgs {
  uint64_t table, order, ids, weights;
  uint64_t x, ldx;
  uint64_t xq, xscale;    // quantised x, by token
  uint64_t h;             // fp32, by place in the order
  uint64_t hq, hscale;    // quantised h
  uint64_t xcopies, hcopies;  // both shifted, where rows of the matrices need it
  uint64_t out;           // experts' results, fp32, by slot
  uint64_t y, ldy;
  uint32_t tokens, k, experts, hidden, ffn, slots;
  uint32_t blocks;        // upper bound of the blocks of places
  uint32_t up_step, down_step;  // classes of the columns of h, of the results (row_pitch)
  int32_t dtype;
  Bank gate, up, down;
};

// The block-th block of places (Blocks): false past the last.
struct Place {
  uint32_t expert, first, last;
};
__device__ __forceinline__ uint32_t block_count(const ExpertArgs& a) {
  return __builtin_amdgcn_readfirstlane(*global<const uint32_t>(a.table));
}
__device__ __forceinline__ Place block_at(const ExpertArgs& a, uint32_t block) {
  const u32x4 v = global<const u32x4>(a.table)[block + 1];
  return {uint32_t(__builtin_amdgcn_readfirstlane(v[0])), uint32_t(__builtin_amdgcn_readfirstlane(v[1])),
          uint32_t(__builtin_amdgcn_readfirstlane(v[2]))};
}

__device__ __forceinline__ uint32_t slot_at(const ExpertArgs& a, uint32_t place) {
  return min(uint32_t(max(global<const int32_t>(a.order)[place], 0)), a.slots - 1);
}

// g / (1 + exp(-g)), with an exponential of 1 ulp and a rounded division.  The unit's own
// exponential, of g log2(e), and reciprocal would be off by 2^-23 (3 + |g|) and save a
// fortieth: 2612 us for 2677 at 4096 tokens of 8 experts of 6144 x 16384, 2 each, 45.0 for
// 46.1 at 203 of 7 of 1537 x 2051, 3 each.
__device__ __forceinline__ float silu(float g) { return g / (1.0f + expf(-g)); }

// 16 columns of an expert's result for up to 16 of its rows: kMats products that
// share their rows (gate and up, or down alone), k split over the waves.  For matrices whose
// rows start at other bytes of a dword than the copies of x, or than each other: each load
// touches sixteen rows, which the L1 cache answers one line at a time.  32 tokens, 2 each, of
// 8 experts of 4096 x 14336, gate a byte on: 292 us up (3.2 TB/s) and 113 down, 418 in all
// against 281 on tiles; 256 tokens of 2048 x 1408 120 against 37.
template <int kMats>
__device__ __forceinline__ void expert_product(global_ptr<const uint8_t> x, const uint64_t (&mats)[2],
                                               uint32_t n, uint32_t k,
                                               int32_t (&part)[kRowWaves][kMats * 256]) {
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, g = lane >> 4;
  global_ptr<const uint8_t> w[kMats];
  i32x4 acc[kMats];
#pragma unroll
  for (int t = 0; t < kMats; t++) {
    w[t] = global<const uint8_t>(mats[t]) + uint64_t(n) * k + g * 32;
    acc[t] = {0, 0, 0, 0};
  }
  const uint32_t whole = k / 128, blocks = (k + 127) / 128;
  const auto step = [&](uint32_t b, int32_t left) {
    const auto p = reinterpret_cast<global_ptr<const i32x4>>(x + g * 32 + uint64_t(b) * 128);
    const i32x4 x0 = p[0], x1 = p[1];
#pragma unroll
    for (int t = 0; t < kMats; t++) {
      const i32x4 w0 = load_codes(w[t] + uint64_t(b) * 128, left);
      const i32x4 w1 = load_codes(w[t] + uint64_t(b) * 128 + 16, left - 16);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w0, x0, acc[t], 0, 0, 0);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w1, x1, acc[t], 0, 0, 0);
    }
  };
  uint32_t b = wave;
  for (; b < whole; b += kRowWaves) step(b, 32);
  if (b < blocks) step(b, int32_t(k - b * 128) - int32_t(g * 32));
#pragma unroll
  for (int t = 0; t < kMats; t++)
#pragma unroll
    for (int i = 0; i < 4; i++) part[wave][t * 256 + i * 64 + lane] = acc[t][i];
  __syncthreads();
}

template <int kMats>
__device__ __forceinline__ int32_t summed(const int32_t (&part)[kRowWaves][kMats * 256], int t,
                                          uint32_t n, uint32_t m) {
  const uint32_t at = uint32_t(t) * 256 + n % 4 * 64 + n / 4 * 16 + m;
  int32_t sum = 0;
#pragma unroll
  for (int v = 0; v < kRowWaves; v++) sum += part[v][at];
  return sum;
}

// h = silu(gate x) * (up x) of 16 columns for up to 16 places of the order.
__global__ __launch_bounds__(64 * kRowWaves) void wc_experts_up_kernel(ExpertArgs a) {
  __shared__ int32_t part[kRowWaves][2 * 256];
  if (blockIdx.x >= block_count(a)) return;
  const auto [e, first, last] = block_at(a, blockIdx.x);
  const uint32_t n0 = blockIdx.y * 16, r = threadIdx.x % 16;
  const uint32_t token = slot_at(a, min(first + r, last - 1)) / a.k;
  const uint64_t mats[2] = {a.gate.w + e * a.gate.stride, a.up.w + e * a.up.stride};
  expert_product<2>(global<const uint8_t>(a.xq) + token * WC_I8_ROW_BYTES(a.hidden), mats,
                    min(n0 + r, a.ffn - 1), a.hidden, part);
  for (uint32_t o = threadIdx.x; o < 256; o += 64 * kRowWaves) {
    const uint32_t n = n0 + o % 16, place = first + o / 16;
    if (n >= a.ffn || place >= last) continue;
    const float xs = global<const float>(a.xscale)[slot_at(a, place) / a.k];
    const uint64_t at = uint64_t(e) * a.ffn + n;
    const float g = float(summed<2>(part, 0, o % 16, o / 16)) * xs *
                    load_float(a.gate.scale, a.gate.scale_dtype, at);
    const float u = float(summed<2>(part, 1, o % 16, o / 16)) * xs *
                    load_float(a.up.scale, a.up.scale_dtype, at);
    global<float>(a.h)[uint64_t(place) * row_pitch(a.ffn, 1) + n] = silu(g) * u;
  }
}

// down(h) of 16 columns for up to 16 places, stored by slot.
__global__ __launch_bounds__(64 * kRowWaves) void wc_experts_down_kernel(ExpertArgs a) {
  __shared__ int32_t part[kRowWaves][256];
  if (blockIdx.x >= block_count(a)) return;
  const auto [e, first, last] = block_at(a, blockIdx.x);
  const uint32_t n0 = blockIdx.y * 16, r = threadIdx.x % 16;
  const uint64_t mats[2] = {a.down.w + e * a.down.stride, 0};
  expert_product<1>(global<const uint8_t>(a.hq) + min(first + r, last - 1) * WC_I8_ROW_BYTES(a.ffn),
                    mats, min(n0 + r, a.hidden - 1), a.ffn, part);
  for (uint32_t o = threadIdx.x; o < 256; o += 64 * kRowWaves) {
    const uint32_t n = n0 + o % 16, place = first + o / 16;
    if (n >= a.hidden || place >= last) continue;
    global<float>(a.out)[uint64_t(slot_at(a, place)) * row_pitch(a.hidden, 1) + n] =
        float(summed<1>(part, 0, o % 16, o / 16)) * global<const float>(a.hscale)[place] *
        load_float(a.down.scale, a.down.scale_dtype, uint64_t(e) * a.hidden + n);
  }
}

// The same from rings of whole lines, for few rows to an expert: bound by reading the
// experts that were hit.  The sixteen rows of a product's W are eight of gate and the same
// eight of up.  16 experts of 2048 x 1024, 8 tokens 4 each: 13.8 us up and 9.0 down, 33 with
// the three launches around them: latencies, at 2.7 TB/s of the weights hit.
template <int kX>
using ExpertRing = Ring<kX, 4, 4>;

template <int kX>
__global__ __launch_bounds__(ExpertRing<kX>::kThreads) void wc_experts_up_ring_kernel(ExpertArgs a) {
  using R = ExpertRing<kX>;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[R::kLds];
  if (blockIdx.x >= block_count(a)) return;
  const auto [e, first, last] = block_at(a, blockIdx.x);
  const uint32_t k = a.hidden, step = a.up_step, blocks = ((a.ffn + step - 1) / step + 7) / 8;
  const uint32_t class0 = blockIdx.y / blocks, r0 = blockIdx.y % blocks * 8;
  const ClassRows G = class_rows(a.gate.w + e * a.gate.stride, k, a.ffn, k, step, class0);
  const ClassRows U = class_rows(a.up.w + e * a.up.stride, k, a.ffn, k, step, class0);
  if (r0 >= G.rows) return;
  const uint32_t n_rows = min(8u, G.rows - r0);
  const Shifted X = shifted(a.xq, a.xcopies, a.tokens, k, G.shift);
  const u32x4 gr = rows_rsrc(G.base + r0 * uint64_t(G.pitch), (n_rows - 1) * G.pitch + G.bytes);
  const u32x4 ur = rows_rsrc(U.base + r0 * uint64_t(G.pitch), (n_rows - 1) * G.pitch + G.bytes);
  const u32x4 xr = rows_rsrc(X.base, a.tokens * X.pitch);
  const uint32_t row = min(R::row_of(), n_rows - 1) * G.pitch;
  const uint32_t woff[2] = {row + R::byte_of(0), row + R::byte_of(1)};
  uint32_t xoff[kX / 8];
#pragma unroll
  for (int i = 0; i < kX / 8; i++)
    xoff[i] = slot_at(a, min(first + 8 * i + R::row_of(), last - 1)) / a.k * X.pitch + R::byte_of(i);
  i32x4 acc;
  R::product(lds, (G.bytes + kStage - 1) / kStage,
             [&](int i, uint32_t at, uint32_t to) { load_lds(xr, to, xoff[i] + at); },
             [&](int i, uint32_t at, uint32_t to) { load_lds(i ? ur : gr, to, woff[i] + at); }, acc,
             [] { return typename R::Held{}; });
  R::gather(lds, acc);
  for (uint32_t o = threadIdx.x; o < 8 * kX; o += R::kThreads) {
    const uint32_t r = o % 8, n = class0 + (r0 + r) * step, place = first + o / 8;
    if (r >= n_rows || place >= last) continue;
    const float xs = global<const float>(a.xscale)[slot_at(a, place) / a.k];
    const uint64_t at = uint64_t(e) * a.ffn + n;
    const float g = float(R::sum(lds, r, o / 8)) * xs * load_float(a.gate.scale, a.gate.scale_dtype, at);
    const float u = float(R::sum(lds, 8 + r, o / 8)) * xs * load_float(a.up.scale, a.up.scale_dtype, at);
    global<float>(a.h)[uint64_t(place) * row_pitch(a.ffn, step) + class0 * class_pitch(a.ffn, step) + r0 + r] =
        silu(g) * u;
  }
}

template <int kX>
__global__ __launch_bounds__(ExpertRing<kX>::kThreads) void wc_experts_down_ring_kernel(ExpertArgs a) {
  using R = ExpertRing<kX>;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[R::kLds];
  if (blockIdx.x >= block_count(a)) return;
  const auto [e, first, last] = block_at(a, blockIdx.x);
  const uint32_t k = a.ffn, step = a.down_step, blocks = ((a.hidden + step - 1) / step + 15) / 16;
  const uint32_t class0 = blockIdx.y / blocks, r0 = blockIdx.y % blocks * 16;
  const ClassRows C = class_rows(a.down.w + e * a.down.stride, k, a.hidden, k, step, class0);
  if (r0 >= C.rows) return;
  const uint32_t n_rows = min(16u, C.rows - r0), m_rows = last - first;
  const Shifted X = shifted(a.hq, a.hcopies, a.slots, k, C.shift);
  const u32x4 wr = rows_rsrc(C.base + r0 * uint64_t(C.pitch), (n_rows - 1) * C.pitch + C.bytes);
  const u32x4 xr = rows_rsrc(X.base + uint64_t(first) * X.pitch, m_rows * X.pitch);
  uint32_t woff[2], xoff[kX / 8];
#pragma unroll
  for (int i = 0; i < 2; i++) woff[i] = min(8 * i + R::row_of(), n_rows - 1) * C.pitch + R::byte_of(i);
#pragma unroll
  for (int i = 0; i < kX / 8; i++) xoff[i] = min(8 * i + R::row_of(), m_rows - 1) * X.pitch + R::byte_of(i);
  i32x4 acc;
  R::product(lds, (C.bytes + kStage - 1) / kStage,
             [&](int i, uint32_t at, uint32_t to) { load_lds(xr, to, xoff[i] + at); },
             [&](int i, uint32_t at, uint32_t to) { load_lds(wr, to, woff[i] + at); }, acc,
             [] { return typename R::Held{}; });
  R::gather(lds, acc);
  for (uint32_t o = threadIdx.x; o < 16 * kX; o += R::kThreads) {
    const uint32_t r = o % 16, n = class0 + (r0 + r) * step, place = first + o / 16;
    if (r >= n_rows || place >= last) continue;
    global<float>(a.out)[uint64_t(slot_at(a, place)) * row_pitch(a.hidden, step) +
                         class0 * class_pitch(a.hidden, step) + r0 + r] =
        float(R::sum(lds, r, o / 16)) * global<const float>(a.hscale)[place] *
        load_float(a.down.scale, a.down.scale_dtype, uint64_t(e) * a.hidden + n);
  }
}

// A few tokens: each slot by itself, with its expert's rows of W read for it alone, in
// two launches.  Every workgroup quantises the row of x, then of h, that it multiplies,
// while its first rows of W are on their way; a token's slots are added where its
// columns' sums meet.  64 experts of 2048 x 1408, one token of 6: 10.0 and 10.2 us
// for 35 and 17 MB, a chain of latencies: the ids, x, its maximum, W, the sums.
using SlotRing = Ring<0, 4, 4>;
using DownSlotRing = Ring<0, 8, 3>;

template <int kType>
__global__ __launch_bounds__(SlotRing::kThreads) void wc_experts_up_slot_kernel(ExpertArgs a) {
  using R = SlotRing;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  __shared__ float scale[1];
  __shared__ uint32_t tops[1];
  const uint32_t slot = blockIdx.y;
  const int32_t id = global<const int32_t>(a.ids)[slot];
  if (id < 0) return;
  const uint32_t e = min(uint32_t(id), a.experts - 1);
  const uint32_t n0 = blockIdx.x * 8, n_rows = min(8u, a.ffn - n0), k = a.hidden;
  const uint32_t row_bytes = uint32_t(WC_I8_ROW_BYTES(k));
  const u32x4 gr = rows_rsrc(a.gate.w + e * a.gate.stride + uint64_t(n0) * k, n_rows * k);
  const u32x4 ur = rows_rsrc(a.up.w + e * a.up.stride + uint64_t(n0) * k, n_rows * k);
  const uint32_t row = min(R::row_of(), n_rows - 1) * k;
  const uint32_t woff[2] = {row + R::byte_of(0), row + R::byte_of(1)};
  i32x4 acc;
  R::product(lds, row_bytes / kStage, [](int, uint32_t, uint32_t) {},
             [&](int i, uint32_t at, uint32_t to) { load_lds(i ? ur : gr, to, woff[i] + at); }, acc, [&] {
               hold_rows<R::kThreads, kType, 2>(
                   1, k, [&](uint32_t) { return a.x + slot / a.k * a.ldx * (kType == WC_FP32 ? 4 : 2); },
                   lds + R::kLds, scale, tops);
               return R::Held{lds + R::kLds, row_bytes, 1};
             });
  R::gather(lds, acc);
  const uint32_t n = n0 + threadIdx.x;
  if (threadIdx.x < 8 && n < a.ffn) {
    const uint64_t at = uint64_t(e) * a.ffn + n;
    const float g = float(R::sum(lds, threadIdx.x, 0)) * scale[0] * load_float(a.gate.scale, a.gate.scale_dtype, at);
    const float u = float(R::sum(lds, 8 + threadIdx.x, 0)) * scale[0] * load_float(a.up.scale, a.up.scale_dtype, at);
    global<float>(a.h)[uint64_t(slot) * row_pitch(a.ffn, 1) + n] = silu(g) * u;
  }
}

constexpr uint32_t kSlots = 32;  // at most, of a token here

__global__ __launch_bounds__(DownSlotRing::kThreads) void wc_experts_down_slot_kernel(ExpertArgs a) {
  using R = DownSlotRing;
  constexpr uint32_t kW = R::kThreads / 64, kS = R::kWave / R::kStageBytes;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  __shared__ float scales[kSlots];
  __shared__ uint32_t tops[kSlots];
  const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t first = blockIdx.y * a.k, n0 = blockIdx.x * 16, n_rows = min(16u, a.hidden - n0);
  const uint32_t k = a.ffn, row_bytes = uint32_t(WC_I8_ROW_BYTES(k)), blocks = row_bytes / kStage;
  // sums by slot, wave and column, after the rings and the rows of h
  int32_t* const part = reinterpret_cast<int32_t*>(lds + R::kLds + a.k * row_bytes);
  for (uint32_t i = threadIdx.x; i < a.k * kW * 16; i += R::kThreads) part[i] = 0;
  uint32_t woff[2];
#pragma unroll
  for (int i = 0; i < 2; i++) woff[i] = min(8 * i + R::row_of(), n_rows - 1) * k + R::byte_of(i);
  uint8_t* const mine = lds + wave * R::kWave;
  const uint32_t base = __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>(
      (__attribute__((address_space(3))) uint8_t*)mine)));
  // lane j: the expert of slot j
  int32_t ids = lane < a.k ? global<const int32_t>(a.ids)[first + lane] : -1;
  asm volatile("" : "+v"(ids));  // here, before loads that should not be waited for
  const auto id_of = [&](uint32_t s) { return __builtin_amdgcn_readlane(ids, int(s)); };
  const uint32_t used = uint32_t(__ballot(ids >= 0));
  const auto start = [&](const SlotBlock& at, uint32_t place) {
    const uint32_t e = min(uint32_t(id_of(at.slot())), a.experts - 1);
    const u32x4 wr = rows_rsrc(a.down.w + e * a.down.stride + uint64_t(n0) * k, n_rows * k);
    const uint32_t to = base + place * R::kStageBytes;
#pragma unroll
    for (int i = 0; i < 2; i++) load_lds(wr, to + i * 1024, woff[i] + at.block * kStage);
  };
  // This wave's blocks of k: every kW-th of all the used slots' blocks.
  SlotBlock ahead = {used, wave};
  settle_block(ahead, blocks);
  SlotBlock here = ahead;
  uint32_t begun = 0;
#pragma unroll
  for (uint32_t j = 0; j < kS - 1; j++)
    if (ahead.left) {
      start(ahead, j);
      ahead.block += kW;
      settle_block(ahead, blocks);
      begun++;
    }
  hold_rows<R::kThreads, WC_FP32, 3>(
      a.k, k, [&](uint32_t r) { return a.h + uint64_t(first + r) * row_pitch(k, 1) * 4; }, lds + R::kLds,
      scales, tops);
  const uint32_t r = lane % 16;
  const uint32_t w0 = r * kStage + ((lane / 16) ^ R::turn(r)) * 16;
  const uint32_t w1 = r * kStage + ((lane / 16 + 4) ^ R::turn(r)) * 16;
  i32x4 acc = {0, 0, 0, 0};
  const auto leave = [&](uint32_t slot) {
    // every column of the products is the one row of h
    if (r == 0)
#pragma unroll
      for (int i = 0; i < 4; i++) part[(slot * kW + wave) * 16 + lane / 16 * 4 + i] = acc[i];
  };
  uint32_t place = 0, done = 0, slot = 0;
  while (here.left) {
    if (ahead.left) {
      start(ahead, place ? place - 1 : kS - 1);
      ahead.block += kW;
      settle_block(ahead, blocks);
      begun++;
    }
    R::wait_for<kS - 1>(min(begun - 1 - done, kS - 1));
    const uint8_t* s = mine + place * R::kStageBytes;
    const uint32_t now = here.slot();
    const uint8_t* x = lds + R::kLds + now * row_bytes + here.block * kStage;
    if (now != slot) {
      if (done) leave(slot);
      acc = {0, 0, 0, 0};
      slot = now;
    }
    const uint32_t turn = now % 8;
    const i32x4 a0 = *reinterpret_cast<const i32x4*>(x + ((lane / 16) ^ turn) * 16);
    const i32x4 a1 = *reinterpret_cast<const i32x4*>(x + ((lane / 16 + 4) ^ turn) * 16);
    const i32x4 b0 = *reinterpret_cast<const i32x4*>(s + w0);
    const i32x4 b1 = *reinterpret_cast<const i32x4*>(s + w1);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b0, a0, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b1, a1, acc, 0, 0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    place = place + 1 < kS ? place + 1 : 0;
    done++;
    here.block += kW;
    settle_block(here, blocks);
  }
  if (done) leave(slot);
  __syncthreads();
  const uint32_t n = n0 + threadIdx.x;
  if (threadIdx.x < 16 && n < a.hidden) {
    float sum = 0.0f;
    for (uint32_t j = 0; j < a.k; j++) {
      const int32_t id = id_of(j);
      float v = 0.0f;
      if (id >= 0) {
        int32_t p = 0;
#pragma unroll
        for (uint32_t w = 0; w < kW; w++) p += part[(j * kW + w) * 16 + threadIdx.x];
        v = float(p) * scales[j] *
            load_float(a.down.scale, a.down.scale_dtype, uint64_t(min(uint32_t(id), a.experts - 1)) * a.hidden + n);
      }
      sum += global<const float>(a.weights)[first + j] * v;
    }
    store_float(a.y, a.dtype, blockIdx.y * a.ldy + n, sum);
  }
}

// The same on tiles through LDS.  A wave's columns of W are 32 of gate and the same 32
// of up, so that both products of a value of h meet in one lane.  With few rows to an
// expert bound by reading W: 8 experts of 6144 x 16384, 32 tokens 2 each, 287 us up (5.6
// TB/s) and 159 down (5.1).  With many by the matrix units: 4096 tokens, 1630 us up (2.0
// POP/s, the units busy 52 % of the cycles at 1.87 GHz; a stage of 128 bytes takes 1.65 us,
// a tile's 48 of them 79 of its some 91) and 855 down (1.9; 864 tiles are 3.4 rounds of workgroups).
template <class T>
__global__ __launch_bounds__(T::kThreads) void wc_experts_up_tile_kernel(ExpertArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
  __shared__ float scales[T::kRows];  // of the tile's rows of x
  static_assert(T::kNT == 2 && T::kRows <= T::kThreads);
  constexpr uint32_t kBM = T::kRows, kCols = T::kWN_ * 32;
  const uint32_t k = a.hidden, step = a.up_step;
  const uint32_t blocks = ((a.ffn + step - 1) / step + kCols - 1) / kCols;
  uint32_t mt, nt;
  if (!tile_at(blockIdx.x, block_count(a), blocks * step, mt, nt)) return;
  const auto [e, first, last] = block_at(a, mt);
  const uint32_t class0 = nt / blocks, r0 = nt % blocks * kCols;
  const ClassRows G = class_rows(a.gate.w + e * a.gate.stride, k, a.ffn, k, step, class0);
  const ClassRows U = class_rows(a.up.w + e * a.up.stride, k, a.ffn, k, step, class0);
  if (r0 >= G.rows) return;
  const uint32_t n_rows = min(kCols, G.rows - r0);
  const Shifted X = shifted(a.xq, a.xcopies, a.tokens, k, G.shift);
  const u32x4 xr = rows_rsrc(X.base, a.tokens * X.pitch);
  uint32_t xoff[T::kXLoads], woff[T::kWLoads];
#pragma unroll
  for (int i = 0; i < T::kXLoads; i++)
    xoff[i] = slot_at(a, min(first + T::row_of(i), last - 1)) / a.k * X.pitch + T::byte_of();
  // a load among the stores at the end would wait for all stores before it
  const float row_scale =
      global<const float>(a.xscale)[slot_at(a, min(first + threadIdx.x % kBM, last - 1)) / a.k];
  // W row r of the tile: column r / 64 * 32 + r mod 32 of gate (r mod 64 < 32) or of up
  u32x4 wr[T::kWLoads];
#pragma unroll
  for (int i = 0; i < T::kWLoads; i++) {
    const uint32_t r = T::row_of(i);
    wr[i] = rows_rsrc((T::first_row(i) & 32 ? U.base : G.base) + r0 * uint64_t(G.pitch),
                      (n_rows - 1) * G.pitch + G.bytes);
    woff[i] = min(r / 64 * 32 + r % 32, n_rows - 1) * G.pitch + T::byte_of();
  }
  i32x16 acc[T::kMT][2];
  T::product(lds, (G.bytes + kStage - 1) / kStage, last - first,
             [&](int i, uint32_t s, uint32_t to) { load_lds(xr, to, xoff[i] + s * kStage); },
             [&](int i, uint32_t s, uint32_t to) { load_lds(wr[i], to, woff[i] + s * kStage); }, acc);
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t column = wave % T::kWN_ * 32 + lane % 8 * 4, row0 = wave / T::kWN_ * (T::kMT * 32);
  float gs[4], us[4];
  const uint32_t out =
      column < n_rows ? (class0 * class_pitch(a.ffn, step) + r0 + column) * 4 : kNowhere;
#pragma unroll
  for (uint32_t i = 0; i < 4; i++) {
    const uint32_t n = class0 + (r0 + column + i) * step;
    const uint64_t at = uint64_t(e) * a.ffn + min(n, a.ffn - 1);
    gs[i] = load_float(a.gate.scale, a.gate.scale_dtype, at);
    us[i] = load_float(a.up.scale, a.up.scale_dtype, at);
  }
  if (threadIdx.x < kBM) scales[threadIdx.x] = row_scale;
  __syncthreads();
  // no branches: rows and columns past the last go nowhere
  const uint32_t pitch = row_pitch(a.ffn, step) * 4;
  const u32x4 to = rows_rsrc(a.h + first * uint64_t(pitch), (last - first) * pitch);
#pragma unroll
  for (int b = 0; b < T::kMT; b++)
    T::template rows_out<32>(
        lds, [&](int c, int i) { return float(acc[b][c][i]); },
        [&](uint32_t r, uint32_t, auto get) {
          const uint32_t row = row0 + b * 32 + r;
          const float xs = scales[row];
          const f32x4 g4 = get(0), u4 = get(32);
          f32x4 h;
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const float g = g4[i] * xs * gs[i], u = u4[i] * xs * us[i];
            h[i] = silu(g) * u;
          }
          store_rows(to, out + row * pitch, __builtin_bit_cast(u32x4, h));
        });
}

template <class T>
__global__ __launch_bounds__(T::kThreads) void wc_experts_down_tile_kernel(ExpertArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
  __shared__ float scales[T::kRows];   // of the tile's rows of h, and their slots
  __shared__ uint32_t slots[T::kRows];
  static_assert(T::kRows <= T::kThreads);
  constexpr uint32_t kBM = T::kRows, kBN = T::kCols;
  const uint32_t k = a.ffn, step = a.down_step;
  const uint32_t blocks = ((a.hidden + step - 1) / step + kBN - 1) / kBN;
  uint32_t mt, nt;
  if (!tile_at(blockIdx.x, block_count(a), blocks * step, mt, nt)) return;
  const auto [e, first, last] = block_at(a, mt);
  const uint32_t class0 = nt / blocks, r0 = nt % blocks * kBN, m_rows = last - first;
  const ClassRows C = class_rows(a.down.w + e * a.down.stride, k, a.hidden, k, step, class0);
  if (r0 >= C.rows) return;
  const uint32_t n_rows = min(kBN, C.rows - r0);
  const Shifted X = shifted(a.hq, a.hcopies, a.slots, k, C.shift);
  const u32x4 xr = rows_rsrc(X.base + uint64_t(first) * X.pitch, m_rows * X.pitch);
  const u32x4 wr = rows_rsrc(C.base + r0 * uint64_t(C.pitch), (n_rows - 1) * C.pitch + C.bytes);
  uint32_t xoff[T::kXLoads], woff[T::kWLoads];
#pragma unroll
  for (int i = 0; i < T::kXLoads; i++) xoff[i] = min(T::row_of(i), m_rows - 1) * X.pitch + T::byte_of();
#pragma unroll
  for (int i = 0; i < T::kWLoads; i++) woff[i] = min(T::row_of(i), n_rows - 1) * C.pitch + T::byte_of();
  // a load among the stores at the end would wait for all stores before it
  const uint32_t place = min(first + threadIdx.x % kBM, last - 1);
  const float row_scale = global<const float>(a.hscale)[place];
  const uint32_t row_slot = slot_at(a, place);
  i32x16 acc[T::kMT][T::kNT];
  T::product(lds, (C.bytes + kStage - 1) / kStage, m_rows,
             [&](int i, uint32_t s, uint32_t to) { load_lds(xr, to, xoff[i] + s * kStage); },
             [&](int i, uint32_t s, uint32_t to) { load_lds(wr, to, woff[i] + s * kStage); }, acc);
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  constexpr int kCols = T::kNT * 32;
  const uint32_t column = wave % T::kWN_ * kCols + lane % (kCols / 4) * 4;
  const uint32_t row0 = wave / T::kWN_ * (T::kMT * 32), pitch = row_pitch(a.hidden, step);
  // no branches: rows and columns past the last go to a row of their own
  const uint64_t nowhere = uint64_t(a.slots) * pitch;
  const bool inside = column < n_rows;
  const uint32_t out = class0 * class_pitch(a.hidden, step) + r0 + column;
  float scale[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; i++) {
    const uint32_t n = class0 + (r0 + column + i) * step;
    scale[i] = load_float(a.down.scale, a.down.scale_dtype, uint64_t(e) * a.hidden + min(n, a.hidden - 1));
  }
  if (threadIdx.x < kBM) {
    scales[threadIdx.x] = row_scale;
    slots[threadIdx.x] = first + threadIdx.x < last ? row_slot : a.slots;
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < T::kMT; b++)
    T::template rows_out<kCols>(
        lds, [&](int c, int i) { return float(acc[b][c][i]); },
        [&](uint32_t r, uint32_t, auto get) {
          const uint32_t row = row0 + b * 32 + r;
          const float hs = scales[row];
          const uint64_t at = uint64_t(slots[row]) * pitch;
          f32x4 v = get(0);
#pragma unroll
          for (int i = 0; i < 4; i++) v[i] = v[i] * hs * scale[i];
          *reinterpret_cast<global_ptr<f32x4>>(global<float>(a.out) + (inside ? at + out : nowhere)) = v;
        });
}

// y of one token, four columns a thread: its slots' results in their order, times
// their weights.  Bound by memory: 4096 tokens of 6144, 2 slots each, 48 us (5.2 TB/s).
__global__ __launch_bounds__(256) void wc_experts_join_kernel(ExpertArgs a) {
  const uint32_t token = blockIdx.x, n = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (n >= a.hidden) return;
  const uint32_t each = class_pitch(a.hidden, a.down_step);
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (uint32_t j = 0; j < a.k; j++) {
    const uint64_t slot = uint64_t(token) * a.k + j;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (global<const int32_t>(a.ids)[slot] >= 0) {
      const auto row = global<const float>(a.out) + slot * (a.down_step * each);
      if (a.down_step == 1) {
        v = *reinterpret_cast<global_ptr<const f32x4>>(row + n);
      } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; i++) v[i] = row[column_at(min(n + i, a.hidden - 1), a.down_step, each)];
      }
    }
    const float w = global<const float>(a.weights)[slot];
#pragma unroll
    for (int i = 0; i < 4; i++) sum[i] += w * v[i];
  }
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (n + i < a.hidden) store_float(a.y, a.dtype, token * a.ldy + n + i, sum[i]);
}

// Blocks of `rows` places: every expert that has places ends in one that may not be full.
uint64_t most_blocks(uint32_t slots, uint32_t experts, uint32_t rows) {
  return uint64_t(slots) / rows + (experts < slots ? experts : slots);
}

struct Workspace {
  uint64_t xq, xscale, wide, hq, hscale, xcopies, hcopies, table, bytes;
};
Workspace layout(uint64_t tokens, uint64_t k, uint64_t experts, uint64_t hidden, uint64_t ffn) {
  Workspace w{};
  uint64_t at = 0;
  const auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at += pad256(bytes);
    return here;
  };
  w.table = take((1 + most_blocks(uint32_t(tokens * k), uint32_t(experts), 8)) * 16);
  w.xq = take(tokens * WC_I8_ROW_BYTES(hidden));
  w.xscale = take(tokens * 4);
  // h, and after its quantisation the experts' results and a row for what is past them
  const uint64_t h = row_pitch(uint32_t(ffn), steps_of(hidden)), out = row_pitch(uint32_t(hidden), steps_of(ffn));
  w.wide = take((tokens * k + 1) * (h > out ? h : out) * 4);
  w.hq = take(tokens * k * WC_I8_ROW_BYTES(ffn));
  w.hscale = take(tokens * k * 4);
  if (hidden % 4) w.xcopies = take(copies_bytes(tokens, hidden));
  if (ffn % 4) w.hcopies = take(copies_bytes(tokens * k, ffn));
  w.bytes = at;
  return w;
}
bool sizes_ok(uint32_t tokens, uint32_t k, uint32_t experts, uint32_t hidden, uint32_t ffn) {
  return k >= 1 && experts >= 1 && experts <= kMaxExperts && k <= experts && hidden >= 1 &&
         hidden <= kMaxK && ffn >= 1 && ffn <= kMaxK && uint64_t(tokens) * k < (1ull << 24);
}
bool bank_ok(const wc_i8_experts* b, uint64_t n, uint64_t k) {
  return b && b->w && b->scale && float_ok(b->scale_dtype) && b->stride >= n * k &&
         !(b->stride >> 40) && reinterpret_cast<uintptr_t>(b->scale) % size_of(b->scale_dtype) == 0;
}
Bank bank(const wc_i8_experts* b) {
  return {reinterpret_cast<uint64_t>(b->w), reinterpret_cast<uint64_t>(b->scale), b->stride,
          b->scale_dtype};
}

// Whether the rows of an expert's matrix start where the workspace has a copy of what
// multiplies them: at whole dwords where k is whole ones.
bool reached(const wc_i8_experts* b, uint32_t k) {
  return k % 4 || (reinterpret_cast<uintptr_t>(b->w) % 4 == 0 && b->stride % 4 == 0);
}

// Slot by slot, while few slots share an expert, whose rows are then read for each (or the
// rows are few): 64 experts of 2048 x 1408, 6 a token, 20.6 us at one token against 25.2 on
// the launches of the general path, 28.2 and 33.7 at two, 43.4 and 52.8 at four; of 4096 x
// 2048, 8 a token, 40.4 and 46.8 at one, 127 (20 experts hit) and 118 (22 hit) at four.  A
// workgroup holds all of a token's h: 8 experts of 6144 x 16384, 2 a token, would take 129
// and take 119.
constexpr uint32_t kSlotTokens = 4, kHoldBytes = 16 * 1024;
constexpr uint64_t kSlotWeights = 64u << 20;

using Tile64 = Tile<64, 128, 1, 2, 3>;
using Tile128 = Tile<128, 128, 2, 2, 3>;
using Tile256 = Tile<256, 256, 2, 4>;
template <class F>
void with_tile(int tile, F f) {
  switch (tile) {
    case 1: return f(Tile64{});
    case 2: return f(Tile128{});
    case 3: return f(Tile256{});
    default: return;
  }
}

uint32_t columns(uint32_t n, uint32_t step, uint32_t each) {
  return step * (((n + step - 1) / step + each - 1) / each);
}
// What a tile's kernels take, in us: a stage of 128 bytes of k, one workgroup's and two's
// where two fit a compute unit, and all else of a round of workgroups.  Taken so that the
// least sum is the fastest tile, or within 2 % of it, at each of these (measured on tiles of
// 64, 128 and 256 places, us; experts, of them a token's, width x inner width, tokens):
//   7, 3, 1537 x 2051: 150 57, 52, 86; 203 58, 66, 88; 330 87, 70, 93
//   7, 3, 2049 x 1365: 77 44, 46, 79; 256 62, 51, 84
//   16, 4, 2048 x 1024: 500 81, 71, 75; 1000 112, 102, 82
//   64, 6, 2048 x 1408: 43 132, 161, 169; 683 202, 205, 214; 1995 342, 330, 287
//   8, 2, 4096 x 14336: 16 274, 269, 392; 128 294, 313, 400; 256 375, 337, 428;
//     600 559, 518, 500; 4096 4370, 3613, 2760
//   8, 2, 6144 x 16384: 32 473, 506, 578
struct ExpertCost {
  int tile;
  uint32_t rows, up_columns, columns;
  double stage, stage_of_two, round;
};
constexpr ExpertCost kExpertCosts[] = {{1, Tile64::kRows, Tile64::kWN_ * 32, Tile64::kCols, 0.55, 0.8, 5},
                                       {2, Tile128::kRows, Tile128::kWN_ * 32, Tile128::kCols, 0.60, 0, 5},
                                       {3, Tile256::kRows, Tile256::kWN_ * 32, Tile256::kCols, 1.55, 0, 9}};
constexpr double kUnits = 256, kReadPerUs = 5e6;

// The kernel, by the rows an expert has on average: a tile (0: none) of `rows` places, or
// rings of 8 or 16, or (0) the one for matrices at any address.
struct Chosen {
  int tile;
  uint32_t rows;
};
Chosen choose(uint64_t tokens, uint32_t slots, uint32_t experts, uint32_t hidden, uint32_t ffn,
              bool direct) {
  // tiles find x by 32-bit offsets
  if (!direct || tokens * WC_I8_ROW_BYTES(hidden + 3) >> 32) return {0, 0};
  const uint32_t average = slots / experts;
  // a token takes an expert once.  Rings and the least tile, us: average 4 of 8 experts of
  // 4096 x 14336 283 and 274, 6 of 64 of 2048 x 1408 152 and 132, 32 of the first 594 and 294
  if (average < 4) return {0, tokens <= 8 ? 8u : 16u};
  Chosen best{0, 0};
  double least = 0;
  const double hit = std::min(experts, slots);
  for (const ExpertCost& c : kExpertCosts) {
    // an expert's last block is half full, on average
    const double blocks = hit * std::max(1.0, double(average) / c.rows + 0.5);
    const auto product = [&](uint32_t n, uint32_t k, uint32_t each, uint32_t matrices) {
      const double groups = blocks * columns(n, steps_of(k), each);
      const bool two = c.stage_of_two > 0 && groups > kUnits;
      const double rounds = groups / (two ? 2 * kUnits : kUnits);
      const double us = (c.round + (k + 127) / 128 * (two ? c.stage_of_two : c.stage)) *
                        // many rounds overlap
                        (rounds < 4 ? std::ceil(rounds) : rounds + 0.5);
      return std::max(us, hit * matrices * double(n) * k / kReadPerUs);
    };
    const double us = product(ffn, hidden, c.up_columns, 2) + product(hidden, ffn, c.columns, 1);
    if (least == 0 || us < least) {
      least = us;
      best = {c.tile, c.rows};
    }
  }
  return best;
}

template <class T>
void start_up(const ExpertArgs& a, hipStream_t st) {
  const dim3 grid(a.blocks * columns(a.ffn, a.up_step, T::kWN_ * 32));
  hipLaunchKernelGGL((wc_experts_up_tile_kernel<T>), grid, dim3(T::kThreads), 0, st, a);
}
template <class T>
void start_down(const ExpertArgs& a, hipStream_t st) {
  const dim3 grid(a.blocks * columns(a.hidden, a.down_step, T::kCols));
  hipLaunchKernelGGL((wc_experts_down_tile_kernel<T>), grid, dim3(T::kThreads), 0, st, a);
}

}  // namespace

extern "C" wc_status wc_experts_i8_workspace_bytes(uint32_t tokens, uint32_t k, uint32_t experts,
                                                   uint32_t hidden, uint32_t ffn, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!sizes_ok(tokens, k, experts, hidden, ffn)) return WC_EINVAL;
  *bytes = layout(tokens, k, experts, hidden, ffn).bytes;
  return WC_OK;
}

extern "C" wc_status wc_experts_i8(const void* dev_x, int32_t dtype, uint32_t tokens, uint64_t ldx,
                                   uint32_t k, uint32_t experts, uint32_t hidden, uint32_t ffn,
                                   const int32_t* dev_ids, const float* dev_weights,
                                   const int32_t* dev_offsets, const int32_t* dev_order,
                                   const wc_i8_experts* gate, const wc_i8_experts* up,
                                   const wc_i8_experts* down, void* dev_y, uint64_t ldy,
                                   void* dev_workspace, uint64_t workspace_bytes, void* stream) {
  if (!sizes_ok(tokens, k, experts, hidden, ffn) || !float_ok(dtype) || ldx < hidden || ldx >> 31 ||
      ldy < hidden || ldy >> 31 || !bank_ok(gate, ffn, hidden) || !bank_ok(up, ffn, hidden) ||
      !bank_ok(down, hidden, ffn))
    return WC_EINVAL;
  if (tokens == 0) return WC_OK;
  const auto off = [](const void* p, uint32_t to) {
    return !p || reinterpret_cast<uintptr_t>(p) % to != 0;
  };
  if (off(dev_x, size_of(dtype)) || off(dev_y, size_of(dtype)) || off(dev_ids, 4) ||
      off(dev_weights, 4) || off(dev_offsets, 4) || off(dev_order, 4))
    return WC_EINVAL;
  const Workspace w = layout(tokens, k, experts, hidden, ffn);
  if (off(dev_workspace, 256) || workspace_bytes < w.bytes) return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const uint64_t ws = reinterpret_cast<uint64_t>(dev_workspace);
  const uint32_t slots = tokens * k;
  ExpertArgs a{};
  a.table = ws + w.table;
  a.order = reinterpret_cast<uint64_t>(dev_order);
  a.ids = reinterpret_cast<uint64_t>(dev_ids);
  a.weights = reinterpret_cast<uint64_t>(dev_weights);
  a.x = reinterpret_cast<uint64_t>(dev_x);
  a.ldx = ldx;
  a.xq = ws + w.xq;
  a.xscale = ws + w.xscale;
  a.h = a.out = ws + w.wide;
  a.hq = ws + w.hq;
  a.hscale = ws + w.hscale;
  a.xcopies = ws + w.xcopies;
  a.hcopies = ws + w.hcopies;
  a.y = reinterpret_cast<uint64_t>(dev_y);
  a.ldy = ldy;
  a.tokens = tokens;
  a.k = k;
  a.experts = experts;
  a.hidden = hidden;
  a.ffn = ffn;
  a.slots = slots;
  a.dtype = dtype;
  a.gate = bank(gate);
  a.up = bank(up);
  a.down = bank(down);
  // gate and up rows of one column share their x, so they have to start alike
  const bool direct = reached(gate, hidden) && reached(up, hidden) && reached(down, ffn) &&
                      (reinterpret_cast<uintptr_t>(gate->w) - reinterpret_cast<uintptr_t>(up->w)) % 4 == 0 &&
                      (gate->stride - up->stride) % 4 == 0;
  const uint64_t hold_x = WC_I8_ROW_BYTES(hidden), hold_h = k * WC_I8_ROW_BYTES(ffn);
  const bool few = tokens == 1 || 2 * slots < experts ||
                   (slots <= experts && 3ull * slots * hidden * ffn <= kSlotWeights);
  if (direct && hidden % 8 == 0 && ffn % 8 == 0 && tokens <= kSlotTokens && few && k <= kSlots &&
      hold_x <= kHoldBytes && hold_h <= kHoldBytes) {
    const dim3 grid((ffn + 7) / 8, slots), block(SlotRing::kThreads);
    const uint32_t held = SlotRing::kLds + uint32_t(hold_x);
    if (dtype == WC_BF16)
      hipLaunchKernelGGL((wc_experts_up_slot_kernel<WC_BF16>), grid, block, held, st, a);
    else if (dtype == WC_FP16)
      hipLaunchKernelGGL((wc_experts_up_slot_kernel<WC_FP16>), grid, block, held, st, a);
    else
      hipLaunchKernelGGL((wc_experts_up_slot_kernel<WC_FP32>), grid, block, held, st, a);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
    hipLaunchKernelGGL(wc_experts_down_slot_kernel, dim3((hidden + 15) / 16, tokens),
                       dim3(DownSlotRing::kThreads),
                       DownSlotRing::kLds + uint32_t(hold_h) + k * DownSlotRing::kThreads, st, a);
    return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
  }
  const Chosen kernel = choose(tokens, slots, experts, hidden, ffn, direct);
  const uint32_t rows = kernel.rows;
  const uint32_t block_rows = rows ? rows : 16;
  a.blocks = uint32_t(most_blocks(slots, experts, block_rows));
  const Blocks blocks = {a.table, reinterpret_cast<uint64_t>(dev_offsets), experts, slots, block_rows,
                         a.blocks};
  if (!launch_quantize(dev_x, dtype, tokens, hidden, ldx, reinterpret_cast<void*>(a.xq),
                       reinterpret_cast<float*>(a.xscale), st, nullptr, &blocks,
                       hidden % 4 ? reinterpret_cast<void*>(a.xcopies) : nullptr))
    return WC_EHIP;
  a.up_step = rows ? steps_of(hidden) : 1;
  a.down_step = rows ? steps_of(ffn) : 1;
  const dim3 up_grid(a.blocks, columns(ffn, a.up_step, rows ? 8 : 16));
  const dim3 down_grid(a.blocks, columns(hidden, a.down_step, 16));
  if (kernel.tile) with_tile(kernel.tile, [&](auto t) { start_up<decltype(t)>(a, st); });
  else if (rows == 16)
    hipLaunchKernelGGL((wc_experts_up_ring_kernel<16>), up_grid, dim3(ExpertRing<16>::kThreads), 0, st, a);
  else if (rows == 8)
    hipLaunchKernelGGL((wc_experts_up_ring_kernel<8>), up_grid, dim3(ExpertRing<8>::kThreads), 0, st, a);
  else
    hipLaunchKernelGGL(wc_experts_up_kernel, up_grid, dim3(64 * kRowWaves), 0, st, a);
  if (hipGetLastError() != hipSuccess) return WC_EHIP;
  if (!launch_quantize(reinterpret_cast<const void*>(a.h), WC_FP32, slots, ffn, row_pitch(ffn, a.up_step),
                       reinterpret_cast<void*>(a.hq), reinterpret_cast<float*>(a.hscale), st,
                       dev_offsets + experts, nullptr,
                       ffn % 4 ? reinterpret_cast<void*>(a.hcopies) : nullptr, a.up_step))
    return WC_EHIP;
  if (kernel.tile) with_tile(kernel.tile, [&](auto t) { start_down<decltype(t)>(a, st); });
  else if (rows == 16)
    hipLaunchKernelGGL((wc_experts_down_ring_kernel<16>), down_grid, dim3(ExpertRing<16>::kThreads), 0, st, a);
  else if (rows == 8)
    hipLaunchKernelGGL((wc_experts_down_ring_kernel<8>), down_grid, dim3(ExpertRing<8>::kThreads), 0, st, a);
  else
    hipLaunchKernelGGL(wc_experts_down_kernel, down_grid, dim3(64 * kRowWaves), 0, st, a);
  if (hipGetLastError() != hipSuccess) return WC_EHIP;
  hipLaunchKernelGGL(wc_experts_join_kernel, dim3(tokens, (hidden + 1023) / 1024), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
}
