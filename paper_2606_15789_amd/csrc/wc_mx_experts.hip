// wc_mx_experts.hip -- mixture layers with MXFP4 experts: wc_experts_mx, wc_moe_mx.
//
// For a token t with experts e_j of weights g_j:
//   h_j = silu(G_ej x_t) * (U_ej x_t),  y_t = sum_j g_j D_ej h_j,
// x_t and every h_j in MXFP4.  The scale of a block of h needs 32 of its columns only, so the
// product that makes them quantises them as well.  Two ways:
//   - up to 16 tokens, which are the columns of a matrix instruction, two kernels: one finds the
//     experts (and chooses them, from logits), multiplies by gate and up and writes h by slot, the
//     other multiplies by down and adds a token's slots;
//   - more tokens, or wider ones: the places of the router's order in blocks of one expert's, on tiles
//     through LDS, each expert's results stored by slot and then added.
#include <algorithm>

#include "wc_choose.h"
#include "wc_mx_tile.h"

namespace {

using namespace wc_mx;
using wc_choose::RouteArgs;

typedef float f32x8 __attribute__((ext_vector_type(8)));

struct Bank {
  uint64_t w, stride;
  Scales scales;
  uint64_t scale_stride;
};
struct ExpertArgs {
  uint64_t table, order, ids, weights;
  uint64_t x, ldx;
  uint64_t xq, hq;  // codes of x, by token, and of h, by place in the order (few tokens: by slot)
  Scales xs, hs;
  uint64_t out;     // experts' results, fp32, by slot, in rows of whole eights
  uint64_t y, ldy;
  uint32_t tokens, k, experts, hidden, ffn, slots;
  int32_t dtype;
  Bank gate, up, down;
};
// Row min(first + r, n - 1) of expert e's matrix.
__device__ __forceinline__ Row row_of(const Bank& b, uint32_t e, uint32_t first, uint32_t r, uint32_t n,
                                      uint32_t blocks) {
  return row_at(b.w + e * b.stride, blocks * 16, Scales{b.scales.at + e * b.scale_stride, b.scales.pitch, b.scales.step},
                first, r, n);
}

// h = silu(g) u in MXFP4.  The borders that a code or a block's scale goes by, 0.25, 0.75, 1.25, 1.75,
// 2.5, 3.5, 5 and 1 times a power of two, have zeros for the low 21 bits of a float.  fp32's h, with
// an exponential of 1 ulp and a rounded sum, division and product, is at most 2.5 * 2^-23 of its size
// off, 5 ulps: where it is further from such a float, it is on the right side of all borders.  Where it
// is not, one value in 160 thousand, and the border is one of its block's, h is found in 64 bits and
// rounded to odd, which leaves it on its side.  (Not so for h of less than 2^-126 and where silu(g)
// underflows, g < -88: those are fp32's.)  us with fp32's h and with this: 16 tokens, 8 of 128 experts of
// 4096 x 1536 159.5 and 159.9; 2000 tokens, 6 of 64 of 2048 x 1408 154.5 and 156.5; 4096 tokens, 2 of 8 of
// 6144 x 16384 1525 and 1535.  With 64 bits for every value near such a float the last took 1560: the
// instructions of that path come from memory.
constexpr uint32_t kUlps = 6;
// ulps past a float with `kBits` zeros, kUlps of them on it, times a power of two
template <int kBits>
__device__ __forceinline__ bool next_to(uint32_t bits) {
  return (bits << (32 - kBits)) + (kUlps << (32 - kBits)) <= 2 * kUlps << (32 - kBits);
}
__device__ __forceinline__ float hidden_fp32(float g, float u) { return g / (1.0f + expf(-g)) * u; }
__device__ __forceinline__ float hidden_odd(float g, float u) {
  const double d = double(g) / (1.0 + exp(-double(g))) * double(u);
  const float f = float(d);
  if (__builtin_isinf(f) || double(f) == d) return f;  // beyond fp32: an infinity
  const uint32_t bits = __float_as_uint(f);
  return __uint_as_float((__builtin_fabs(double(f)) > __builtin_fabs(d) ? bits - 1 : bits) | 1u);
}
// Codes of eight values from h[i] on, times `by`.
template <class V>
__device__ __forceinline__ uint32_t eight_codes(const V& h, int i, float scale, float by) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, h[i] * by, h[i + 1] * by, scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, h[i + 2] * by, h[i + 3] * by, scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, h[i + 4] * by, h[i + 5] * by, scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, h[i + 6] * by, h[i + 7] * by, scale, 3);
}
template <int kN>
struct Hidden {
  uint32_t byte, codes[kN / 8];
};
// A lane's kN values: those of a row have in(i), the others are zeros; `across` gives the greatest of
// the lanes that share a block.  Of lanes without `live` any.
template <int kN, class V, class In, class Across>
__device__ __forceinline__ Hidden<kN> hidden(const V& g, const V& u, bool live, In in, Across across) {
  V h;
  uint32_t least = ~0u;
#pragma unroll
  for (int i = 0; i < kN; i++) {
    h[i] = hidden_fp32(g[i], u[i]);
    least = min(least, (__float_as_uint(h[i]) << 11) + (kUlps << 11));
    if (!in(i)) h[i] = 0.0f;
  }
  Hidden<kN> r;
  for (bool sure = false;; sure = true) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kN; i++) top = max(top, __float_as_uint(h[i]) & 0x7FFFFFFFu);
    top = across(top);
    r.byte = scale_byte(top);
    const float scale = scale_value(r.byte);
#pragma unroll
    for (int i = 0; i < kN; i += 8) r.codes[i / 8] = r.byte == 255 ? 0u : eight_codes(h, i, scale, 1.0f);
    if (sure || __builtin_expect(!__ballot(live && least <= 2 * kUlps << 11), 1)) return r;
    uint32_t apart = top && next_to<23>(top);
#pragma unroll
    for (int i = 0; i < kN; i += 8)
      apart |= eight_codes(h, i, scale, 1 - 0x1p-20f) ^ eight_codes(h, i, scale, 1 + 0x1p-20f);
    if (__builtin_expect(!__ballot(live && apart), 1)) return r;
    uint32_t near = 0;  // bit i: h[i]
#pragma unroll
    for (int i = 0; i < kN; i++)
      if (next_to<21>(__float_as_uint(h[i])) && in(i)) near |= 1u << i;
    if (!live || !apart) near = 0;
#pragma unroll 1
    for (; __ballot(near != 0); near &= near - 1) {
      const int at = near ? __builtin_ctz(near) : kN;
      float gi = 0.0f, ui = 0.0f;
#pragma unroll
      for (int i = 0; i < kN; i++) {
        gi = at == i ? g[i] : gi;
        ui = at == i ? u[i] : ui;
      }
      const float v = hidden_odd(gi, ui);
#pragma unroll
      for (int i = 0; i < kN; i++) h[i] = at == i ? v : h[i];
    }
  }
}

// Codes and scales of row `at` of h.
__device__ __forceinline__ uint64_t h_codes(const ExpertArgs& a, uint64_t at, uint32_t block) {
  return a.hq + (at * ((a.ffn + 31) / 32) + block) * 16;
}
// A block's scale; after a row's last one zeros to a whole word.
__device__ __forceinline__ void store_h_scale(const ExpertArgs& a, uint64_t at, uint32_t block, uint32_t byte) {
  const auto to = global<uint8_t>(a.hs.at + at * a.hs.pitch + uint64_t(block / 16) * a.hs.step + block % 16);
  *to = uint8_t(byte);
  if (block + 1 == (a.ffn + 31) / 32)
    for (uint32_t i = 1; (block + i) % 4; i++) to[i] = 0;
}
// --- few tokens ---------------------------------------------------------------

constexpr uint32_t kFew = 16;            // tokens
constexpr uint32_t kFewHidden = 8192;    // width of x that a workgroup holds in LDS
constexpr int kFewWaves = 8;

inline bool is_few(uint64_t tokens, uint64_t k, uint64_t hidden) {
  return tokens <= kFew && k <= wc_choose::kMaxChosen && hidden <= kFewHidden;
}
// The tokens' experts in a workgroup's LDS.
constexpr uint32_t kFewThreads = 64 * kFewWaves;
struct Chosen {
  int32_t ids[kFew][wc_choose::kMaxChosen];
  float weights[kFew][wc_choose::kMaxChosen];
  uint8_t hit[kMaxExperts];
  uint16_t list[kMaxExperts];  // the experts hit, in order
  uint32_t count;
};
// Lists the experts that ids name.
template <uint32_t kThreads>
__device__ __forceinline__ void list_experts(Chosen& c, const ExpertArgs& a) {
  for (uint32_t e = threadIdx.x; e < kMaxExperts; e += kThreads) c.hit[e] = 0;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < a.slots; i += kThreads) {
    const int32_t id = c.ids[i / a.k][i % a.k];
    if (id >= 0) c.hit[id] = 1;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    uint32_t count = 0;
    for (uint32_t e0 = 0; e0 < a.experts; e0 += 64) {
      const bool on = c.hit[e0 + threadIdx.x];
      const uint64_t all = __ballot(on);
      if (on) c.list[count + uint32_t(__popcll(all & ((1ull << threadIdx.x) - 1)))] = uint16_t(e0 + threadIdx.x);
      count += uint32_t(__popcll(all));
    }
    if (threadIdx.x == 0) c.count = count;
  }
  __syncthreads();
}
template <uint32_t kThreads>
__device__ __forceinline__ void load_choice(Chosen& c, const ExpertArgs& a) {
  for (uint32_t i = threadIdx.x; i < a.slots; i += kThreads) {
    const int32_t id = global<const int32_t>(a.ids)[i];
    c.ids[i / a.k][i % a.k] = id < 0 ? -1 : min(id, int32_t(a.experts) - 1);
    c.weights[i / a.k][i % a.k] = global<const float>(a.weights)[i];
  }
}
// The first slot of a token with expert e, -1 if none.
__device__ __forceinline__ int32_t slot_of(const Chosen& c, const ExpertArgs& a, uint32_t token, uint32_t e) {
  int32_t slot = -1;
  if (token < a.tokens)
    for (int32_t j = int32_t(a.k) - 1; j >= 0; j--)
      if (c.ids[token][j] == int32_t(e)) slot = int32_t(token * a.k) + j;
  return slot;
}

// The greatest of the four lanes 16 apart that hold a token's columns.
__device__ __forceinline__ uint32_t top_of_column(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(b[0], b[1]);
}
// A wave's 32 columns of h for 16 rows of x: the lane's two groups of four from gate's and up's sums
// (columns 4 (lane / 16) on, and 16 further), quantised and stored for row `at` if `live`.
__device__ __forceinline__ void store_h(const ExpertArgs& a, const f32x4 (&g)[2], const f32x4 (&u)[2], uint64_t at,
                                        uint32_t block, bool live) {
  const uint32_t quarter = threadIdx.x % 64 / 16;
  const auto h = hidden<8>(
      __builtin_shufflevector(g[0], g[1], 0, 1, 2, 3, 4, 5, 6, 7),
      __builtin_shufflevector(u[0], u[1], 0, 1, 2, 3, 4, 5, 6, 7), live,
      [&](uint32_t i) { return block * 32 + 16 * (i / 4) + 4 * quarter + i % 4 < a.ffn; }, top_of_column);
  if (!live) return;
  const auto to = global<uint16_t>(h_codes(a, at, block)) + quarter;
  to[0] = uint16_t(h.codes[0]);
  to[4] = uint16_t(h.codes[0] >> 16);
  if (quarter == 0) store_h_scale(a, at, block, h.byte);
}

// 32 columns of h at a time, for all tokens of one expert; the tokens are the columns of the matrix
// instruction, whether they have the expert or not.  kPer: registers of logits to a lane of the
// choice, 0 where the ids are given.  Bound by reading the experts hit: 16 tokens, 8 of 128 experts
// of 4096 x 1536 in groups, 73 to 76 us for the 350 MB of the some 53 that are hit, 4.7 TB/s; one token, 6
// of 64 of 2048 x 1408, 13.0, a chain of latencies (x, the logits, the choice, W, the sums).  With the
// choice by a workgroup for every tile, 16 tokens of 128 experts without groups took 389 us, 267
// from a plan.  Two waves to a SIMD: past 256 registers, one workgroup of four waves to a compute unit,
// one token's layer took 26 us instead of 20.
template <int kType, int kPer, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void wc_moe_mx_up_kernel(ExpertArgs a, RouteArgs route) {
  using S = Stream<4, kWaves>;
  __shared__ typename S::Shared sh;
  __shared__ Chosen c;
  extern __shared__ u32x4 held[];  // x; only its own wave reads a part
  const uint32_t lane = threadIdx.x % 64, r = lane % 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t blocks = (a.hidden + 31) / 32, supers = (blocks + kSuper - 1) / kSuper;
  // the first token's logits are on their way to the cache while x is quantised
  float logit = 0.0f;
  if constexpr (kPer > 0)
    logit = load_float(route.logits, route.dtype, min(wave, a.tokens - 1) * route.ld + min(lane, a.experts - 1));
  for (uint32_t super = wave; super < supers; super += kWaves)
    hold_part(held, super,
              quantize_part<kType>(a.x + r * a.ldx * (kType == WC_FP32 ? 4 : 2), r < a.tokens, super, a.hidden));
  asm volatile("" ::"v"(logit));
  if constexpr (kPer > 0) {
    // the sums' place in LDS is free until then
    static_assert(sizeof(float) * kWaves * 64 * (kPer ? kPer : 1) <= sizeof(sh));
    float* const scratch = reinterpret_cast<float*>(&sh) + wave * (64 * kPer);
    for (uint32_t token = wave; token < a.tokens; token += kWaves) {
      int32_t id;
      float weight;
      wc_choose::choose<64, kPer>(route, token, scratch, id, weight);
      if (lane < a.k) {
        c.ids[token][lane] = id;
        c.weights[token][lane] = weight;
      }
      if (blockIdx.x == 0) wc_choose::store_choice<64>(route, token, id, weight);
    }
  } else {
    load_choice<64 * kWaves>(c, a);
  }
  __syncthreads();
  list_experts<64 * kWaves>(c, a);
  const uint32_t each = (a.ffn + 31) / 32, tiles = c.count * each;
  if (blockIdx.x >= tiles) return;
  S::run(
      sh, blockIdx.x, tiles, gridDim.x, blocks,
      [&](uint32_t tile, Row(&w)[4]) {
        const uint32_t e = __builtin_amdgcn_readfirstlane(c.list[tile / each]), n0 = tile % each * 32;
#pragma unroll
        for (uint32_t n = 0; n < 2; n++) {
          w[n] = row_of(a.gate, e, n0 + 16 * n, r, a.ffn, blocks);
          w[n + 2] = row_of(a.up, e, n0 + 16 * n, r, a.ffn, blocks);
        }
      },
      [&](uint32_t super) { return held_part(held, super); },
      [&](uint32_t tile, auto sum) {
        if (wave) return;
        const int32_t slot = slot_of(c, a, r, c.list[tile / each]);
        const f32x4 g[2] = {sum(lane), sum(64 + lane)}, u[2] = {sum(128 + lane), sum(192 + lane)};
        store_h(a, g, u, uint32_t(slot), tile % each, slot >= 0);
      });
}

// 16 columns of y for all tokens: parts of 512 of every expert hit, spread over the waves.  Each
// expert's first slot and weight of a token stand in a table in LDS.  33 to 35 us (5 TB/s) and 7.5 after
// the calls above.
__global__ __launch_bounds__(64 * kFewWaves) void wc_moe_mx_down_kernel(ExpertArgs a) {
  __shared__ Chosen c;
  __shared__ f32x4 part[kFewWaves][64];
  extern __shared__ float table[];  // weights, then slots
  load_choice<kFewThreads>(c, a);
  __syncthreads();
  list_experts<kFewThreads>(c, a);
  float* const weights = table;
  int16_t* const slots = reinterpret_cast<int16_t*>(table + c.count * 16);
  for (uint32_t i = threadIdx.x; i < c.count * 16; i += kFewThreads) {
    const int32_t e = c.list[i / 16];
    const uint32_t token = i % 16;
    int32_t slot = -1;
    float weight = 0.0f;
    if (token < a.tokens)
      for (uint32_t j = 0; j < a.k; j++)
        if (c.ids[token][j] == e) {
          if (slot < 0) slot = int32_t(token * a.k + j);
          weight += c.weights[token][j];
        }
    weights[i] = weight;
    slots[i] = int16_t(slot);
  }
  __syncthreads();
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, r = lane % 16;
  const uint32_t blocks = (a.ffn + 31) / 32, supers = (blocks + kSuper - 1) / kSuper;
  const uint32_t n0 = blockIdx.x * 16, all = c.count * supers;
  const uint32_t first = uint32_t(uint64_t(all) * wave / kFewWaves);
  const uint32_t last = uint32_t(uint64_t(all) * (wave + 1) / kFewWaves);
  // the part that is on its way: of expert `at` of the list
  uint32_t at = first / supers, super = first % supers;
  int32_t slot = -1;
  Row w{}, x{};
  RawPart next_w, next_x = {};
  const auto begin = [&] {
    const uint32_t e = __builtin_amdgcn_readfirstlane(c.list[at]);
    w = row_of(a.down, e, n0, r, a.hidden, blocks);
    slot = slots[at * 16 + r];
    x = {h_codes(a, max(slot, 0), 0), a.hs.at + uint64_t(max(slot, 0)) * a.hs.pitch, a.hs.step, 0, 0};
  };
  const auto load = [&] {
    next_w = load_raw<false>(w, super, blocks);
    if (slot >= 0) next_x = load_raw<true>(x, super, blocks);
  };
  f32x4 y = {0, 0, 0, 0}, acc = {0, 0, 0, 0};
  if (first < last) {
    begin();
    load();
  }
  for (uint32_t u = first; u < last; u++) {
    const Part wp = next_w.part(), xp = next_x.part();
    const bool mine = slot >= 0;
    const uint32_t here = at;
    if (u + 1 < last) {
      if (++super == supers) {
        super = 0;
        at++;
        begin();
      }
      load();
    }
    multiply(wp, xp, acc);
    if (at != here || u + 1 == last) {
      // an expert that a token lacks adds nothing, not even a NaN of its scales
      const float weight = weights[here * 16 + r];
      if (mine)
#pragma unroll
        for (int i = 0; i < 4; i++) y[i] += weight * acc[i];
      acc = f32x4{0, 0, 0, 0};
    }
  }
  part[wave][lane] = y;
  __syncthreads();
  if (threadIdx.x >= 64 || r >= a.tokens) return;
  f32x4 v = part[0][lane];
#pragma unroll
  for (int i = 1; i < kFewWaves; i++)
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] += part[i][lane][j];
  // slots without an expert: a NaN weight makes the token's results NaN
  for (uint32_t j = 0; j < a.k; j++)
    if (c.ids[r][j] < 0)
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] += c.weights[r][j] * 0.0f;
  const uint32_t n = n0 + lane / 16 * 4;
  if (n < a.hidden) store_four(a.y, a.dtype, r * a.ldy + n, v, a.hidden - n);
}

// --- any number of tokens -----------------------------------------------------

// The block-th block of places (Blocks).
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

__host__ __device__ constexpr uint32_t out_pitch(uint32_t hidden) { return (hidden + 7) & ~7u; }

// 32 columns of h for a block of 16 places, quantised.
__global__ __launch_bounds__(512) void wc_experts_mx_up_slim_kernel(ExpertArgs a) {
  using S = Slim<4, 1, 8>;
  __shared__ typename S::Shared sh;
  const uint32_t block = blockIdx.x;
  if (block >= block_count(a)) return;
  const auto [e, first, last] = block_at(a, block);
  const uint32_t lane = threadIdx.x % 64, r = lane % 16, n0 = blockIdx.y * 32, blocks = (a.hidden + 31) / 32;
  Row w[4];
#pragma unroll
  for (uint32_t n = 0; n < 2; n++) {
    w[n] = row_of(a.gate, e, n0 + 16 * n, r, a.ffn, blocks);
    w[n + 2] = row_of(a.up, e, n0 + 16 * n, r, a.ffn, blocks);
  }
  const uint64_t token = slot_at(a, min(first + r, last - 1)) / a.k;
  const Row x = {a.xq + token * blocks * 16, a.xs.at + token * a.xs.pitch, a.xs.step, 0, 0};
  S::product(sh, w, blocks, [&](int, uint32_t super) { return load_part<true>(x, super, blocks); });
  if (threadIdx.x >= 64) return;
  const f32x4 g[2] = {S::sum(sh, lane), S::sum(sh, 64 + lane)}, u[2] = {S::sum(sh, 128 + lane), S::sum(sh, 192 + lane)};
  store_h(a, g, u, first + r, blockIdx.y, first + r < last);
}

// down(h) of 32 columns for a block of places, stored by slot.
__global__ __launch_bounds__(512) void wc_experts_mx_down_slim_kernel(ExpertArgs a) {
  using S = Slim<2, 1, 8>;
  __shared__ typename S::Shared sh;
  const uint32_t block = blockIdx.x;
  if (block >= block_count(a)) return;
  const auto [e, first, last] = block_at(a, block);
  const uint32_t r = threadIdx.x % 16, n0 = blockIdx.y * 32, blocks = (a.ffn + 31) / 32;
  Row w[2];
#pragma unroll
  for (uint32_t n = 0; n < 2; n++) w[n] = row_of(a.down, e, n0 + 16 * n, r, a.hidden, blocks);
  const uint64_t place = min(first + r, last - 1);
  const Row x = {h_codes(a, place, 0), a.hs.at + place * a.hs.pitch, a.hs.step, 0, 0};
  S::product(sh, w, blocks, [&](int, uint32_t super) { return load_part<true>(x, super, blocks); });
  if (threadIdx.x >= S::kPart) return;
  const uint32_t n = n0 + threadIdx.x / 64 * 16 + threadIdx.x % 64 / 16 * 4;
  if (first + r < last && n < a.hidden)
    store_four(a.out, WC_FP32, uint64_t(slot_at(a, first + r)) * out_pitch(a.hidden) + n, S::sum(sh, threadIdx.x), 4);
}

// The same on tiles through LDS: kCols / 2 columns of h, for which W's rows are those of gate and the
// same of up, so that both products of a value of h meet in one lane, and a block of 32 of
// its columns in two: the scale of a block of h is found where its values are, and h is never stored
// in more than 4 bits.  32 tokens, 2 each, of 8 experts of 6144 x 16384 163 us up and 86 to 97 down
// (4.4 to 5.2 TB/s of the weights); 4096 tokens 1016 and 515: 3.3 and 3.2 PFLOP/s, in 36 blocks of
// places where 32 full ones would do.
template <class T>
__global__ __launch_bounds__(T::kThreads) void wc_experts_mx_up_tile_kernel(ExpertArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
  constexpr uint32_t kBM = T::kRows, kColumns = T::kCols / 2;
  static_assert(T::kNT % 2 == 0 && kColumns % 64 == 0 && kColumns % T::kStep == 0);
  uint32_t mt, nt;
  if (!tile_at(blockIdx.x, block_count(a), (a.ffn + kColumns - 1) / kColumns, mt, nt)) return;
  const auto [e, first, last] = block_at(a, mt);
  const uint32_t n0 = nt * kColumns, n_rows = min(kColumns, a.ffn - n0);
  const uint32_t blocks = (a.hidden + 31) / 32, words = (blocks + 3) / 4, pitch = blocks * 16;
  const auto matrix = [&](const Bank& b) {
    return rows_of(b.w + e * b.stride, pitch, Scales{b.scales.at + e * b.scale_stride, b.scales.pitch, b.scales.step}, n0,
                   n_rows, blocks);
  };
  const RowsOf G = matrix(a.gate), U = matrix(a.up);
  const RowsOf X = rows_of(a.xq, pitch, a.xs, 0, a.tokens, blocks);
  const uint32_t chunk = T::chunk_of(), woff = T::row_of(0) * pitch + chunk * 16;
  const auto token_of = [&](uint32_t row) { return slot_at(a, min(first + row, last - 1)) / a.k; };
  uint32_t xoff[T::kXLoads];
#pragma unroll
  for (int i = 0; i < T::kXLoads; i++) xoff[i] = token_of(T::row_of(i)) * pitch + chunk * 16;
  ScaleLoad scales[T::kSLoads];
#pragma unroll
  for (int j = 0; j < T::kSLoads; j++) {
    const uint32_t row = T::scale_row(j), at = T::first_scale_row(j);
    if (at < kBM) scales[j].set(X, token_of(row));
    else if (at < kBM + kColumns) scales[j].set(G, row - kBM);
    else scales[j].set(U, row - kBM - kColumns);
  }
  f32x16 acc[T::kMT][T::kNT];
  T::product(
      lds, T::stages_of(blocks), last - first, words,
      [&](int i, uint32_t s, uint32_t to) {
        load_lds(X.codes, to, (s * T::kBlocks + chunk < blocks ? xoff[i] : kNowhere) + s * T::kBytes);
      },
      [&](int i, uint32_t s, uint32_t to) {
        constexpr int kHalf = int(kColumns / T::kStep);
        load_lds(i < kHalf ? G.codes : U.codes, to, woff + (i % kHalf * T::kStep * pitch + s * T::kBytes));
      },
      [&](int j, uint32_t s, uint32_t to) { scales[j](s / T::kGroup, to); }, acc);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const uint32_t wm0 = wave / T::kWN_ * (T::kMT * 32), wn0 = wave % T::kWN_ * (T::kNT * 16);
#pragma unroll
  for (int nb = 0; nb < T::kNT / 2; nb++)
#pragma unroll
    for (int mb = 0; mb < T::kMT; mb++) {
      const uint32_t place = first + wm0 + mb * 32 + lane % 32, c0 = n0 + wn0 + nb * 32, block = c0 / 32;
      if (first + wm0 + mb * 32 >= last || c0 >= a.ffn) continue;
      const auto h = hidden<16>(
          acc[mb][nb], acc[mb][nb + T::kNT / 2], true,
          [&](uint32_t i) { return c0 + i / 4 * 8 + lane / 32 * 4 + i % 4 < a.ffn; },
          [](uint32_t top) {
            const auto both = __builtin_amdgcn_permlane32_swap(top, top, false, false);
            return max(both[0], both[1]);
          });
      // this lane's codes of every eight columns are two bytes, the other lane's the next two
      u32x4 codes;
#pragma unroll
      for (int p = 0; p < 2; p++) {
        const auto v = __builtin_amdgcn_permlane32_swap(h.codes[p], h.codes[p], false, false);
        codes[2 * p] = (v[0] & 0xFFFFu) | v[1] << 16;       // the lower lanes' own, the upper lanes'
        codes[2 * p + 1] = v[0] >> 16 | (v[1] & 0xFFFF0000u);
      }
      if (lane < 32 && place < last) {
        *global<u32x4>(h_codes(a, place, block)) = codes;
        store_h_scale(a, place, block, h.byte);
      }
    }
}

// down(h) of a block of places on tiles, stored by slot.
template <class T>
__global__ __launch_bounds__(T::kThreads) void wc_experts_mx_down_tile_kernel(ExpertArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
  constexpr uint32_t kBM = T::kRows, kBN = T::kCols;
  uint32_t mt, nt;
  if (!tile_at(blockIdx.x, block_count(a), (a.hidden + kBN - 1) / kBN, mt, nt)) return;
  const auto [e, first, last] = block_at(a, mt);
  const uint32_t n0 = nt * kBN, n_rows = min(kBN, a.hidden - n0);
  const uint32_t blocks = (a.ffn + 31) / 32, words = (blocks + 3) / 4, pitch = blocks * 16;
  const Bank& b = a.down;
  const RowsOf W = rows_of(b.w + e * b.stride, pitch,
                           Scales{b.scales.at + e * b.scale_stride, b.scales.pitch, b.scales.step}, n0, n_rows, blocks);
  const RowsOf X = rows_of(a.hq, pitch, a.hs, first, last - first, blocks);
  const uint32_t chunk = T::chunk_of(), off = T::row_of(0) * pitch + chunk * 16;
  ScaleLoad scales[T::kSLoads];
#pragma unroll
  for (int j = 0; j < T::kSLoads; j++)
    if (T::first_scale_row(j) < kBM) scales[j].set(X, T::scale_row(j));
    else scales[j].set(W, T::scale_row(j) - kBM);
  f32x16 acc[T::kMT][T::kNT];
  T::product(
      lds, T::stages_of(blocks), last - first, words,
      [&](int i, uint32_t s, uint32_t to) {
        load_lds(X.codes, to, (s * T::kBlocks + chunk < blocks ? off : kNowhere) + (i * T::kStep * pitch + s * T::kBytes));
      },
      [&](int i, uint32_t s, uint32_t to) { load_lds(W.codes, to, off + (i * T::kStep * pitch + s * T::kBytes)); },
      [&](int j, uint32_t s, uint32_t to) { scales[j](s / T::kGroup, to); }, acc);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const uint32_t wm0 = wave / T::kWN_ * (T::kMT * 32), c0 = n0 + wave % T::kWN_ * (T::kNT * 32);
#pragma unroll
  for (int mb = 0; mb < T::kMT; mb++) {
    const uint32_t place = first + wm0 + mb * 32 + lane % 32;
    if (first + wm0 + mb * 32 >= last) break;
    const uint64_t row = uint64_t(slot_at(a, min(place, last - 1))) * out_pitch(a.hidden);
#pragma unroll
    for (int nb = 0; nb < T::kNT; nb++)
      rows_out(acc[mb][nb], [&](uint32_t column, f32x4 low, f32x4 high) {
        const uint32_t n = c0 + nb * 32 + column;
        if (place >= last || n >= a.hidden) return;
        const auto to = global<f32x4>(a.out + (row + n) * 4);
        to[0] = low;
        to[1] = high;
      });
  }
}

// y of one token, four columns a thread: its slots' results in their order, times their weights.
// Bound by memory: 4096 tokens of 6144, 2 slots each, 46 us (5.5 TB/s).
__global__ __launch_bounds__(256) void wc_experts_mx_join_kernel(ExpertArgs a) {
  const uint32_t n = (blockIdx.y * 256 + threadIdx.x) * 4;
  const uint64_t token = blockIdx.x;
  if (n >= a.hidden) return;
  const uint32_t left = a.hidden - n;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (uint32_t j = 0; j < a.k; j++) {
    const uint64_t slot = token * a.k + j;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (global<const int32_t>(a.ids)[slot] >= 0) v = *global<const f32x4>(a.out + (slot * out_pitch(a.hidden) + n) * 4);
    const float w = global<const float>(a.weights)[slot];
#pragma unroll
    for (int i = 0; i < 4; i++) sum[i] += w * v[i];
  }
  store_four(a.y, a.dtype, token * a.ldy + n, sum, left);
}

// Blocks of `rows` places: every expert that has places ends in one that may not be full.
uint64_t most_blocks(uint32_t slots, uint32_t experts, uint32_t rows) {
  return uint64_t(slots) / rows + std::min(experts, slots);
}
struct Workspace {
  uint64_t table, xq, xs, hq, hs, out, gate, up, down, bytes;  // gate, up, down: copies of scales
};
Workspace layout(uint64_t tokens, uint64_t k, uint32_t experts, uint32_t hidden, uint32_t ffn) {
  Workspace w{};
  const auto take = [&](uint64_t bytes) {
    const uint64_t here = w.bytes;
    w.bytes += pad256(bytes);
    return here;
  };
  w.hq = take(tokens * k * WC_MX_ROW_BYTES(ffn));
  w.hs = take(own_scales_bytes(tokens * k, ffn));
  if (is_few(tokens, k, hidden)) return w;
  w.table = take((1 + most_blocks(uint32_t(tokens * k), experts, 16)) * 16);
  w.xq = take(tokens * WC_MX_ROW_BYTES(hidden));
  w.xs = take(own_scales_bytes(tokens, hidden));
  w.out = take(tokens * k * out_pitch(hidden) * 4);
  // room for the copies at any alignment of the scales
  w.gate = take(own_scales_bytes(uint64_t(experts) * ffn, hidden));
  w.up = take(own_scales_bytes(uint64_t(experts) * ffn, hidden));
  w.down = take(own_scales_bytes(uint64_t(experts) * hidden, ffn));
  return w;
}
bool sizes_ok(uint32_t tokens, uint32_t k, uint32_t experts, uint32_t hidden, uint32_t ffn) {
  return k >= 1 && experts >= 1 && experts <= kMaxExperts && k <= experts && hidden >= 1 &&
         hidden <= kMaxK && ffn >= 1 && ffn <= kMaxK && uint64_t(tokens) * k < (1ull << 24);
}
bool bank_ok(const wc_mx_experts* b, uint64_t n, uint32_t k) {
  return b && !off(b->w, 16) && b->scale && b->stride % 16 == 0 && b->stride >= n * WC_MX_ROW_BYTES(k) &&
         b->scale_stride >= n * WC_MX_BLOCKS(k) && !(b->stride >> 40) && !(b->scale_stride >> 40);
}
Bank bank(const wc_mx_experts* b, uint32_t k) {
  return {reinterpret_cast<uint64_t>(b->w), b->stride,
          {reinterpret_cast<uint64_t>(b->scale), blocks_of(k), 16}, b->scale_stride};
}
bool tensors_ok(const void* x, int32_t dtype, uint32_t tokens, uint64_t ldx, uint32_t hidden, uint32_t ffn,
                const wc_mx_experts* gate, const wc_mx_experts* up, const wc_mx_experts* down, const void* y,
                uint64_t ldy) {
  return float_ok(dtype) && ldx >= hidden && !(ldx >> 31) && ldy >= hidden && !(ldy >> 31) &&
         bank_ok(gate, ffn, hidden) && bank_ok(up, ffn, hidden) && bank_ok(down, hidden, ffn) &&
         (tokens == 0 || (!off(x, size_of(dtype)) && !off(y, size_of(dtype))));
}
ExpertArgs args_of(const void* x, int32_t dtype, uint32_t tokens, uint64_t ldx, uint32_t k, uint32_t experts,
                   uint32_t hidden, uint32_t ffn, const wc_mx_experts* gate, const wc_mx_experts* up,
                   const wc_mx_experts* down, void* y, uint64_t ldy, const Workspace& w, uint64_t ws) {
  ExpertArgs a{};
  a.table = ws + w.table;
  a.x = reinterpret_cast<uint64_t>(x);
  a.ldx = ldx;
  a.xq = ws + w.xq;
  a.xs = own_scales(ws + w.xs, tokens, hidden);
  a.hq = ws + w.hq;
  a.hs = own_scales(ws + w.hs, uint64_t(tokens) * k, ffn);
  a.out = ws + w.out;
  a.y = reinterpret_cast<uint64_t>(y);
  a.ldy = ldy;
  a.tokens = tokens;
  a.k = k;
  a.experts = experts;
  a.hidden = hidden;
  a.ffn = ffn;
  a.slots = tokens * k;
  a.dtype = dtype;
  a.gate = bank(gate, hidden);
  a.up = bank(up, hidden);
  a.down = bank(down, ffn);
  return a;
}

template <int kType, int kPer>
void start_up(const ExpertArgs& a, const RouteArgs& route, hipStream_t st) {
  const uint32_t most = (a.ffn + 31) / 32 * std::min(a.slots, a.experts);
  const uint32_t held = uint32_t(groups_of(a.hidden)) * kHeldPart;
  // two workgroups of four waves to a compute unit, or one of eight
  if (a.hidden <= 2048)
    hipLaunchKernelGGL((wc_moe_mx_up_kernel<kType, kPer, 4>), dim3(std::min(most, 512u)), dim3(256), held, st, a, route);
  else
    hipLaunchKernelGGL((wc_moe_mx_up_kernel<kType, kPer, 8>), dim3(std::min(most, 256u)), dim3(512), held, st, a, route);
}
template <int kType>
void start_up(const ExpertArgs& a, const RouteArgs* route, hipStream_t st) {
  if (!route) start_up<kType, 0>(a, RouteArgs{}, st);
  else if (a.experts <= 64) start_up<kType, 1>(a, *route, st);
  else if (a.experts <= 128) start_up<kType, 2>(a, *route, st);
  else if (a.experts <= 256) start_up<kType, 4>(a, *route, st);
  else start_up<kType, 8>(a, *route, st);
}
// Few tokens, by `route` or the ids that a names.
wc_status few(const ExpertArgs& a, const RouteArgs* route, hipStream_t st) {
  if (a.dtype == WC_BF16) start_up<WC_BF16>(a, route, st);
  else if (a.dtype == WC_FP16) start_up<WC_FP16>(a, route, st);
  else start_up<WC_FP32>(a, route, st);
  if (hipGetLastError() != hipSuccess) return WC_EHIP;
  hipLaunchKernelGGL(wc_moe_mx_down_kernel, dim3((a.hidden + 15) / 16), dim3(64 * kFewWaves),
                     std::min(a.slots, a.experts) * 16 * 6, st, a);
  return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
}

// tokens * k < 2^24: at most 2^20 + 512 blocks, of less than 2^32 threads, a grid axis's limit.
bool start_slim(const ExpertArgs& a, uint32_t most, hipStream_t st) {
  hipLaunchKernelGGL(wc_experts_mx_up_slim_kernel, dim3(most, (a.ffn + 31) / 32), dim3(512), 0, st, a);
  if (hipGetLastError() != hipSuccess) return false;
  hipLaunchKernelGGL(wc_experts_mx_down_slim_kernel, dim3(most, (a.hidden + 31) / 32), dim3(512), 0, st, a);
  return hipGetLastError() == hipSuccess;
}

// Tiles by the places of a block: up's columns are half of gate's and half of up's.
template <int kPlaces>
struct Tiles;
template <>
struct Tiles<64> {
  using Up = MxTile<64, 128, 2, 2, 2, true>;
  using Down = MxTile<64, 128, 2, 2, 2>;
};
template <>
struct Tiles<128> {
  using Up = MxTile<128, 128, 2, 2, 2, true>;
  using Down = MxTile<128, 128, 2, 2, 2>;
};
template <>
struct Tiles<256> {
  using Up = MxTile<256, 256, 2, 4, 2, true>;
  using Down = MxTile<256, 256, 2, 4, 2>;
};
uint32_t tiles(uint32_t n, uint32_t each) { return (n + each - 1) / each; }
// Scales that the tiles cannot load as they are: their copies instead.
void copy_of(Bank& b, uint64_t to, uint32_t experts, uint32_t n, uint32_t k, ScaleCopies& copies) {
  if (whole_words(reinterpret_cast<const void*>(b.scales.at), blocks_of(k), k) && b.scale_stride % 4 == 0) return;
  const Scales own = own_scales(to, uint64_t(experts) * n, k);
  copies.add(b.scales.at, blocks_of(k), n, b.scale_stride, uint64_t(experts) * n, k, own);
  b.scales = own;
  b.scale_stride = uint64_t(n) * own.pitch;
}
template <int kPlaces>
bool start_tiles(const ExpertArgs& a, uint32_t most, hipStream_t st) {
  using Up = typename Tiles<kPlaces>::Up;
  using Down = typename Tiles<kPlaces>::Down;
  hipLaunchKernelGGL(wc_experts_mx_up_tile_kernel<Up>, dim3(most * tiles(a.ffn, Up::kCols / 2)), dim3(Up::kThreads), 0,
                     st, a);
  if (hipGetLastError() != hipSuccess) return false;
  hipLaunchKernelGGL(wc_experts_mx_down_tile_kernel<Down>, dim3(most * tiles(a.hidden, Down::kCols)),
                     dim3(Down::kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess;
}
// Places to a block; 16: straight from memory to registers, at any sizes.  Up to 16 tokens, which are all
// the places that an expert has, us with 16 and 64: 8 experts, 2 a token, of 8224 x 16384: 1 token 115,
// 190; 2 196, 249; 4 363, 337; 16 418, 475; 64, 6, 8224 x 2048: 1 58, 121; 16 333, 340; 4, 1, 12288 x
// 4096: 1 33, 50; 8 78, 84; 16 89, 86; 1, 1, 16384 x 53248: 3 316, 376.  More with 64, 128 and 256:
//   8 experts, 2 a token, of 4096 x 14336: 64 tokens 172, 181, 215; 128 177, 192, 226; 256 217,
//     203, 236; 600 (tiles of 64 with two waves less) 426, 275, 270; 1500 876, 518, 384
//   64, 6, 2048 x 1408: 60 78, 80, 89; 200 83, 84, 92; 700 123, 103, 111; 2000 293, 175, 156
//   7, 3, 2049 x 1365: 77 39, 40, 47; 256 43, 45, 54
//   128, 8, 4096 x 1536: 40 248, 254, 283; 1000 403, 367, 387
uint32_t places(const ExpertArgs& a) {
  // on tiles x lies within 32-bit offsets, its scales group by group; a grid's axis has less than 2^32 threads
  if (a.tokens <= kFew || a.tokens * WC_MX_ROW_BYTES(a.hidden) >> 31 || own_scales_bytes(a.tokens, a.hidden) >> 30 ||
      most_blocks(a.slots, a.experts, 64) * std::max(tiles(a.ffn, 64), tiles(a.hidden, 128)) * 256 >> 32)
    return 16;
  const uint32_t average = a.slots / a.experts;
  return average < 48 ? 64 : average < 160 ? 128 : 256;
}

wc_status experts(ExpertArgs a, const Workspace& w, const int32_t* offsets, hipStream_t st) {
  if (is_few(a.tokens, a.k, a.hidden)) return few(a, nullptr, st);
  const uint32_t rows = places(a), most = uint32_t(most_blocks(a.slots, a.experts, rows));
  const Blocks blocks = {a.table, reinterpret_cast<uint64_t>(offsets), a.experts, a.slots, rows, most};
  ScaleCopies copies;
  copies.n = copies.groups = 0;
  const uint64_t ws = a.hq - w.hq;
  if (rows >= 64) {
    copy_of(a.gate, ws + w.gate, a.experts, a.ffn, a.hidden, copies);
    copy_of(a.up, ws + w.up, a.experts, a.ffn, a.hidden, copies);
    copy_of(a.down, ws + w.down, a.experts, a.hidden, a.ffn, copies);
  }
  if (!launch_quantize(reinterpret_cast<const void*>(a.x), a.dtype, a.tokens, a.hidden, a.ldx,
                       reinterpret_cast<void*>(a.xq), WC_MX_ROW_BYTES(a.hidden), a.xs,
                       uint32_t(groups_of(a.hidden)) * 16, st, &blocks, &copies))
    return WC_EHIP;
  const bool started = rows == 16   ? start_slim(a, most, st)
                       : rows == 64 ? start_tiles<64>(a, most, st)
                       : rows == 128 ? start_tiles<128>(a, most, st)
                                     : start_tiles<256>(a, most, st);
  if (!started) return WC_EHIP;
  hipLaunchKernelGGL(wc_experts_mx_join_kernel, dim3(a.tokens, (a.hidden + 1023) / 1024), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
}

// What wc_moe_mx keeps of the routing, before the rest.
struct RouteSpace {
  uint64_t ids, weights, offsets, order, scratch, scratch_bytes, bytes;
};
RouteSpace route_layout(uint32_t tokens, const wc_route_params* p, uint32_t hidden) {
  RouteSpace r{};
  const auto take = [&](uint64_t bytes) {
    const uint64_t here = r.bytes;
    r.bytes += pad256(bytes);
    return here;
  };
  const uint64_t slots = uint64_t(tokens) * p->k;
  r.ids = take(slots * 4);
  r.weights = take(slots * 4);
  if (is_few(tokens, p->k, hidden)) return r;
  r.offsets = take((p->experts + 1) * 4);
  r.order = take(slots * 4);
  wc_route_workspace_bytes(tokens, p, &r.scratch_bytes);
  r.scratch = take(r.scratch_bytes);
  return r;
}

}  // namespace

extern "C" wc_status wc_experts_mx_workspace_bytes(uint32_t tokens, uint32_t k, uint32_t experts,
                                                   uint32_t hidden, uint32_t ffn, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!sizes_ok(tokens, k, experts, hidden, ffn)) return WC_EINVAL;
  *bytes = layout(tokens, k, experts, hidden, ffn).bytes;
  return WC_OK;
}

extern "C" wc_status wc_experts_mx(const void* dev_x, int32_t dtype, uint32_t tokens, uint64_t ldx, uint32_t k,
                                   uint32_t n_experts, uint32_t hidden, uint32_t ffn, const int32_t* dev_ids,
                                   const float* dev_weights, const int32_t* dev_offsets,
                                   const int32_t* dev_order, const wc_mx_experts* gate, const wc_mx_experts* up,
                                   const wc_mx_experts* down, void* dev_y, uint64_t ldy, void* dev_workspace,
                                   uint64_t workspace_bytes, void* stream) {
  if (!sizes_ok(tokens, k, n_experts, hidden, ffn) ||
      !tensors_ok(dev_x, dtype, tokens, ldx, hidden, ffn, gate, up, down, dev_y, ldy))
    return WC_EINVAL;
  if (tokens == 0) return WC_OK;
  if (off(dev_ids, 4) || off(dev_weights, 4) || off(dev_offsets, 4) || off(dev_order, 4)) return WC_EINVAL;
  const Workspace w = layout(tokens, k, n_experts, hidden, ffn);
  if (off(dev_workspace, 256) || workspace_bytes < w.bytes) return WC_EINVAL;
  ExpertArgs a = args_of(dev_x, dtype, tokens, ldx, k, n_experts, hidden, ffn, gate, up, down, dev_y, ldy, w,
                         reinterpret_cast<uint64_t>(dev_workspace));
  a.order = reinterpret_cast<uint64_t>(dev_order);
  a.ids = reinterpret_cast<uint64_t>(dev_ids);
  a.weights = reinterpret_cast<uint64_t>(dev_weights);
  return experts(a, w, dev_offsets, reinterpret_cast<hipStream_t>(stream));
}

extern "C" wc_status wc_moe_mx_workspace_bytes(uint32_t tokens, const wc_route_params* p, uint32_t hidden,
                                               uint32_t ffn, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!wc_choose::params_ok(tokens, p) || !sizes_ok(tokens, p->k, p->experts, hidden, ffn)) return WC_EINVAL;
  *bytes = route_layout(tokens, p, hidden).bytes + layout(tokens, p->k, p->experts, hidden, ffn).bytes;
  return WC_OK;
}

extern "C" wc_status wc_moe_mx(const void* dev_x, int32_t dtype, uint32_t tokens, uint64_t ldx,
                               const void* dev_logits, int32_t logits_dtype, uint64_t ld,
                               const wc_route_params* p, const float* dev_bias, uint32_t hidden, uint32_t ffn,
                               const wc_mx_experts* gate, const wc_mx_experts* up, const wc_mx_experts* down,
                               void* dev_y, uint64_t ldy, void* dev_workspace, uint64_t workspace_bytes,
                               void* stream) {
  uint64_t need = 0;
  if (wc_moe_mx_workspace_bytes(tokens, p, hidden, ffn, &need) != WC_OK ||
      !tensors_ok(dev_x, dtype, tokens, ldx, hidden, ffn, gate, up, down, dev_y, ldy) ||
      !float_ok(logits_dtype) || ld < p->experts || ld >> 31 || (dev_bias && off(dev_bias, 4)))
    return WC_EINVAL;
  if (tokens == 0) return WC_OK;
  if (off(dev_logits, size_of(logits_dtype)) || off(dev_workspace, 256) || workspace_bytes < need) return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const uint64_t ws = reinterpret_cast<uint64_t>(dev_workspace);
  const RouteSpace r = route_layout(tokens, p, hidden);
  const Workspace w = layout(tokens, p->k, p->experts, hidden, ffn);
  ExpertArgs a = args_of(dev_x, dtype, tokens, ldx, p->k, p->experts, hidden, ffn, gate, up, down, dev_y, ldy, w,
                         ws + r.bytes);
  a.ids = ws + r.ids;
  a.weights = ws + r.weights;
  if (is_few(tokens, p->k, hidden)) {
    const RouteArgs route = {reinterpret_cast<uint64_t>(dev_logits), reinterpret_cast<uint64_t>(dev_bias),
                             a.ids, a.weights, ld, tokens, p->experts, p->k, p->groups, p->top_groups,
                             p->group_top, 0, logits_dtype, p->score, p->renormalize, p->scale};
    return few(a, &route, st);
  }
  a.order = ws + r.order;
  const wc_status s = wc_route(dev_logits, logits_dtype, tokens, ld, p, dev_bias,
                               reinterpret_cast<int32_t*>(a.ids), reinterpret_cast<float*>(a.weights),
                               reinterpret_cast<int32_t*>(ws + r.offsets), reinterpret_cast<int32_t*>(a.order),
                               reinterpret_cast<void*>(ws + r.scratch), r.scratch_bytes, stream);
  return s == WC_OK ? experts(a, w, reinterpret_cast<const int32_t*>(ws + r.offsets), st) : s;
}
