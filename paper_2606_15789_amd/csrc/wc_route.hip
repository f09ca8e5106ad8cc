// wc_route.hip -- routing to experts: wc_route.
#include <cmath>

#include "wc_i8.h"

namespace {

using namespace wc_i8;

constexpr int kTokenWaves = 4;         // tokens to a workgroup of the choice
constexpr uint32_t kSortThreads = 1024;
constexpr uint32_t kSortSlots = 2048;  // slots to a workgroup of the sort
constexpr uint32_t kMaxChosen = 32;

struct RouteArgs {
  uint64_t logits, bias, ids, weights, ld;
  uint32_t tokens, experts, k, groups, top_groups, group_top;
  int32_t dtype, score, renormalize;
  float scale;
};

struct Best {
  float key;
  uint32_t at;
};
// The larger key, the lower index among equals.
__device__ __forceinline__ Best better(Best a, Best b) {
  return b.key > a.key || (b.key == a.key && b.at < a.at) ? b : a;
}
__device__ __forceinline__ Best wave_best(Best b) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
    b = better(b, {__shfl_xor(b.key, d), uint32_t(__shfl_xor(int(b.at), d))});
  return b;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// One wave a token, experts lane + 64 i in its registers.  A softmax without a
// bias chooses by the logits, which are in the scores' order, so no two of them
// fall together by rounding.
template <int kPer>
__global__ __launch_bounds__(64 * kTokenWaves) void wc_route_choose_kernel(RouteArgs a) {
  __shared__ float keys[kTokenWaves][64 * kPer];
  __shared__ uint8_t kept[kTokenWaves][64 * kPer];
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t token = blockIdx.x * kTokenWaves + wave;
  const bool live = token < a.tokens;
  const float ninf = -__builtin_inff();
  float s[kPer], key[kPer];
  bool bad = false;
  float top = ninf;
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    const uint32_t e = lane + 64 * i;
    float x = ninf, b = 0.0f;
    if (live && e < a.experts) {
      x = load_float(a.logits, a.dtype, token * a.ld + e);
      if (a.bias) b = global<const float>(a.bias)[e];
    }
    if (b == ninf) x = ninf;
    s[i] = x;
    key[i] = b;
    if (x != ninf) bad = bad || x != x || b != b;
    top = fmaxf(top, x);
  }
  const bool soft = a.score == WC_SCORE_SOFTMAX;
  if (soft) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  }
  const bool by_logits = soft && !a.bias && (a.groups == 1 || a.group_top == 1);
  float total = 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    const float x = s[i];
    const bool off = x == ninf;
    s[i] = off ? 0.0f : soft ? expf(x - top) : 1.0f / (1.0f + expf(-x));
    total += s[i];
    if (by_logits) key[i] = x;
    else if (!soft) key[i] = off ? ninf : s[i] + key[i];
    else if (off) key[i] = ninf;
  }
  if (soft) {
    total = wave_sum(total);
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      s[i] = total != 0.0f ? s[i] / total : 0.0f;
      if (!by_logits && key[i] != ninf) key[i] += s[i];
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; i++)
    if (key[i] != key[i]) key[i] = ninf;
  if (a.groups > 1) {
    const uint32_t per = a.experts / a.groups;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      keys[wave][lane + 64 * i] = key[i];
      kept[wave][lane + 64 * i] = 0;
    }
    __syncthreads();
    float best[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const uint32_t g = lane + 64 * i;
      float first = ninf, second = ninf;
      if (g < a.groups)
        for (uint32_t j = 0; j < per; j++) {
          const float v = keys[wave][g * per + j];
          second = fmaxf(second, fminf(first, v));
          first = fmaxf(first, v);
        }
      best[i] = a.group_top == 2 ? first + second : first;
    }
    uint32_t taken = 0;  // bit i: group lane + 64 i
    for (uint32_t n = 0; n < a.top_groups; n++) {
      Best b = {ninf, 0xFFFFFFFFu};
#pragma unroll
      for (int i = 0; i < kPer; i++)
        if (lane + 64 * i < a.groups && !(taken >> i & 1)) b = better(b, {best[i], lane + 64 * i});
      b = wave_best(b);
      if (b.at % 64 == lane && b.at < a.groups) {
        taken |= 1u << (b.at / 64);
        kept[wave][b.at] = 1;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const uint32_t e = lane + 64 * i;
      if (e < a.experts && !kept[wave][e / per]) key[i] = ninf;
    }
  }
  int32_t id = -1;
  float weight = 0.0f;
  for (uint32_t n = 0; n < a.k; n++) {
    Best b = {ninf, 0xFFFFFFFFu};
#pragma unroll
    for (int i = 0; i < kPer; i++) b = better(b, {key[i], lane + 64 * i});
    b = wave_best(b);
    if (b.key == ninf) break;
    float mine = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; i++)
      if (b.at == lane + 64 * i) {
        mine = s[i];
        key[i] = ninf;
      }
    mine = __shfl(mine, int(b.at % 64));
    if (lane == n) {
      id = int32_t(b.at);
      weight = mine;
    }
  }
  if (a.renormalize) {
    const float sum = wave_sum(weight);
    weight = sum != 0.0f ? weight / sum : 0.0f;
  }
  weight *= a.scale;
  if (__ballot(bad)) weight = __builtin_nanf("");
  if (live && lane < a.k) {
    const uint64_t at = uint64_t(token) * a.k + lane;
    global<int32_t>(a.ids)[at] = id;
    global<float>(a.weights)[at] = weight;
  }
}

struct SortArgs {
  uint64_t ids, offsets, order, hist;
  uint32_t slots, experts, blocks;
};
__device__ __forceinline__ uint32_t class_of(const SortArgs& a, uint32_t slot) {
  const int32_t id = global<const int32_t>(a.ids)[slot];
  return id < 0 ? a.experts : uint32_t(id);
}

// How many slots of each block of kSortSlots each expert has (and how many have none).
__global__ __launch_bounds__(kSortThreads) void wc_route_count_kernel(SortArgs a) {
  __shared__ uint32_t count[kMaxExperts + 1];
  for (uint32_t e = threadIdx.x; e <= a.experts; e += kSortThreads) count[e] = 0;
  __syncthreads();
  const uint32_t first = blockIdx.x * kSortSlots, left = min(kSortSlots, a.slots - first);
  for (uint32_t i = threadIdx.x; i < left; i += kSortThreads)
    atomicAdd(&count[class_of(a, first + i)], 1u);
  __syncthreads();
  for (uint32_t e = threadIdx.x; e <= a.experts; e += kSortThreads)
    global<uint32_t>(a.hist)[uint64_t(blockIdx.x) * (a.experts + 1) + e] = count[e];
}

// The stable order of one block's slots: each expert's first place (all experts
// before it, all blocks before this one, all waves before this wave), then the
// rank of a slot among its wave's with the same expert.
__global__ __launch_bounds__(kSortThreads) void wc_route_order_kernel(SortArgs a) {
  constexpr uint32_t kWaves = kSortThreads / 64, kEach = kSortSlots / kWaves;
  __shared__ uint32_t next[kWaves][kMaxExperts + 1], wave_total[kWaves];
  const uint32_t t = threadIdx.x, lane = t % 64, wave = t / 64, classes = a.experts + 1;
  for (uint32_t w = 0; w < kWaves; w++)
    for (uint32_t e = t; e < classes; e += kSortThreads) next[w][e] = 0;
  __syncthreads();
  const uint32_t first = blockIdx.x * kSortSlots + wave * kEach;
  uint32_t mine[kEach / 64];
#pragma unroll
  for (uint32_t i = 0; i < kEach / 64; i++) {
    const uint32_t slot = first + i * 64 + lane;
    mine[i] = slot < a.slots ? class_of(a, slot) : 0xFFFFFFFFu;
    if (slot < a.slots) atomicAdd(&next[wave][mine[i]], 1u);
  }
  __syncthreads();
  // a thread an expert: its slots in all blocks, and in the blocks before this one
  uint32_t all = 0, before = 0;
  if (t < classes) {
    if (a.blocks == 1) {
      for (uint32_t w = 0; w < kWaves; w++) all += next[w][t];
    } else {
      for (uint32_t b = 0; b < a.blocks; b++) {
        const uint32_t n = global<const uint32_t>(a.hist)[uint64_t(b) * classes + t];
        all += n;
        before += b < blockIdx.x ? n : 0;
      }
    }
  }
  // exclusive scan over the experts
  uint32_t sum = all;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t v = uint32_t(__shfl_up(int(sum), d));
    if (lane >= uint32_t(d)) sum += v;
  }
  if (lane == 63) wave_total[wave] = sum;
  __syncthreads();
  uint32_t start = sum - all;
  for (uint32_t w = 0; w < wave; w++) start += wave_total[w];
  if (t < classes) {
    if (blockIdx.x == 0) global<int32_t>(a.offsets)[t] = int32_t(start);
    uint32_t at = start + before;
    for (uint32_t w = 0; w < kWaves; w++) {
      const uint32_t n = next[w][t];
      next[w][t] = at;
      at += n;
    }
  }
  __syncthreads();
  volatile uint32_t* const mine_next = next[wave];  // lanes read what another lane wrote
#pragma unroll
  for (uint32_t i = 0; i < kEach / 64; i++) {
    const bool on = mine[i] != 0xFFFFFFFFu;
    uint64_t same = __ballot(on);
    for (uint32_t bit = 1; bit < classes; bit *= 2) {
      const uint64_t set = __ballot((mine[i] & bit) != 0);
      same &= mine[i] & bit ? set : ~set;
    }
    if (on) {
      const uint32_t rank = uint32_t(__popcll(same & ((1ull << lane) - 1)));
      const uint32_t place = mine_next[mine[i]] + rank;
      global<int32_t>(a.order)[place] = int32_t(first + i * 64 + lane);
    }
    __builtin_amdgcn_wave_barrier();
    if (on && !(same >> lane >> 1))
      mine_next[mine[i]] = mine_next[mine[i]] + uint32_t(__popcll(same));
    __builtin_amdgcn_wave_barrier();
  }
}

bool params_ok(uint32_t tokens, const wc_route_params* p) {
  return p && p->experts >= 1 && p->experts <= kMaxExperts && p->k >= 1 && p->k <= p->experts &&
         p->k <= kMaxChosen && (p->score == WC_SCORE_SOFTMAX || p->score == WC_SCORE_SIGMOID) &&
         p->groups >= 1 && p->experts % p->groups == 0 && p->top_groups >= 1 &&
         p->top_groups <= p->groups && p->group_top >= 1 && p->group_top <= 2 &&
         p->group_top <= p->experts / p->groups && std::isfinite(p->scale) &&
         uint64_t(tokens) * p->k < (1ull << 31);
}
uint32_t sort_blocks(uint32_t slots) { return slots ? (slots + kSortSlots - 1) / kSortSlots : 1; }

}  // namespace

extern "C" wc_status wc_route_workspace_bytes(uint32_t tokens, const wc_route_params* p,
                                              uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!params_ok(tokens, p)) return WC_EINVAL;
  const uint32_t blocks = sort_blocks(tokens * p->k);
  if (blocks > 1) *bytes = uint64_t(blocks) * (p->experts + 1) * 4;
  return WC_OK;
}

extern "C" wc_status wc_route(const void* dev_logits, int32_t dtype, uint32_t tokens, uint64_t ld,
                              const wc_route_params* p, const float* dev_bias, int32_t* dev_ids,
                              float* dev_weights, int32_t* dev_offsets, int32_t* dev_order,
                              void* dev_workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (wc_route_workspace_bytes(tokens, p, &need) != WC_OK || !float_ok(dtype) || ld < p->experts ||
      ld >> 31 || !dev_offsets)
    return WC_EINVAL;
  const auto off = [](const void* ptr, uint32_t to) {
    return reinterpret_cast<uintptr_t>(ptr) % to != 0;
  };
  if (off(dev_offsets, 4) || off(dev_bias, 4)) return WC_EINVAL;
  if (tokens && (!dev_logits || !dev_ids || !dev_weights || !dev_order ||
                 off(dev_logits, size_of(dtype)) || off(dev_ids, 4) || off(dev_weights, 4) ||
                 off(dev_order, 4)))
    return WC_EINVAL;
  if (need && (!dev_workspace || off(dev_workspace, 16) || workspace_bytes < need)) return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const RouteArgs a = {reinterpret_cast<uint64_t>(dev_logits), reinterpret_cast<uint64_t>(dev_bias),
                       reinterpret_cast<uint64_t>(dev_ids), reinterpret_cast<uint64_t>(dev_weights),
                       ld, tokens, p->experts, p->k, p->groups, p->top_groups, p->group_top, dtype,
                       p->score, p->renormalize, p->scale};
  if (tokens) {
    const dim3 grid((tokens + kTokenWaves - 1) / kTokenWaves), block(64 * kTokenWaves);
    switch ((p->experts + 63) / 64) {
      case 1: hipLaunchKernelGGL((wc_route_choose_kernel<1>), grid, block, 0, st, a); break;
      case 2: hipLaunchKernelGGL((wc_route_choose_kernel<2>), grid, block, 0, st, a); break;
      case 3: case 4: hipLaunchKernelGGL((wc_route_choose_kernel<4>), grid, block, 0, st, a); break;
      default: hipLaunchKernelGGL((wc_route_choose_kernel<8>), grid, block, 0, st, a); break;
    }
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
  }
  const SortArgs s = {a.ids, reinterpret_cast<uint64_t>(dev_offsets),
                      reinterpret_cast<uint64_t>(dev_order),
                      reinterpret_cast<uint64_t>(dev_workspace), tokens * p->k, p->experts,
                      sort_blocks(tokens * p->k)};
  if (s.blocks > 1) {
    hipLaunchKernelGGL(wc_route_count_kernel, dim3(s.blocks), dim3(kSortThreads), 0, st, s);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
  }
  hipLaunchKernelGGL(wc_route_order_kernel, dim3(s.blocks), dim3(kSortThreads), 0, st, s);
  return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
}
