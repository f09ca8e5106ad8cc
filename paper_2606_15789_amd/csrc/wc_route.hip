// wc_route.hip -- routing to experts: wc_route.
#include <algorithm>
#include <cmath>

#include "wc_i8.h"

namespace {

using namespace wc_i8;

constexpr int kTokenWaves = 4;         // waves to a workgroup of the choice
constexpr uint32_t kSortThreads = 1024;
constexpr uint32_t kSortSlots = 2048;  // slots to a workgroup of the sort
constexpr uint32_t kMaxChosen = 32;
constexpr uint32_t kLaunchTokens = 1u << 24;  // a grid's axis has less than 2^32 threads
// Blocks of the sort up to which each counts all slots itself, in place of a launch that
// counts: 512 tokens of 8 slots (2 blocks) 13.9 us against 15.0, 1500 (6) 17.7 and 16.5,
// but the host has a launch less.
constexpr uint32_t kSelfCount = 4;
// Counts (blocks of the sort times experts and one) from which they are summed up once, by a
// launch more, and no longer by every block for itself.  With the launch and without, us: 8
// experts 39.5 and 38.0 at 768 blocks, 65.9 and 70.0 at 1536; 61 experts 28.1 and 27.4 at 192,
// 43.9 and 45.1 at 384; 256 experts 28.5 and 30.5 at 64; 512 experts 27.9 and 32.8 at 32.
constexpr uint64_t kSumCounts = 16384;
// Tokens from which four share a wave where they fit: 32768 of 61 experts 20.3 us against
// 24.0, 4096 11.7 and 11.1.
constexpr uint32_t kManyTokens = 16384;

struct RouteArgs {
  uint64_t logits, bias, ids, weights, ld;
  uint32_t tokens, experts, k, groups, top_groups, group_top;
  uint32_t first;  // this launch's first token
  int32_t dtype, score, renormalize;
  float scale;
};

// Reductions over kLanes neighbouring lanes (16, 32 or 64), every lane gets the result:
// rotations within the sixteen lanes of a row, then the rows by readlane.
template <int kLanes, class Op>
__device__ __forceinline__ uint32_t reduced(uint32_t v, Op op) {
  v = op(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xF, 0xF, false)));
  v = op(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xF, 0xF, false)));
  v = op(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xF, 0xF, false)));
  v = op(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xF, 0xF, false)));
  if constexpr (kLanes == 16) return v;
  const auto row = [&](int lane) { return uint32_t(__builtin_amdgcn_readlane(int(v), lane)); };
  const uint32_t low = op(row(0), row(16)), high = op(row(32), row(48));
  if constexpr (kLanes == 32) return threadIdx.x % 64 < 32 ? low : high;
  return op(low, high);
}
template <int kLanes>
__device__ __forceinline__ uint32_t top_of(uint32_t v) {
  return reduced<kLanes>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
template <int kLanes>
__device__ __forceinline__ float sum_of(float v) {
  return __uint_as_float(reduced<kLanes>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
// The lanes of this lane's group for which `on` holds, from bit 0 on.
template <int kLanes>
__device__ __forceinline__ uint64_t votes(bool on) {
  const uint64_t all = __ballot(on);
  if constexpr (kLanes == 64) return all;
  return all >> (threadIdx.x % 64 / kLanes * kLanes) & ((1ull << kLanes) - 1);
}
// Numbers in order as unsigned ones; -0 as 0, NaN as -inf.
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t b = __float_as_uint(f == f ? f + 0.0f : -__builtin_inff());
  return b >> 31 ? ~b : b | 0x80000000u;
}
constexpr uint32_t kNone = 0x007FFFFFu;  // ordered(-inf)

// The greatest of all the lanes' key[i] (the expert or group lane + kLanes i), the lowest
// index among equals; its place, or -1 if nothing is above -inf (`floor`).  That key is
// taken out.
template <int kLanes, int kPer>
__device__ __forceinline__ int32_t take_best(uint32_t (&key)[kPer], uint32_t floor) {
  uint32_t best = key[0];
#pragma unroll
  for (int i = 1; i < kPer; i++) best = max(best, key[i]);
  best = top_of<kLanes>(best);
  int32_t at = -1;
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    const uint64_t v = votes<kLanes>(key[i] == best);
    if (at < 0 && v) at = i * kLanes + __builtin_ctzll(v);
  }
  if (best <= floor) at = -1;
  const int32_t lane = int32_t(threadIdx.x % kLanes);
#pragma unroll
  for (int i = 0; i < kPer; i++)
    if (at == i * kLanes + lane) key[i] = 0;
  return at;
}

// The choice of one token by kLanes lanes: expert lane + kLanes i in register i.  A softmax
// without a bias chooses by the logits, which are in the scores' order, so no two of them
// fall together by rounding.  Lane j < k gets slot j's expert and weight.  All lanes of a wave
// work on as many tokens as fit it.  32771 tokens of 61 experts, 6 of them, 11.0 us: bound by
// issuing vector instructions, 91 % of the cycles (a ballot and a select for each register,
// k times).  4096 of 256 experts, 8 of 4 of 8 groups, 11.9 us: 58 % of the cycles, with four
// waves to a SIMD; the groups' keys read from LDS a fifth of them, two thirds of that in bank
// conflicts (8 lanes, 32 words apart).
template <int kLanes, int kPer>
__device__ __forceinline__ void choose(const RouteArgs& a, uint32_t token, float* scratch,
                                       int32_t& id, float& weight) {
  const uint32_t lane = threadIdx.x % kLanes;
  const bool live = token < a.tokens;
  const float ninf = -__builtin_inff();
  float s[kPer], key[kPer];
  const bool soft = a.score == WC_SCORE_SOFTMAX;
  bool bad = false;  // the weights are NaN; the choice goes by the other logits
  float top = ninf;
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    const uint32_t e = lane + kLanes * i;
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
  if (soft) {
    const uint32_t best = top_of<kLanes>(ordered(top));
    top = __uint_as_float(best >> 31 ? best & 0x7FFFFFFFu : ~best);
    bad = bad || top == -ninf;
  }
  const bool by_logits = soft && !a.bias && (a.groups == 1 || a.group_top == 1);
  float total = 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    const float x = s[i];
    const bool off = !(x > ninf);  // a NaN too: in no sum, and not chosen
    // an infinite logit's x - top is a NaN, which the least of it and 0 is not
    s[i] = off ? 0.0f : soft ? expf(fminf(x - top, 0.0f)) : 1.0f / (1.0f + expf(-x));
    total += s[i];
    if (by_logits) key[i] = x;
    else if (!soft) key[i] = off ? ninf : s[i] + key[i];
    else if (off) key[i] = ninf;
  }
  if (soft) {
    total = sum_of<kLanes>(total);
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      s[i] = total != 0.0f ? s[i] / total : 0.0f;
      if (!by_logits && key[i] != ninf) key[i] += s[i];
    }
  }
  uint32_t rank[kPer];
#pragma unroll
  for (int i = 0; i < kPer; i++) rank[i] = ordered(key[i]);
  if (a.groups > 1) {
    // the keys, then a flag for each group, in LDS of this token's own
    const uint32_t per = a.experts / a.groups;
#pragma unroll
    for (int i = 0; i < kPer; i++) scratch[lane + kLanes * i] = key[i] == key[i] ? key[i] : ninf;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    uint32_t best[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const uint32_t g = lane + kLanes * i;
      float first = ninf, second = ninf;
      if (g < a.groups)
#pragma unroll 4
        for (uint32_t j = 0; j < per; j++) {
          const float v = scratch[g * per + j];
          second = fmaxf(second, fminf(first, v));
          first = fmaxf(first, v);
        }
      best[i] = g < a.groups ? ordered(a.group_top == 2 ? first + second : first) : 0;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < kPer; i++) scratch[lane + kLanes * i] = 0.0f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (uint32_t n = 0; n < a.top_groups; n++) {
      const int32_t g = take_best<kLanes, kPer>(best, 0);
      if (g >= 0) scratch[g] = 1.0f;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const uint32_t e = lane + kLanes * i;
      if (e < a.experts && scratch[e / per] == 0.0f) rank[i] = kNone;
    }
  }
  id = -1;
  weight = 0.0f;
  for (uint32_t n = 0; n < a.k; n++) {
    const int32_t at = take_best<kLanes, kPer>(rank, kNone);
    if (lane == n) id = at;
  }
  // its score lies in register id / kLanes of lane id % kLanes
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    const float there = __shfl(s[i], id & (kLanes - 1), kLanes);
    if (id >= 0 && id / kLanes == i) weight = there;
  }
  if (a.renormalize) {
    // lanes past k have none
    const float sum = sum_of<kLanes>(weight);
    weight = sum != 0.0f ? weight / sum : 0.0f;
  }
  weight *= a.scale;
  if (votes<kLanes>(bad)) weight = __builtin_nanf("");
  if (live && lane < a.k) {
    const uint64_t at = uint64_t(token) * a.k + lane;
    global<int32_t>(a.ids)[at] = id;
    global<float>(a.weights)[at] = weight;
  }
}

template <int kLanes, int kPer>
__global__ __launch_bounds__(64 * kTokenWaves) void wc_route_choose_kernel(RouteArgs a) {
  constexpr uint32_t kTokens = 64 * kTokenWaves / kLanes;
  __shared__ float scratch[kTokens][kLanes * kPer];
  const uint32_t t = threadIdx.x / kLanes;
  int32_t id;
  float weight;
  choose<kLanes, kPer>(a, a.first + blockIdx.x * kTokens + t, scratch[t], id, weight);
}

struct SortArgs {
  uint64_t ids, offsets, order, hist;
  uint32_t slots, experts, blocks;
  uint32_t summed;  // hist holds sums over the blocks before each, and over all in one more row
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

// Sums of the counts over the blocks, in place: 16 experts a workgroup, kSets runs of blocks.
// What every block adds up for itself grows with the square of the blocks: 2^27 slots of 256
// experts took 893 ms in all, and take 16.4.
__global__ __launch_bounds__(kSortThreads) void wc_route_sum_kernel(SortArgs a) {
  constexpr uint32_t kSets = kSortThreads / 16;
  __shared__ uint32_t sums[kSets][16];
  const uint32_t classes = a.experts + 1, set = threadIdx.x / 16, column = threadIdx.x % 16;
  const uint32_t e = blockIdx.x * 16 + column, each = (a.blocks + kSets - 1) / kSets;
  const uint32_t first = min(set * each, a.blocks), last = min(first + each, a.blocks);
  const auto hist = global<uint32_t>(a.hist) + min(e, a.experts);
  uint32_t sum = 0;
#pragma unroll 8
  for (uint32_t b = first; b < last; b++) sum += hist[uint64_t(b) * classes];
  sums[set][column] = sum;
  __syncthreads();
  if (e >= classes) return;
  uint32_t before = 0;
  for (uint32_t s = 0; s < set; s++) before += sums[s][column];
#pragma unroll 8
  for (uint32_t b = first; b < last; b++) {
    const uint32_t n = hist[uint64_t(b) * classes];
    hist[uint64_t(b) * classes] = before;
    before += n;
  }
  if (set == kSets - 1) hist[uint64_t(a.blocks) * classes] = before;
}

// The stable order of one block's slots: each expert's first place (all experts
// before it, all blocks before this one, all waves before this wave), then the
// rank of a slot among its wave's with the same expert.  `class_at(slot)` is a slot's
// expert.
struct SortShared {
  uint32_t next[kSortThreads / 64][kMaxExperts + 1];
  uint32_t all[kMaxExperts + 1], before[kMaxExperts + 1], wave_total[kSortThreads / 64];
};
template <class ClassAt>
__device__ __forceinline__ void sort_block(const SortArgs& a, SortShared& sh, uint32_t block,
                                           ClassAt class_at) {
  constexpr uint32_t kWaves = kSortThreads / 64, kEach = kSortSlots / kWaves;
  const uint32_t t = threadIdx.x, lane = t % 64, wave = t / 64, classes = a.experts + 1;
  for (uint32_t w = 0; w < kWaves; w++)
    for (uint32_t e = t; e < classes; e += kSortThreads) sh.next[w][e] = 0;
  for (uint32_t e = t; e < classes; e += kSortThreads) sh.all[e] = sh.before[e] = 0;
  __syncthreads();
  const uint32_t first = block * kSortSlots + wave * kEach;
  uint32_t mine[kEach / 64];
#pragma unroll
  for (uint32_t i = 0; i < kEach / 64; i++) {
    const uint32_t slot = first + i * 64 + lane;
    mine[i] = slot < a.slots ? class_at(slot) : 0xFFFFFFFFu;
    if (slot < a.slots) atomicAdd(&sh.next[wave][mine[i]], 1u);
  }
  if (a.blocks > 1 && !a.hist) {
    // few blocks: each counts them all for itself
    const uint32_t mine_from = block * kSortSlots;
#pragma unroll 4
    for (uint32_t slot = t; slot < a.slots; slot += kSortThreads) {
      const uint32_t c = class_at(slot);
      atomicAdd(slot < mine_from ? &sh.before[c] : &sh.all[c], 1u);
    }
  } else if (a.summed) {
    if (t < classes) {
      const auto hist = global<const uint32_t>(a.hist) + t;
      const uint32_t before = hist[uint64_t(block) * classes];
      sh.before[t] = before;
      sh.all[t] = hist[uint64_t(a.blocks) * classes] - before;
    }
  } else if (a.blocks > 1) {
    // each expert's slots in all blocks, and in those before this one: the blocks over as
    // many threads to an expert as there are
    const uint32_t sets = kSortThreads / classes, set = t / classes, e = t - set * classes;
    if (set < sets) {
      uint32_t all = 0, before = 0;
#pragma unroll 4
      for (uint32_t b = set; b < a.blocks; b += sets) {
        const uint32_t n = global<const uint32_t>(a.hist)[uint64_t(b) * classes + e];
        (b < block ? before : all) += n;
      }
      atomicAdd(&sh.all[e], all);
      atomicAdd(&sh.before[e], before);
    }
  }
  __syncthreads();
  uint32_t all = 0;
  if (t < classes) {
    if (a.blocks > 1)
      all = sh.all[t] + sh.before[t];
    else
      for (uint32_t w = 0; w < kWaves; w++) all += sh.next[w][t];
  }
  // exclusive scan over the experts
  uint32_t sum = all;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t v = uint32_t(__shfl_up(int(sum), d));
    if (lane >= uint32_t(d)) sum += v;
  }
  if (lane == 63) sh.wave_total[wave] = sum;
  __syncthreads();
  uint32_t start = sum - all;
  for (uint32_t w = 0; w < wave; w++) start += sh.wave_total[w];
  if (t < classes) {
    if (block == 0) global<int32_t>(a.offsets)[t] = int32_t(start);
    uint32_t at = start + sh.before[t];
    for (uint32_t w = 0; w < kWaves; w++) {
      const uint32_t n = sh.next[w][t];
      sh.next[w][t] = at;
      at += n;
    }
  }
  __syncthreads();
  volatile uint32_t* const next = sh.next[wave];  // lanes read what another lane wrote
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
      const uint32_t place = next[mine[i]] + rank;
      global<int32_t>(a.order)[place] = int32_t(first + i * 64 + lane);
    }
    __builtin_amdgcn_wave_barrier();
    if (on && !(same >> lane >> 1)) next[mine[i]] = next[mine[i]] + uint32_t(__popcll(same));
    __builtin_amdgcn_wave_barrier();
  }
}

// 16 blocks of 257 classes 7.1 us, 97 of 62 6.8, with 4 each for the counts: chains of
// latencies.  Counts from the choice's own workgroups save that launch, but make rows of
// counts of 16 to 64 tokens, which this kernel then reads for 5 us and more.
__global__ __launch_bounds__(kSortThreads) void wc_route_order_kernel(SortArgs a) {
  __shared__ SortShared sh;
  sort_block(a, sh, blockIdx.x, [&](uint32_t slot) { return class_of(a, slot); });
}

// Few tokens: all of it by one workgroup.
template <int kLanes, int kPer>
__global__ __launch_bounds__(kSortThreads) void wc_route_small_kernel(RouteArgs a, SortArgs s) {
  constexpr uint32_t kTokens = kSortThreads / kLanes;
  __shared__ SortShared sh;
  __shared__ float scratch[kTokens][kLanes * kPer];
  __shared__ uint16_t classes[kSortSlots];
  const uint32_t t = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  for (uint32_t first = 0; first < a.tokens; first += kTokens) {
    int32_t id;
    float weight;
    choose<kLanes, kPer>(a, first + t, scratch[t], id, weight);
    if (first + t < a.tokens && lane < a.k)
      classes[(first + t) * a.k + lane] = uint16_t(id < 0 ? int32_t(a.experts) : id);
  }
  __syncthreads();
  sort_block(s, sh, 0, [&](uint32_t slot) { return uint32_t(classes[slot]); });
}

template <int kLanes, int kPer>
void start_choice(RouteArgs a, const SortArgs& s, bool small, hipStream_t st) {
  constexpr uint32_t kTokens = 64 * kTokenWaves / kLanes;
  if (small) {
    hipLaunchKernelGGL((wc_route_small_kernel<kLanes, kPer>), dim3(1), dim3(kSortThreads), 0, st, a, s);
    return;
  }
  for (; a.first < a.tokens; a.first += kLaunchTokens) {
    const uint32_t tokens = std::min(a.tokens - a.first, kLaunchTokens);
    hipLaunchKernelGGL((wc_route_choose_kernel<kLanes, kPer>), dim3((tokens + kTokens - 1) / kTokens),
                       dim3(64 * kTokenWaves), 0, st, a);
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
bool summed(uint32_t blocks, uint32_t experts) {
  return blocks > kSelfCount && uint64_t(blocks) * (experts + 1) >= kSumCounts;
}

}  // namespace

extern "C" wc_status wc_route_workspace_bytes(uint32_t tokens, const wc_route_params* p,
                                              uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!params_ok(tokens, p)) return WC_EINVAL;
  const uint32_t blocks = sort_blocks(tokens * p->k);
  if (blocks > kSelfCount) *bytes = uint64_t(blocks + summed(blocks, p->experts)) * (p->experts + 1) * 4;
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
                       ld, tokens, p->experts, p->k, p->groups, p->top_groups, p->group_top, 0, dtype,
                       p->score, p->renormalize, p->scale};
  const SortArgs s = {a.ids, reinterpret_cast<uint64_t>(dev_offsets),
                      reinterpret_cast<uint64_t>(dev_order),
                      need ? reinterpret_cast<uint64_t>(dev_workspace) : 0, tokens * p->k, p->experts,
                      sort_blocks(tokens * p->k), summed(sort_blocks(tokens * p->k), p->experts)};
  const uint32_t e = p->experts;
  // small: one workgroup's round of choices, or two where a token takes one register (32
  // tokens of 64 experts 8.4 us against 6.7 in two launches, which the host takes 4 us
  // more for)
  const uint32_t lanes = e <= 16 && p->k <= 16 ? 16 : e <= 32 ? 32 : 64;
  const bool small = tokens <= (e <= 64 ? 2u : 1u) * kSortThreads / lanes && s.slots <= kSortSlots;
  if (tokens) {
    if (lanes == 16) start_choice<16, 1>(a, s, small, st);
    else if (lanes == 32) start_choice<32, 1>(a, s, small, st);
    else if (e <= 64 && p->k <= 16 && tokens >= kManyTokens) start_choice<16, 4>(a, s, false, st);
    else if (e <= 64) start_choice<64, 1>(a, s, small, st);
    else if (e <= 128) start_choice<64, 2>(a, s, small, st);
    else if (e <= 256) start_choice<64, 4>(a, s, small, st);
    else start_choice<64, 8>(a, s, small, st);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
    if (small) return WC_OK;
  }
  if (s.hist) {
    hipLaunchKernelGGL(wc_route_count_kernel, dim3(s.blocks), dim3(kSortThreads), 0, st, s);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
  }
  if (s.summed) {
    hipLaunchKernelGGL(wc_route_sum_kernel, dim3((e + 16) / 16), dim3(kSortThreads), 0, st, s);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
  }
  hipLaunchKernelGGL(wc_route_order_kernel, dim3(s.blocks), dim3(kSortThreads), 0, st, s);
  return hipGetLastError() == hipSuccess ? WC_OK : WC_EHIP;
}
