// wc_choose.h -- one token's experts and their weights, from its logits: what wc_route and
// the mixture layers that route by themselves share.
#pragma once

#include <cmath>

#include "wc_i8.h"

namespace wc_choose {

using namespace wc_i8;

constexpr uint32_t kMaxChosen = 32;

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
}
// Lane j's slot of a token to memory.
template <int kLanes>
__device__ __forceinline__ void store_choice(const RouteArgs& a, uint32_t token, int32_t id, float weight) {
  const uint32_t lane = threadIdx.x % kLanes;
  if (token < a.tokens && lane < a.k) {
    const uint64_t at = uint64_t(token) * a.k + lane;
    global<int32_t>(a.ids)[at] = id;
    global<float>(a.weights)[at] = weight;
  }
}

inline bool params_ok(uint32_t tokens, const wc_route_params* p) {
  return p && p->experts >= 1 && p->experts <= kMaxExperts && p->k >= 1 && p->k <= p->experts &&
         p->k <= kMaxChosen && (p->score == WC_SCORE_SOFTMAX || p->score == WC_SCORE_SIGMOID) &&
         p->groups >= 1 && p->experts % p->groups == 0 && p->top_groups >= 1 &&
         p->top_groups <= p->groups && p->group_top >= 1 && p->group_top <= 2 &&
         p->group_top <= p->experts / p->groups && std::isfinite(p->scale) &&
         uint64_t(tokens) * p->k < (1ull << 31);
}

}  // namespace wc_choose
