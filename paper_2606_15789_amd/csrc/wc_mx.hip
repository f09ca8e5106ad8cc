// wc_mx.hip -- microscaled 4-bit (MXFP4) linear layers: wc_quantize_mx, wc_dequantize_mx,
// wc_matmul_mx, wc_linear_mx.
#include <algorithm>

#include "wc_mx.h"

namespace {

using namespace wc_mx;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kLaunchRows = 1u << 23;  // a grid's axis has less than 2^32 threads

struct QuantArgs {
  uint64_t x, ldx, q, ldq, scale, lds;
  uint32_t m, k, each, groups;  // rows to a workgroup; workgroups of rows
  Blocks blocks;
};

// Four lanes to a block of 32, eight elements each: loads and stores of neighbouring lanes are
// next to each other. Rows of less than a workgroup's elements share one.
template <int kType>
__global__ __launch_bounds__(kThreads) void wc_quantize_mx_kernel(QuantArgs a) {
  if (blockIdx.x == a.groups) {
    __shared__ uint32_t starts[kMaxExperts + 1];
    if (blockIdx.y == 0) write_blocks<kThreads>(a.blocks, starts);
    return;
  }
  const uint32_t units = (a.k + 31) / 32 * 4;
  uint32_t row = blockIdx.x, unit = blockIdx.y * kThreads + threadIdx.x;
  if (a.each > 1) {
    row = blockIdx.x * a.each + threadIdx.x / units;
    unit = threadIdx.x / units < a.each ? threadIdx.x % units : units;
  }
  const bool live = row < a.m && unit < units;
  Eight<kType> e = load_eight<kType>(a.x + (row * a.ldx + unit * 8) * (kType == WC_FP32 ? 4 : 2),
                                     live ? int32_t(a.k) - int32_t(unit * 8) : 0);
  uint32_t top = float_bits<kType>(e.top());
  top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0xB1, 0xF, 0xF, false)));  // lane ^ 1
  top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0x4E, 0xF, 0xF, false)));  // lane ^ 2
  if (!live) return;
  const uint32_t byte = scale_byte(top);
  global<uint32_t>(a.q + row * a.ldq)[unit] = byte == 255 ? 0u : e.codes(scale_value(byte));
  if (unit % 4 == 0) global<uint8_t>(a.scale + row * a.lds)[unit / 4] = uint8_t(byte);
}

struct DequantArgs {
  uint64_t q, ldq, scale, lds, y, ldy;
  uint32_t m, k, each;
};

// The same the other way: eight codes a lane.  Values are exact in fp32, and rounded once to
// y's type.
template <int kType>
__global__ __launch_bounds__(kThreads) void wc_dequantize_mx_kernel(DequantArgs a) {
  const uint32_t units = (a.k + 7) / 8;
  uint32_t row = blockIdx.x, unit = blockIdx.y * kThreads + threadIdx.x;
  if (a.each > 1) {
    row = blockIdx.x * a.each + threadIdx.x / units;
    unit = threadIdx.x / units < a.each ? threadIdx.x % units : units;
  }
  if (row >= a.m || unit >= units) return;
  const uint32_t codes = global<const uint32_t>(a.q + row * a.ldq)[unit];
  const uint32_t byte = global<const uint8_t>(a.scale + row * a.lds)[unit / 4];
  const float scale = byte == 255 ? __builtin_nanf("") : scale_value(byte);
  f32x4 v[2];
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const f32x2 p = j == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0)
                    : j == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1)
                    : j == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2)
                             : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    v[j / 2][j % 2 * 2] = p[0] * scale;
    v[j / 2][j % 2 * 2 + 1] = p[1] * scale;
  }
  const uint32_t left = a.k - unit * 8;
  const uint64_t at = row * a.ldy + unit * 8, to = a.y + at * (kType == WC_FP32 ? 4 : 2);
  if (kType != WC_FP32 && left >= 8 && to % 16 == 0) {
    u32x4 h;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const float low = v[j / 2][j % 2 * 2], high = v[j / 2][j % 2 * 2 + 1];
      h[j] = kType == WC_BF16 ? floats_to_bf16(low, high) : float_to_fp16(low) | float_to_fp16(high) << 16;
    }
    *global<u32x4>(to) = h;
    return;
  }
  store_four(a.y, kType, at, v[0], left);
  if (left > 4) store_four(a.y, kType, at + 4, v[1], left - 4);
}

struct MatJob {
  uint64_t w, scale, bias, y, ldw, lds, ldy;
  uint32_t n, first;  // its first tile
  int32_t bias_dtype, y_dtype;
};
struct MatArgs {
  uint64_t x, ldx, xs, ldxs;  // rows of codes and scales, or of elements (ldx in bytes)
  uint32_t m, k, n_jobs;
  MatJob job[kMaxJobs];
};
__device__ __forceinline__ uint32_t job_of(const MatArgs& a, uint32_t tile) {
  uint32_t j = 0;
  for (uint32_t i = 1; i < a.n_jobs; i++)
    if (tile >= a.job[i].first) j = i;
  return j;
}

// 16 kN rows of W by 16 kM rows of x, kType the elements of x, or 0: quantised.
template <int kN, int kM, int kWaves, int kType>
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
    w[n] = {J.w + row * J.ldw, J.scale + row * J.lds};
  }
  const uint32_t blocks = (a.k + 31) / 32;
  S::product(sh, w, blocks, [&](int m, uint32_t super) {
    const uint64_t row = m0 + 16 * uint32_t(m) + r;
    if constexpr (kType == 0) {
      const uint64_t at = min(row, uint64_t(a.m - 1));
      return load_part<true>(Row{a.x + at * a.ldx, a.xs + at * a.ldxs}, super, blocks);
    } else {
      return quantize_part<kType>(a.x + row * a.ldx, super, row < a.m ? a.k : 0);
    }
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

// What a call does, by the sizes alone.
struct Plan {
  bool inside;        // the product's kernel quantises x itself
  uint64_t parts;     // bytes of the workspace, without the quantised x
};
Plan plan_of(uint32_t m, uint32_t, uint32_t, const wc_mx_job*) { return {m <= 16, 0}; }
uint64_t quantized_bytes(uint32_t m, uint32_t k) {
  return pad256(uint64_t(m) * WC_MX_ROW_BYTES(k)) + pad256(uint64_t(m) * WC_MX_BLOCKS(k));
}
bool workspace_ok(const void* p, uint64_t bytes, uint64_t need) {
  return need == 0 || (!off(p, 256) && bytes >= need);
}

template <int kM, int kType>
void start_slim(uint32_t tiles, const MatArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((wc_matmul_mx_slim_kernel<2, kM, 8, kType>), dim3(tiles, (a.m + 16 * kM - 1) / (16 * kM)),
                     dim3(512), 0, st, a);
}

wc_status matmul(const void* x, uint64_t ldx, const void* xs, uint64_t ldxs, int32_t x_dtype, uint32_t m,
                 uint32_t k, uint32_t n_jobs, const wc_mx_job* jobs, hipStream_t st) {
  MatArgs a{};
  a.x = reinterpret_cast<uint64_t>(x);
  a.ldx = ldx;
  a.xs = reinterpret_cast<uint64_t>(xs);
  a.ldxs = ldxs;
  a.k = k;
  a.n_jobs = n_jobs;
  uint32_t tiles = 0;
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_mx_job& J = jobs[i];
    a.job[i] = {reinterpret_cast<uint64_t>(J.w), reinterpret_cast<uint64_t>(J.scale),
                reinterpret_cast<uint64_t>(J.bias), reinterpret_cast<uint64_t>(J.y),
                J.ldw, J.lds, J.ldy, J.n, tiles, J.bias_dtype, J.y_dtype};
    tiles += (J.n + 31) / 32;
  }
  // a grid's second axis holds 65535 blocks of 64 rows
  constexpr uint32_t kSlice = 65535u * 64;
  for (uint32_t m0 = 0; m0 < m; m0 += kSlice) {
    a.m = std::min(m - m0, kSlice);
    if (x_dtype == WC_BF16) start_slim<1, WC_BF16>(tiles, a, st);
    else if (x_dtype == WC_FP16) start_slim<1, WC_FP16>(tiles, a, st);
    else if (x_dtype == WC_FP32) start_slim<1, WC_FP32>(tiles, a, st);
    else if (a.m <= 16) start_slim<1, 0>(tiles, a, st);
    else if (a.m <= 32) start_slim<2, 0>(tiles, a, st);
    else start_slim<4, 0>(tiles, a, st);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
    a.x += uint64_t(a.m) * ldx;
    a.xs += uint64_t(a.m) * ldxs;
    for (uint32_t i = 0; i < n_jobs; i++)
      a.job[i].y += uint64_t(a.m) * a.job[i].ldy * size_of(a.job[i].y_dtype);
  }
  return WC_OK;
}

}  // namespace

namespace wc_mx {

bool launch_quantize(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ldx, void* q,
                     uint64_t ldq, void* scale, uint64_t lds, hipStream_t stream, const Blocks* blocks) {
  const uint32_t units = blocks_of(k) * 4, each = units < kThreads ? kThreads / units : 1;
  for (uint32_t first = 0; first < m; first += kLaunchRows) {
    const uint32_t rows = std::min(m - first, kLaunchRows), groups = (rows + each - 1) / each;
    const bool table = blocks && first == 0;
    const QuantArgs a = {reinterpret_cast<uint64_t>(x) + first * ldx * size_of(dt), ldx,
                         reinterpret_cast<uint64_t>(q) + first * ldq, ldq,
                         reinterpret_cast<uint64_t>(scale) + first * lds, lds, rows, k, each, groups,
                         table ? *blocks : Blocks{}};
    const dim3 grid(groups + table, (units + kThreads - 1) / kThreads), block(kThreads);
    if (dt == WC_BF16) hipLaunchKernelGGL((wc_quantize_mx_kernel<WC_BF16>), grid, block, 0, stream, a);
    else if (dt == WC_FP16) hipLaunchKernelGGL((wc_quantize_mx_kernel<WC_FP16>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((wc_quantize_mx_kernel<WC_FP32>), grid, block, 0, stream, a);
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
  return launch_quantize(dev_x, x_dtype, m, k, ldx, dev_q, ldq, dev_scale, lds,
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
  for (uint32_t first = 0; first < m; first += kLaunchRows) {
    const uint32_t rows = std::min(m - first, kLaunchRows);
    const DequantArgs a = {reinterpret_cast<uint64_t>(dev_q) + first * ldq, ldq,
                           reinterpret_cast<uint64_t>(dev_scale) + first * lds, lds,
                           reinterpret_cast<uint64_t>(dev_y) + first * ldy * size_of(y_dtype), ldy, rows, k, each};
    const dim3 grid((rows + each - 1) / each, (units + kThreads - 1) / kThreads), block(kThreads);
    if (y_dtype == WC_BF16) hipLaunchKernelGGL((wc_dequantize_mx_kernel<WC_BF16>), grid, block, 0, st, a);
    else if (y_dtype == WC_FP16) hipLaunchKernelGGL((wc_dequantize_mx_kernel<WC_FP16>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((wc_dequantize_mx_kernel<WC_FP32>), grid, block, 0, st, a);
    if (hipGetLastError() != hipSuccess) return WC_EHIP;
  }
  return WC_OK;
}

extern "C" wc_status wc_matmul_mx_workspace_bytes(uint32_t m, uint32_t k, uint32_t n_jobs,
                                                  const wc_mx_job* jobs, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  *bytes = plan_of(m, k, n_jobs, jobs).parts;
  return WC_OK;
}

extern "C" wc_status wc_matmul_mx(const uint8_t* dev_q, uint64_t ldq, const uint8_t* dev_scale, uint64_t lds,
                                  uint32_t m, uint32_t k, uint32_t n_jobs, const wc_mx_job* jobs,
                                  void* dev_workspace, uint64_t workspace_bytes, void* stream) {
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!coded_ok(dev_q, ldq, dev_scale, lds, k)) return WC_EINVAL;
  const Plan p = plan_of(m, k, n_jobs, jobs);
  if (!workspace_ok(dev_workspace, workspace_bytes, p.parts)) return WC_EINVAL;
  return matmul(dev_q, ldq, dev_scale, lds, 0, m, k, n_jobs, jobs, reinterpret_cast<hipStream_t>(stream));
}

extern "C" wc_status wc_linear_mx_workspace_bytes(uint32_t m, uint32_t k, uint32_t n_jobs,
                                                  const wc_mx_job* jobs, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  const Plan p = plan_of(m, k, n_jobs, jobs);
  *bytes = p.parts + (p.inside ? 0 : quantized_bytes(m, k));
  return WC_OK;
}

extern "C" wc_status wc_linear_mx(const void* dev_x, int32_t x_dtype, uint32_t m, uint32_t k, uint64_t ldx,
                                  uint32_t n_jobs, const wc_mx_job* jobs, void* dev_workspace,
                                  uint64_t workspace_bytes, void* stream) {
  if (!rows_ok(dev_x, x_dtype, m, k, ldx) || !jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  const Plan p = plan_of(m, k, n_jobs, jobs);
  if (!workspace_ok(dev_workspace, workspace_bytes, p.parts + (p.inside ? 0 : quantized_bytes(m, k))))
    return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (p.inside)
    return matmul(dev_x, ldx * size_of(x_dtype), nullptr, 0, x_dtype, m, k, n_jobs, jobs, st);
  uint8_t* q = static_cast<uint8_t*>(dev_workspace);
  uint8_t* scale = q + pad256(uint64_t(m) * WC_MX_ROW_BYTES(k));
  if (!launch_quantize(dev_x, x_dtype, m, k, ldx, q, WC_MX_ROW_BYTES(k), scale, WC_MX_BLOCKS(k), st))
    return WC_EHIP;
  return matmul(q, WC_MX_ROW_BYTES(k), scale, WC_MX_BLOCKS(k), 0, m, k, n_jobs, jobs, st);
}
