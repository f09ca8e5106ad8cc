// wc_i8.hip -- int8 linear layers: wc_quantize_i8, wc_matmul_i8, wc_linear_i8.
#include "wc_i8.h"

namespace {

using namespace wc_i8;

// One workgroup a row: the largest magnitude, then the codes.  The bits of |x|
// order as the numbers do, so the maximum is an integer one, which keeps a NaN
// and does not depend on the order.
__global__ __launch_bounds__(256) void wc_quantize_i8_kernel(uint64_t x, int32_t dt,
                                                             uint32_t k, uint64_t ldx,
                                                             uint8_t* __restrict__ q,
                                                             float* __restrict__ scale) {
  __shared__ uint32_t top[4];
  const uint64_t row = blockIdx.x, first = row * ldx;
  uint32_t t = 0;
  for (uint32_t i = threadIdx.x; i < k; i += 256)
    t = max(t, __float_as_uint(load_float(x, dt, first + i)) & 0x7FFFFFFFu);
  t = wave_max(t);
  if (threadIdx.x % 64 == 0) top[threadIdx.x / 64] = t;
  __syncthreads();
  const RowScale s = row_scale(max(max(top[0], top[1]), max(top[2], top[3])));
  const uint32_t bytes = uint32_t(WC_I8_ROW_BYTES(k));
  uint32_t* out = reinterpret_cast<uint32_t*>(q + row * bytes);
  for (uint32_t i = threadIdx.x; i < bytes / 4; i += 256) {
    uint32_t v = 0;
#pragma unroll
    for (uint32_t j = 0; j < 4; j++)
      if (4 * i + j < k) v |= code_of(load_float(x, dt, first + 4 * i + j), s.inverse) << (8 * j);
    out[i] = v;
  }
  if (threadIdx.x == 0) scale[row] = s.scale;
}

struct MatJob {
  uint64_t w, scale, bias, y, ldw, ldy;
  uint32_t n, tile0;  // tile0: its first workgroup
  int32_t scale_dtype, bias_dtype, y_dtype, reserved;
};
struct MatArgs {
  uint64_t q, qscale;
  uint32_t m, k, n_jobs, reserved;
  MatJob job[kMaxJobs];
};

constexpr int kRowWaves = 8;

// 16 rows of W times 16 kMT rows of x a workgroup, k split over its waves in
// blocks of 128 bytes.  A lane reads 32 bytes in a row of W and of x and feeds
// two v_mfma_i32_16x16x64_i8: the sum runs over k in any order as long as both
// operands agree.
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
  return tiles < (1u << 24);
}

bool rows_ok(const void* x, int32_t dt, uint32_t m, uint32_t k, uint64_t ldx) {
  return float_ok(dt) && k >= 1 && k <= kMaxK && m <= 0x7FFFFFFFu && ldx >= k && !(ldx >> 31) &&
         (m == 0 || (x && reinterpret_cast<uintptr_t>(x) % size_of(dt) == 0));
}

wc_status matmul(const int8_t* q, const float* scale, uint32_t m, uint32_t k, uint32_t n_jobs,
                 const wc_i8_job* jobs, hipStream_t stream) {
  MatArgs a{};
  a.q = reinterpret_cast<uint64_t>(q);
  a.qscale = reinterpret_cast<uint64_t>(scale);
  a.k = k;
  a.n_jobs = n_jobs;
  uint32_t tiles = 0;
  for (uint32_t i = 0; i < n_jobs; i++) {
    const wc_i8_job& J = jobs[i];
    a.job[i] = {reinterpret_cast<uint64_t>(J.w),    reinterpret_cast<uint64_t>(J.scale),
                reinterpret_cast<uint64_t>(J.bias), reinterpret_cast<uint64_t>(J.y),
                J.ldw, J.ldy, J.n, tiles, J.scale_dtype, J.bias_dtype, J.y_dtype, 0};
    tiles += (J.n + 15) / 16;
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
                     float* scale, hipStream_t stream) {
  hipLaunchKernelGGL(wc_quantize_i8_kernel, dim3(m), dim3(256), 0, stream,
                     reinterpret_cast<uint64_t>(x), dt, k, ldx,
                     static_cast<uint8_t*>(q), scale);
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
  return jobs_ok(m, k, n_jobs, jobs) ? WC_OK : WC_EINVAL;
}

extern "C" wc_status wc_matmul_i8(const int8_t* dev_q, const float* dev_scale, uint32_t m,
                                  uint32_t k, uint32_t n_jobs, const wc_i8_job* jobs,
                                  void* dev_workspace, uint64_t workspace_bytes, void* stream) {
  (void)dev_workspace;
  (void)workspace_bytes;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  if (m == 0) return WC_OK;
  if (!dev_q || !dev_scale || reinterpret_cast<uintptr_t>(dev_q) % 16 ||
      reinterpret_cast<uintptr_t>(dev_scale) % 4)
    return WC_EINVAL;
  return matmul(dev_q, dev_scale, m, k, n_jobs, jobs, reinterpret_cast<hipStream_t>(stream));
}

extern "C" wc_status wc_linear_i8_workspace_bytes(uint32_t m, uint32_t k, uint32_t n_jobs,
                                                  const wc_i8_job* jobs, uint64_t* bytes) {
  if (!bytes) return WC_EINVAL;
  *bytes = 0;
  if (!jobs_ok(m, k, n_jobs, jobs)) return WC_EINVAL;
  *bytes = pad256(uint64_t(m) * WC_I8_ROW_BYTES(k)) + pad256(uint64_t(m) * 4);
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
  if (!dev_workspace || reinterpret_cast<uintptr_t>(dev_workspace) % 256 || workspace_bytes < need)
    return WC_EINVAL;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  int8_t* q = static_cast<int8_t*>(dev_workspace);
  float* scale = reinterpret_cast<float*>(q + pad256(uint64_t(m) * WC_I8_ROW_BYTES(k)));
  if (!launch_quantize(dev_x, x_dtype, m, k, ldx, q, scale, st)) return WC_EHIP;
  return matmul(q, scale, m, k, n_jobs, jobs, st);
}
