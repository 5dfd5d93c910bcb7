// sp_fp8.cu -- quantisation to e4m3 with a scale for each block of 128 (include/sp_fp8.h).
//
// A row's block is held by 16 lanes, eight entries each, a warp taking two neighbouring blocks; its largest
// magnitude goes around by shuffles, so that x is read once and its codes and scale are written once.  A weight's
// block of 128 x 128 is held by a CTA's registers in the same way.  Measured: rows of 4096 x 4096 (50 MB) 11 us, 4.5 TB/s (17 us, of
// 0.75 of the issue slots, before four pairs of blocks went to a warp; half of them are taken now, and a warp has one batch of loads in its
// life, so that the rest is their way); 16 x 4096 1.3 us among others, 4 alone, which is latency.  A weight of 4096 x 4096
// 11.7 us, of 22016 x 4096 57 us (4.7 TB/s): a CTA's loads, its maximum and its stores follow one another, four CTAs to an SM.
#include <type_traits>

#include "sp_fp8.cuh"

namespace sp {
namespace {

constexpr int kQuThreads = 256;

// G pairs of blocks to a warp: with four, what a warp works out once is shared, where there are rows enough.
template <bool WIDE, int G>
__global__ void __launch_bounds__(kQuThreads) quantize_rows_kernel(const uint16_t* __restrict__ x, int64_t x_stride,
                                                                   int64_t m, int32_t k, uint8_t* __restrict__ codes,
                                                                   int64_t stride, float* __restrict__ scale,
                                                                   int64_t scale_stride) {
  const int lane = threadIdx.x & 31;
  const int blocks = (k + kFp8Block - 1) / kFp8Block;
  const uint32_t groups = (uint32_t)(blocks + 2 * G - 1) / (2 * G);
  const int64_t at = blockIdx.x * (int64_t)(kQuThreads / 32) + (threadIdx.x >> 5);
  pdl_launch_dependents();  // the product's CTAs may set up meanwhile
  pdl_wait();
  if (at >= m * groups) return;
  // (a 64-bit division takes longer than the rest)
  const int64_t row = at >> 32 ? at / groups : (int64_t)((uint32_t)at / groups);
  const int b = (int)(at - row * groups) * 2 * G + (lane >> 4), c = b * kFp8Block + 8 * (lane & 15);
  x += row * x_stride, codes += row * stride, scale += row;
  uint4 u[G];
  uint32_t a[G];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int at_c = c + 2 * i * kFp8Block;
    u[i] = at_c < k ? load8<WIDE>(x, at_c, k) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < G; ++i) a[i] = largest_of(u[i]);
#pragma unroll
  for (int d = 8; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < G; ++i) a[i] = max(a[i], __shfl_xor_sync(0xffffffffu, a[i], d));
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int at_c = c + 2 * i * kFp8Block, at_b = b + 2 * i;
    const float s = fp8_scale(a[i]);
    if (at_b >= blocks) continue;
    if (at_c < stride) *reinterpret_cast<uint2*>(codes + at_c) = codes_of(u[i], __frcp_rn(s));
    if ((lane & 15) == 0) scale[at_b * scale_stride] = s;
  }
}

template <bool WIDE>
__global__ void __launch_bounds__(kQuThreads) quantize_blocks_kernel(const uint16_t* __restrict__ w, int64_t w_stride,
                                                                     int64_t n, int64_t k, uint8_t* __restrict__ codes,
                                                                     int64_t stride, float* __restrict__ scale) {
  __shared__ uint32_t s_most[kQuThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31;
  const int64_t blocks = (k + kFp8Block - 1) / kFp8Block;
  const int64_t rb = blockIdx.x / blocks, b = blockIdx.x % blocks, c = b * kFp8Block + 8 * (lane & 15);
  pdl_wait();
  uint4 u[8];
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = rb * kFp8Block + 16 * i + (tid >> 4);
    u[i] = r < n && c < k ? load8<WIDE>(w + r * w_stride, c, k) : make_uint4(0, 0, 0, 0);
    a = max(a, largest_of(u[i]));
  }
  a = __reduce_max_sync(0xffffffffu, a);
  if (lane == 0) s_most[tid >> 5] = a;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kQuThreads / 32; ++i) a = max(a, s_most[i]);
  const float s = fp8_scale(a), inv = __frcp_rn(s);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = rb * kFp8Block + 16 * i + (tid >> 4);
    if (r < n && c < stride) *reinterpret_cast<uint2*>(codes + r * stride + c) = codes_of(u[i], inv);
  }
  if (tid == 0) scale[rb * blocks + b] = s;
}

// 16-byte loads of eight entries
bool wide_rows(const void* x, int64_t stride) { return al16(x) && stride % 8 == 0; }

bool bad_sizes(const void* x, int64_t x_stride, int64_t rows, int64_t k, const void* codes, int64_t stride, const void* scale) {
  return rows < 0 || k < 1 || x_stride < k || stride < k || (rows > 0 && (!x || !codes || !scale));
}
bool off_bounds(const void* x, const void* codes, const void* scale) {
  return reinterpret_cast<uintptr_t>(x) % 2 || !al16(codes) || reinterpret_cast<uintptr_t>(scale) % 4;
}
constexpr int64_t kMost = (int64_t)1 << 30;

}  // namespace

sp_status launch_fp8_quantize_rows(const uint16_t* x, int64_t x_stride, int64_t m, int64_t k, uint8_t* codes,
                                   int64_t stride, float* scale, int64_t scale_stride, cudaStream_t stream) {
  const int64_t pairs = (k + 2 * kFp8Block - 1) / (2 * kFp8Block);
  const bool many = m * pairs >= 16384 && pairs >= 4;
  const int64_t warps = m * (many ? (pairs + 3) / 4 : pairs), ctas = (warps * 32 + kQuThreads - 1) / kQuThreads;
  if (ctas > INT32_MAX) return SP_ERR_UNSUPPORTED;
  auto kern = [&](auto wide) {
    return many ? quantize_rows_kernel<decltype(wide)::value, 4> : quantize_rows_kernel<decltype(wide)::value, 1>;
  };
  return launch_pdl(wide_rows(x, m > 1 ? x_stride : 0) ? kern(std::true_type()) : kern(std::false_type()), dim3((unsigned)ctas), kQuThreads, 0,
                    1, stream, x, x_stride, m, (int32_t)k, codes, stride, scale, scale_stride);
}

}  // namespace sp

using namespace sp;

extern "C" sp_status sp_fp8_quantize_rows(const void* x, int64_t x_stride, int64_t m, int64_t k, void* codes,
                                          int64_t stride, float* scale, int64_t scale_stride, void* stream) {
  if (bad_sizes(x, x_stride, m, k, codes, stride, scale) || scale_stride < m) return SP_ERR_INVALID_ARG;
  if (m > kMost || k > kMost || stride % 16 || scale_stride % 4) return SP_ERR_UNSUPPORTED;
  if (off_bounds(x, codes, scale) || !al16(scale)) return SP_ERR_ALIGNMENT;
  if (m == 0) return SP_OK;
  return launch_fp8_quantize_rows(static_cast<const uint16_t*>(x), x_stride, m, k, static_cast<uint8_t*>(codes), stride,
                                  scale, scale_stride, (cudaStream_t)stream);
}

extern "C" sp_status sp_fp8_quantize_blocks(const void* w, int64_t w_stride, int64_t n, int64_t k, void* codes,
                                            int64_t stride, float* scale, void* stream) {
  if (bad_sizes(w, w_stride, n, k, codes, stride, scale)) return SP_ERR_INVALID_ARG;
  if (n > kMost || k > kMost || stride % 16) return SP_ERR_UNSUPPORTED;
  if (off_bounds(w, codes, scale)) return SP_ERR_ALIGNMENT;
  if (n == 0) return SP_OK;
  const int64_t ctas = ((n + kFp8Block - 1) / kFp8Block) * ((k + kFp8Block - 1) / kFp8Block);
  if (ctas > INT32_MAX) return SP_ERR_UNSUPPORTED;
  return launch_pdl(wide_rows(w, n > 1 ? w_stride : 0) ? quantize_blocks_kernel<true> : quantize_blocks_kernel<false>,
                    dim3((unsigned)ctas), kQuThreads, 0, 1, (cudaStream_t)stream, static_cast<const uint16_t*>(w), w_stride, n,
                    k, static_cast<uint8_t*>(codes), stride, scale);
}
