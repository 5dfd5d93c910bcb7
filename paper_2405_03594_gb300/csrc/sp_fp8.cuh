// sp_fp8.cuh -- what the 8-bit kernels share: quantisation of a block, the parameters of a product, the tensor
// cores' 8-bit form.
#pragma once

#include "../../include/sp_fp8.h"
#include "sp_attend.cuh"
#include "sp_tcgen05.cuh"

namespace sp {

constexpr int kFp8Block = 128;  // rows and columns of a weight's block, columns of a row's

// A block's scale from the bits of its largest magnitude (a NaN's bits are above infinity's), and 1 / scale.
__device__ __forceinline__ float fp8_scale(uint32_t largest) {
  const float s = __fmul_rn(__uint_as_float(largest), 1.f / 448.f);
  return s != s ? s : fmaxf(s, 0x1p-100f);
}
__device__ __forceinline__ uint16_t fp8_codes(float lo, float hi) {  // two codes, limited to +-448; NaN stays NaN
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t fp8_codes4(float a, float b, float c, float d, float inv) {
  return (uint32_t)fp8_codes(__fmul_rn(a, inv), __fmul_rn(b, inv)) |
         ((uint32_t)fp8_codes(__fmul_rn(c, inv), __fmul_rn(d, inv)) << 16);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Instruction descriptor, kind::f8f6f4: D fp32, A and B e4m3, both K-major, M = m, N = n.
__host__ __device__ constexpr uint32_t idesc_e4m3(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// D[tmem] (+)= A[smem] * B[smem], 32 columns of e4m3.
__device__ __forceinline__ void mma_fp8(uint32_t d_taddr, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_taddr),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The same on a pair of CTAs, each with 128 rows of A and of D and half of B's rows; issued by the first CTA.
__device__ __forceinline__ void mma_fp8_pair(uint32_t d_taddr, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_taddr),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}

// Bounded wait as mbar_wait, for waits that end within a microsecond: it looks at the barrier many times before it
// asks for the time, which takes longer than such a wait.
__device__ __forceinline__ bool mbar_wait_short(uint64_t* bar, uint32_t parity, uint64_t timeout_ns) {
  for (int i = 0; i < 128; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  return mbar_wait(bar, parity, timeout_ns);
}

// Whether the phase is complete now.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

// c += a * s; volatile, so that it stays behind the wait for what was loaded.
__device__ __forceinline__ void fma_behind(float& c, uint32_t a, float s) {
  asm volatile("fma.rn.f32 %0, %1, %2, %0;" : "+f"(c) : "f"(__uint_as_float(a)), "f"(s));
}
// The same for two numbers at once. Where a thread's registers are nearly all taken the pairs cost moves: 256 columns of a tile
// take 300 us of 4096 x 22016 x 4096 one by one and 370 in pairs, 128 columns 397 and 356.
__device__ __forceinline__ void fma2_behind(float& c0, float& c1, uint32_t a0, uint32_t a1, float s) {
  asm volatile(
      "{\n\t.reg .b64 c, a, s;\n\t"
      "mov.b64 c, {%0, %1};\n\t"
      "mov.b64 a, {%2, %3};\n\t"
      "mov.b64 s, {%4, %4};\n\t"
      "fma.rn.f32x2 c, a, s, c;\n\t"
      "mov.b64 {%0, %1}, c;\n\t}"
      : "+f"(c0), "+f"(c1)
      : "f"(__uint_as_float(a0)), "f"(__uint_as_float(a1)), "f"(s));
}

// A warpgroup's registers per thread, of those that the block was launched with.
template <int R>
__device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R>
__device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }

// The rows of a product, quantised.
struct Fp8Rows {
  const uint8_t* codes;
  const float* scale;
  int64_t stride, scale_stride;
};

sp_status launch_fp8_quantize_rows(const uint16_t* x, int64_t x_stride, int64_t m, int64_t k, uint8_t* codes,
                                   int64_t stride, float* scale, int64_t scale_stride, cudaStream_t stream);

}  // namespace sp
