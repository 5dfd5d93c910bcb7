// sp_attend.cuh -- what the two attention kernels share: their parameters and number formats.
#pragma once

#include "sp_kv4.cuh"

namespace sp {

struct AttendParams {
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;
  Kv4 cache;
  const int32_t *table, *lens, *cu_q, *work;
  int32_t requests, width, group;
  int32_t max_new;
  int32_t alone;  // attend_kernel: no attend_rows_kernel was launched before it
  int64_t tokens;
  int32_t group_inverse;  // 2^16 / group, rounded up
  float scale_log2;
  float* part;    // attend_kernel: [2 grid][8 NT] of (D sums, maximum, sum of weights, unused);
                  // attend_rows_kernel: [items][split] of 256 columns of (D sums, maximum, sum of weights)
  int32_t split, parts;  // attend_rows_kernel: shares of an item, at most; shares that `part` holds
  int* cnt;     // attend_kernel: [grid] arrivals; attend_rows_kernel: its next item, CTAs that are done
  int32_t* status;
  uint64_t timeout_ns;
  uint32_t expire_cta;  // in the variants of sp_test_expired_attend: the warp that gives up
  int32_t expire_warp;
};

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Two fp32 numbers in one register pair, and arithmetic on both at once.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void apart(uint64_t x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// attend_rows_kernel over the requests that the plan gave to it (sp_attend_rows.cu); expire: the variant of
// sp_test_expired_attend, for head_dim 64.
sp_status launch_attend_rows(AttendParams p, int head_dim, bool expire, cudaStream_t stream);
size_t attend_rows_part_bytes(int head_dim, int sms);  // of the shares that it joins

}  // namespace sp
