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

// Eight entries of a row from column c on; 0 behind the end.
template <bool WIDE>
__device__ __forceinline__ uint4 load8(const uint16_t* row, int64_t c, int64_t k) {
  if (WIDE && c + 8 <= k) return __ldg(reinterpret_cast<const uint4*>(row + c));
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < k) w[i >> 1] |= (uint32_t)__ldg(row + c + i) << (16 * (i & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint32_t largest_of(const uint4& u) {  // fp32 bits
  uint32_t m = 0;
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max((w[i] << 16) & 0x7fffffffu, w[i] & 0x7fff0000u));
  return m;
}
__device__ __forceinline__ uint2 codes_of(const uint4& u, float inv) {
  auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
  auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
  return make_uint2(fp8_codes4(lo(u.x), hi(u.x), lo(u.y), hi(u.y), inv),
                    fp8_codes4(lo(u.z), hi(u.z), lo(u.w), hi(u.w), inv));
}

// A tile asked into L2: a hint that may come before what it reads is ordered behind an earlier launch.
__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap* map, int c0, int c1) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0),
               "r"(c1)
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
// The same for two numbers at once. Where a thread's registers are nearly all taken the pairs cost moves: with 256 columns a tile
// 4096 x 22016 x 4096 takes 301 us one by one and 306 in pairs (4096 x 19456 x 8192: 468 and 528), with 128 columns 401 and 367.
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

// c += a * s for two numbers each, behind the wait.
__device__ __forceinline__ void add_behind(uint64_t& c, uint32_t a0, uint32_t a1, uint64_t s) {
  asm volatile("{\n\t.reg .b64 a;\n\tmov.b64 a, {%1, %2};\n\tfma.rn.f32x2 %0, a, %3, %0;\n\t}" : "+l"(c) : "r"(a0), "r"(a1), "l"(s));
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

// What sp_test_expired_fp8 makes expire: the waits of a warp of a CTA, from its block `block` on.
struct Fp8Expire {
  int32_t cta, warp, block;
  uint64_t wait_ns;
};

// In the variants of sp_test_expired_fp8: whether this warp gives up before its block b.  (p: a kernel's parameters)
template <bool kExpire, typename P>
__device__ __forceinline__ bool gives_up(const P& p, int b, uint64_t* never) {
  if constexpr (kExpire)
    return b == p.expire_block && (int)blockIdx.x == p.expire_cta && (int)(threadIdx.x >> 5) == p.expire_warp && !mbar_wait(never, 0, p.timeout_ns);
  else
    return false;
}

// fp8_few_kernel: up to kFewTokens rows.
constexpr int kFewTokens = 64;
inline int few_box(int64_t m) { return m <= 16 ? 16 : m <= 32 ? 32 : 64; }  // rows of x in a tile, of map_x's box
constexpr int kFewCtas = 2;  // of its CTAs on an SM
// CTAs that share a tile: as many as the SMs hold at once, with two blocks each at least. Tiles of 64 tokens keep an SM busy alone, and take
// two CTAs to one only for short stretches. Measured, us: 1 x 4096 x 4096 with eight 5.9, with four 6.3; 64 x 4096 x 4096 with eight 11.2, four
// (an SM each) 12.8; 64 x 12288 x 4096 with one 17.9, two 20.6, three 21.8; 24 x 5120 x 5120 with four 10.8, with seven, for which there is less
// room than eight CTAs' worth, 14.5.
inline int few_cluster(int64_t m, int64_t n, int64_t blocks, int sms) {
  const int64_t tiles = (n + kFp8Block - 1) / kFp8Block;
  int c = 1;
  while (c < 8 && tiles * c * 2 <= (int64_t)kFewCtas * sms && blocks >= 4 * c &&
         (m <= 32 || tiles * c * 2 <= sms || blocks <= 24 * c))
    c *= 2;
  return c;
}
// Whether that kernel quantises x itself, which every tile then does again (rows: NULL; no workspace): up to eight rows, and up
// to ten pairs of rows of a block for each of its four warps. Measured, us, so / by a launch before: 8 x 4096 x 4096 (four) 7.5 / 9.0,
// 8 x 22016 x 4096 (32) 27.0 / 19.7; 1 x 32000 x 4096 (eight) 22.3 / 24.6.
inline bool few_fused(int64_t m, int64_t n, int64_t k, int sms) {
  const int64_t blocks = (k + kFp8Block - 1) / kFp8Block, c = few_cluster(m, n, blocks, sms);
  return m <= 8 && (m + 1) / 2 * ((blocks + c - 1) / c) <= 40;
}
// expire: the variant of sp_test_expired_fp8, for up to 16 rows.
sp_status launch_fp8_few(const sp_fp8_linear_args& a, const Fp8Rows* rows, const CUtensorMap& map_w, const CUtensorMap& map_x,
                         int sms, const Fp8Expire* expire, cudaStream_t stream);

sp_status launch_fp8_quantize_rows(const uint16_t* x, int64_t x_stride, int64_t m, int64_t k, uint8_t* codes,
                                   int64_t stride, float* scale, int64_t scale_stride, cudaStream_t stream);

}  // namespace sp
