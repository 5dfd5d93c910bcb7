// sp_probs.cu -- probabilities from logits, with a temperature for each row (include/sp_serve.h):
//     z = (x - max x) / T,   p = exp(z) / sum(exp(z)) over the entries with z >= ln(min_p).
//
// A row is read once: its 16-byte pieces stay in the threads' registers while the row's
// maximum and then its sum go around, within the CTA and, where rows are few or long, among the CTAs of a
// cluster.  Pieces beyond what the registers hold are read again, from L2.  The bound is the
// row's bytes in and out.  Pieces begin at the row's first 16-byte boundary; the entries before it and behind the last piece
// go to rank 0's first threads.  Rows of logits and of probabilities that lie as densely have their boundaries at the same
// entries, so that the pieces of both are aligned.
//
// Measured: 320 rows of 131071, fp32 (168 MB in, 168 out) 79 us, 4.2 TB/s: a row's exchanges, during which its CTAs neither load nor
// write, and half of it read again (clusters of four 85 us, of two 120). The same rows in bf16 (84 MB in, 168 out) 87 us, 2.9 TB/s, 2048 rows of
// 32000 131 us (105 in fp32): their exponentials are worked out twice, as the logits are what is kept, and 144 bytes of a thread do not fit
// its 64 registers. Five rows of 32000, bf16, 4.5 us. The first form, which put
// misaligned pieces together from two loads and worked out the exponentials twice, took 130 and 7.2.
#include <cmath>

#include "sp_attend.cuh"

namespace sp {
namespace {

constexpr int kPrThreads = 256;  // (512 with as many pieces each: 320 rows of 131071 82.8 us, 81.2 so)
constexpr int kPrCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;

struct ProbsParams {
  const void* logits;
  const float* temperature;  // or NULL
  float one_temperature;
  float least;  // ln(min_p)
  int64_t stride, vocab, out_stride;
  float* out;
  int32_t cluster;
};

template <typename T>
struct Piece;
template <>
struct Piece<uint16_t> {
  static constexpr int N = 8;
  static constexpr int kKept = 4;  // pieces that a thread keeps, as logits
  static constexpr uint32_t kNothing = 0xff80ff80u;  // -inf
  static __device__ __forceinline__ float one(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ void get(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static constexpr int kKept = 8;  // as logits, then as exponentials
  static constexpr uint32_t kNothing = 0xff800000u;
  static __device__ __forceinline__ float one(float v) { return v; }
  static __device__ __forceinline__ void get(const uint4& u, float (&v)[4]) {
    v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
  }
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct PrShared {
  float warp[kPrThreads / 32];
  uint32_t warp_at[kPrThreads / 32];
  float cta[2];  // this CTA's maximum, its sum
  uint32_t cta_at;
};

// The row's value of `v` by f, in every thread: warps, the CTA, the cluster's CTAs in order.
template <typename F>
__device__ __forceinline__ float over_row(float v, PrShared& sh, int which, int cluster, F f) {
  constexpr int W = kPrThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, d));
  __syncthreads();  // (the array's last readers)
  if (lane == 0) sh.warp[warp] = v;
  __syncthreads();
  v = sh.warp[lane & (W - 1)];
#pragma unroll
  for (int d = W / 2; d > 0; d >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, d));
  if (cluster > 1) {
    if (threadIdx.x == 0) sh.cta[which] = v;
    cluster_sync_all();
    float u = ld_cluster_f32(cluster_map(smem_u32(&sh.cta[which]), (uint32_t)(lane % cluster)));
    v = __shfl_sync(0xffffffffu, u, 0);
    for (int r = 1; r < cluster; ++r) v = f(v, __shfl_sync(0xffffffffu, u, r));
  }
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kPrThreads, 4) probs_kernel(const __grid_constant__ ProbsParams p) {
  constexpr int N = Piece<T>::N, kKept = Piece<T>::kKept, W = kPrThreads / 32;
  __shared__ PrShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = p.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t row = blockIdx.x / p.cluster;
  pdl_wait();
  const T* x = static_cast<const T*>(p.logits) + row * p.stride;
  float* out = p.out + row * p.out_stride;
  const float t = p.temperature ? p.temperature[row] : p.one_temperature;
  // entries before the first 16-byte boundary, whole pieces, entries behind the last
  const int vocab = (int)p.vocab;
  const int head = min((int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / sizeof(T)), vocab);
  const int pieces = (vocab - head) / N, tail = head + pieces * N;
  const int c0 = (int)((int64_t)pieces * rank / p.cluster), c1 = (int)((int64_t)pieces * (rank + 1) / p.cluster);
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  float* ov = out + head;
  const bool aligned = (reinterpret_cast<uintptr_t>(ov) & 15u) == 0;
  // a loose entry of this thread: its index, or -1
  const int loose = rank != 0 ? -1 : tid < head ? tid : tid < head + (vocab - tail) ? tail + (tid - head) : -1;
  const float lone = loose >= 0 ? Piece<T>::one(x[loose]) : -INFINITY;

  uint4 kept[kKept];
#pragma unroll
  for (int j = 0; j < kKept; ++j) {
    const int c = c0 + tid + j * kPrThreads;
    kept[j] = make_uint4(Piece<T>::kNothing, Piece<T>::kNothing, Piece<T>::kNothing, Piece<T>::kNothing);
    if (c < c1) kept[j] = __ldcs(xv + c);
  }
  const int more = c0 + tid + kKept * kPrThreads;  // pieces that are read again
  float best = lone;
  auto lift = [&](const uint4& u) {
    float v[N];
    Piece<T>::get(u, v);
#pragma unroll
    for (int i = 0; i < N; ++i) best = max_nan(best, v[i]);
  };
#pragma unroll
  for (int j = 0; j < kKept; ++j) lift(kept[j]);
  for (int c = more; c < c1; c += kPrThreads) lift(__ldg(xv + c));
  best = over_row(best, sh, 0, p.cluster, [](float a, float b) { return max_nan(a, b); });

  // This CTA has read the others' numbers.  It says so before it writes: behind its stores a barrier would wait for them.
  auto leave = [] {
    __syncwarp();
    cluster_arrive_release();
  };
  auto write = [&](int c, const float (&v)[N]) {
    float* o = ov + (int64_t)c * N;
    if (aligned) {
#pragma unroll
      for (int i = 0; i < N; i += 4)  // (kept in L2, where the verification reads them; streamed past it 320 rows take 83.6 us for 79.4)
        *reinterpret_cast<float4*>(o + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = v[i];
    }
  };

  if (!(t > 0.f)) {  // the first of the best entries (the same branch in the whole cluster)
    uint32_t at = loose >= 0 && lone == best ? (uint32_t)loose : 0xffffffffu;
    auto look = [&](int c, const uint4& u) {
      float v[N];
      Piece<T>::get(u, v);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (v[i] == best) at = min(at, (uint32_t)(head + c * N + i));
    };
#pragma unroll
    for (int j = 0; j < kKept; ++j)
      if (c0 + tid + j * kPrThreads < c1) look(c0 + tid + j * kPrThreads, kept[j]);
    for (int c = more; c < c1; c += kPrThreads) look(c, __ldg(xv + c));
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) sh.warp_at[warp] = at;
    __syncthreads();
    at = __reduce_min_sync(0xffffffffu, sh.warp_at[lane & (W - 1)]);
    if (p.cluster > 1) {
      if (tid == 0) sh.cta_at = at;
      cluster_sync_all();
      for (int r = 0; r < p.cluster; ++r)
        at = min(at, __float_as_uint(ld_cluster_f32(cluster_map(smem_u32(&sh.cta_at), (uint32_t)r))));
      leave();
    }
    // (a NaN, as a logit or as the temperature, makes the row NaN, and so does nothing above -inf: there is no best entry)
    const bool sound = best > -INFINITY && t == t;
    const float nothing = sound ? 0.f : __uint_as_float(0x7fffffffu);
    for (int c = c0 + tid; c < c1; c += kPrThreads) {
      float v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = sound && (uint32_t)(head + c * N + i) == at ? 1.f : nothing;
      write(c, v);
    }
    if (loose >= 0) out[loose] = sound && (uint32_t)loose == at ? 1.f : nothing;
  } else {
    // 1 / T, at most 2^120: 0 times it is 0
    const float inv = __frcp_rn(fmaxf(t, 0x1p-120f));
    // exp(z), or 0 where z is below the least that is kept; a NaN (-inf at an infinite temperature, or a
    // row's only value) is not kept either
    const uint64_t down = two(-best, -best), inv2 = two(inv, inv), log2e = two(kLog2e, kLog2e);
    auto exp_of = [&](const uint4& u, float (&v)[N]) {
      Piece<T>::get(u, v);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const uint64_t z = mul2(add2(two(v[i], v[i + 1]), down), inv2);
        float z0, z1, y0, y1;
        apart(z, z0, z1);
        apart(mul2(z, log2e), y0, y1);
        v[i] = z0 >= p.least ? ex2(y0) : 0.f;
        v[i + 1] = z1 >= p.least ? ex2(y1) : 0.f;
      }
    };
    auto sum_of = [&](const float (&v)[N]) {
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) a += v[i];
      return a;
    };
    const float zl = __fmul_rn(__fsub_rn(lone, best), inv), el = loose >= 0 && zl >= p.least ? ex2(zl * kLog2e) : 0.f;
    float s = el;
#pragma unroll
    for (int j = 0; j < kKept; ++j) {  // (what a thread does not have is -inf: 0, or NaN, which is not kept)
      float v[N];
      exp_of(kept[j], v);
      if (c0 + tid + j * kPrThreads < c1) s += sum_of(v);
      if constexpr (N == 4)  // fp32: the exponentials stay in the logits' place
        kept[j] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    for (int c = more; c < c1; c += kPrThreads) {
      float v[N];
      exp_of(__ldg(xv + c), v);
      s += sum_of(v);
    }
    s = over_row(s, sh, 1, p.cluster, [](float a, float b) { return a + b; });
    if (p.cluster > 1) leave();
    // a row without a largest number (a NaN, +inf, nothing above -inf) is NaN
    const float f = s > 0.f ? 1.f / s : __uint_as_float(0x7fffffffu);
    auto share = [&](int c, float (&v)[N]) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] *= f;
      write(c, v);
    };
#pragma unroll
    for (int j = 0; j < kKept; ++j) {
      const int c = c0 + tid + j * kPrThreads;
      if (c >= c1) continue;
      float v[N];
      if constexpr (N == 4) Piece<T>::get(kept[j], v);
      else exp_of(kept[j], v);
      share(c, v);
    }
    for (int c = more; c < c1; c += kPrThreads) {
      float v[N];
      exp_of(__ldg(xv + c), v);
      share(c, v);
    }
    if (loose >= 0) out[loose] = el * f;
  }
  if (p.cluster > 1) cluster_wait();  // the other CTAs have read this one's numbers
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" sp_status sp_token_probs(const void* logits, sp_logits_dtype dtype, int64_t stride, int64_t tokens,
                                    int64_t vocab, const float* temperature, float one_temperature, double min_p,
                                    float* out, int64_t out_stride, void* stream) {
  if (dtype != SP_LOGITS_BF16 && dtype != SP_LOGITS_F32) return SP_ERR_INVALID_ARG;
  if (tokens < 0 || vocab < 1 || stride < vocab || out_stride < vocab || !(min_p >= 0 && min_p <= 1))
    return SP_ERR_INVALID_ARG;
  if (!temperature && one_temperature != one_temperature) return SP_ERR_INVALID_ARG;
  if (vocab >= (int64_t)1 << 31) return SP_ERR_UNSUPPORTED;
  if (tokens == 0) return SP_OK;
  if (!logits || !out) return SP_ERR_INVALID_ARG;
  const int64_t es = dtype == SP_LOGITS_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(out) % 4 ||
      reinterpret_cast<uintptr_t>(temperature) % 4)
    return SP_ERR_ALIGNMENT;
  // (pieces of a row may be read again while others are written, and a row's temperature once other rows are)
  const uintptr_t in0 = reinterpret_cast<uintptr_t>(logits), out0 = reinterpret_cast<uintptr_t>(out), t0 = reinterpret_cast<uintptr_t>(temperature);
  const uintptr_t out1 = out0 + 4 * ((uintptr_t)(tokens - 1) * out_stride + vocab);
  if (in0 < out1 && out0 < in0 + es * ((uintptr_t)(tokens - 1) * stride + vocab)) return SP_ERR_INVALID_ARG;
  if (temperature && t0 < out1 && out0 < t0 + 4 * (uintptr_t)tokens) return SP_ERR_INVALID_ARG;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  const int64_t pieces = (vocab * es + 15) / 16;
  const int kept = dtype == SP_LOGITS_BF16 ? Piece<uint16_t>::kKept : Piece<float>::kKept;
  int cluster = 1;
  while (cluster < kPrCluster && (pieces > (int64_t)cluster * kept * kPrThreads || (tokens * cluster * 2 <= sms && pieces >= (int64_t)cluster * 512)))
    cluster *= 2;
  if (tokens * cluster > ((int64_t)1 << 31) - 1) return SP_ERR_UNSUPPORTED;
  ProbsParams p = {};
  p.logits = logits;
  p.temperature = temperature;
  p.one_temperature = one_temperature;
  p.least = (float)std::log(min_p);  // -inf for 0
  p.stride = stride;
  p.vocab = vocab;
  p.out = out;
  p.out_stride = out_stride;
  p.cluster = cluster;
  return launch_pdl(dtype == SP_LOGITS_BF16 ? probs_kernel<uint16_t> : probs_kernel<float>, dim3((unsigned)(tokens * cluster)),
                    kPrThreads, 0, cluster, (cudaStream_t)stream, p);
}
