// sp_probs.cu -- probabilities from logits, with a temperature for each row (include/sp_serve.h):
//     z = (x - max x) / T,   p = exp(z) / sum(exp(z)) over the entries with z >= ln(min_p).
//
// A row is read once: its 16-byte pieces stay in the threads' registers (eight each) while the row's
// maximum and then its sum go around, within the CTA and, where rows are few or long, among the CTAs of a
// cluster.  Pieces beyond what the registers hold are read again, from L2.  The bound is the
// row's bytes in and out.  A piece is eight entries (bf16) or four (fp32) counted from the row's first, so
// that the output's vectors are aligned whatever the logits' rows are; a piece that straddles a
// 16-byte boundary of the logits is put together from two loads.
#include <cmath>

#include "sp_attend.cuh"

namespace sp {
namespace {

constexpr int kPrThreads = 512;
constexpr int kPrWarps = kPrThreads / 32;
constexpr int kKept = 8;  // pieces that a thread keeps
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
  int32_t out_aligned;  // rows of `out` start at multiples of 16 bytes
};

template <typename T>
struct Piece;
template <>
struct Piece<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float at(const uint4& u, int i) {
    const uint32_t w = i < 2 ? u.x : i < 4 ? u.y : i < 6 ? u.z : u.w;
    return __uint_as_float((i & 1) ? w & 0xffff0000u : w << 16);
  }
  static __device__ __forceinline__ float one(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static constexpr uint32_t kNothing = 0xff80ff80u;  // -inf
  static __device__ __forceinline__ void put(uint32_t (&w)[4], int i, uint16_t v) {
    w[i >> 1] = (i & 1) ? (w[i >> 1] & 0xffffu) | ((uint32_t)v << 16) : (w[i >> 1] & 0xffff0000u) | v;
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float at(const uint4& u, int i) {
    return __uint_as_float(i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w);
  }
  static __device__ __forceinline__ float one(float v) { return v; }
  static constexpr uint32_t kNothing = 0xff800000u;
  static __device__ __forceinline__ void put(uint32_t (&w)[4], int i, float v) { w[i] = __float_as_uint(v); }
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Piece c of the row x of `vocab` entries; entries behind the end are -inf.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* x, int64_t vocab, int64_t c) {
  constexpr int N = Piece<T>::N;
  const T* at = x + c * N;
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15u);
  const T* lo = reinterpret_cast<const T*>(reinterpret_cast<uintptr_t>(at) - off);
  // every byte of what is loaded belongs to the row
  if (off == 0 && (c + 1) * N <= vocab) return __ldcs(reinterpret_cast<const uint4*>(at));
  if (off != 0 && lo >= x && lo + 2 * N <= x + vocab) {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(lo)), b = __ldg(reinterpret_cast<const uint4*>(lo) + 1);
    const uint32_t sh = (off & 3u) * 8u;
    uint32_t w[5];
    const uint32_t s = off >> 2;
    w[0] = s == 0 ? a.x : s == 1 ? a.y : s == 2 ? a.z : a.w;
    w[1] = s == 0 ? a.y : s == 1 ? a.z : s == 2 ? a.w : b.x;
    w[2] = s == 0 ? a.z : s == 1 ? a.w : s == 2 ? b.x : b.y;
    w[3] = s == 0 ? a.w : s == 1 ? b.x : s == 2 ? b.y : b.z;
    w[4] = s == 0 ? b.x : s == 1 ? b.y : s == 2 ? b.z : b.w;
    return make_uint4(__funnelshift_r(w[0], w[1], sh), __funnelshift_r(w[1], w[2], sh),
                      __funnelshift_r(w[2], w[3], sh), __funnelshift_r(w[3], w[4], sh));
  }
  uint32_t w[4] = {Piece<T>::kNothing, Piece<T>::kNothing, Piece<T>::kNothing, Piece<T>::kNothing};
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c * N + i < vocab) Piece<T>::put(w, i, at[i]);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct PrShared {
  float warp[kPrWarps];
  int64_t warp_at[kPrWarps];
  float cta[2];  // this CTA's maximum, its sum
  int64_t cta_at;
};

// The row's value of `v` by f, in every thread: warps, the CTA, the cluster's CTAs in order.
template <typename F>
__device__ __forceinline__ float over_row(float v, PrShared& sh, int which, int cluster, F f) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, d));
  __syncthreads();  // (the array's last readers)
  if (lane == 0) sh.warp[warp] = v;
  __syncthreads();
  v = sh.warp[lane & (kPrWarps - 1)];
#pragma unroll
  for (int d = kPrWarps / 2; d > 0; d >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, d));
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
__global__ void __launch_bounds__(kPrThreads, 2) probs_kernel(const __grid_constant__ ProbsParams p) {
  constexpr int N = Piece<T>::N;
  __shared__ PrShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = p.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t row = blockIdx.x / p.cluster;
  pdl_wait();
  const T* x = static_cast<const T*>(p.logits) + row * p.stride;
  float* out = p.out + row * p.out_stride;
  const float t = p.temperature ? p.temperature[row] : p.one_temperature;
  const int64_t pieces = (p.vocab + N - 1) / N;
  const int64_t c0 = pieces * rank / p.cluster, c1 = pieces * (rank + 1) / p.cluster;

  uint4 kept[kKept];
  float best = -INFINITY;
  auto lift = [&](const uint4& u) {
#pragma unroll
    for (int i = 0; i < N; ++i) best = max_nan(best, Piece<T>::at(u, i));
  };
#pragma unroll
  for (int j = 0; j < kKept; ++j) {
    const int64_t c = c0 + tid + (int64_t)j * kPrThreads;
    kept[j] = make_uint4(Piece<T>::kNothing, Piece<T>::kNothing, Piece<T>::kNothing, Piece<T>::kNothing);
    if (c < c1) kept[j] = load_piece(x, p.vocab, c);
  }
#pragma unroll
  for (int j = 0; j < kKept; ++j) lift(kept[j]);
  for (int64_t c = c0 + tid + (int64_t)kKept * kPrThreads; c < c1; c += kPrThreads) lift(load_piece(x, p.vocab, c));
  best = over_row(best, sh, 0, p.cluster, [](float a, float b) { return max_nan(a, b); });

  auto write = [&](int64_t c, const float (&v)[N]) {
    if (p.out_aligned && (c + 1) * N <= p.vocab) {
#pragma unroll
      for (int i = 0; i < N; i += 4)
        __stcs(reinterpret_cast<float4*>(out + c * N + i), make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (c * N + i < p.vocab) out[c * N + i] = v[i];
    }
  };
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < kKept; ++j) {
      const int64_t c = c0 + tid + (int64_t)j * kPrThreads;
      if (c < c1) f(c, kept[j]);
    }
    for (int64_t c = c0 + tid + (int64_t)kKept * kPrThreads; c < c1; c += kPrThreads) f(c, load_piece(x, p.vocab, c));
  };

  if (!(t > 0.f)) {  // the first of the best entries (the same branch in the whole cluster)
    int64_t at = INT64_MAX;
    each([&](int64_t c, const uint4& u) {
#pragma unroll
      for (int i = N - 1; i >= 0; --i)
        if (c * N + i < p.vocab && Piece<T>::at(u, i) == best) at = min(at, c * N + i);
    });
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) at = min(at, __shfl_xor_sync(0xffffffffu, at, d));
    if (lane == 0) sh.warp_at[warp] = at;
    __syncthreads();
    for (int w = 0; w < kPrWarps; ++w) at = min(at, sh.warp_at[w]);
    if (p.cluster > 1) {
      if (tid == 0) sh.cta_at = at;
      cluster_sync_all();
      for (int r = 0; r < p.cluster; ++r) {
        uint64_t v;
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_map(smem_u32(&sh.cta_at), (uint32_t)r)) : "memory");
        at = min(at, (int64_t)v);
      }
    }
    // (a NaN, as a logit or as the temperature, makes the row NaN)
    const float nothing = best == best && t == t ? 0.f : __uint_as_float(0x7fffffffu);
    each([&](int64_t c, const uint4&) {
      float v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = c * N + i == at && nothing == 0.f ? 1.f : nothing;
      write(c, v);
    });
  } else {
    // 1 / T, at most 2^120: 0 times it is 0
    const float inv = __frcp_rn(fmaxf(t, 0x1p-120f));
    // exp(z), or 0 where z is below the least that is kept; a NaN (-inf at an infinite temperature, or a
    // row's only value) is not kept either
    auto e_of = [&](float v) {
      const float z = __fmul_rn(__fsub_rn(v, best), inv);
      return z >= p.least ? ex2(z * kLog2e) : 0.f;
    };
    float s = 0.f;
    each([&](int64_t c, const uint4& u) {
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) a += e_of(Piece<T>::at(u, i));
      s += a;
    });
    s = over_row(s, sh, 1, p.cluster, [](float a, float b) { return a + b; });
    // a row without a largest number (a NaN, +inf, nothing above -inf) is NaN
    const float f = s > 0.f ? 1.f / s : __uint_as_float(0x7fffffffu);
    each([&](int64_t c, const uint4& u) {
      float v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = e_of(Piece<T>::at(u, i)) * f;
      write(c, v);
    });
  }
  if (p.cluster > 1) cluster_sync_all();  // the other CTAs have read this one's numbers
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
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  const int64_t pieces = (vocab * es + 15) / 16;
  int cluster = 1;
  while (cluster < kPrCluster && (pieces > (int64_t)cluster * kKept * kPrThreads ||
                                  (tokens * cluster * 2 <= sms && pieces >= (int64_t)cluster * kPrThreads)))
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
  p.out_aligned = al16(out) && (out_stride % 4 == 0 || tokens == 1);
  return launch_pdl(dtype == SP_LOGITS_BF16 ? probs_kernel<uint16_t> : probs_kernel<float>,
                    dim3((unsigned)(tokens * cluster)), kPrThreads, 0, cluster, (cudaStream_t)stream, p);
}
