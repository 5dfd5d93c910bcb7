// sp_logprobs.cu -- log probabilities of given tokens, the entropy of each row and its most likely
// entries (include/sp_serve.h).
//
// One pass over the row keeps, per thread and around its running maximum m,
//     s = sum 2^d,   z = sum d 2^d,   d = (x - m) log2(e),
// which join as sums do once rescaled to the larger maximum; then
//     log p(i) = (x_i - m) - log s,   H = log s - log(2) z / s.
// The pass is bound by reading the row.  A row goes to one CTA, or, where rows are few, to a cluster
// of up to eight that exchange their sums through shared memory.
//
// The most likely entries need no second pass over the row: of the threads' own maxima, some k are at
// least tau (a binary search by block-wide counts), so the k best entries are all at least tau, and
// only a thread whose maximum is at least tau can hold one.  Those few threads look at their
// entries again (L2 has them) and the handful that reach tau are ranked by counting.
//
// Measured: 2048 rows of 32000, bf16 (131 MB) 23.6 us, 5.6 TB/s; 64 rows of 131071, fp32 (34 MB) with twenty entries
// 13.6 us, 8.8 without them (the search for tau is block-wide counts, one after the other); one row of 32000
// with five 6.1 us, 3.9 without.
#include <cfloat>

#include "sp_attend.cuh"

namespace sp {
namespace {

// Threads of a row's CTA: few where rows are many, as 16 such CTAs are resident at a time (2048 rows of 32000,
// bf16: 23.6 us; with 12 of them, which leaves 40 registers a thread and a second wave, 26.5).  Else by the
// 16-byte vectors that the CTA has (one row of 32000 and its best five: 6.1 us by 256 threads, 7.0 by 512; one
// row of 131071 in fp32: 7.9 and 7.3).
constexpr int kFewThreads = 128, kSomeThreads = 256, kManyThreads = 512;
constexpr int64_t kManyVectors = 2048;
constexpr int kMaxTop = 64;
constexpr int kMaxCluster = 8;
constexpr int kCandidates = 1024;
constexpr float kLog2e = 1.4426950408889634f;

// Keys in the order of the numbers, -0 below +0 and NaN above all; none is 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  if (k == 0xffffffffu) return __uint_as_float(0x7fffffffu);
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct Stat {
  float m, s, z;
};
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  const float da = a.m == -INFINITY ? 0.f : (a.m - r.m) * kLog2e, db = b.m == -INFINITY ? 0.f : (b.m - r.m) * kLog2e;
  const float fa = ex2(da), fb = ex2(db);
  // a side that has seen nothing but -inf has s = z = 0; one so far below that its factor is 0 may
  // be an infinite distance below, and adds nothing (a NaN stays in s)
  r.s = a.s * fa + b.s * fb;
  r.z = (fa > 0.f ? fmaf(a.s, da, a.z) * fa : 0.f) + (fb > 0.f ? fmaf(b.s, db, b.z) * fb : 0.f);
  return r;
}

template <typename T>
struct Vec;
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t kNothing = 0xff80ff80u;  // -inf
  static __device__ __forceinline__ float one(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
  static __device__ __forceinline__ float2 two_of(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  template <int W>
  static __device__ __forceinline__ float largest(const uint32_t (&w)[W]) {
    uint32_t m = w[0];
#pragma unroll
    for (int i = 1; i < W; ++i) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i]));
    const float2 x = two_of(m);
    return max_nan(x.x, x.y);
  }
  static __device__ __forceinline__ void get(const uint4& u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = two_of(w[i]);
      x[2 * i] = y.x, x[2 * i + 1] = y.y;
    }
  }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kNothing = 0xff800000u;
  static __device__ __forceinline__ float one(float u) { return u; }
  template <int W>
  static __device__ __forceinline__ float largest(const uint32_t (&w)[W]) {
    float m[2] = {__uint_as_float(w[0]), __uint_as_float(w[1])};
#pragma unroll
    for (int i = 2; i < W; ++i) m[i & 1] = max_nan(m[i & 1], __uint_as_float(w[i]));
    return max_nan(m[0], m[1]);
  }
  static __device__ __forceinline__ void get(const uint4& u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
  }
};

// A thread's numbers, the sums in pairs.
struct Running {
  float m, top;  // maximum of the numbers (m: so far as the sums know it; top: a NaN if there is one)
  uint64_t s, z;
  __device__ __forceinline__ void lift(float vm) {
    top = max_nan(top, vm);
    if (vm > m) {  // (never for a NaN, which makes s NaN below)
      const float d = m == -INFINITY ? 0.f : (m - vm) * kLog2e, f = ex2(d);
      const uint64_t f2 = two(f, f);
      z = f > 0.f ? mul2(fma2(s, two(d, d), z), f2) : 0;
      s = mul2(s, f2);
      m = vm;
    }
  }
  // Two numbers, neither above m.  The distance is bounded so that an infinite one adds nothing
  // (2^-150 is 0 here), and a NaN stays one.
  __device__ __forceinline__ void add(float a, float b, uint64_t minus) {
    float x, y;
    apart(mul2(add2(two(a, b), minus), two(kLog2e, kLog2e)), x, y);
    x = max_nan(x, -150.f), y = max_nan(y, -150.f);
    const uint64_t e = two(ex2(x), ex2(y));
    s = add2(s, e);
    z = fma2(e, two(x, y), z);
  }
  __device__ __forceinline__ uint64_t minus() const { return two(m == -INFINITY ? 0.f : -m, m == -INFINITY ? 0.f : -m); }
  __device__ __forceinline__ Stat stat() const {
    float s0, s1, z0, z1;
    apart(s, s0, s1);
    apart(z, z0, z1);
    return Stat{m, s0 + s1, z0 + z1};
  }
};

struct LogprobParams {
  const void* logits;
  int64_t stride, vocab;
  const int64_t* ids;
  int32_t top, cluster;
  float *logp, *entropy, *top_logp;
  int64_t* top_ids;
  int32_t* status;
};

__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t caddr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(caddr) : "memory");
  return v;
}

// The warp's lanes joined, in every lane: the maximum first, then one rescaling and plain sums.
__device__ __forceinline__ Stat join_warp(Stat a) {
  float m = a.m;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  const float d = a.m == -INFINITY ? 0.f : (a.m - m) * kLog2e, f = ex2(d);
  uint64_t sz = two(a.s * f, f > 0.f ? fmaf(a.s, d, a.z) * f : 0.f);
#pragma unroll
  for (int d2 = 16; d2 > 0; d2 >>= 1) sz = add2(sz, __shfl_xor_sync(0xffffffffu, sz, d2));
  Stat r;
  r.m = m;
  apart(sz, r.s, r.z);
  return r;
}

template <typename T, int kLpThreads>
__global__ void __launch_bounds__(kLpThreads, (kLpThreads == kFewThreads ? 2048 : 1536) / kLpThreads)
    logprobs_kernel(const __grid_constant__ LogprobParams p) {
  constexpr int kLpWarps = kLpThreads / 32;
  using V = Vec<T>;
  constexpr int N = V::N;
  __shared__ uint64_t s_cand[kCandidates];
  __shared__ uint64_t s_top[kMaxTop];
  __shared__ Stat s_stat[kLpWarps > kMaxCluster ? kLpWarps : kMaxCluster];
  __shared__ Stat s_row;
  __shared__ uint32_t s_keys[kLpWarps][2];  // the least and the largest of the warp's threads' best
  __shared__ float s_lse[2];
  __shared__ int s_count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = p.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t row = blockIdx.x / p.cluster;
  pdl_wait();
  const T* x = static_cast<const T*>(p.logits) + row * p.stride;
  // entries before the first 16-byte boundary, whole vectors, entries behind the last
  const int64_t head = min((int64_t)(((16 - (reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / sizeof(T)), p.vocab);
  const int64_t vecs = (p.vocab - head) / N, tail = head + vecs * N;
  const int64_t v0 = vecs * rank / p.cluster, v1 = vecs * (rank + 1) / p.cluster;
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  // the loose entries, at most N - 1 on either side, go to rank 0's first threads
  const int loose = rank == 0 ? (int)(head + (p.vocab - tail)) : 0;
  auto loose_at = [&](int i) { return i < head ? (int64_t)i : tail + (i - head); };

  Running run = {-INFINITY, -INFINITY, 0, 0};
  bool any = false;
  constexpr int kBatch = 4;
  for (int64_t i = v0 + tid; i < v1; i += kBatch * kLpThreads) {
    uint32_t u[4 * kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      uint4 v = make_uint4(V::kNothing, V::kNothing, V::kNothing, V::kNothing);
      if (i + j * kLpThreads < v1) v = __ldg(xv + i + j * kLpThreads);
      u[4 * j] = v.x, u[4 * j + 1] = v.y, u[4 * j + 2] = v.z, u[4 * j + 3] = v.w;
    }
    any = true;
    run.lift(V::largest(u));
    const uint64_t minus = run.minus();
    if constexpr (N == 8) {
#pragma unroll
      for (int j = 0; j < 4 * kBatch; ++j) {
        const float2 y = V::two_of(u[j]);
        run.add(y.x, y.y, minus);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4 * kBatch; j += 2) run.add(__uint_as_float(u[j]), __uint_as_float(u[j + 1]), minus);
    }
  }
  if (tid < loose) {
    const float f = V::one(x[loose_at(tid)]);
    any = true;
    run.lift(f);
    run.add(f, -INFINITY, run.minus());
  }
  const float top = run.top;
  Stat w = join_warp(run.stat());
  const uint32_t own = any ? key_of(top) : 0u;  // the thread's best key
  if (p.top > 0) {
    const uint32_t least = __reduce_min_sync(0xffffffffu, any ? own : 0xffffffffu), best = __reduce_max_sync(0xffffffffu, own);
    if (lane == 0) s_keys[warp][0] = least, s_keys[warp][1] = best;
  }
  if (lane == 0) s_stat[warp] = w;
  if (tid == 0) s_count = 0;
  if (tid < kMaxTop) s_top[tid] = 0;
  __syncthreads();
  if (warp == 0) {
    w = join_warp(lane < kLpWarps ? s_stat[lane] : Stat{-INFINITY, 0.f, 0.f});
    if (lane == 0) s_row = w;
  }

  if (p.top > 0) {
    // tau: a key that at least `top` threads reach, and few more, between the least and the largest of
    // the threads' maxima (0 if there are not so many threads with entries)
    uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int i = 0; i < kLpWarps; ++i) lo = min(lo, s_keys[i][0]), hi = max(hi, s_keys[i][1]);
    if (__syncthreads_count(any) < p.top) lo = hi = 0;
    while (lo < hi) {
      const uint32_t mid = hi - (hi - lo) / 2;
      const int n = __syncthreads_count(own >= mid);
      if (n >= p.top) {
        lo = mid;
        if (n <= p.top + 8) break;
      } else {
        hi = mid - 1;
      }
    }
    const uint32_t tau = lo;
    auto offer = [&](float f, int64_t at) {
      const uint32_t k = key_of(f);
      if (k >= tau) {
        const int c = atomicAdd(&s_count, 1);
        if (c < kCandidates) s_cand[c] = ((uint64_t)k << 32) | (uint32_t)~(uint32_t)at;
      }
    };
    // the entries of the threads that reach tau: looked at by the thread where it has few vectors, else by
    // its whole warp, a vector per lane (2048 rows of 32000, one entry: 31 us against 55; 16 rows, 64
    // entries, a vector a thread: 20 us by the threads, 23 by the warps)
    auto look_at = [&](int64_t i) {
      float f[N];
      V::get(__ldg(xv + i), f);
#pragma unroll
      for (int j = 0; j < N; ++j) offer(f[j], head + i * N + j);
    };
    if (v1 - v0 <= 4 * kLpThreads) {
      if (any && own >= tau)
        for (int64_t i = v0 + tid; i < v1; i += kLpThreads) look_at(i);
    } else {
      for (unsigned hit = __ballot_sync(0xffffffffu, any && own >= tau); hit; hit &= hit - 1) {
        const int64_t of = v0 + warp * 32 + __ffs(hit) - 1;
#pragma unroll 1
        for (int64_t i = of + (int64_t)lane * kLpThreads; i < v1; i += 32 * kLpThreads) look_at(i);
      }
    }
    if (tid < loose && own >= tau) offer(V::one(x[loose_at(tid)]), loose_at(tid));
    __syncthreads();
    int n = s_count;
    if (n > kCandidates) {
      // as many equal entries: the best ones one after the other, each below the one before
      uint64_t below = 0;
      for (int r = 0; r < p.top; ++r) {
        uint64_t best = 0;
        auto look = [&](float f, int64_t at) {
          const uint64_t k = ((uint64_t)key_of(f) << 32) | (uint32_t)~(uint32_t)at;
          if (k > best && (r == 0 || k < below)) best = k;  // (a NaN at index 0 is ~0)
        };
        if (any && own >= tau) {
          for (int64_t i = v0 + tid; i < v1; i += kLpThreads) {
            float f[N];
            V::get(__ldg(xv + i), f);
#pragma unroll
            for (int j = 0; j < N; ++j) look(f[j], head + i * N + j);
          }
          if (tid < loose) look(V::one(x[loose_at(tid)]), loose_at(tid));
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, d));
        if (lane == 0) s_cand[warp] = best;
        __syncthreads();
        best = s_cand[lane & (kLpWarps - 1)];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, d));
        if (tid == 0) s_top[r] = best;
        below = best;
        __syncthreads();
      }
    } else {
      for (int c = tid; c < n; c += kLpThreads) {
        const uint64_t k = s_cand[c];
        int above = 0;
        for (int j = 0; j < n; ++j) above += s_cand[j] > k ? 1 : 0;
        if (above < p.top) s_top[above] = k;
      }
    }
  }
  __syncthreads();

  if (p.cluster > 1) {
    cluster_sync_all();
    if (rank == 0) {
      if (tid < p.cluster) {
        const uint32_t a = cluster_map(smem_u32(&s_row), (uint32_t)tid);
        s_stat[tid] = Stat{ld_cluster_f32(a), ld_cluster_f32(a + 4), ld_cluster_f32(a + 8)};
      }
      const int n = p.cluster * p.top;
      for (int i = tid; i < n; i += kLpThreads)
        s_cand[i] = ld_cluster_u64(cluster_map(smem_u32(&s_top[i % p.top]), (uint32_t)(i / p.top)));
      __syncthreads();
      if (tid == 0) {
        Stat a = s_stat[0];
        for (int i = 1; i < p.cluster; ++i) a = join(a, s_stat[i]);
        s_row = a;
      }
      for (int c = tid; c < n; c += kLpThreads) {
        const uint64_t k = s_cand[c];
        int above = 0;
        for (int j = 0; j < n; ++j) above += s_cand[j] > k ? 1 : 0;
        if (k != 0 && above < p.top) s_top[above] = k;
      }
      __syncthreads();
    }
    // (the other CTAs' shared memory has been read once all are here)
    cluster_sync_all();
    if (rank != 0) return;
  }
  if (tid == 0) {
    const Stat a = s_row;
    const float ls = logf(a.s);
    const bool empty = a.m == -INFINITY && a.s == 0.f;
    s_lse[0] = a.m;
    s_lse[1] = ls;
    p.entropy[row] = empty ? 0.f : ls - a.z / a.s * 0.6931471805599453f;
    const int64_t id = p.ids[row];
    float r = 0.f;
    if (id >= p.vocab) {
      set_status(p.status, kStatusBadIndex);
      r = __uint_as_float(0x7fffffffu);
    } else if (id >= 0) {
      r = empty ? -INFINITY : (V::one(x[id]) - a.m) - ls;
    }
    p.logp[row] = r;
  }
  if (p.top > 0) {
    __syncthreads();
    if (tid < p.top) {
      const uint64_t k = s_top[tid];
      const float f = of_key((uint32_t)(k >> 32)), m = s_lse[0];
      p.top_logp[row * p.top + tid] = m == -INFINITY && f == -INFINITY && s_lse[1] == -INFINITY ? -INFINITY : (f - m) - s_lse[1];
      p.top_ids[row * p.top + tid] = (int64_t)(uint32_t)~(uint32_t)k;
    }
  }
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" sp_status sp_token_logprobs(const void* logits, sp_logits_dtype dtype, int64_t stride, int64_t tokens,
                                       int64_t vocab, const int64_t* ids, int32_t top, float* logp_out,
                                       float* entropy_out, float* top_logp_out, int64_t* top_ids_out, void* stream) {
  if (dtype != SP_LOGITS_BF16 && dtype != SP_LOGITS_F32) return SP_ERR_INVALID_ARG;
  if (tokens < 0 || vocab < 1 || stride < vocab || top < 0 || top > kMaxTop || top > vocab) return SP_ERR_INVALID_ARG;
  if (vocab >= (int64_t)1 << 31) return SP_ERR_UNSUPPORTED;
  if (tokens == 0) return SP_OK;
  if (!logits || !ids || !logp_out || !entropy_out || (top > 0 && (!top_logp_out || !top_ids_out)))
    return SP_ERR_INVALID_ARG;
  const int64_t es = dtype == SP_LOGITS_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es) return SP_ERR_ALIGNMENT;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  // as many CTAs per row as the SMs have room for at once (two each), each with a vector for half
  // its threads
  int cluster = 1;
  while (cluster < kMaxCluster && tokens * cluster * 2 <= 2 * sms &&
         vocab * es / 16 >= (int64_t)cluster * 2 * (kSomeThreads / 2))
    cluster *= 2;
  const bool few = tokens >= 4 * sms;
  if (tokens * cluster > ((int64_t)1 << 31) - 1) return SP_ERR_UNSUPPORTED;
  LogprobParams p = {};
  p.logits = logits;
  p.stride = stride;
  p.vocab = vocab;
  p.ids = ids;
  p.top = top;
  p.cluster = cluster;
  p.logp = logp_out;
  p.entropy = entropy_out;
  p.top_logp = top_logp_out;
  p.top_ids = top_ids_out;
  p.status = device_status_ptr();
  const int threads = few ? kFewThreads : vocab * es / 16 / cluster < kManyVectors ? kSomeThreads : kManyThreads;
  auto kern = [&](auto x) {
    using T = decltype(x);
    return threads == kFewThreads    ? logprobs_kernel<T, kFewThreads>
           : threads == kSomeThreads ? logprobs_kernel<T, kSomeThreads>
                                     : logprobs_kernel<T, kManyThreads>;
  };
  return launch_pdl(dtype == SP_LOGITS_BF16 ? kern(uint16_t()) : kern(float()), dim3((unsigned)(tokens * cluster)), threads, 0, cluster,
                    (cudaStream_t)stream, p);
}
