// sp_verify.cu -- verification of drafted tokens from given random numbers (include/sp_serve.h).
//
// Draft i of a request is kept while u q < p for its token; behind the last kept one a token is drawn from
// the target's distribution p, or, where a draft was refused, from max(p - q, 0): that makes the
// answer's distribution the target's (speculative sampling: Leviathan et al., Chen et al., 2023).
// Drawing is the inversion of the cumulated weights.  The weights are whole numbers, floor(2^40 w), and so are
// their sums: no order of adding changes the token, and the same numbers give the same token on any machine.
//
// A request has a CTA, or a cluster where requests are few.  It looks at its drafts (a few loads that wait for one
// another), then reads one row of p and one of q: every warp adds up a stretch of its own, the totals go
// around, and the warp in whose stretch the drawn number falls goes over it again for the entry.
#include "sp_kv4.cuh"

namespace sp {
namespace {

constexpr int kVeThreads = 512;
constexpr int kVeWarps = kVeThreads / 32;
constexpr int kVeCluster = 8;
constexpr int64_t kVeMostVocab = (int64_t)1 << 22;  // sums of weights of up to 2^40 stay below 2^63

struct VerifyParams {
  const void *probs, *draft;  // draft: NULL where drafts are certain
  int64_t stride, draft_stride, rows, vocab;
  const int64_t* ids;
  const int32_t *cu_q, *drafts;
  const float *accept, *sample;
  int32_t *accepted, *rejected;
  int64_t* next;
  int32_t cluster;
  int32_t* status;
};

template <typename T>
__device__ __forceinline__ float number(T v);
template <>
__device__ __forceinline__ float number<float>(float v) { return v; }
template <>
__device__ __forceinline__ float number<uint16_t>(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

template <typename T>
__device__ __forceinline__ void load4(const T* x, int64_t i, float (&v)[4]);
template <>
__device__ __forceinline__ void load4<float>(const float* x, int64_t i, float (&v)[4]) {
  const float4 u = __ldg(reinterpret_cast<const float4*>(x + i));
  v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
}
template <>
__device__ __forceinline__ void load4<uint16_t>(const uint16_t* x, int64_t i, float (&v)[4]) {
  const uint2 u = __ldg(reinterpret_cast<const uint2*>(x + i));
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
}

__device__ __forceinline__ uint64_t weight(float w) {  // (a NaN counts as 0)
  return (uint64_t)__float2ull_rz(__saturatef(w) * 1099511627776.f);
}

template <typename T, typename Q>
struct Rows {
  const T* p;
  const Q* q;    // or NULL
  int64_t not_this, vocab;
  bool wide;     // both rows start at a vector's boundary
  // entries i .. i + 3 of the row (0 behind the end)
  __device__ __forceinline__ void get(int64_t i, uint64_t (&w)[4]) const {
    float a[4], b[4] = {0.f, 0.f, 0.f, 0.f};
    if (wide && i + 4 <= vocab) {
      load4(p, i, a);
      if (q) load4(q, i, b);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = i + j < vocab ? number(p[i + j]) : 0.f;
        if (q && i + j < vocab) b[j] = number(q[i + j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i + j == not_this) b[j] = 1.f;
      w[j] = weight(__fsub_rn(a[j], b[j]));
    }
  }
};

__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

template <typename T, typename Q>
__global__ void __launch_bounds__(kVeThreads, 2) verify_kernel(const __grid_constant__ VerifyParams p) {
  __shared__ uint64_t s_warp[kVeWarps];
  __shared__ uint64_t s_total[2];  // this CTA's, of either try
  __shared__ int s_accepted, s_bad;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = p.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t b = blockIdx.x / p.cluster;
  pdl_wait();
  const int64_t r0 = p.cu_q[b], r1 = p.cu_q[b + 1];
  const int64_t n = p.drafts[b];
  // (the same in every CTA of the cluster, so that all leave here or none)
  const bool sound = r0 >= 0 && r1 >= r0 && r1 <= p.rows && n >= 0 && (r1 == r0 ? n == 0 : n < r1 - r0);
  if (!sound || r1 == r0) {
    if (rank == 0 && tid == 0) {
      p.accepted[b] = p.rejected[b] = 0;
      p.next[b] = -1;
      if (!sound) set_status(p.status, kStatusBadIndex);
    }
    return;
  }
  const int64_t first = r1 - 1 - n;
  const T* probs = static_cast<const T*>(p.probs);
  const Q* draft = static_cast<const Q*>(p.draft);
  if (warp == 0) {  // 32 drafts at a time
    int64_t a = 0;
    bool bad = false;
    for (; a < n; a += 32) {
      bool ok = true;
      if (a + lane < n) {
        const int64_t row = first + a + lane, id = p.ids[row + 1];
        ok = id >= 0 && id < p.vocab;
        bad |= !ok;
        if (ok) {
          const float q = draft ? number(draft[row * p.draft_stride + id]) : 1.f;
          ok = __fmul_rn(p.accept[row], q) < number(probs[row * p.stride + id]);
        }
      }
      const unsigned no = __ballot_sync(0xffffffffu, !ok);
      if (no) {
        a += __ffs(no) - 1;
        break;
      }
    }
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) s_accepted = (int)min(a, n), s_bad = bad;
  }
  __syncthreads();
  const int64_t a = s_accepted, row = first + a;
  const bool less = a < n;
  Rows<T, Q> rows;
  rows.p = probs + row * p.stride;
  rows.vocab = p.vocab;
  const uint32_t u24 = (uint32_t)(fminf(fmaxf(p.sample[b], 0.f), 0.99999994f) * 16777216.f);
  const int64_t quads = (p.vocab + 3) / 4;
  const int64_t parts = (int64_t)p.cluster * kVeWarps, part = (int64_t)rank * kVeWarps + warp;
  const int64_t q0 = quads * part / parts, q1 = quads * (part + 1) / parts;

  uint64_t total = 0, before = 0, own = 0;
  for (int attempt = 0; attempt < 2; ++attempt) {
    rows.q = less && draft && attempt == 0 ? draft + row * p.draft_stride : nullptr;
    rows.not_this = less && !draft && attempt == 0 ? p.ids[row + 1] : -1;
    rows.wide = (reinterpret_cast<uintptr_t>(rows.p) % (4 * sizeof(T)) == 0) &&
                (reinterpret_cast<uintptr_t>(rows.q) % (4 * sizeof(Q)) == 0);
    uint64_t s = 0;
#pragma unroll 4
    for (int64_t i = q0 + lane; i < q1; i += 32) {
      uint64_t w[4];
      rows.get(4 * i, w);
      s += w[0] + w[1] + w[2] + w[3];
    }
    own = warp_sum(s);
    if (lane == 0) s_warp[warp] = own;
    __syncthreads();
    before = total = 0;  // weights before the warp's stretch, and all
#pragma unroll
    for (int w = 0; w < kVeWarps; ++w) {
      if (w < warp) before += s_warp[w];
      total += s_warp[w];
    }
    if (p.cluster > 1) {
      if (tid == 0) s_total[attempt] = total;
      cluster_sync_all();
      total = 0;
      for (int r = 0; r < p.cluster; ++r) {
        uint64_t v;
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_map(smem_u32(&s_total[attempt]), (uint32_t)r)) : "memory");
        if (r < rank) before += v;
        total += v;
      }
    }
    if (total > 0 || !less) break;
    __syncthreads();  // (s_warp is written again)
  }
  // floor(total * u): total < 2^63, u in 24 bits
  const uint64_t t = __umul64hi(total, (uint64_t)u24 << 40);
  if (total > 0 && t >= before && t - before < own) {  // one warp of the cluster
    uint64_t sum = before;
    for (int64_t i = q0; i < q1; i += 32) {
      uint64_t w[4] = {0, 0, 0, 0};
      if (i + lane < q1) rows.get(4 * (i + lane), w);
      uint64_t incl = w[0] + w[1] + w[2] + w[3];
      const uint64_t mine = incl;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint64_t v = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += v;
      }
      const uint64_t end = sum + __shfl_sync(0xffffffffu, incl, 31);
      if (t < end) {
        uint64_t at = sum + incl - mine;
        if (t >= at && t - at < mine) {
          int j = 0;
          while (j < 3 && t - at >= w[j]) at += w[j++];
          p.next[b] = 4 * (i + lane) + j;
        }
        break;
      }
      sum = end;
    }
  }
  if (rank == 0 && tid == 0) {
    p.accepted[b] = (int32_t)a;
    p.rejected[b] = (int32_t)(n - a);
    if (total == 0) p.next[b] = -1;
    if (total == 0 || s_bad) set_status(p.status, kStatusBadIndex);
  }
  if (p.cluster > 1) cluster_sync_all();  // the other CTAs have read this one's totals
}

template <typename T>
void (*kernel_for(sp_logits_dtype draft))(const VerifyParams) {
  return draft == SP_LOGITS_BF16 ? verify_kernel<T, uint16_t> : verify_kernel<T, float>;
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" sp_status sp_verify_drafts(const sp_verify_args* a, void* stream) {
  if (!a || a->requests < 0 || a->rows < 0 || a->vocab < 1 || a->stride < a->vocab || a->reserved != 0)
    return SP_ERR_INVALID_ARG;
  for (int32_t d : {a->dtype, a->draft_dtype})
    if (d != SP_LOGITS_BF16 && d != SP_LOGITS_F32) return SP_ERR_INVALID_ARG;
  if (a->draft_probs && a->draft_stride < a->vocab) return SP_ERR_INVALID_ARG;
  if (a->vocab > kVeMostVocab) return SP_ERR_UNSUPPORTED;
  if (a->requests == 0) return SP_OK;
  if (!a->cu_q || !a->drafts || !a->sample || !a->accepted || !a->rejected || !a->next ||
      (a->rows > 0 && (!a->probs || !a->ids || !a->accept)))
    return SP_ERR_INVALID_ARG;
  auto off = [](const void* p, int32_t dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == SP_LOGITS_BF16 ? 2 : 4) != 0; };
  if (off(a->probs, a->dtype) || off(a->draft_probs, a->draft_dtype)) return SP_ERR_ALIGNMENT;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  int cluster = 1;
  while (cluster < kVeCluster && (int64_t)a->requests * cluster * 2 <= 2 * sms && a->vocab >= (int64_t)cluster * 2 * 4 * kVeThreads)
    cluster *= 2;
  if ((int64_t)a->requests * cluster > ((int64_t)1 << 31) - 1) return SP_ERR_UNSUPPORTED;
  VerifyParams p = {};
  p.probs = a->probs;
  p.draft = a->draft_probs;
  p.stride = a->stride;
  p.draft_stride = a->draft_stride;
  p.rows = a->rows;
  p.vocab = a->vocab;
  p.ids = a->ids;
  p.cu_q = a->cu_q;
  p.drafts = a->drafts;
  p.accept = a->accept;
  p.sample = a->sample;
  p.accepted = a->accepted;
  p.rejected = a->rejected;
  p.next = a->next;
  p.cluster = cluster;
  p.status = device_status_ptr();
  auto kern = a->dtype == SP_LOGITS_BF16 ? kernel_for<uint16_t>((sp_logits_dtype)a->draft_dtype)
                                         : kernel_for<float>((sp_logits_dtype)a->draft_dtype);
  return launch_pdl(kern, dim3((unsigned)(a->requests * cluster)), kVeThreads, 0, cluster, (cudaStream_t)stream, p);
}
