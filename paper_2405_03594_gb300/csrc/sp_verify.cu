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
// around, and the CTA in one of whose stretches the drawn number falls shares that one out among its warps until one looks at it
// whole.
//
// Measured: one request with four drafts over 32000 entries 4.6 us; 64 requests over 131071 (34 MB of p, fp32, and 17 of q, bf16) 17.4 us, of
// which the rows take 11.6 (4.3 TB/s: four batches of loads a thread, one after the other), the search for the entry 1.7, the launch and the
// loads before the rows 4; 256 rows of 32000 without drafts (33 MB) 11.4 us, the rows 5.6 of them.
#include <type_traits>

#include "sp_kv4.cuh"

namespace sp {
namespace {

constexpr int kVeThreads = 256;
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
__device__ __forceinline__ void load4(const T* x, int i, float (&v)[4]);
template <>
__device__ __forceinline__ void load4<float>(const float* x, int i, float (&v)[4]) {
  const float4 u = __ldg(reinterpret_cast<const float4*>(x + i));
  v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
}
template <>
__device__ __forceinline__ void load4<uint16_t>(const uint16_t* x, int i, float (&v)[4]) {
  const uint2 u = __ldg(reinterpret_cast<const uint2*>(x + i));
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
}

// floor(2^40 w), w limited to [0, 1] (a NaN counts as 0), in two parts: floor(2^17 w) are the last bits of 64 + w rounded towards zero,
// and what is left of w, below 2^-17, gives floor(2^40 rest) as those of 2^-17 + rest. A conversion to 64 bits takes the SM
// several times as long: 256 rows of 32000 24.2 us so, 29.7 at first.
struct Parts {
  uint32_t hi, lo;  // sums of the parts' bits, with what belongs to 64 and 2^-17 (modulo 2^32)
  __device__ __forceinline__ void add(float w) {
    w = __saturatef(w);
    const float t = __fadd_rz(w, 64.f);
    hi += __float_as_uint(t);
    lo += __float_as_uint(__fadd_rz(__fsub_rn(w, __fsub_rn(t, 64.f)), 0x1p-17f));
  }
  // the sum of n weights, n up to 511
  __device__ __forceinline__ uint64_t sum(uint32_t n) const {
    return ((uint64_t)(hi - n * 0x42800000u) << 23) + (lo - n * 0x37000000u);
  }
};
__device__ __forceinline__ uint64_t weight(float w) {
  Parts p = {0, 0};
  p.add(w);
  return p.sum(1);
}

struct Certain {};  // the type of the drafts' probabilities where there are none

// A row in quads: quad i is the entries 4 i - shift .. 4 i - shift + 3, of which those of the row count, and shift puts the quads
// of the target's row on 16-byte boundaries.
template <typename T, typename Q>
struct Rows {
  static constexpr bool kDraft = !std::is_same<Q, Certain>::value;
  static constexpr int kBatch = 4;  // quads of a lane under way at a time (without drafts eight: 13.3 us for 11.0, 256 rows of 32000)
  const T* p;
  const Q* q;    // or NULL
  int not_this, vocab, shift;
  bool wide;     // the draft's quads are aligned too; otherwise shift is 0
  __device__ __forceinline__ void set(const T* p_, const Q* q_) {
    p = p_, q = q_;
    shift = (int)(reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) / sizeof(T));
    wide = true;
    if constexpr (kDraft)
      if (q && reinterpret_cast<uintptr_t>(q - shift) % (4 * sizeof(Q))) wide = false, shift = 0;
  }
  __device__ __forceinline__ int quads() const { return (vocab + shift + 3) >> 2; }
  __device__ __forceinline__ float draft(int i) const {
    if constexpr (kDraft)
      if (q) return number(__ldg(q + i));
    return 0.f;
  }
  __device__ __forceinline__ float left(int i, float a, float b) const {
    if constexpr (!kDraft) return i == not_this ? __fsub_rn(a, 1.f) : a;
    return __fsub_rn(a, b);
  }
  __device__ __forceinline__ float left_at(int i) const { return i >= 0 && i < vocab ? left(i, number(__ldg(p + i)), draft(i)) : 0.f; }
  __device__ __forceinline__ void load(int quad, float (&a)[4], float (&b)[4]) const {  // a whole one
    load4(p, 4 * quad - shift, a);
    if constexpr (kDraft)
      if (q) load4(q, 4 * quad - shift, b);
  }
  // the weights of a quad
  __device__ __forceinline__ void get(int quad, uint64_t (&w)[4]) const {
    const int i = 4 * quad - shift;
    if (wide && i >= 0 && i + 4 <= vocab) {
      float a[4], b[4] = {0.f, 0.f, 0.f, 0.f};
      load(quad, a, b);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = weight(left(i + j, a[j], b[j]));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = weight(left_at(i + j));
    }
  }
  // this lane's share of the sum over the quads [q0, q1), which the warp takes together: by quads, or, where rows start
  // anywhere, by single entries side by side (in quads of single loads four lanes' sectors would be asked for four times)
  __device__ __forceinline__ uint64_t sum(int q0, int q1, int lane) const {
    uint64_t s = 0;
    const int e0 = max(4 * q0 - shift, 0), e1 = min(4 * q1 - shift, vocab);  // entries
    if (!kDraft || wide) {
      const int w0 = (e0 + shift + 3) >> 2, w1 = (e1 + shift) >> 2;  // whole quads
      for (int i = w0 + lane; i < w1; i += 32 * kBatch) {
        float a[kBatch][4], b[kBatch][4];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
#pragma unroll
          for (int j = 0; j < 4; ++j) a[k][j] = b[k][j] = 0.f;
          if (i + 32 * k < w1) load(i + 32 * k, a[k], b[k]);
        }
        Parts sums = {0, 0};  // (entries behind the end are 0)
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) sums.add(left(4 * (i + 32 * k) - shift + j, a[k][j], b[k][j]));
        s += sums.sum(4 * kBatch);
      }
      // up to three entries at either end
      const int before = min(4 * w0 - shift, e1) - e0, behind = w1 < w0 ? 0 : e1 - (4 * w1 - shift);
      if (lane < before) s += weight(left_at(e0 + lane));
      if (lane < behind) s += weight(left_at(e1 - 1 - lane));
    } else {
      constexpr int N = 4 * kBatch;
      for (int i = e0 + lane; i < e1; i += 32 * N) {
        float a[N], b[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          a[k] = i + 32 * k < e1 ? number(__ldg(p + i + 32 * k)) : 0.f;
          b[k] = i + 32 * k < e1 ? draft(i + 32 * k) : 0.f;
        }
        Parts sums = {0, 0};
#pragma unroll
        for (int k = 0; k < N; ++k) sums.add(left(i + 32 * k, a[k], b[k]));
        s += sums.sum(N);
      }
    }
    return s;
  }
};

__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

template <typename T, typename Q>
__global__ void __launch_bounds__(kVeThreads, 4) verify_kernel(const __grid_constant__ VerifyParams p) {
  constexpr bool kDraft = Rows<T, Q>::kDraft;
  constexpr int kBatch = Rows<T, Q>::kBatch;
  __shared__ uint64_t s_warp[kVeWarps];
  __shared__ uint64_t s_total[2];  // this CTA's, of either try
  __shared__ int s_accepted, s_bad, s_owner;
  __shared__ int s_range[2];
  __shared__ uint64_t s_before;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = p.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t b = blockIdx.x / p.cluster;
  pdl_launch_dependents();
  pdl_wait();
  const int64_t r0 = p.cu_q[b], r1 = p.cu_q[b + 1];
  const int64_t n = p.drafts[b];
  // (the same in every CTA of the cluster, so that all leave here or none)
  const bool sound = r0 >= 0 && r1 >= r0 && r1 <= p.rows && (r1 == r0 || (n >= 0 && n < r1 - r0));
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
          float q = 1.f;
          if constexpr (kDraft) q = number(draft[row * p.draft_stride + id]);
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
  int not_this = -1;  // (an index outside the vocabulary is none of its entries)
  if (less && !kDraft) {
    const int64_t id = p.ids[row + 1];
    not_this = id >= 0 && id < p.vocab ? (int)id : -1;
  }
  Rows<T, Q> rows;
  rows.vocab = (int)p.vocab;
  const uint32_t u24 = (uint32_t)(fminf(fmaxf(p.sample[b], 0.f), 0.99999994f) * 16777216.f);
  const int parts = p.cluster * kVeWarps, part = rank * kVeWarps + warp;
  int q0 = 0, q1 = 0;  // the warp's stretch (quads up to 2^20, parts up to 2^7)
  uint64_t total = 0, before = 0, own = 0;
  for (int attempt = 0; attempt < 2; ++attempt) {
    if constexpr (kDraft) rows.set(probs + row * p.stride, less && attempt == 0 ? draft + row * p.draft_stride : nullptr);
    else rows.set(probs + row * p.stride, nullptr);
    rows.not_this = attempt == 0 ? not_this : -1;
    q0 = rows.quads() * part / parts, q1 = rows.quads() * (part + 1) / parts;
    own = warp_sum(rows.sum(q0, q1, lane));
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
  // the warp in whose stretch it falls; all warps of its CTA then share that stretch, until a warp looks at it whole
  if (tid == 0) s_owner = -1;
  __syncthreads();
  if (lane == 0 && total > 0 && t >= before && t - before < own) {
    s_owner = warp;
    s_range[0] = q0, s_range[1] = q1, s_before = before;
  }
  __syncthreads();
  if (s_owner >= 0) {
    int f0 = s_range[0], f1 = s_range[1];
    uint64_t up = s_before;  // weights before f0: t is at least this
    while (f1 - f0 > 32 * kBatch) {
      const int n = f1 - f0;
      const uint64_t part_sum = warp_sum(rows.sum(f0 + n * warp / kVeWarps, f0 + n * (warp + 1) / kVeWarps, lane));
      if (lane == 0) s_warp[warp] = part_sum;
      __syncthreads();
      int w = 0;
      while (w < kVeWarps - 1 && t - up >= s_warp[w]) up += s_warp[w++];
      f1 = f0 + n * (w + 1) / kVeWarps;
      f0 += n * w / kVeWarps;
      __syncthreads();
    }
    if (warp == 0) {  // kBatch quads in a row of each lane
      uint64_t w[kBatch][4], mine = 0;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int i = f0 + kBatch * lane + k;
        w[k][0] = w[k][1] = w[k][2] = w[k][3] = 0;
        if (i < f1) rows.get(i, w[k]);
        mine += w[k][0] + w[k][1] + w[k][2] + w[k][3];
      }
      uint64_t incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint64_t v = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += v;
      }
      uint64_t at = up + incl - mine;
      if (t >= at && t - at < mine) {
        int found = -1;
#pragma unroll
        for (int k = 0; k < 4 * kBatch; ++k) {
          if (found < 0 && t - at < w[k / 4][k % 4]) found = k;
          at += w[k / 4][k % 4];
        }
        p.next[b] = 4 * (f0 + kBatch * lane) - rows.shift + found;
      }
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
void (*kernel_for(const sp_verify_args* a))(const VerifyParams) {
  return !a->draft_probs ? verify_kernel<T, Certain> : a->draft_dtype == SP_LOGITS_BF16 ? verify_kernel<T, uint16_t> : verify_kernel<T, float>;
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
  auto off = [](const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size != 0; };
  if (off(a->probs, a->dtype == SP_LOGITS_BF16 ? 2 : 4) || off(a->draft_probs, a->draft_dtype == SP_LOGITS_BF16 ? 2 : 4))
    return SP_ERR_ALIGNMENT;
  if (off(a->ids, 8) || off(a->next, 8)) return SP_ERR_ALIGNMENT;
  for (const void* p : {(const void*)a->cu_q, (const void*)a->drafts, (const void*)a->accept, (const void*)a->sample,
                        (const void*)a->accepted, (const void*)a->rejected})
    if (off(p, 4)) return SP_ERR_ALIGNMENT;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  int cluster = 1;
  // (four CTAs to an SM, a few quads for each thread; 512 threads, two to an SM: one request 5.1 us for 4.6, 64 requests 18.1 for 17.4)
  while (cluster < kVeCluster && (int64_t)a->requests * cluster * 2 <= 4 * sms && a->vocab >= (int64_t)cluster * 2 * 4 * kVeThreads)
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
  auto kern = a->dtype == SP_LOGITS_BF16 ? kernel_for<uint16_t>(a) : kernel_for<float>(a);
  return launch_pdl(kern, dim3((unsigned)(a->requests * cluster)), kVeThreads, 0, cluster, (cudaStream_t)stream, p);
}
