// sp_kv_plan.cu -- the tables of a serving step (include/sp_serve.h): pages, slots, positions and
// the shares of the attention kernels, from the lengths of the requests.
//
// A few kilobytes move, so the time is latency: one CTA takes the requests 1024 at a time, two
// passes over their lengths.  The first adds up what the step needs, and whether it fits; the second
// has the exclusive sums (one shuffle scan for all five quantities) at which each request's pages
// and tokens begin, and puts the pages of ended requests on the stack.  Slots are filled by token, where
// there are many by a grid of their own; a token whose page is new finds it on the stack, and the page's
// first token writes it to the table.  A warp looks for the request of its first token among 32
// shares at a time, and then among 32 requests, so that a search is few loads.
//
// Tokens that a step's verification refused give their pages back by a kernel of the same kind: 64 requests 2.6 us, 1000 requests with
// up to three pages each 4.5 us.
//
// Measured: 64 requests with a token each 4.5 us; 1000 requests with up to 256 new tokens each, some of them ended,
// 13.2 us: the one CTA's loads and scans, which wait for one another, then the slots' grid.
#include <climits>

#include "sp_kv4.cuh"

namespace sp {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int64_t kFillHere = 4096;  // tokens that the planning CTA fills itself
constexpr int kCuShared = 4096;      // requests whose sums fit its shared memory

struct Request {
  int64_t len, add;  // tokens after the step, new ones
  int64_t before, after;  // pages
  bool gone;
  int bad;
};

__device__ __forceinline__ Request request_at(const sp_kv_plan_args& a, int shift, int b) {
  Request r;
  const int64_t cached = a.cached[b], add = a.new_tokens[b];
  const int64_t room = min((int64_t)a.width << shift, (int64_t)INT_MAX);
  r.gone = add < 0;
  r.add = r.gone ? 0 : add;
  r.len = r.gone ? 0 : cached + r.add;
  r.bad = cached < 0 || cached > room ? SP_PLAN_INPUT : r.len > room ? SP_PLAN_WIDTH : 0;
  const int64_t p1 = ((int64_t)1 << shift) - 1;
  if (r.bad == SP_PLAN_INPUT) r.len = r.add = 0;
  r.before = r.bad == SP_PLAN_INPUT ? 0 : (cached + p1) >> shift;
  r.after = (r.len + p1) >> shift;
  return r;
}

// Shares of the attention kernel: for every tile of kRowTile query rows, units of kUnitKeys keys and what
// a tile costs beside them.
__device__ __forceinline__ int64_t units_of(const Request& r, int group) {
  if (r.add == 0 || r.add * group >= kManyRows) return 0;
  return (r.add * group + kRowTile - 1) / kRowTile * ((r.len + kUnitKeys - 1) / kUnitKeys + kSetupUnits);
}

// Pairs of tiles of the kernel for many rows.
__device__ __forceinline__ int64_t pairs_of(const Request& r, int group) {
  return r.add * group >= kManyRows ? (r.add * group + kPairRows - 1) / kPairRows : 0;
}

// f(j) for j in [0, n) of each lane's own n: long ranges by the whole warp, one after the other.
template <typename F>
__device__ __forceinline__ void each_page(int n, int64_t key, F f) {
  const int lane = threadIdx.x & 31;
  unsigned big = __ballot_sync(0xffffffffu, n > 4);
  while (big) {
    const int src = __ffs(big) - 1;
    big &= big - 1;
    const int m = __shfl_sync(0xffffffffu, n, src);
    const int64_t k = __shfl_sync(0xffffffffu, key, src);
    for (int j = lane; j < m; j += 32) f(k, j);
  }
  if (n <= 4)
    for (int j = 0; j < n; ++j) f(key, j);
}

// Slot and position of the warp's tokens t (one per lane, in a row); cu[0..requests] are the sums.
__device__ __forceinline__ void fill_tokens(const sp_kv_plan_args& a, int shift, const int32_t* cu, int64_t t) {
  const int lane = threadIdx.x & 31, total = cu[a.requests];
  const int64_t t0 = t - lane;
  if (t0 < total) {
    // the first token's request: among 32 shares at a time, then 32 requests, one per lane
    int lo = 0, n = a.requests;
    while (n > 32) {
      const int step = (n + 31) / 32, at = min(n, (lane + 1) * step);
      const unsigned past = __ballot_sync(0xffffffffu, cu[lo + at] > t0);
      const int k = __ffs(past) - 1;
      lo += k * step;
      n = min(step, n - k * step);
    }
    const int end = cu[min(lo + lane + 1, a.requests)];
    int b = 0;  // requests of the 32 that end at or before the lane's token
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
      if (__shfl_sync(0xffffffffu, end, b + d - 1) <= t) b += d;
    if (__shfl_sync(0xffffffffu, end, 31) <= t) b = 32;
    b += lo;
    if (t < total) {
      if (b == lo + 32) {  // further on
        int hi = a.requests;
        while (hi - b > 1) {
          const int mid = (b + hi) >> 1;
          if (cu[mid] <= t) b = mid;
          else hi = mid;
        }
      }
      const int32_t *lens = a.lens, *work = a.work, *free_pages = a.free_pages;
      const int len = lens[b], at = cu[b], pos = len - (cu[b + 1] - (int)t), j = pos >> shift;
      int32_t* entry = a.table + (int64_t)b * a.width + j;
      int page;
      // a page that begins among the new tokens comes off the stack; its first token extends the table
      const int cached = pos - ((int)t - at);
      if (free_pages && j >= (int)(((int64_t)cached + ((int64_t)1 << shift) - 1) >> shift)) {
        page = free_pages[work[2 * (a.requests + 1) + b] - j];
        if ((pos & ((1 << shift) - 1)) == 0) *entry = page;
      } else {
        page = *entry;
      }
      a.slots[t] = ((int64_t)page << shift) + (pos & ((1 << shift) - 1));
      a.positions[t] = pos;
      return;
    }
  }
  if (t < a.max_tokens) {
    a.slots[t] = -1;
    a.positions[t] = 0;
  }
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ sp_kv_plan_args a, int shift,
                                                            bool fill) {
  __shared__ int64_t s_sum[4];     // pages needed, pages given back, new tokens, units
  __shared__ int s_bad;
  __shared__ int s_warp[32][5];
  __shared__ int32_t s_cu[kCuShared + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  const bool allocate = a.free_pages != nullptr;
  const int64_t height = allocate ? *a.free_count : 0;
  if (tid < 4) s_sum[tid] = 0;
  if (tid == 0) s_bad = height < 0 || height > a.pages ? SP_PLAN_INPUT : 0;
  __syncthreads();
  Request own = {};  // of a batch of one chunk, read once
  {
    int64_t sum[4] = {};
    int bad = 0;
    for (int b = tid; b < a.requests; b += kPlanThreads) {
      const Request r = request_at(a, shift, b);
      own = r;
      bad |= r.bad;
      if (allocate && !r.gone) sum[0] += r.after - r.before;
      if (allocate && r.gone) sum[1] += r.before;
      sum[2] += r.add;
      sum[3] += units_of(r, a.group);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], d);
      if (lane == 0 && sum[k]) atomicAdd(reinterpret_cast<unsigned long long*>(&s_sum[k]), (unsigned long long)sum[k]);
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    if (lane == 0 && bad) atomicOr(&s_bad, bad);
  }
  __syncthreads();
  int bad = s_bad;
  const int64_t top = height + s_sum[1];  // of the stack once the ended requests' pages are on it
  if (top > a.pages && allocate) bad |= SP_PLAN_INPUT;
  if (s_sum[0] > top) bad |= SP_PLAN_PAGES;
  if (s_sum[2] > a.max_tokens) bad |= SP_PLAN_TOKENS;
  if (s_sum[3] > INT_MAX / 64) bad |= SP_PLAN_WIDTH;  // more shares than the attention kernel counts
  if (tid == 0) {
    *a.status = bad;
    if (allocate) *a.next_count = bad ? (int32_t)height : (int32_t)(top - s_sum[0]);
    a.cu_q[0] = 0;
    a.work[0] = 0;
    a.work[a.requests + 1] = 0;
    s_cu[0] = 0;
  }
  int base[5];  // pages taken, pages given back, tokens, units, pairs of the chunks before
  const bool one = a.requests <= kPlanThreads;
  for (int phase = s_sum[1] > 0 ? 0 : 1; phase < 2; ++phase) {
    // phase 0: pages given back; phase 1, behind a barrier: everything else
    base[0] = base[1] = base[2] = base[3] = base[4] = 0;
    for (int b0 = 0; b0 < a.requests; b0 += kPlanThreads) {
      const int b = b0 + tid;
      Request r = {};
      if (b < a.requests && !bad) r = one ? own : request_at(a, shift, b);
      const int v[5] = {allocate && !r.gone ? (int)(r.after - r.before) : 0, allocate && r.gone ? (int)r.before : 0,
                        (int)r.add, (int)units_of(r, a.group), (int)pairs_of(r, a.group)};
      int x[5];
#pragma unroll
      for (int k = 0; k < 5; ++k) {
        int s = v[k];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, s, d);
          if (lane >= d) s += u;
        }
        x[k] = s - v[k];
        if (lane == 31) s_warp[warp][k] = s;
      }
      __syncthreads();
      if (warp < 5) {  // a warp per quantity
        int s = s_warp[lane][warp];
        const int own = s;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, s, d);
          if (lane >= d) s += u;
        }
        __syncwarp();
        s_warp[lane][warp] = s - own;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 5; ++k) x[k] += base[k] + s_warp[warp][k];
      if (phase == 0)
        each_page(v[1], ((int64_t)b << 32) | (uint32_t)x[1], [&](int64_t key, int j) {
          a.free_pages[height + (int32_t)key + j] = a.table[(key >> 32) * a.width + j];
        });
      if (phase == 1) {
        if (b < a.requests) {
          a.cu_q[b + 1] = x[2] + v[2];
          a.work[b + 1] = x[3] + v[3];
          a.work[a.requests + 2 + b] = x[4] + v[4];
          // where its new pages are on the stack: page j of the request at this less j
          a.work[2 * (a.requests + 1) + b] = (int32_t)(top - 1 - x[0] + r.before);
          if (b < kCuShared) s_cu[b + 1] = x[2] + v[2];
        }
      }
      if (!one) {  // the chunk's sums
        __syncthreads();
        if (tid == kPlanThreads - 1) {
#pragma unroll
          for (int k = 0; k < 5; ++k) s_warp[0][k] = x[k] + v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 5; ++k) base[k] = s_warp[0][k];
        __syncthreads();
      }
    }
    __syncthreads();
  }
  // lengths last: they may be written over the ones that the passes above read
  for (int b = tid; b < a.requests; b += kPlanThreads)
    a.lens[b] = bad ? a.cached[b] : (int32_t)(one ? own : request_at(a, shift, b)).len;
  __syncthreads();
  if (fill) {
    const int32_t* cu = a.requests <= kCuShared ? s_cu : a.cu_q;
    for (int64_t t = tid; t < (a.max_tokens + 31) / 32 * 32; t += kPlanThreads) fill_tokens(a, shift, cu, t);
  }
}

__global__ void __launch_bounds__(kFillThreads) fill_kernel(const __grid_constant__ sp_kv_plan_args a, int shift) {
  pdl_wait();
  fill_tokens(a, shift, a.cu_q, blockIdx.x * (int64_t)kFillThreads + threadIdx.x);
}

// What is taken back from request b: its length before and after, its pages (retract_kernel).
struct Kept {
  int64_t cached, len;
  int before, after;
  bool bad;
};
__device__ __forceinline__ Kept kept_at(const sp_kv_retract_args& a, int shift, int64_t b) {
  Kept r;
  const int64_t drop = a.drop[b], p1 = ((int64_t)1 << shift) - 1;
  r.cached = a.cached[b];
  r.bad = r.cached < 0 || r.cached > min((int64_t)a.width << shift, (int64_t)INT_MAX) || drop < 0 || drop > r.cached;
  r.len = r.bad ? r.cached : r.cached - drop;
  r.before = r.bad ? 0 : (int)((r.cached + p1) >> shift);
  r.after = r.bad ? 0 : (int)((r.len + p1) >> shift);
  return r;
}

// One CTA, as the plan of a step: a sum of the pages and whether all is sound, then the exclusive sums at
// which each request's pages go on the stack.
__global__ void __launch_bounds__(kPlanThreads) retract_kernel(const __grid_constant__ sp_kv_retract_args a, int shift) {
  __shared__ unsigned long long s_pages;
  __shared__ int s_bad, s_warp[32], s_base;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  const bool release = a.free_pages != nullptr;
  const int64_t height = release ? *a.free_count : 0;
  if (tid == 0) s_pages = 0, s_base = 0, s_bad = height < 0 || height > a.pages;
  __syncthreads();
  Kept own = {};
  const bool one = a.requests <= kPlanThreads;
  {
    int64_t pages = 0;
    bool bad = false;
    for (int64_t b = tid; b < a.requests; b += kPlanThreads) {
      own = kept_at(a, shift, b);
      pages += own.before - own.after;
      bad |= own.bad;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) pages += __shfl_xor_sync(0xffffffffu, pages, d);
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0 && pages) atomicAdd(&s_pages, (unsigned long long)pages);
    if (lane == 0 && bad) s_bad = 1;
  }
  __syncthreads();
  const int64_t top = height + (int64_t)s_pages;
  const bool bad = s_bad || (release && top > a.pages);
  if (tid == 0) {
    if (bad) *a.status |= SP_PLAN_INPUT;  // (what the step's plan said stays)
    if (release) *a.next_count = (int32_t)(bad ? height : top);
  }
  if (release && !bad && top > height) {
    for (int64_t b0 = 0; b0 < a.requests; b0 += kPlanThreads) {
      const int64_t b = b0 + tid;
      Kept r = {};
      if (b < a.requests) r = one ? own : kept_at(a, shift, b);
      const int n = r.before - r.after;
      int s = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += u;
      }
      if (lane == 31) s_warp[warp] = s;
      __syncthreads();
      if (warp == 0) {
        int t = s_warp[lane];
        const int own_t = t;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, t, d);
          if (lane >= d) t += u;
        }
        s_warp[lane] = t - own_t;
      }
      __syncthreads();
      const int at = s_base + s_warp[warp] + s - n;
      // page j of those that b gives back, from table entry after + j: a few by the request's lane, all asked for before the
      // first is written (by the warp, one request after the other: 1000 requests 13.1 us), many by the warp
      const int64_t from = b * a.width + r.after, to = height + at;
      int few[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < n && n <= 4) few[j] = a.table[from + j];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < n && n <= 4) a.free_pages[to + j] = few[j];
      for (unsigned todo = __ballot_sync(0xffffffffu, n > 4); todo; todo &= todo - 1) {
        const int src = __ffs(todo) - 1;
        const int m = __shfl_sync(0xffffffffu, n, src);
        const int64_t f = __shfl_sync(0xffffffffu, from, src), o = __shfl_sync(0xffffffffu, to, src);
        for (int j = lane; j < m; j += 32) a.free_pages[o + j] = a.table[f + j];
      }
      __syncthreads();
      if (tid == kPlanThreads - 1) s_base = at + n;
      __syncthreads();
    }
  }
  // lengths last: they may be written over the ones that the passes above read
  __syncthreads();
  for (int64_t b = tid; b < a.requests; b += kPlanThreads) {
    const Kept r = one ? own : kept_at(a, shift, b);
    a.lens[b] = (int32_t)(bad ? r.cached : r.len);
  }
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" sp_status sp_kv_retract(const sp_kv_retract_args* a, void* stream) {
  if (!a || a->requests < 0 || a->width < 0 || a->pages < 0 || a->page_size <= 0 || (a->page_size & (a->page_size - 1)) ||
      a->page_size > 1 << 16 || a->reserved != 0)
    return SP_ERR_INVALID_ARG;
  if (!a->status || (a->requests > 0 && (!a->cached || !a->drop || !a->lens))) return SP_ERR_INVALID_ARG;
  if (a->free_pages && (!a->free_count || !a->next_count || (a->requests > 0 && !a->table))) return SP_ERR_INVALID_ARG;
  if (a->pages > INT_MAX || a->requests > INT_MAX / 4) return SP_ERR_UNSUPPORTED;
  auto off = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; };
  if (off(a->cached) || off(a->drop) || off(a->lens) || off(a->status)) return SP_ERR_ALIGNMENT;
  if (a->free_pages && (off(a->free_pages) || off(a->free_count) || off(a->next_count) || off(a->table))) return SP_ERR_ALIGNMENT;
  return launch_pdl(retract_kernel, dim3(1), kPlanThreads, 0, 1, (cudaStream_t)stream, *a, page_shift(a->page_size));
}

extern "C" sp_status sp_kv_plan(const sp_kv_plan_args* a, void* stream) {
  if (!a || a->requests < 0 || a->width < 0 || a->max_tokens < 0 || a->pages < 0 || a->page_size <= 0 ||
      (a->page_size & (a->page_size - 1)) || a->page_size > 1 << 16 || a->group < 1 || a->group > kMaxGroup)
    return SP_ERR_INVALID_ARG;
  if (!a->cu_q || !a->work || !a->status) return SP_ERR_INVALID_ARG;
  if (a->requests > 0 && (!a->cached || !a->new_tokens || !a->lens || !a->table)) return SP_ERR_INVALID_ARG;
  if (a->max_tokens > 0 && (!a->slots || !a->positions)) return SP_ERR_INVALID_ARG;
  if (a->free_pages && (!a->free_count || !a->next_count)) return SP_ERR_INVALID_ARG;
  if (a->max_tokens > INT_MAX || a->pages > INT_MAX || a->requests > INT_MAX / 4) return SP_ERR_UNSUPPORTED;
  const int shift = page_shift(a->page_size);
  const bool fill = a->max_tokens <= kFillHere;
  sp_status st = launch_pdl(plan_kernel, dim3(1), kPlanThreads, 0, 1, (cudaStream_t)stream, *a, shift, fill);
  if (st != SP_OK || fill) return st;
  return launch_pdl(fill_kernel, dim3((unsigned)((a->max_tokens + kFillThreads - 1) / kFillThreads)), kFillThreads, 0,
                    1, (cudaStream_t)stream, *a, shift);
}
