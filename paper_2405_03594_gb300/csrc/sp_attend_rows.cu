// sp_attend_rows.cu -- attention over the cache held in 4 bits (include/sp_serve.h) for requests with
// many new tokens: prompts, and chunks of prompts behind a cached prefix.
//
// The products are large, so they run on the 5th-generation tensor cores: S = Q . K^T and O += P . V,
// 128 query rows by 128 keys a step, fp16 with fp32 sums in tensor memory.  Per step and 128 rows
// the tensor core needs 1024 clocks (D = 128); the exponentials, and the expansion of codes to
// fp16, need issue slots of the same order.  So a CTA takes 256 query rows, two tiles that share
// every expanded key and value and alternate: while one tile's scores are turned into weights, the
// other's products run.
//
//   warps 0-3, 4-7   a tile of query rows each, thread = row: scores out of tensor memory, weights back
//                    into their place as fp16 (an operand of the second product), row sums
//   warps 8-11       codes to fp16 operands in shared memory: rows of keys and of values in
//                    128-byte-swizzled panels of 64 channels
//   warps 12, 13     issue a tile's products each
//   warp 14          copies of the codes, the keys' sixteen more columns, and the next item
//
// Measured, 32 heads of 128, two prompts of up to 2048 tokens behind a prefix (4 x 24e9 operations): 149 us,
// 0.65 PFLOP/s, 0.34 of the measured bf16 rate; the tensor pipe is active 35 % of the time.  No part alone bounds
// it.  With the products cut to an eighth it takes 148 us, without exponentials no less than with them, without the
// expansion of the codes and its stores 139, without the expansion and with an eighth of the products 130 (the same
// kernel with that part left out, wrong results).  What is left is a tile's chain in each step, whose links wait
// for one another: scores out of tensor memory, maximum, weights and their stores, the products of the weights, the
// next scores, four barriers.
//
// Split.  Pairs of tiles are taken from one list, those that see more first.  Where there are
// fewer pairs than SMs, each one's steps of keys are cut into shares, whose sums join_rows_kernel adds up
// in order: a chunk of 64 tokens behind 8000, 8 key heads of 128 with four query heads each, 142 us uncut, 46 in
// shares.  The host, which sees no lengths, cuts by the most pairs that so many rows of q can make, so beside many
// single tokens, or in a padded q, such a chunk stays uncut.
//
// Numbers.  A value s n + m is rounded once to fp16 (the cache holds |x| <= 2^15), which is an eighth of what the
// output's rounding to bf16 takes from it.  A key is not: its offset may be a thousand times its step s, and rounded with
// it would lose the codes (keys 1000 from zero, s = 0.3: outputs off by a tenth).  So the operand is s (n - 8), and
// sixteen more columns hold m and 8 s, which are fp16 numbers, against the queries' sum as three fp16 numbers: 33 bits
// of it (2 % of the time: 148.9 us against 146).  The queries, bf16, enter exactly but for entries below 2^-24 of their row's
// largest, each row scaled by a power of two that keeps its sum below 2^15.  The running maximum of a row moves only when
// a weight would pass 2^8, so the sums in tensor memory are rarely touched by the rows' threads.  The channels
// stand in the order in which a word's codes come out, i and i + 4 as a pair, in the queries
// too; the output is put in order on its way out.
#include <algorithm>
#include <climits>

#include "sp_attend.cuh"
#include "sp_lookup.h"
#include "sp_tcgen05.cuh"

namespace sp {
namespace {

constexpr int kTile = 128;                // keys of a step, query rows of a tile
constexpr int kRowThreads = 256;          // two tiles' rows
constexpr int kFillWarps = 4;
constexpr int kBusyThreads = kRowThreads + 32 * kFillWarps + 96;
constexpr int kThreads = 512;             // whole warpgroups, as the division of the registers wants them
constexpr int kStages = 2;
constexpr int kMostShares = 16;
constexpr int kShareSteps = 3;            // of keys, least of a share where an item is cut
constexpr int kMaxDevices = 64;
constexpr float kFarScore = 1048576.f;    // 2^20: half a unit of such a score is 2^-4
constexpr uint32_t kPanel = kTile * 128;  // 128 rows of 64 columns

template <int D>
struct Smem {
  static constexpr uint32_t kQ = D / 64 * kPanel;              // a tile of queries, a step's keys
  static constexpr uint32_t kV = kQ;                           // a step's values
  static constexpr uint32_t kRaw = kTile * (D / 2 + 4);        // a step's codes and parameters of one of them
  static constexpr uint32_t kMore = kTile * 32;                // sixteen more columns of either
  static constexpr uint32_t kBytes = 2 * kQ + kStages * (kQ + kV) + 2 * kRaw + (2 + kStages) * kMore;
  static constexpr size_t kTotal = 1024 + kBytes;              // + base alignment
  static_assert(kTotal + 1024 <= 227 * 1024, "beside them a kilobyte at most of barriers, items and the like");
};

__device__ __forceinline__ void mma_ss(uint32_t d_taddr, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_taddr),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
// Instruction descriptor, kind::f16: D fp32, A and B fp16, both K-major.
constexpr uint32_t idesc_f16(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

// B held as rows of 64 of its N columns, one row per K (128-byte swizzle): eight rows 1024 bytes apart
// make the next eight of K (stride byte offset), the next 64 columns lie a panel on (leading byte offset).
constexpr uint32_t kRowsAlongK = 1u << 16;
__device__ __forceinline__ uint64_t smem_desc_rows_along_k(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
  d |= (uint64_t)((kPanel >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)((1024u >> 4) & 0x3FFFu) << 32;
  d |= (uint64_t)1u << 46;
  d |= (uint64_t)2u << 61;
  return d;
}

// The sixteen more columns: two blocks of 8 rows by 16 bytes side by side, 128 bytes each (no swizzle).
__device__ __forceinline__ uint64_t smem_desc_more(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
  d |= (uint64_t)(128u >> 4) << 16;
  d |= (uint64_t)(256u >> 4) << 32;
  d |= (uint64_t)1u << 46;
  return d;
}
__device__ __forceinline__ uint4* more_columns(uint8_t* base, int row) {  // the first eight of a row
  return reinterpret_cast<uint4*>(base + (row >> 3) * 256 + (row & 7) * 16);
}

__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// s n + m of the nibbles i and i + 4 of w: a code's bits under the exponent of 1024, the 1024 taken off
// again, then one rounding.
__device__ __forceinline__ uint32_t value_lo(uint32_t w, uint32_t s, uint32_t m) {  // i = 0 (2, of w >> 8)
  return hfma2(hsub2((w & 0x000f000fu) | 0x64006400u, 0x64006400u), s, m);
}
__device__ __forceinline__ uint32_t value_hi(uint32_t w, uint32_t s, uint32_t m) {  // i = 1 (3): 1024 + 16 n
  return hfma2(hfma2((w & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd400d400u), s, m);
}

// 256 query rows of a request and key head.
struct Item {
  int b, h;
  int q0;           // row of q of the request's first new token
  int row0, rows;   // first query row among the request's, query rows
  int sees0;        // keys that new token 0 sees
  int len;
  int j0, j1;       // steps of keys of this share
  int part;         // the share's place in the workspace; -1: it holds all steps
};

// Steps of keys that the rows of the item's tile i see, all shares together.
__device__ __forceinline__ int all_steps(const AttendParams& p, const Item& it, int i) {
  const int rows = min(it.rows - i * kTile, kTile);
  return rows > 0 ? (it.sees0 + (it.row0 + i * kTile + rows - 1) / p.group + kTile - 1) / kTile : 0;
}
// Of them, those of this share.
__device__ __forceinline__ int steps_of(const AttendParams& p, const Item& it, int i) {
  return max(0, min(all_steps(p, it, i), it.j1) - it.j0);
}

// Item i of the list: pairs of tiles of all requests, later rows, which see more, first.  Rows 0 behind the
// last, -1 where the shares do not belong to the lengths.  shares: into how many its steps are cut.
__device__ __forceinline__ Item item_at(const AttendParams& p, int64_t i, int& shares) {
  const int32_t* share = p.work + p.requests + 1;  // pairs of tiles of the requests before each
  const int heads = p.cache.heads;
  Item it;
  it.rows = 0;
  shares = 1;
  if (i >= (int64_t)share[p.requests] * heads) return it;
  const int pair = (int)(i / heads);
  int lo = 0, hi = p.requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (share[mid] <= pair) lo = mid;
    else hi = mid;
  }
  it.b = lo;
  it.h = (int)(i % heads);
  it.q0 = p.cu_q[lo];
  it.len = p.lens[lo];
  const int fresh = p.cu_q[lo + 1] - it.q0, pairs = share[lo + 1] - share[lo];
  const int64_t all = (int64_t)fresh * p.group;
  if (fresh <= 0 || it.len < fresh || fresh > p.max_new || it.q0 < 0 || it.q0 + (int64_t)fresh > p.tokens ||
      (all + 2 * kTile - 1) / (2 * kTile) != pairs) {
    set_status(p.status, kStatusBadIndex);
    it.rows = -1;
    return it;
  }
  it.row0 = (pairs - 1 - (pair - share[lo])) * 2 * kTile;
  it.rows = (int)min(all - it.row0, (int64_t)(2 * kTile));
  it.sees0 = it.len - fresh + 1;
  it.j0 = 0;
  it.j1 = max(all_steps(p, it, 0), all_steps(p, it, 1));
  it.part = -1;
  shares = min(p.split, (it.j1 + kShareSteps - 1) / kShareSteps);
  if (shares > 1 && (i + 1) * p.split > p.parts) {  // rows of q that the host did not count
    set_status(p.status, kStatusBadIndex);
    shares = 1;
  }
  return it;
}

// Item i, by a warp, where every item is a whole one and up to 32 requests have more items than there are
// CTAs: most steps first, whatever request they belong to, so that the CTAs finish together (two prompts, of
// 24 to 17 and 18 to 10 steps, over 152 SMs: the last one ends after 51 steps, in the list's order
// after 55).  A lane per request counts its pairs of at least so many steps, and a search over the steps finds the item.
__device__ __forceinline__ Item item_by_steps(const AttendParams& p, int64_t i) {
  const int32_t* share = p.work + p.requests + 1;
  const int lane = threadIdx.x & 31, heads = p.cache.heads;
  int shares;
  if (p.requests > 32 || (int64_t)share[p.requests] * heads <= gridDim.x) return item_at(p, i, shares);
  Item it;
  it.rows = 0;
  int pairs = 0, q0 = 0, len = 0, fresh = 0;
  if (lane < p.requests) {
    q0 = p.cu_q[lane];
    len = p.lens[lane];
    fresh = p.cu_q[lane + 1] - q0;
    pairs = share[lane + 1] - share[lane];
    if (pairs != 0 && (fresh <= 0 || len < fresh || fresh > p.max_new || q0 < 0 || q0 + (int64_t)fresh > p.tokens ||
                       ((int64_t)fresh * p.group + 2 * kTile - 1) / (2 * kTile) != pairs)) {
      set_status(p.status, kStatusBadIndex);
      pairs = 0;
    }
  }
  const int64_t rows = (int64_t)fresh * p.group;
  const int k = (int)(i / heads);  // pairs of tiles before this one
  auto of_steps = [&](int steps) {  // of the lane's request: pairs of at least so many
    const int64_t row = ((int64_t)(steps - 1) * kTile - (len - fresh)) * p.group;  // the first row that needs them
    return pairs == 0 || row >= rows ? 0 : row <= 0 ? pairs : pairs - (int)(row / (2 * kTile));
  };
  int lo = 1, hi = (int)__reduce_max_sync(0xffffffffu, pairs ? (unsigned)((len + kTile - 1) / kTile) : 0u) + 1;
  if (__reduce_add_sync(0xffffffffu, pairs) <= k) return it;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__reduce_add_sync(0xffffffffu, of_steps(mid)) > k) lo = mid;
    else hi = mid;
  }
  const int more = of_steps(lo + 1), own = of_steps(lo) - more;
  int before = own;  // own pairs of the requests up to this one
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, before, d);
    if (lane >= d) before += x;
  }
  const int rank = k - __reduce_add_sync(0xffffffffu, more);
  const int b = __ffs(__ballot_sync(0xffffffffu, before > rank)) - 1;
  const int from_end = __shfl_sync(0xffffffffu, more + rank - (before - own), b);
  it.b = b;
  it.h = (int)(i % heads);
  it.q0 = __shfl_sync(0xffffffffu, q0, b);
  it.len = __shfl_sync(0xffffffffu, len, b);
  fresh = __shfl_sync(0xffffffffu, fresh, b);
  it.row0 = (__shfl_sync(0xffffffffu, pairs, b) - 1 - from_end) * 2 * kTile;
  it.rows = (int)min((int64_t)fresh * p.group - it.row0, (int64_t)(2 * kTile));
  it.sees0 = it.len - fresh + 1;
  it.j0 = 0;
  it.j1 = max(all_steps(p, it, 0), all_steps(p, it, 1));
  it.part = -1;
  return it;
}

struct Barriers {
  uint64_t q_full, k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  uint64_t s_full[2], p_full[2], o_done[2];
  uint64_t raw_full[2], raw_empty[2];  // keys, values
  uint64_t turn[2];          // the other tile's products of its step have been issued
  uint64_t probe;            // kExpire: nothing arrives here
  uint64_t drained[2];       // where a wait has expired: a tile's products on their way are done
};

struct Shared {
  Barriers bar;
  uint32_t tmem;
  uint32_t nan[kStages][4];  // keys of the step whose values are not finite
  Item item[2];
  unsigned pages[2];         // of the raw keys and values: the pages that exist
};

// A bounded wait of a whole warp; nothing is waited for once one has expired.  (The sleeping wait is a
// short loop.  mbar_wait's polls, unrolled at every wait, were more code than the SM's instruction
// cache holds beside the roles' own: 165 us against 140 for the prefill measured below.)
struct Wait {
  const AttendParams& p;
  bool dead;
  __device__ __forceinline__ void operator()(uint64_t* bar, uint32_t parity) {
    if (dead) return;
    if (!__all_sync(0xffffffffu, mbar_wait_sleep(bar, parity, p.timeout_ns))) {
      if ((threadIdx.x & 31) == 0) set_status(p.status, kStatusTimeout);
      dead = true;
    }
  }
};

// The end of an item for every warp that works on it; false, in all of them alike, once a wait has expired.
__device__ __forceinline__ bool end_item(const Wait& wait) {
  tc_fence_before();
  const bool dead = named_bar_or(1, kBusyThreads, wait.dead);
  tc_fence_after();
  return !dead;
}

// ------------------------------------------------------------------ rows: scores to weights, and the output
template <int D>
__device__ __forceinline__ void rows_role(const AttendParams& p, Shared& sh, uint8_t* s_q, uint8_t* s_more, uint32_t tmem,
                                          bool gone) {
  using L = Smem<D>;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int i = warp >> 2;  // tile
  const int r = tid & (kTile - 1);
  const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t t_s = tmem + lanes + i * kTile, t_o = tmem + lanes + 2 * kTile + i * D;
  Wait wait{p, gone};
  uint32_t steps = 0, done = 0;
  for (uint32_t round = 0;; ++round) {
    const Item& it = sh.item[round & 1];  // (in shared memory: registers are what this role is short of)
    if (it.rows <= 0) break;
    const int n = steps_of(p, it, i);
    int limit;  // keys of the share that the row sees
    float cr;   // log2 score = cr * product
    {
      const bool there = i * kTile + r < it.rows;
      const int row = it.row0 + i * kTile + r, token = row / p.group;
      const int64_t col = (int64_t)(it.h * p.group + row - token * p.group) * D;
      limit = there ? it.sees0 + token - it.j0 * kTile : 0;
      const uint4* src = reinterpret_cast<const uint4*>(p.q + (it.q0 + (int64_t)token) * p.q_stride + col);
      uint4 u[D / 8];
      uint32_t big = 0;
#pragma unroll
      for (int c = 0; c < D / 8; ++c) u[c] = there ? src[c] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        const uint32_t x[4] = {u[c].x, u[c].y, u[c].z, u[c].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) big = max(big, max(x[j] & 0x7fffu, (x[j] >> 16) & 0x7fffu));
      }
      // 2^(134 - e): the row's largest entry, of biased exponent e, comes to 2^7 ... 2^8, their sum below 2^15
      const uint32_t e = max(15u, min(254u, big >> 7));
      const float f = copysignf(__uint_as_float((261u - e) << 23), p.scale_log2);
      // (not 0, which would make NaN of what the row does not see)
      cr = fmaxf(__uint_as_float((e - 7u) << 23) * fabsf(p.scale_log2), 1e-37f);
      uint8_t* dst = s_q + i * L::kQ + r * 128;
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        const uint32_t x[4] = {u[c].x, u[c].y, u[c].z, u[c].w};
        float y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[2 * j] = __uint_as_float(x[j] << 16) * f;
          y[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u) * f;
          sum[0] += y[2 * j], sum[1] += y[2 * j + 1];
        }
        *reinterpret_cast<uint4*>(dst + (c >> 3) * kPanel + (((c & 7) ^ (r & 7)) << 4)) =
            make_uint4(pack_f16(y[0], y[4]), pack_f16(y[1], y[5]), pack_f16(y[2], y[6]), pack_f16(y[3], y[7]));
      }
      // the sum in three fp16 numbers, against the keys' minima and scales
      const float h0 = __half2float(__float2half_rn(sum[0] + sum[1])), r1 = sum[0] + sum[1] - h0;
      const float h1 = __half2float(__float2half_rn(r1)), h2 = r1 - h1;
      *more_columns(s_more + i * L::kMore, r) = make_uint4(pack_f16(h0, h1), pack_f16(h2, h0), pack_f16(h1, h2), 0);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.bar.q_full);
    float m = -INFINITY;
    uint64_t l = 0;
    bool poisoned = false;
    for (int j = 0; j < n; ++j) {
      wait(&sh.bar.s_full[i], (done + j) & 1);
      if (wait.dead) break;
      tc_fence_after();
      uint32_t u[kTile];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_load32(t_s + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(u + 32 * c));
      tmem_load_wait();
      const int seen = limit - j * kTile;  // of the step's keys
      if (__any_sync(0xffffffffu, seen < kTile)) {
#pragma unroll
        for (int k = 0; k < kTile; ++k)
          if (k >= seen) u[k] = 0xff800000u;
      }
      float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int k = 0; k < kTile; ++k) t4[k & 3] = fmaxf(t4[k & 3], __uint_as_float(u[k]));
      float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
      top *= cr;
      if (__any_sync(0xffffffffu, top > m + 8.f)) {
        const float up = top > m + 8.f ? top : m;
        const float alpha = up == m ? 1.f : m == -INFINITY ? 0.f : ex2(m - up);
        m = up;
        if (j > 0) {
          const uint64_t a2 = two(alpha, alpha);
          l = mul2(l, a2);
          wait(&sh.bar.o_done[i], (done + j - 1) & 1);
          if (wait.dead) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t v[16];
            tmem_load16(t_o + 16 * c, v);
            tmem_load_wait();
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * alpha);
            tmem_store16(t_o + 16 * c, v);
          }
        }
      }
      const float minus = m == -INFINITY ? 0.f : -m;
      float c = cr;
      // The maximum is a rounded product, the exponents below are not: off by half a unit of the scores, all by
      // the same, which is nothing up to here and would pass fp16 from 2^28 on.  So far away the scores are rounded first.
      if (__any_sync(0xffffffffu, fabsf(minus) > kFarScore)) {
        c = 1.f;
#pragma unroll
        for (int k = 0; k < kTile; ++k) u[k] = __float_as_uint(__uint_as_float(u[k]) * cr);
      }
      const uint64_t c2 = two(c, c), m2 = two(minus, minus);
      uint64_t sum[2] = {0, 0};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          float a, b;
          apart(fma2(two(__uint_as_float(u[32 * c + k]), __uint_as_float(u[32 * c + k + 1])), c2, m2), a, b);
          a = ex2(a), b = ex2(b);
          sum[(k >> 1) & 1] = add2(sum[(k >> 1) & 1], two(a, b));
          w[k / 2] = pack_f16(a, b);
        }
        tmem_store16(t_s + 16 * c, w);
      }
      l = add2(l, add2(sum[0], sum[1]));
      // a value row that is not finite entered as zeros: it makes NaN of the rows that see it
      const int st = (steps + j) % kStages;
      wait(&sh.bar.v_full[st], ((steps + j) / kStages) & 1);
      if (wait.dead) break;
      const volatile uint32_t* bad = sh.nan[st];
      const uint32_t x[4] = {bad[0], bad[1], bad[2], bad[3]};
      if (x[0] | x[1] | x[2] | x[3]) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int sc = seen - 32 * c;
          if (x[c] & (sc >= 32 ? ~0u : sc <= 0 ? 0u : (1u << sc) - 1u)) poisoned = true;
        }
      }
      tmem_store_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.bar.p_full[i]);
    }
    if (n > 0) wait(&sh.bar.o_done[i], (done + n - 1) & 1);
    tc_fence_after();
    if (wait.dead) {
      tmem_store_wait();  // (this thread's, before the columns are given back)
    } else {
      float a, b;
      apart(l, a, b);
      a += b;
      if (poisoned) a = __uint_as_float(0x7fffffffu);
      if (it.part < 0) {
        const bool there = i * kTile + r < it.rows;  // (worked out again: not kept over the steps)
        const int row = it.row0 + i * kTile + r, token = row / p.group;
        const int64_t col = (int64_t)(it.h * p.group + row - token * p.group) * D;
        const float inv = a == 0.f ? 0.f : 1.f / a;
        uint16_t* dst = p.out + (it.q0 + (int64_t)token) * p.out_stride + col;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_load32(t_o + 32 * c, v);
          tmem_load_wait();
          if (there) {
#pragma unroll
            for (int k = 0; k < 32; k += 8) {
              uint32_t w[4];
#pragma unroll
              for (int x = 0; x < 4; ++x) {  // channels 0, 4, 1, 5, 2, 6, 3, 7 of eight
                const int y = k + (x & 1) * 4 + (x >> 1);
                w[x] = pack_bf16(__uint_as_float(v[y]) * inv, __uint_as_float(v[y + 2]) * inv);
              }
              *reinterpret_cast<uint4*>(dst + 32 * c + k) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
      } else {  // a column per row: D sums, the maximum, the sum of weights
        float* dst = p.part + (int64_t)it.part * (D + 2) * kPairRows + i * kTile + r;
#pragma unroll 1
        for (int c = 0; c < D; c += 16) {
          uint32_t v[16];
          if (n > 0) tmem_load16(t_o + c, v);
          tmem_load_wait();
#pragma unroll
          for (int k = 0; k < 16; ++k) __stcg(dst + (c + k) * kPairRows, n > 0 ? __uint_as_float(v[k]) : 0.f);
        }
        __stcg(dst + D * kPairRows, m);
        __stcg(dst + (D + 1) * kPairRows, a);
      }
    }
    steps += max(steps_of(p, it, 0), steps_of(p, it, 1));
    done += n;
    if (!end_item(wait)) break;
  }
}

// ------------------------------------------------------------------ keys and values: copies of the codes
// A step's codes and parameters come to shared memory as they are, by one bulk copy per page, as soon as
// the step before is expanded.  Where a wait has expired, none is on its way any more when the CTA ends.
template <int D, class Fetch>
__device__ __forceinline__ void copy_role(const AttendParams& p, Shared& sh, uint8_t* s_raw, uint8_t* s_more, Fetch fetch, bool gone) {
  using L = Smem<D>;
  const int lane = threadIdx.x & 31;
  const int shift = p.cache.shift, heads = p.cache.heads, pages = kTile >> shift;
  const int64_t block = kv4_block_bytes<D>(shift);
  Wait wait{p, gone};
  uint32_t steps = 0, sent = 0;  // sent: copies of keys and values, one after the other
  for (uint32_t round = 0;; ++round) {
    const Item it = sh.item[round & 1];
    if (it.rows <= 0) break;
    const int n = max(steps_of(p, it, 0), steps_of(p, it, 1));
    const int32_t* table = p.table + (int64_t)it.b * p.width;
    auto page_of = [&](int j) {  // a lane per page of step j
      const int at = (it.j0 + j) * pages + lane;
      return j < n && lane < pages && ((int64_t)at << shift) < it.len ? (at < p.width ? table[at] : -1) : INT_MIN;
    };
    int next = page_of(0);
    {
      Item after;  // the item after this one
      do fetch(after);
      while (after.rows < 0);
      if (lane == 0) sh.item[(round + 1) & 1] = after;
    }
    __syncwarp();
    for (int j = 0; j < n && !wait.dead; ++j) {
      int page = next;
      next = page_of(j + 1);
      if (page < 0 || page >= p.cache.pages) {
        if (page != INT_MIN) set_status(p.status, kStatusBadIndex);
        page = -1;
      }
      const unsigned ok = __ballot_sync(0xffffffffu, page >= 0);
      const uint8_t* src = p.cache.data + ((int64_t)max(page, 0) * heads + it.h) * block;
#pragma unroll 1
      for (int which = 0; which < 2; ++which) {
        wait(&sh.bar.raw_empty[which], ((steps + j) & 1) ^ 1);
        if (wait.dead) break;
        uint64_t* full = &sh.bar.raw_full[which];
        if (lane == 0) {
          sh.pages[which] = ok;
          mbar_arrive_expect_tx(full, __popc(ok) * ((uint32_t)(D / 2 + 4) << shift));
        }
        __syncwarp();
        if (page >= 0) {
          uint8_t* dst = s_raw + which * L::kRaw;
          bulk_g2s(dst + ((lane * (D / 2)) << shift), src + (which ? kv4_value_codes<D>(shift) : 0), (D / 2) << shift, full);
          bulk_g2s(dst + kTile * (D / 2) + ((lane * 4) << shift),
                   src + (which ? kv4_value_params<D>(shift) : kv4_key_params<D>(shift)), 4 << shift, full);
        }
        ++sent;
      }
      // the keys' sixteen more columns: their minima and eight times their scales, three times each
      const int st = (steps + j) % kStages;
      wait(&sh.bar.raw_full[0], (steps + j) & 1);
      wait(&sh.bar.k_empty[st], (((steps + j) / kStages) & 1) ^ 1);
      if (wait.dead) break;
      const uint32_t* raw_par = reinterpret_cast<const uint32_t*>(s_raw + kTile * (D / 2));
      const int left = it.len - (it.j0 + j) * kTile;
#pragma unroll
      for (int x = 0; x < kTile; x += 32) {
        const int key = x + lane;
        uint32_t y = raw_par[key];
        if (key >= left || !(ok >> (key >> shift) & 1)) y = 0;  // what no token was written to may hold anything
        const uint32_t s8 = hfma2(y, 0x48004800u, 0);
        *more_columns(s_more + (2 + st) * L::kMore, key) =
            make_uint4(__byte_perm(y, y, 0x3232), __byte_perm(y, s8, 0x5432), __byte_perm(s8, s8, 0x1010), 0);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.bar.k_full[st]);
      }
    }
    steps += n;
    if (!end_item(wait)) {
      for (uint32_t which = 0; which < 2 && which < sent; ++which)
        mbar_wait_sleep(&sh.bar.raw_full[which], ((sent - 1 - which) >> 1) & 1, p.timeout_ns);
      break;
    }
  }
}

// ------------------------------------------------------------------ keys and values: codes to operands
template <int D>
__device__ __forceinline__ void fill_role(const AttendParams& p, Shared& sh, uint8_t* s_k, uint8_t* s_v, const uint8_t* s_raw,
                                          bool gone) {
  using L = Smem<D>;
  const int f = threadIdx.x - kRowThreads, lane = threadIdx.x & 31;
  const int shift = p.cache.shift;
  constexpr int KP = D / 32;  // 16-byte pieces of a row: a lane takes one of row f / KP, then of rows further on
  const int piece = f % KP;
  // The pieces of a row that lie in the second panel are stored in another order, so that eight
  // lanes' 16 bytes, of two rows, never share a bank.
  const int turn = piece >> 1 << 1;
  Wait wait{p, gone};
  bool alive = true;
  uint32_t steps = 0;
  for (uint32_t round = 0;; ++round) {
    const Item& it = sh.item[round & 1];
    if (it.rows <= 0) break;
    const int keys = it.len - it.j0 * kTile;  // from the share's first on
    const int n = max(steps_of(p, it, 0), steps_of(p, it, 1));
    for (int j = 0; j < n; ++j) {
      const int st = (steps + j) % kStages;
      const uint32_t ph = ((steps + j) / kStages) & 1;
#pragma unroll 1
      for (int which = 0; which < 2; ++which) {
        wait(&sh.bar.raw_full[which], (steps + j) & 1);
        wait(which ? &sh.bar.v_empty[st] : &sh.bar.k_empty[st], ph ^ 1);
        if (!wait.dead) {
          const uint8_t* raw = s_raw + which * L::kRaw;
          const uint32_t* raw_par = reinterpret_cast<const uint32_t*>(raw + kTile * (D / 2));
          uint8_t* dst = which ? s_v + st * L::kV : s_k + st * L::kQ;
          const unsigned ok = sh.pages[which];
          const int left = keys - j * kTile;
          uint4 c4[KP];
          uint32_t par[KP];
#pragma unroll
          for (int x = 0; x < KP; ++x) {
            const int key = x * (kTile / KP) + f / KP;
            c4[x] = *reinterpret_cast<const uint4*>(raw + (x * 128 + f) * 16);
            par[x] = raw_par[key];
            if (key >= left || !(ok >> (key >> shift) & 1)) par[x] = 0;  // what no token was written to may hold anything
          }
          if (which) {
            auto finite = [](uint32_t y) { return (y & 0x7c00u) != 0x7c00u && (y & 0x7c000000u) != 0x7c000000u; };
#pragma unroll
            for (int x = 0; x < KP; ++x)
              if (!finite(par[x])) par[x] = 0;
            if (f < 32) {
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int key = 32 * x + lane;
                const bool bad = key < left && (ok >> (key >> shift) & 1) && !finite(raw_par[key]);
                const unsigned bits = __ballot_sync(0xffffffffu, bad);
                if (lane == 0) sh.nan[st][x] = bits;  // (read before the stage was handed back)
              }
            }
          }
#pragma unroll
          for (int x = 0; x < KP; ++x) {
            const int key = x * (kTile / KP) + f / KP;
            const uint32_t s = __byte_perm(par[x], par[x], 0x1010);
            // (of keys s (n - 8): the rest, which may be far larger than it, is in the other columns)
            const uint32_t m = which ? __byte_perm(par[x], par[x], 0x3232) : hfma2(s, 0xc800c800u, 0);
            const uint32_t w[4] = {turn ? c4[x].z : c4[x].x, turn ? c4[x].w : c4[x].y, turn ? c4[x].x : c4[x].z,
                                   turn ? c4[x].y : c4[x].w};
            uint8_t* row = dst + key * 128 + (piece >> 1) * kPanel;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int c = (4 * (piece & 1) + y) ^ turn;  // eight channels
              const uint32_t h = w[y] >> 8;
              *reinterpret_cast<uint4*>(row + ((c ^ (key & 7)) << 4)) =
                  make_uint4(value_lo(w[y], s, m), value_hi(w[y], s, m), value_lo(h, s, m), value_hi(h, s, m));
            }
          }
          fence_proxy_async_smem();
        }
        // All of the raw rows have been read, all operands written.  (A warp whose wait expired has made none, but it
        // comes here as often as the others, who would wait without a bound; the launch has been reported then.)
        named_bar_sync(2, 32 * kFillWarps);
        if (f == 0 && !wait.dead) {
          mbar_arrive(which ? &sh.bar.v_full[st] : &sh.bar.k_full[st]);
          mbar_arrive(&sh.bar.raw_empty[which]);
        }
      }
    }
    steps += n;
    alive = end_item(wait);
    if (!alive) break;
  }
  if (f < 32 && alive) {  // the products' last arrivals on this CTA's barriers
    for (uint32_t x = steps > kStages ? steps - kStages : 0; x < steps; ++x) {
      wait(&sh.bar.k_empty[x % kStages], (x / kStages) & 1);
      wait(&sh.bar.v_empty[x % kStages], (x / kStages) & 1);
    }
  }
}

// ------------------------------------------------------------------ the products of tile i
template <int D>
__device__ __forceinline__ void product_role(const AttendParams& p, Shared& sh, uint8_t* s_q, uint8_t* s_k, uint8_t* s_v,
                                             uint8_t* s_more, uint32_t tmem, int i, bool gone) {
  using L = Smem<D>;
  Wait wait{p, gone};
  // operand descriptors; a piece further on is a larger start address, in units of 16 bytes
  const uint64_t d_q = smem_desc_sw128(smem_u32(s_q + i * L::kQ)), d_k = smem_desc_sw128(smem_u32(s_k)),
                 d_v = smem_desc_rows_along_k(smem_u32(s_v)), d_qm = smem_desc_more(smem_u32(s_more + i * L::kMore)),
                 d_km = smem_desc_more(smem_u32(s_more + 2 * L::kMore));
  const uint32_t t_s = tmem + i * kTile, t_o = tmem + 2 * kTile + i * D;
  uint32_t steps = 0, done = 0, turns = 0;
  for (uint32_t round = 0;; ++round) {
    if (sh.item[round & 1].rows <= 0) break;
    const int n = steps_of(p, sh.item[round & 1], i);
    const int n_all = max(n, steps_of(p, sh.item[round & 1], 1 - i));
    wait(&sh.bar.q_full, round & 1);
    // step j: O += P_(j-1) . V_(j-1), then S = Q . K_j^T, whose columns P has left by then
    // The tiles take turns, so that one's products run while the other's weights are made; without
    // that both wait at the same time.  The weights are waited for last: all else is there by then.
    for (int j = 0; j <= n_all && !wait.dead; ++j, ++turns) {
      const uint32_t vs = (steps + j - 1) % kStages, ks = (steps + j) % kStages;
      if (j > 0) wait(&sh.bar.v_full[vs], ((steps + j - 1) / kStages) & 1);
      if (j < n_all) wait(&sh.bar.k_full[ks], ((steps + j) / kStages) & 1);
      if (i == 1 || turns > 0) wait(&sh.bar.turn[i], (i == 1 ? turns : turns - 1) & 1);
      if (j > 0 && j - 1 < n) wait(&sh.bar.p_full[i], (done + j - 1) & 1);
      if (wait.dead) break;
      tc_fence_after();
      if (elect_one()) {
        if (j > 0 && j - 1 < n) {
          const uint64_t b = d_v + (uint64_t)(vs * (L::kV >> 4));
#pragma unroll
          for (int kk = 0; kk < kTile / 16; ++kk)  // 16 keys' rows
            mma_ts(t_o, t_s + kk * 8, b + ((kk * 16 * 128) >> 4), idesc_f16(kTile, D) | kRowsAlongK,
                   (j > 1 || kk > 0) ? 1u : 0u);
          mma_commit(&sh.bar.o_done[i]);
        }
        if (j < n) {
          const uint64_t b = d_k + (uint64_t)(ks * (L::kQ >> 4));
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t off = ((kk >> 2) * kPanel + (kk & 3) * 32) >> 4;
            mma_ss(t_s, d_q + off, b + off, idesc_f16(kTile, kTile), kk > 0 ? 1u : 0u);
          }
          mma_ss(t_s, d_qm, d_km + (uint64_t)(ks * (L::kMore >> 4)), idesc_f16(kTile, kTile), 1u);
          mma_commit(&sh.bar.s_full[i]);
        }
        mbar_arrive(&sh.bar.turn[1 - i]);
        // the stages are free once these products are done (or were not needed: the other tile has more steps)
        if (j > 0) mma_commit(&sh.bar.v_empty[vs]);
        if (j < n_all) mma_commit(&sh.bar.k_empty[ks]);
      }
      __syncwarp();
    }
    steps += n_all;
    done += n;
    if (!end_item(wait)) {
      if (elect_one()) mma_commit(&sh.bar.drained[i]);
      __syncwarp();
      mbar_wait_sleep(&sh.bar.drained[i], 0, p.timeout_ns);
      break;
    }
  }
}

// kExpire: a variant for sp_test_expired_attend, whose warp p.expire_warp of CTA p.expire_cta first waits for what
// never comes and gives up.
template <int D, bool kExpire = false>
__global__ void __launch_bounds__(kThreads, 1) attend_rows_kernel(const __grid_constant__ AttendParams p) {
  using L = Smem<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* s_q = smem;
  uint8_t* s_v = smem + 2 * L::kQ;
  uint8_t* s_k = s_v + kStages * L::kV;
  uint8_t* s_raw = s_k + kStages * L::kQ;
  uint8_t* s_more = s_raw + 2 * L::kRaw;  // of two tiles of queries, of the stages' keys
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5;
  if (tid == 0) {
    mbar_init(&sh.bar.q_full, kRowThreads / 32);
    mbar_init(&sh.bar.probe, 1);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.bar.k_full[i], 2);
      mbar_init(&sh.bar.v_full[i], 1);
      mbar_init(&sh.bar.k_empty[i], 2);
      mbar_init(&sh.bar.v_empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.bar.s_full[i], 1);
      mbar_init(&sh.bar.p_full[i], 4);
      mbar_init(&sh.bar.o_done[i], 1);
      mbar_init(&sh.bar.raw_full[i], 1);
      mbar_init(&sh.bar.raw_empty[i], 1);
      mbar_init(&sh.bar.turn[i], 1);
      mbar_init(&sh.bar.drained[i], 1);
    }
    fence_barrier_init();
  }
  for (uint32_t i = tid; i < (2 + kStages) * L::kMore / 16; i += kThreads)
    reinterpret_cast<uint4*>(s_more)[i] = make_uint4(0, 0, 0, 0);  // (the second eight columns stay so)
  fence_proxy_async_smem();
  pdl_wait();
  // the next share of the list, by a warp
  auto fetch = [&](Item& it) {
    int next = 0;
    if ((tid & 31) == 0) next = atomicAdd(&p.cnt[0], 1);
    const int64_t i = (int64_t)__shfl_sync(0xffffffffu, next, 0);
    if (p.split == 1) {
      it = item_by_steps(p, i);
      return;
    }
    int shares;
    it = item_at(p, i / p.split, shares);
    if (it.rows <= 0 || shares == 1) {
      if (i % p.split > 0 && it.rows > 0) it.rows = -1;  // (its first share takes all)
      return;
    }
    const int x = (int)(i % p.split), n = it.j1;
    if (x >= shares) {
      it.rows = -1;
      return;
    }
    it.j0 = (int)((int64_t)x * n / shares);
    it.j1 = (int)((int64_t)(x + 1) * n / shares);
    it.part = (int)i;
  };
  if (warp == kBusyThreads / 32 - 1) {
    Item it;
    do fetch(it);
    while (it.rows < 0);
    if (tid == kBusyThreads - 32) sh.item[0] = it;
  }
  if (warp == 0) {
    tmem_alloc(&sh.tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  bool gone = false;
  if constexpr (kExpire) {
    if (blockIdx.x == p.expire_cta && warp == p.expire_warp && tid < kBusyThreads && sh.item[0].rows > 0) {
      Wait wait{p, false};
      wait(&sh.bar.probe, 0);
      gone = wait.dead;
    }
  }
  // registers: 128 a thread at launch, (176 + 176 + 88 + 72) / 4 from here on
  if (warp < kRowThreads / 32) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    rows_role<D>(p, sh, s_q, s_more, tmem, gone);
  } else if (warp < kRowThreads / 32 + kFillWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    fill_role<D>(p, sh, s_k, s_v, s_raw, gone);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    const int x = warp - kRowThreads / 32 - kFillWarps;
    if (x < 2) product_role<D>(p, sh, s_q, s_k, s_v, s_more, tmem, x, gone);
    if (x == 2) copy_role<D>(p, sh, s_raw, s_more, fetch, gone);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  // the last CTA leaves the counters at zero
  if (tid == 0) {
    __threadfence();
    if (atomicAdd(&p.cnt[1], 1) == (int)gridDim.x - 1) {
      p.cnt[0] = 0;
      p.cnt[1] = 0;
    }
  }
}

// The shares of an item joined: a warp takes 32 rows, a lane each, and 16 of their channels.
template <int D>
__global__ void __launch_bounds__(128) join_rows_kernel(const __grid_constant__ AttendParams p) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t items = (int64_t)p.work[2 * p.requests + 1] * p.cache.heads;
  constexpr int kGroups = kPairRows / 32, kUnits = kGroups * (D / 16);
  for (int64_t u = blockIdx.x * 4 + (threadIdx.x >> 5); u < items * kUnits; u += gridDim.x * 4) {
    const int64_t i = u / kUnits;
    const int r0 = (int)(u % kUnits) % kGroups * 32, c0 = (int)(u % kUnits) / kGroups * 16;
    int shares;
    const Item it = item_at(p, i, shares);
    if (it.rows <= r0 || shares == 1) continue;
    const float* src = p.part + i * p.split * (D + 2) * kPairRows + r0 + lane;
    constexpr int64_t kNext = (int64_t)(D + 2) * kPairRows;
    float m = -INFINITY;
    for (int x = 0; x < shares; ++x) m = fmaxf(m, __ldcg(src + x * kNext + D * kPairRows));
    const float safe = m == -INFINITY ? 0.f : m;
    float sum = 0.f, acc[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) acc[k] = 0.f;
#pragma unroll 2
    for (int x = 0; x < shares; ++x) {
      const float* s = src + x * kNext;
      const float f = ex2(__ldcg(s + D * kPairRows) - safe);
      sum = fmaf(__ldcg(s + (D + 1) * kPairRows), f, sum);
#pragma unroll
      for (int k = 0; k < 16; ++k) acc[k] = fmaf(__ldcg(s + (c0 + k) * kPairRows), f, acc[k]);
    }
    if (r0 + lane >= it.rows) continue;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int row = it.row0 + r0 + lane, token = row / p.group;
    uint16_t* dst = p.out + (it.q0 + (int64_t)token) * p.out_stride + (int64_t)(it.h * p.group + row - token * p.group) * D + c0;
#pragma unroll
    for (int k = 0; k < 16; k += 8) {
      uint32_t w[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // channels 0, 4, 1, 5, 2, 6, 3, 7 of eight
        const int y = k + (x & 1) * 4 + (x >> 1);
        w[x] = pack_bf16(acc[y] * inv, acc[y + 2] * inv);
      }
      *reinterpret_cast<uint4*>(dst + k) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

template <int D, bool kExpire = false>
sp_status launch(const AttendParams& p, int sms, cudaStream_t stream) {
  static std::atomic<int> set[kMaxDevices] = {};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
    cudaGetLastError();
    return SP_ERR_CUDA;
  }
  const int ok = kept_or_looked_up(set[dev], [] {
    if (cudaFuncSetAttribute(attend_rows_kernel<D, kExpire>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)Smem<D>::kTotal) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    return 1;
  });
  if (!ok) return SP_ERR_CUDA;
  const sp_status st = launch_pdl(attend_rows_kernel<D, kExpire>, dim3((unsigned)sms), kThreads, Smem<D>::kTotal, 1, stream, p);
  if (st != SP_OK || p.split == 1) return st;
  return launch_pdl(join_rows_kernel<D>, dim3((unsigned)sms * 4), 128, 0, 1, stream, p);
}

}  // namespace

size_t attend_rows_part_bytes(int head_dim, int sms) {
  return (size_t)sms * kPairRows * (size_t)(head_dim + 2) * sizeof(float);
}

// Where there are fewer items than SMs, the steps of keys are cut into shares.  The host does not
// see the lengths: it goes by the most items that so many tokens can make (R requests of kManyRows
// rows or more have sum ceil(rows / 256) <= (all rows + 255 R) / 256).
sp_status launch_attend_rows(AttendParams p, int head_dim, bool expire, cudaStream_t stream) {
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  const int64_t rows = p.tokens * p.group, most = std::min<int64_t>(p.requests, rows / kManyRows);
  const int64_t items = (rows + (kPairRows - 1) * most) / kPairRows * p.cache.heads;
  p.parts = sms;
  p.split = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kMostShares, sms / std::max<int64_t>(items, 1)));
  if (expire) return launch<64, true>(p, sms, stream);
  return head_dim == 64 ? launch<64>(p, sms, stream) : launch<128>(p, sms, stream);
}

}  // namespace sp
