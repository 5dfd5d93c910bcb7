// sp_attend.cu -- attention over the cache held in 4 bits (include/sp_serve.h): single tokens and
// short runs of tokens of many requests.
//
// Mathematics.  With codes n, scale s and minimum m per key, and c = scale * log2(e):
//     log2 score   x_k = c s_k (q . n) + c m_k sum(q)
//     out          = (sum_k (e_k s_k) n + sum_k e_k m_k) / sum_k e_k,    e_k = 2^(x_k - M)
// so both products run on the codes.  A code's four bits, wherever they lie in the low byte of a
// 16-bit half, are an fp16 subnormal, n 2^-24 or n 2^-20, which the tensor cores multiply exactly:
// one AND per two codes is all the expansion there is.  The queries enter as fp16 too: each row is
// scaled by the power of two that brings its own largest entry to 2^14 ... 2^15, half of its channels
// by 1/16 of that, which is exact (bf16 has fewer bits) but for entries below 2^-27 of the largest; those
// round to 2^-35 of it, far below the fp32 sums' own rounding.  The weights e_k s_k of the values are
// rounded to fp16; M is a running maximum of x_k + log2(s_k), so that they stay below 2^8 and their large
// ones keep 11 bits whatever the scales are.  M moves only when a weight would pass 2^8, so most steps
// rescale nothing.
//
// Layout.  A warp takes units of 32 keys.  Both products have the codes as the wide operand of
// m16n8k16 (keys, then channels, along M) and up to 8 NT query rows -- the heads that share the key
// head, times the new tokens -- along N.  The channels of a key, and the keys of a channel, may be
// taken in any order in a sum, so a lane's operand is 16 consecutive bytes of a key, or 8 of four
// keys.  The scores' transposition between the products is movmatrix.  Each warp copies its own units
// into a ring in shared memory (bulk copies: a unit's keys, values and parameters are contiguous).
//
// Split.  The units of all requests, key heads and row tiles form one list, cut into equal ranges,
// first among CTAs (one per SM), then among their warps, whatever the lengths of the requests are.  A
// warp finishes the segments (units of one request, head and row tile) that it holds whole; of the
// others it leaves sums and maxima in shared memory, which the CTA joins at its end, and where a
// segment spans CTAs the last of them joins their parts from the workspace, in order.
//
// Measured (GPU time of one call among others).  One request behind 4096 tokens, 32 key heads of 128 (17.9 MB):
// 12.5 us.  64 requests of 100 to 16384 tokens, 8 key heads of 128 with four query heads each (207 MB): 49.9 us,
// 4.2 TB/s over the whole, 5.7 while it streams.  16 requests of 500 to 6000 tokens with five new ones, 8 key
// heads of 64 with four each (21 MB): 22.9 us.  Bound by what lies around the stream: 4 us to the first
// copies (lengths, table and pages are loads that wait for one another), 2 to 3 to the first unit, 4 to 8 for the
// last units and the joins; with many rows a unit (24: 840 instructions, some 80 % of the issue slots) the products
// and softmax take longer than its bytes.
#include <algorithm>
#include <climits>

#include "sp_attend.cuh"
#include "sp_lookup.h"

namespace sp {
namespace {

constexpr int kMaxDevices = 64;
constexpr int kMinUnits = 8;  // units of a CTA, before more CTAs share the work

// Warps of a CTA, stages of a warp's ring and place of its query operands, for NT tiles of eight query
// rows: what the registers and shared memory of an SM hold.
constexpr int warps_of(int d, int nt) { return nt == 1 || d == 64 ? 12 : nt < 4 ? 8 : 6; }
constexpr int stages_of(int d, int nt) {
  return d == 64 ? (nt == 4 ? 2 : nt == 3 ? 3 : 4) : nt == 1 || nt == 4 ? 3 : nt == 2 ? 4 : 2;
}
constexpr bool queries_shared(int d, int nt) { return nt > 2; }

__device__ __forceinline__ float lg2(float x) {
  float r;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// fp16 pairs of the nibbles i and i + 4 of w: n 2^-24 for i = 0 (and 2, of w >> 8), n 2^-20 for i = 1 (3)
__device__ __forceinline__ uint32_t nib_lo(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t nib_hi(uint32_t w) { return w & 0x00f000f0u; }
constexpr float kLo = 16777216.f, kHi = 1048576.f;

template <int W>
__device__ __forceinline__ void load_words(uint32_t (&d)[W], const uint8_t* p) {
  if constexpr (W == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    d[0] = u.x, d[1] = u.y, d[2] = u.z, d[3] = u.w;
  } else if constexpr (W == 2) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    d[0] = u.x, d[1] = u.y;
  } else {
    d[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// The list of units in equal ranges: part i of n takes [begin(i), begin(i + 1)).
struct Ranges {
  int each, more;  // the first `more` parts take one unit more
  __device__ __forceinline__ Ranges(int units, int n) : each(units / n), more(units % n) {}
  __device__ __forceinline__ int begin(int i) const { return i * each + min(i, more); }
  __device__ __forceinline__ int owner(int u) const {
    const int cut = more * (each + 1);
    return u < cut ? u / (each + 1) : more + (u - cut) / each;
  }
};

// A segment: the units of one request, key head and row tile.
struct Segment {
  int vis0;         // its first unit's place in the list
  int seen;         // its units that any of its rows sees
  int h;            // key head
  int q0, head0;    // row of q and head, among the group's, of its first query row
  int rows;         // query rows
  int sees;         // keys that its first row sees
};

// What a stage of a ring holds.
struct Meta {
  int u, ok, opens;  // the unit, its halves that have a page, whether a segment begins
  Segment s;         // that segment
};

// What a warp leaves in shared memory of a segment that it does not hold whole.
struct PartInfo {
  int vis0, seen, rows;  // rows == 0: nothing
  int h, q0, head0;
};

// One row of n parts, by L lanes: its maximum and sum of weights (in each of them), and of its sums the
// quadruples that begin at 4 (lane % L + L i).  A warp joins 32 / L rows side by side: a row's joining is a
// chain of waits whatever its lanes, so many rows take eight lanes each (20 rows of 5 tokens over 4 heads of
// D = 128, 16 requests: 23.9 us, by whole warps 25.8) and few rows, at most one a warp, as many as a row
// has quadruples (one request: 12.55 us, by half warps 13.2).
template <int Q>
struct Row {
  float m, sum;
  float4 acc[Q];
};
template <int Q, int L, class Stat, class Sums>
__device__ __forceinline__ Row<Q> join(int n, Stat stat_at, Sums sums_at) {
  constexpr int B = L == 8 ? 4 : 8;  // parts whose loads are in flight at a time
  const int lane = threadIdx.x & 31, sub = lane & (L - 1);
  Row<Q> r;
  // the first L parts' numbers stay in registers
  const float2 own = sub < n ? stat_at(sub) : make_float2(-INFINITY, 0.f);
  r.m = own.x;
  for (int k = sub + L; k < n; k += L) r.m = fmaxf(r.m, stat_at(k).x);
#pragma unroll
  for (int d = L / 2; d > 0; d >>= 1) r.m = fmaxf(r.m, __shfl_xor_sync(0xffffffffu, r.m, d));
  const float safe = r.m == -INFINITY ? 0.f : r.m;
  r.sum = 0.f;
#pragma unroll
  for (int i = 0; i < Q; ++i) r.acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int most = __reduce_max_sync(0xffffffffu, n);  // (the warp's rows may belong to two segments)
  for (int k0 = 0; k0 < most; k0 += L) {
    float f = 0.f;
    if (k0 + sub < n) {
      const float2 st = k0 == 0 ? own : stat_at(k0 + sub);
      f = ex2(st.x - safe);
      r.sum = fmaf(st.y, f, r.sum);
    }
    const int kn = min(L, most - k0);
    for (int k = 0; k < kn; k += B) {
      float4 a[B][Q];
#pragma unroll
      for (int j = 0; j < B; ++j)
#pragma unroll
        for (int i = 0; i < Q; ++i)
          if (k0 + k + j < n) a[j][i] = sums_at(k0 + k + j, 4 * (sub + L * i));
#pragma unroll
      for (int j = 0; j < B; ++j) {
        const float fk = __shfl_sync(0xffffffffu, f, (lane & (32 - L)) + ((k + j) & (L - 1)));
        if (k0 + k + j < n) {
#pragma unroll
          for (int i = 0; i < Q; ++i) {
            r.acc[i].x = fmaf(a[j][i].x, fk, r.acc[i].x), r.acc[i].y = fmaf(a[j][i].y, fk, r.acc[i].y);
            r.acc[i].z = fmaf(a[j][i].z, fk, r.acc[i].z), r.acc[i].w = fmaf(a[j][i].w, fk, r.acc[i].w);
          }
        }
      }
    }
  }
#pragma unroll
  for (int d = L / 2; d > 0; d >>= 1) r.sum += __shfl_xor_sync(0xffffffffu, r.sum, d);
  return r;
}

// kExpire: a variant for sp_test_expired_attend, whose warp p.expire_warp of CTA p.expire_cta first waits for
// what never comes and gives up.
template <int D, int NT, bool kExpire = false>
__global__ void __launch_bounds__(32 * warps_of(D, NT), 1) attend_kernel(const __grid_constant__ AttendParams p) {
  constexpr int KW = D / 32, VW = D / 64;  // words of a lane: keys, values
  constexpr int MT = D / 16;               // channel tiles
  constexpr int R = 8 * NT;                // query rows
  constexpr int W = warps_of(D, NT), S = stages_of(D, NT);
  constexpr bool kQShared = queries_shared(D, NT);
  constexpr int kCodes = kUnitKeys * D / 2;
  constexpr int kStage = 2 * kCodes + 2 * kUnitKeys * 4;
  constexpr int kRow = D + 4;              // floats of a row of a part: sums, maximum, weights
  constexpr int kPartBytes = R * kRow * 4;
  constexpr int kQBytes = kQShared ? 32 * NT * KW * 16 : 0;  // query operands of a warp
  static_assert(S * kStage + kQBytes >= kPartBytes, "a warp's last part takes the place of its ring");
  constexpr int kFirst = S * kStage + kQBytes, kWarpBytes = kFirst + kPartBytes;
  extern __shared__ __align__(128) uint8_t smem[];  // [W] of (ring, query operands, first part)
  __shared__ uint64_t s_bar[W][S];
  __shared__ Meta s_meta[W][S];
  __shared__ PartInfo s_info[W][2];
  __shared__ __align__(8) float s_back[W][R];  // c / the scaling of each query row, where registers are short
  __shared__ int s_last[2], s_order[2 * W], s_row0[2 * W], s_parts, s_rows;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int kg = g ^ ((g >> 1) & 1);  // key of operand row g: neighbours in different halves of the banks
  uint8_t* ring = smem + warp * kWarpBytes;
  uint4* q_shared = reinterpret_cast<uint4*>(ring + S * kStage) + lane;
  uint64_t* bar = s_bar[warp];
  if (lane == 0) {
    for (int i = 0; i < S; ++i) mbar_init(&bar[i], 1);
    fence_barrier_init();
    s_info[warp][0].rows = s_info[warp][1].rows = 0;
  }
  __syncwarp();
  pdl_wait();

  // 32 requests from wb on, one per lane: where their units end, lengths, rows of q
  int wb = 0, w_end, w_len, w_q0, w_q1, w_base;
  auto window = [&] {
    const int b = wb + lane;
    w_base = p.work[wb];
    w_end = b < p.requests ? p.work[b + 1] : INT_MAX;
    w_len = b < p.requests ? p.lens[b] : 0;
    w_q0 = b < p.requests ? p.cu_q[b] : 0;
    w_q1 = b < p.requests ? p.cu_q[b + 1] : 0;
  };
  // the loads that do not need the list's length go out with the one that gives it
  const int step0 = (p.requests + 31) / 32;
  int probe = 0;
  if (p.requests > 32) probe = p.work[min(p.requests, (lane + 1) * step0)];
  else window();
  const int heads = p.cache.heads;
  const int64_t all = (int64_t)p.work[p.requests] * heads;
  int others = 0;  // requests of more new tokens than the call was told of: loaded here, looked at at the end
  if (p.alone && blockIdx.x == 0 && tid == 0)
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(others) : "l"(p.work + 2 * p.requests + 1));
  const int total = (int)min(all, (int64_t)INT_MAX);
  if (total != all && tid == 0) set_status(p.status, kStatusBadIndex);
  const int ctas = max(1, min((int)gridDim.x, total / kMinUnits));
  if (blockIdx.x >= ctas) return;
  const Ranges by_cta(total, ctas);
  const int c0 = by_cta.begin(blockIdx.x), c1 = by_cta.begin(blockIdx.x + 1);
  const Ranges by_warp(c1 - c0, W);
  const int w0 = c0 + by_warp.begin(warp), w1 = c0 + by_warp.begin(warp + 1);
  const int shift = p.cache.shift;
  const int64_t block = kv4_block_bytes<D>(shift);
  // the token of query row x, counted from the head 0 of a token (x < 2^7, so the quotient is exact)
  auto token_of = [&](int x) { return x * p.group_inverse >> 16; };
  // row r of a segment in q or out
  auto q_row = [&](int q0, int h, int head0, int r, auto* base, int64_t stride) {
    const int token = token_of(head0 + r);
    return base + (int64_t)(q0 + token) * stride + (int64_t)(h * p.group + head0 + r - token * p.group) * D;
  };

  if (w0 < w1) {
    // ---------------------------------------------------------------- the copies
    if (p.requests > 32) {
      // a window that holds the first unit's request: 32 shares at a time
      int lo = 0, n = p.requests;
      const int first = w0 / heads;
      for (int step = step0;;) {
        const unsigned past = __ballot_sync(0xffffffffu, probe > first);
        const int k = past ? __ffs(past) - 1 : 31;
        n = min(step, n - min(n, k * step));
        lo += k * step;
        if (n <= 32) break;
        step = (n + 31) / 32;
        probe = p.work[lo + min(n, (lane + 1) * step)];
      }
      wb = max(0, min(lo, p.requests - 1));
      window();
    }
    Segment ps = {};
    int pw = w0, p_end = w0, pu = 0;         // the next unit; where its segment ends; its place there
    int p_b = 0, p_len = 0;                  // its request, that one's tokens
    int pg_from = 0, page[2] = {-1, -1};       // pages of 32 units, one per lane, from pg_from on
    bool opens = false;
    int pstage = 0, pending = 0;
    // the segment that holds unit pw; a share that does not belong to the lengths is passed over
    auto find = [&] {
      unsigned past;
      while (!(past = __ballot_sync(0xffffffffu, (int64_t)w_end * heads > pw))) {
        wb += 32;
        window();
      }
      const int k = __ffs(past) - 1;
      const int end = __shfl_sync(0xffffffffu, w_end, k);
      const int before = __shfl_sync(0xffffffffu, w_end, max(k - 1, 0));
      const int begin = (k == 0 ? w_base : before) * heads;
      p_len = __shfl_sync(0xffffffffu, w_len, k);
      const int q0 = __shfl_sync(0xffffffffu, w_q0, k), fresh = __shfl_sync(0xffffffffu, w_q1, k) - q0;
      p_b = wb + k;
      const int units = (p_len + kUnitKeys - 1) / kUnitKeys + kSetupUnits;
      const int tiles = (int)(((int64_t)fresh * p.group + kRowTile - 1) / kRowTile);
      opens = true;
      if (p_b >= p.requests || pw < begin || tiles <= 0 || p_len < fresh || fresh > p.max_new || q0 < 0 ||
          q0 + (int64_t)fresh > p.tokens || (int64_t)tiles * units != (int64_t)end - begin / heads) {
        if (lane == 0) set_status(p.status, kStatusBadIndex);
        p_end = p_b >= p.requests ? w1 : (int)min((int64_t)w1, (int64_t)end * heads);
        pu = ps.seen = 0;
        return;
      }
      const int idx = (pw - begin) / units;  // (row tile, key head)
      const int at = begin + idx * units;
      const int tile = idx / heads, row0 = tile * kRowTile, token = row0 / p.group;
      ps.h = idx - tile * heads;
      ps.q0 = q0 + token;
      ps.head0 = row0 - token * p.group;
      ps.rows = min(min(fresh * p.group - row0, kRowTile), R);
      ps.sees = p_len - fresh + token + 1;
      ps.seen = (ps.sees + token_of(ps.head0 + ps.rows - 1) + kUnitKeys - 1) / kUnitKeys;
      ps.vis0 = at + kSetupUnits;
      p_end = at + units;
      pu = max(0, pw - ps.vis0);
      pw = max(pw, ps.vis0);
      // its queries, on their way while its pages are looked up
      for (int i = lane; i < ps.rows * (D / 64); i += 32) {
        const uint16_t* q = q_row(ps.q0, ps.h, ps.head0, i / (D / 64), p.q, p.q_stride) + i % (D / 64) * 64;
        asm volatile("prefetch.global.L1 [%0];" ::"l"(q));
      }
    };
    // copies the next unit of the range that any row sees (or only says which it is); nothing where there is none
    auto issue = [&](bool copies) {
      while (pu >= ps.seen || pw >= p_end) {
        pw = max(pw, p_end);
        if (pw >= w1) return;
        find();
      }
      if (pw >= w1) return;
      if (opens || pu >= pg_from + 32) {
        pg_from = pu;
        const int32_t* row = p.table + (int64_t)p_b * p.width;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int64_t k0 = (int64_t)(pu + lane) * kUnitKeys + 16 * i;
          const int at = (int)(k0 >> shift);
          page[i] = -1;
          if (k0 < p_len) {
            if (at < p.width) page[i] = row[at];
            if (page[i] < 0 || page[i] >= p.cache.pages) {
              page[i] = -1;
              set_status(p.status, kStatusBadIndex);
            }
          }
        }
      }
      const int pg0 = __shfl_sync(0xffffffffu, page[0], pu - pg_from), pg1 = __shfl_sync(0xffffffffu, page[1], pu - pg_from);
      if (lane == 0) {
        uint8_t* dst = ring + pstage * kStage;
        uint64_t* full = &bar[pstage];
        const uint8_t* b0 = p.cache.data + ((int64_t)pg0 * heads + ps.h) * block;
        Meta& m = s_meta[warp][pstage];
        m.u = pu;
        m.ok = shift >= 5 ? (pg0 >= 0 ? 3 : 0) : (pg0 >= 0 ? 1 : 0) | (pg1 >= 0 ? 2 : 0);
        m.opens = opens;
        if (opens) m.s = ps;
        if (copies && shift >= 5) {  // the unit lies in one page
          if (pg0 >= 0) {
            const int in = (pu * kUnitKeys) & ((1 << shift) - 1);
            mbar_arrive_expect_tx(full, kStage);
            bulk_g2s(dst, b0 + in * (D / 2), kCodes, full);
            bulk_g2s(dst + kCodes, b0 + kv4_value_codes<D>(shift) + in * (D / 2), kCodes, full);
            bulk_g2s(dst + 2 * kCodes, b0 + kv4_key_params<D>(shift) + in * 4, kUnitKeys * 4, full);
            bulk_g2s(dst + 2 * kCodes + kUnitKeys * 4, b0 + kv4_value_params<D>(shift) + in * 4, kUnitKeys * 4, full);
          } else {
            mbar_arrive(full);
          }
        } else if (copies) {
          const uint8_t* b1 = p.cache.data + ((int64_t)pg1 * heads + ps.h) * block;
          mbar_arrive_expect_tx(full, (pg0 >= 0 ? kStage / 2 : 0) + (pg1 >= 0 ? kStage / 2 : 0));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if ((i ? pg1 : pg0) < 0) continue;
            const uint8_t* bl = i ? b1 : b0;
            bulk_g2s(dst + i * (kCodes / 2), bl, kCodes / 2, full);
            bulk_g2s(dst + kCodes + i * (kCodes / 2), bl + kv4_value_codes<D>(shift), kCodes / 2, full);
            bulk_g2s(dst + 2 * kCodes + i * 64, bl + kv4_key_params<D>(shift), 64, full);
            bulk_g2s(dst + 2 * kCodes + kUnitKeys * 4 + i * 64, bl + kv4_value_params<D>(shift), 64, full);
          }
        }
      }
      opens = false;
      if (++pstage == S) pstage = 0;
      ++pu;
      ++pw;
      ++pending;
    };
#pragma unroll 1
    for (int i = 0; i < S; ++i) issue(true);
    __syncwarp();

    // ---------------------------------------------------------------- the segments of the range
    // the copies on their way, from stage i on, have landed
    auto drain = [&](int i, uint32_t parity) {
      for (int k = 0; k < pending; ++k) {
        mbar_wait_sleep(&bar[i], parity, p.timeout_ns);
        if (++i == S) i = 0, parity ^= 1u;
      }
    };
    int stage = 0;
    uint32_t phase = 0;
    bool dead = false;
    if constexpr (kExpire) {
      __shared__ uint64_t s_probe;
      if (blockIdx.x == p.expire_cta && warp == p.expire_warp) {
        if (lane == 0) {
          mbar_init(&s_probe, 1);
          fence_barrier_init();
        }
        __syncwarp();
        dead = !__all_sync(0xffffffffu, mbar_wait_sleep(&s_probe, 0, p.timeout_ns));
        if (dead && lane == 0) set_status(p.status, kStatusTimeout);
        if (dead) drain(0, 0);
      }
    }
    while (pending > 0) {
      const Segment s = s_meta[warp][stage].s;
      int u = s_meta[warp][stage].u;
      const int u0 = u;
      // queries: fp16 operand registers, and sums over the channels
      uint32_t qf[kQShared ? 1 : NT][KW][4];
      uint64_t qsum[NT];  // of query rows 2t, 2t + 1: c sum(q)
      uint64_t rs;        // of the same, where NT is 1: c / the row's scaling
      int limit[NT][2];   // keys that they see
      {
        auto load = [&](int nt, uint4(&x)[KW]) {
          const uint16_t* src = q_row(s.q0, s.h, s.head0, nt * 8 + g, p.q, p.q_stride) + t * (D / 4);
#pragma unroll
          for (int i = 0; i < KW; ++i) {
            x[i] = make_uint4(0, 0, 0, 0);
            if (nt * 8 + g < s.rows) x[i] = *(reinterpret_cast<const uint4*>(src) + i);
          }
        };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint4 x4[KW];
          load(nt, x4);
          // each row by its own power of two, so that no other row takes bits from it
          uint32_t big = 0;  // the row's largest magnitude, as bf16 bits
#pragma unroll
          for (int i = 0; i < KW; ++i) {
            const uint32_t x[4] = {x4[i].x, x4[i].y, x4[i].z, x4[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) big = max(big, max(x[j] & 0x7fffu, (x[j] >> 16) & 0x7fffu));
          }
          big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
          big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
          // 2^(141 - e): the largest entry, of biased exponent e, comes to 2^14 ... 2^15
          const uint32_t e = max(15u, min(254u, big >> 7));
          const float f = __uint_as_float((268u - e) << 23);
          const float back = __uint_as_float((e - 14u) << 23) * p.scale_log2;
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < KW; ++i) {
            const uint32_t x[4] = {x4[i].x, x4[i].y, x4[i].z, x4[i].w};
            float y[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              y[2 * j] = __uint_as_float(x[j] << 16);
              y[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u);
              sum += y[2 * j] + y[2 * j + 1];
            }
            const float f2 = f * 0.0625f;
            const uint4 v = make_uint4(pack_f16(y[0] * f, y[4] * f), pack_f16(y[1] * f2, y[5] * f2),
                                       pack_f16(y[2] * f, y[6] * f), pack_f16(y[3] * f2, y[7] * f2));
            if constexpr (kQShared) {
              q_shared[(i * NT + nt) * 32] = v;  // (read by the lane that writes it)
            } else {
              qf[nt][i][0] = v.x, qf[nt][i][1] = v.y, qf[nt][i][2] = v.z, qf[nt][i][3] = v.w;
            }
          }
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
          sum *= p.scale_log2;
          qsum[nt] = two(__shfl_sync(0xffffffffu, sum, 8 * t), __shfl_sync(0xffffffffu, sum, 8 * t + 4));
          if (NT == 1) rs = two(__shfl_sync(0xffffffffu, back, 8 * t), __shfl_sync(0xffffffffu, back, 8 * t + 4));
          else if (t == 0) s_back[warp][nt * 8 + g] = back;
#pragma unroll
          for (int c = 0; c < 2; ++c) limit[nt][c] = s.sees + token_of(s.head0 + nt * 8 + 2 * t + c);
        }
      }
      if (NT > 1) __syncwarp();  // (s_back)
      float o[NT][MT][4];
      float mx[NT][2];
      uint64_t l[NT], off[NT];  // sums of the weights, and of the weights times the values' minima
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
#pragma unroll
        for (int c = 0; c < 2; ++c) mx[nt][c] = -INFINITY;
        l[nt] = off[nt] = 0;
      }

      for (; !dead; ++u) {
        if (!__all_sync(0xffffffffu, mbar_wait_sleep(&bar[stage], phase, p.timeout_ns))) {
          if (lane == 0) set_status(p.status, kStatusTimeout);
          dead = true;
          drain(stage, phase);
          break;
        }
        const uint8_t* st = ring + stage * kStage;
        const int ok = s_meta[warp][stage].ok;

        float x[NT][2][4];  // scores: [16 keys][key g row 2t, row 2t + 1, key g + 8 ...]
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t k0[KW], k1[KW];
          load_words<KW>(k0, st + (16 * i + kg) * (D / 2) + t * (D / 8));
          load_words<KW>(k1, st + (16 * i + 8 + kg) * (D / 2) + t * (D / 8));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) x[nt][i][0] = x[nt][i][1] = x[nt][i][2] = x[nt][i][3] = 0.f;
#pragma unroll
          for (int j = 0; j < KW; ++j) {
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
              const uint32_t y0 = hh ? k0[j] >> 8 : k0[j], y1 = hh ? k1[j] >> 8 : k1[j];
              const uint32_t a0 = nib_lo(y0), a1 = nib_lo(y1), a2 = nib_hi(y0), a3 = nib_hi(y1);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if constexpr (kQShared) {
                  const uint2 b = *(reinterpret_cast<const uint2*>(q_shared + (j * NT + nt) * 32) + hh);
                  mma_f16(x[nt][i], a0, a1, a2, a3, b.x, b.y);
                } else {
                  mma_f16(x[nt][i], a0, a1, a2, a3, qf[nt][j][2 * hh], qf[nt][j][2 * hh + 1]);
                }
              }
            }
          }
        }
        float ks[2][2], km[2][2], vs[2][2], vm[2][2], vl[2][2];
        const __half2* kp = reinterpret_cast<const __half2*>(st + 2 * kCodes);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 a = __half22float2(kp[16 * i + 8 * j + kg]);
            const float2 v = __half22float2(kp[kUnitKeys + 16 * i + 8 * j + kg]);
            ks[i][j] = a.x * kLo, km[i][j] = a.y;
            vs[i][j] = v.x, vm[i][j] = v.y;
            vl[i][j] = lg2(fmaxf(v.x, 1.f / kLo));
          }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          // (32 rows a tile: 240 us for 63 requests of a token behind 1000 to 8000, 267 with the factors in registers;
          // 8 rows: 73.9 and 72.4)
          if (NT > 1) rs = *reinterpret_cast<const uint64_t*>(&s_back[warp][nt * 8 + 2 * t]);
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float *y = &x[nt][i][2 * j], k2 = ks[i][j], m2 = km[i][j];
              // (the row's factor last: with the key's it could leave fp32's range)
              apart(fma2(mul2(two(y[0], y[1]), two(k2, k2)), rs, mul2(two(m2, m2), qsum[nt])), y[0], y[1]);
            }
        }
        const bool edge = (u + 1) * kUnitKeys > s.sees || ok != 3;  // some row does not see all of the unit
        if (edge) {
          const int key = u * kUnitKeys + kg;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (key + 16 * i + 8 * (j >> 1) >= limit[nt][j & 1] || !(ok >> i & 1)) x[nt][i][j] = -INFINITY;
        }
        uint32_t pt[NT][2][2];  // weights, transposed: query row g, keys 2t, 2t + 1 of eight
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float a, b;
              apart(add2(two(x[nt][i][2 * j], x[nt][i][2 * j + 1]), two(vl[i][j], vl[i][j])), a, b);
              top[0] = fmaxf(top[0], a), top[1] = fmaxf(top[1], b);
            }
          if (__any_sync(0xffffffffu, top[0] > mx[nt][0] + 8.f || top[1] > mx[nt][1] + 8.f)) {
            float alpha[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 4));
              top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 8));
              top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 16));
              top[c] = fmaxf(top[c], mx[nt][c]);
              alpha[c] = mx[nt][c] == -INFINITY ? 0.f : ex2(mx[nt][c] - top[c]);
              mx[nt][c] = top[c];
            }
            const uint64_t a2 = two(alpha[0], alpha[1]);
            l[nt] = mul2(l[nt], a2);
            off[nt] = mul2(off[nt], a2);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              apart(mul2(two(o[nt][i][0], o[nt][i][1]), a2), o[nt][i][0], o[nt][i][1]);
              apart(mul2(two(o[nt][i][2], o[nt][i][3]), a2), o[nt][i][2], o[nt][i][3]);
            }
          }
          const uint64_t m2 = two(mx[nt][0] == -INFINITY ? 0.f : -mx[nt][0], mx[nt][1] == -INFINITY ? 0.f : -mx[nt][1]);
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float a, b;
              apart(add2(two(x[nt][i][2 * j], x[nt][i][2 * j + 1]), m2), a, b);
              const uint64_t e = two(ex2(a), ex2(b));
              l[nt] = add2(l[nt], e);
              uint64_t om = mul2(e, two(vm[i][j], vm[i][j])), os = mul2(e, two(vs[i][j], vs[i][j]));
              if (edge) {  // what a row does not see may hold anything, in its parameters too
                float m0, m1, s0, s1;
                apart(om, m0, m1);
                apart(os, s0, s1);
                if (a == -INFINITY) m0 = s0 = 0.f;
                if (b == -INFINITY) m1 = s1 = 0.f;
                om = two(m0, m1);
                os = two(s0, s1);
              }
              off[nt] = add2(off[nt], om);
              apart(os, a, b);
              pt[nt][i][j] = transpose8x8(pack_f16(a, b));
            }
        }
        const uint8_t* vc = st + kCodes + g * (D / 16);
        const int v0 = 2 * t ^ (t & 1), v1 = (2 * t + 1) ^ (t & 1);  // keys of operand columns 2t, 2t + 1
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t v[4][VW];
          load_words<VW>(v[0], vc + (16 * i + v0) * (D / 2));
          load_words<VW>(v[1], vc + (16 * i + v1) * (D / 2));
          load_words<VW>(v[2], vc + (16 * i + 8 + v0) * (D / 2));
          load_words<VW>(v[3], vc + (16 * i + 8 + v1) * (D / 2));
#pragma unroll
          for (int y = 0; y < VW; ++y) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t sel = half ? 0x7632u : 0x5410u;
              const uint32_t w01 = __byte_perm(v[0][y], v[1][y], sel), w23 = __byte_perm(v[2][y], v[3][y], sel);
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                const uint32_t y01 = z ? w01 >> 8 : w01, y23 = z ? w23 >> 8 : w23;
                const uint32_t a0 = nib_lo(y01), a1 = nib_hi(y01), a2 = nib_lo(y23), a3 = nib_hi(y23);
                const int mt = 4 * y + 2 * half + z;  // channels D/8 g + 2 mt (rows g), + 1 (rows g + 8)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][mt], a0, a1, a2, a3, pt[nt][i][0], pt[nt][i][1]);
              }
            }
          }
        }
        __syncwarp();  // the stage has been read
        --pending;
        issue(true);
        __syncwarp();
        if (++stage == S) {
          stage = 0;
          phase ^= 1u;
        }
        if (pending == 0 || s_meta[warp][stage].opens) break;
      }

      // A warp that gave up goes on through its range without copies and sums: the CTAs that share a segment
      // count one another, on a counter that the next call finds as this one leaves it.
      if (dead) {
        for (;; ++u) {
          --pending;
          issue(false);
          __syncwarp();
          if (++stage == S) stage = 0;
          if (pending == 0 || s_meta[warp][stage].opens) break;
        }
      }

      // the segment's sums: to `out` if the warp held all of it, else to shared memory
      const bool first = u0 > 0, last = u < s.seen - 1;
      if (!dead || first || last) {
        float* dst = reinterpret_cast<float*>(last ? ring : ring + kFirst);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) {
            l[nt] = add2(l[nt], __shfl_xor_sync(0xffffffffu, l[nt], d));
            off[nt] = add2(off[nt], __shfl_xor_sync(0xffffffffu, off[nt], d));
          }
          float ls[2], as[2];
          apart(l[nt], ls[0], ls[1]);
          apart(off[nt], as[0], as[1]);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int r = nt * 8 + 2 * t + c;
            if (r >= s.rows) continue;
            if (!first && !last) {
              const float inv = ls[c] == 0.f ? 0.f : 1.f / ls[c];
              uint16_t* y = q_row(s.q0, s.h, s.head0, r, p.out, p.out_stride) + g * (D / 8);
#pragma unroll
              for (int mt = 0; mt < MT; mt += 4) {
                uint32_t v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  v[i] = pack_bf16(fmaf(o[nt][mt + i][c], kLo, as[c]) * inv, fmaf(o[nt][mt + i][2 + c], kHi, as[c]) * inv);
                *reinterpret_cast<uint4*>(y + 2 * mt) = make_uint4(v[0], v[1], v[2], v[3]);
              }
            } else {
              float* y = dst + r * kRow + g * (D / 8);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
                *reinterpret_cast<float2*>(y + 2 * mt) =
                    make_float2(fmaf(o[nt][mt][c], kLo, as[c]), fmaf(o[nt][mt][2 + c], kHi, as[c]));
              if (g == 0) *reinterpret_cast<float2*>(dst + r * kRow + D) = make_float2(mx[nt][c], ls[c]);
            }
          }
        }
        if ((first || last) && lane == 0) s_info[warp][last ? 1 : 0] = PartInfo{s.vis0, s.seen, s.rows, s.h, s.q0, s.head0};
      }
    }
  }

  if (others != 0) set_status(p.status, kStatusBadIndex);

  // ------------------------------------------------------------------ segments shared by warps
  __syncthreads();
  if (warp == 0) {  // the parts in order, and the rows of the segments that begin among them
    const PartInfo mine = lane < 2 * W ? s_info[lane >> 1][lane & 1] : PartInfo{};
    const unsigned m = __ballot_sync(0xffffffffu, mine.rows > 0), below = m & ((1u << lane) - 1u);
    const int prev = __shfl_sync(0xffffffffu, mine.vis0, below ? 31 - __clz(below) : 0);
    const bool opens = mine.rows > 0 && (below == 0 || prev != mine.vis0);
    int rows = opens ? mine.rows : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, rows, d);
      if (lane >= d) rows += x;
    }
    if (mine.rows > 0) {
      const int at = __popc(below);
      s_order[at] = lane;
      s_row0[at] = opens ? rows - mine.rows : -1;
    }
    if (lane == 31) s_parts = __popc(m), s_rows = rows;
  }
  __syncthreads();
  constexpr int L = NT == 1 ? D / 4 : 8;  // lanes of a row
  constexpr int Q = D / 4 / L;            // quadruples of a lane
  constexpr int A = 32 / L;               // rows of a warp
  const int sub = lane & (L - 1), side = lane / L;
  auto write_out = [&](const PartInfo& s, int r, const Row<Q>& x) {
    const float inv = x.sum == 0.f ? 0.f : 1.f / x.sum;
    uint16_t* dst = q_row(s.q0, s.h, s.head0, r, p.out, p.out_stride) + 4 * sub;
#pragma unroll
    for (int i = 0; i < Q; ++i)
      *reinterpret_cast<uint2*>(dst + 4 * L * i) = make_uint2(pack_bf16(x.acc[i].x * inv, x.acc[i].y * inv),
                                                           pack_bf16(x.acc[i].z * inv, x.acc[i].w * inv));
  };
  const int parts = s_parts;
  int open[2] = {-1, -1};  // a part of the segment shared with the CTAs before, after
  if (parts > 0) {
    const int i = s_order[0], j = s_order[parts - 1];
    const PartInfo a = s_info[i >> 1][i & 1], b = s_info[j >> 1][j & 1];
    if (a.vis0 < c0) open[0] = i;
    if (b.vis0 >= c0 && b.vis0 + b.seen > c1) open[1] = j;
  }
  const int own0 = lane < parts ? s_row0[lane] : -1;
  const unsigned opening = __ballot_sync(0xffffffffu, own0 >= 0);
  for (int x0 = A * warp; x0 < s_rows; x0 += A * W) {
    const int x = min(x0 + side, s_rows - 1);  // (a lane past the last row repeats it)
    unsigned m = 0;                            // the parts whose segment opens at or before x
#pragma unroll
    for (int k = 0; k < A; ++k) {
      const unsigned o = __ballot_sync(0xffffffffu, own0 >= 0 && own0 <= x0 + k);
      if (k == side) m = o;
    }
    const int i = 31 - __clz(m);  // the segment's first part
    const unsigned after = opening & ~((2u << i) - 1u);
    const int n = (after ? __ffs(after) - 1 : parts) - i;
    const int r = x - __shfl_sync(0xffffffffu, own0, i);
    const PartInfo s = s_info[s_order[i] >> 1][s_order[i] & 1];
    auto at = [&](int k) {
      const int o = s_order[i + k];
      return reinterpret_cast<const float*>(smem + (o >> 1) * kWarpBytes + ((o & 1) ? 0 : kFirst)) + r * kRow;
    };
    const Row<Q> y = join<Q, L>(
        n, [&](int k) { return *reinterpret_cast<const float2*>(at(k) + D); },
        [&](int k, int c) { return *reinterpret_cast<const float4*>(at(k) + c); });
    if (x0 + side >= s_rows) continue;
    if (s.vis0 >= c0 && s.vis0 + s.seen <= c1) {
      write_out(s, r, y);
    } else {
      float* part = p.part + (((int64_t)blockIdx.x * 2 + (s.vis0 < c0 ? 0 : 1)) * R + r) * kRow;
#pragma unroll
      for (int c = 0; c < Q; ++c) __stcg(reinterpret_cast<float4*>(part + 4 * (sub + L * c)), y.acc[c]);
      if (sub == 0) __stcg(reinterpret_cast<float2*>(part + D), make_float2(y.m, y.sum));
    }
  }
  // ------------------------------------------------------------------ segments shared by CTAs
  if (open[0] < 0 && open[1] < 0) return;
  __threadfence();
  __syncthreads();
  auto ctas_of = [&](int which, int& f, int& e) {
    const PartInfo s = s_info[open[which] >> 1][open[which] & 1];
    f = by_cta.owner(s.vis0);
    e = by_cta.owner(s.vis0 + s.seen - 1);
  };
  if (tid < 2) {
    s_last[tid] = 0;
    if ((tid == 0 ? open[0] : open[1]) >= 0) {
      int f, e;
      ctas_of(tid, f, e);
      s_last[tid] = atomicAdd(&p.cnt[f], 1) == e - f ? 1 : 0;
    }
  }
  __syncthreads();
  if (!s_last[0] && !s_last[1]) return;
  __threadfence();
  PartInfo s[2];
  int f[2], e[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    s[i].rows = 0;
    if (s_last[i]) {
      s[i] = s_info[open[i] >> 1][open[i] & 1];
      ctas_of(i, f[i], e[i]);
    }
  }
  const int all_rows = s[0].rows + s[1].rows;
  for (int x0 = A * warp; x0 < all_rows; x0 += A * W) {
    const int x = min(x0 + side, all_rows - 1);
    const int i = x < s[0].rows ? 0 : 1, r = x - (i ? s[0].rows : 0);
    const int first = i ? f[1] : f[0], n = (i ? e[1] : e[0]) - first + 1;
    // the segment is the first CTA's second part and the others' first
    auto at = [&](int k) { return p.part + (((int64_t)(first + k) * 2 + (k == 0 ? 1 : 0)) * R + r) * kRow; };
    const Row<Q> y = join<Q, L>(
        n, [&](int k) { return __ldcg(reinterpret_cast<const float2*>(at(k) + D)); },
        [&](int k, int c) { return __ldcg(reinterpret_cast<const float4*>(at(k) + c)); });
    if (x0 + side < all_rows) write_out(i ? s[1] : s[0], r, y);
  }
  if (tid < 2 && s_last[tid]) atomicExch(&p.cnt[tid ? f[1] : f[0]], 0);
}

template <int D, int NT>
constexpr size_t smem_bytes() {
  return (size_t)warps_of(D, NT) * (stages_of(D, NT) * (kUnitKeys * D + 2 * kUnitKeys * 4) +
                                    (queries_shared(D, NT) ? 32 * NT * (D / 32) * 16 : 0) + 8 * NT * (D + 4) * 4);
}

// CTAs of a full grid; 0 if a lookup failed.
template <int D, int NT, bool kExpire = false>
int grid_of() {
  static std::atomic<int> kept[kMaxDevices] = {};
  int dev = -1;
  const int sms = current_sms();
  if (sms == 0 || cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
    cudaGetLastError();
    return 0;
  }
  return kept_or_looked_up(kept[dev], [sms] {
    int n = 0;
    if (cudaFuncSetAttribute(attend_kernel<D, NT, kExpire>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)smem_bytes<D, NT>()) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, attend_kernel<D, NT, kExpire>, 32 * warps_of(D, NT),
                                                      smem_bytes<D, NT>()) !=
            cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    return n > 0 ? sms : 0;  // one CTA per SM
  });
}

size_t workspace_bytes(int head_dim, int sms) {
  return ws_counter_bytes(sms) + std::max((size_t)sms * 2 * kRowTile * (size_t)(head_dim + 4) * sizeof(float),
                                          attend_rows_part_bytes(head_dim, sms));
}

template <int D, int NT, bool kExpire = false>
sp_status launch(AttendParams p, cudaStream_t stream) {
  const int ctas = grid_of<D, NT, kExpire>();
  if (ctas == 0) return SP_ERR_CUDA;
  return launch_pdl(attend_kernel<D, NT, kExpire>, dim3((unsigned)ctas), 32 * warps_of(D, NT), smem_bytes<D, NT>(), 1, stream,
                    p);
}

}  // namespace
}  // namespace sp

using namespace sp;

namespace {

// What sp_test_expired_attend makes expire.
struct Expire {
  int32_t cta, warp;
  uint64_t wait_ns;
};

sp_status attend(const sp_attend_args* a, void* workspace_dev, size_t workspace_size, const Expire* expire, void* stream) {
  if (!a || !a->cache || !a->cache->data || !kv4_positive(a->cache) || a->cache->reserved != 0 || a->reserved != 0)
    return SP_ERR_INVALID_ARG;
  if (a->requests < 0 || a->width < 0 || a->tokens < 0 || a->max_new < 0 || !(a->scale - a->scale == 0.f))
    return SP_ERR_INVALID_ARG;
  const int kv = a->cache->kv_heads;
  if (a->heads < kv || a->heads % kv != 0) return SP_ERR_INVALID_ARG;
  if (!kv4_supported(a->cache) || a->heads / kv > kMaxGroup) return SP_ERR_UNSUPPORTED;
  if (a->requests == 0 || a->tokens == 0 || a->max_new == 0) return SP_OK;
  if (!a->q || !a->out || !a->table || !a->lens || !a->cu_q || !a->work) return SP_ERR_INVALID_ARG;
  const int64_t row = (int64_t)a->heads * a->cache->head_dim;
  if (a->q_stride < row || a->out_stride < row) return SP_ERR_INVALID_ARG;
  if (a->q_stride % 8 || a->out_stride % 8) return SP_ERR_UNSUPPORTED;
  if (!al16(a->q) || !al16(a->out) || !al16(a->cache->data) || !al16(workspace_dev)) return SP_ERR_ALIGNMENT;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  const int d = a->cache->head_dim;
  if (!workspace_dev || workspace_size < workspace_bytes(d, sms)) return SP_ERR_WORKSPACE;
  AttendParams p = {};
  p.q = static_cast<const uint16_t*>(a->q);
  p.out = static_cast<uint16_t*>(a->out);
  p.q_stride = a->q_stride;
  p.out_stride = a->out_stride;
  p.cache = kv4_view(a->cache);
  p.table = a->table;
  p.lens = a->lens;
  p.cu_q = a->cu_q;
  p.work = a->work;
  p.requests = a->requests;
  p.width = a->width;
  p.group = a->heads / kv;
  p.group_inverse = (65536 + p.group - 1) / p.group;
  p.max_new = a->max_new;
  p.tokens = a->tokens;
  p.scale_log2 = a->scale * 1.4426950408889634f;
  p.cnt = static_cast<int*>(workspace_dev);
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace_dev) + ws_counter_bytes(sms));
  p.status = device_status_ptr();
  p.timeout_ns = wait_timeout_ns();
  cudaStream_t s = (cudaStream_t)stream;
  const int64_t most = (int64_t)a->max_new * p.group;
  if (expire) {
    p.timeout_ns = expire->wait_ns;
    p.expire_cta = (uint32_t)expire->cta;
    p.expire_warp = expire->warp;
  }
  p.alone = most < kManyRows;
  if (expire) {
    if (d != 64 || (most > 8 && most <= 24)) return SP_ERR_UNSUPPORTED;
    if (p.alone) return most <= 8 ? launch<64, 1, true>(p, s) : launch<64, 4, true>(p, s);
  }
  if (!p.alone) {
    const sp_status st = launch_attend_rows(p, d, expire != nullptr, s);
    if (st != SP_OK) return st;
  }
  const int64_t rows = std::min<int64_t>(most, kRowTile);
  const int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : rows <= 24 ? 3 : 4;
  switch (nt) {
    case 1: return d == 64 ? launch<64, 1>(p, s) : launch<128, 1>(p, s);
    case 2: return d == 64 ? launch<64, 2>(p, s) : launch<128, 2>(p, s);
    case 3: return d == 64 ? launch<64, 3>(p, s) : launch<128, 3>(p, s);
  }
  return d == 64 ? launch<64, 4>(p, s) : launch<128, 4>(p, s);
}

}  // namespace

extern "C" {

sp_status sp_kv4_attend_workspace_size(int32_t head_dim, size_t* bytes) {
  if (!bytes) return SP_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return SP_ERR_UNSUPPORTED;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  *bytes = workspace_bytes(head_dim, sms);
  return SP_OK;
}

sp_status sp_kv4_attend(const sp_attend_args* a, void* workspace_dev, size_t workspace_size, void* stream) {
  return attend(a, workspace_dev, workspace_size, nullptr, stream);
}

sp_status sp_test_expired_attend(const sp_attend_args* a, void* workspace_dev, size_t workspace_size, int32_t cta,
                                 int32_t warp, uint32_t wait_ms, void* stream) {
  if (cta < 0 || warp < 0 || wait_ms < 1 || wait_ms > 10000) return SP_ERR_INVALID_ARG;
  const Expire e = {cta, warp, (uint64_t)wait_ms * 1000000ull};
  return attend(a, workspace_dev, workspace_size, &e, stream);
}

}  // extern "C"
