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
//   warps 8-15       codes to fp16 operands in shared memory: K rows as [key][channel], V rows as
//                    [channel][key], both in 128-byte-swizzled panels of 64 columns
//   warp 16          issues the products
//
// Numbers.  s n + m is rounded once to fp16 (the cache holds |x| <= 2^15); the queries, bf16, enter
// exactly, each row scaled by a power of two.  The running maximum of a row moves only when
// a weight would pass 2^8, so the sums in tensor memory are rarely touched by the rows' threads.  A key
// row's channels may be in any order that the queries share, which saves their permutation: of the
// eight codes of a word, i and i + 4 come out as a pair.
#include <algorithm>
#include <climits>

#include "sp_attend.cuh"
#include "sp_lookup.h"
#include "sp_tcgen05.cuh"

namespace sp {
namespace {

constexpr int kTile = 128;                // keys of a step, query rows of a tile
constexpr int kRowThreads = 256;          // two tiles' rows
constexpr int kFillWarps = 8;
constexpr int kFillThreads = 32 * kFillWarps;
constexpr int kThreads = kRowThreads + kFillThreads + 32;
constexpr int kStages = 2;
constexpr int kMaxDevices = 64;
constexpr uint32_t kPanel = kTile * 128;  // 128 rows of 64 columns

template <int D>
struct Smem {
  static constexpr uint32_t kQ = D / 64 * kPanel;              // a tile of queries, a step's keys
  static constexpr uint32_t kV = 2 * D * 128;                  // a step's values: two panels of D channels
  static constexpr uint32_t kBytes = 2 * kQ + kStages * (kQ + kV);
  static constexpr size_t kTotal = 1024 + kBytes;              // + base alignment
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
// Instruction descriptor, kind::f16: D fp32, A and B fp16, both K-major.
constexpr uint32_t idesc_f16(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

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
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1) attend_rows_kernel(const __grid_constant__ AttendParams p) {
  using L = Smem<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* s_q = smem;
  uint8_t* s_k = smem + 2 * L::kQ;
  uint8_t* s_v = s_k + kStages * L::kQ;
  __shared__ uint64_t q_full, k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  __shared__ uint64_t s_full[2], p_full[2], o_done[2];
  __shared__ uint32_t s_tmem;
  __shared__ uint32_t s_nan[kStages][4];  // keys of the step whose values are not finite
  __shared__ Item s_item[2];
  __shared__ int s_dead;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(&q_full, kRowThreads / 32);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&k_full[i], kFillWarps);
      mbar_init(&v_full[i], kFillWarps);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 4);
      mbar_init(&o_done[i], 1);
    }
    fence_barrier_init();
    s_dead = 0;
  }
  pdl_wait();
  const int32_t* share = p.work + p.requests + 1;  // pairs of tiles of the requests before each
  const int heads = p.cache.heads;
  const int64_t items = (int64_t)share[p.requests] * heads;
  // the next item: later rows, which see more, first
  auto fetch = [&](Item& it) {
    it.rows = 0;
    const int64_t i = (int64_t)atomicAdd(&p.cnt[0], 1);
    if (i >= items) return;
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
      set_status(p.status, kStatusBadIndex);  // shares that do not belong to the lengths
      it.rows = -1;
      return;
    }
    it.row0 = (pairs - 1 - (pair - share[lo])) * 2 * kTile;
    it.rows = (int)min(all - it.row0, (int64_t)(2 * kTile));
    it.sees0 = it.len - fresh + 1;
  };
  if (tid == kThreads - 32) {
    Item it;
    do fetch(it);
    while (it.rows < 0);
    s_item[0] = it;
  }
  if (warp == 0) {
    tmem_alloc(&s_tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const int shift = p.cache.shift;
  const int64_t block = kv4_block_bytes<D>(shift);

  // phases of the barriers, counted over all items: steps of keys, and of either tile
  uint32_t steps = 0, done[2] = {0, 0}, round = 0;
  for (;; ++round) {
    const Item it = s_item[round & 1];
    if (it.rows <= 0) break;
    // steps that either tile's last row sees
    int n[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int rows = min(it.rows - i * kTile, kTile);
      n[i] = rows > 0 ? (it.sees0 + (it.row0 + i * kTile + rows - 1) / p.group + kTile - 1) / kTile : 0;
    }
    const int n_all = max(n[0], n[1]);
    bool dead = false;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (dead) return;
      if (!__all_sync(0xffffffffu, mbar_wait(bar, parity, p.timeout_ns))) {
        if (lane == 0) set_status(p.status, kStatusTimeout);
        dead = true;
      }
    };

    if (warp < kRowThreads / 32) {
      // -------------------------------------------------------------- rows
      const int i = warp >> 2;  // tile
      const int r = tid & (kTile - 1);
      const bool there = i * kTile + r < it.rows;
      const int row = it.row0 + i * kTile + r, token = row / p.group;
      const int limit = there ? it.sees0 + token : 0;  // keys that the row sees
      const int64_t col = (int64_t)(it.h * p.group + row - token * p.group) * D;
      float cr;  // log2 score = cr * product
      {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (it.q0 + (int64_t)token) * p.q_stride + col);
        uint32_t big = 0;
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          const uint4 u = there ? src[c] : make_uint4(0, 0, 0, 0);
          const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) big = max(big, max(x[j] & 0x7fffu, (x[j] >> 16) & 0x7fffu));
        }
        // 2^(141 - e): the row's largest entry, of biased exponent e, comes to 2^14 ... 2^15
        const uint32_t e = max(15u, min(254u, big >> 7));
        const float f = copysignf(__uint_as_float((268u - e) << 23), p.scale_log2);
        cr = __uint_as_float((e - 14u) << 23) * fabsf(p.scale_log2);
        uint8_t* dst = s_q + i * L::kQ + r * 128;
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          const uint4 u = there ? src[c] : make_uint4(0, 0, 0, 0);
          const uint32_t x[4] = {u.x, u.y, u.z, u.w};
          float y[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            y[2 * j] = __uint_as_float(x[j] << 16) * f;
            y[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u) * f;
          }
          *reinterpret_cast<uint4*>(dst + (c >> 3) * kPanel + (((c & 7) ^ (r & 7)) << 4)) =
              make_uint4(pack_f16(y[0], y[4]), pack_f16(y[1], y[5]), pack_f16(y[2], y[6]), pack_f16(y[3], y[7]));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full);
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t t_s = tmem + lanes + i * kTile, t_o = tmem + lanes + 2 * kTile + i * D;
      float m = -INFINITY;
      float l = 0.f;
      for (int j = 0; j < n[i]; ++j) {
        wait(&s_full[i], (done[i] + j) & 1);
        if (dead) break;
        tc_fence_after();
        const bool edge = (j + 1) * kTile > limit;  // the row does not see all of the step
        const bool cut = __any_sync(0xffffffffu, edge);
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t u[32];
          tmem_load32(t_s + 32 * c, u);
          tmem_load_wait();
          if (cut) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (j * kTile + 32 * c + k < limit) top = fmaxf(top, __uint_as_float(u[k]));
          } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) top = fmaxf(top, __uint_as_float(u[k]));
          }
        }
        top *= cr;  // (-inf stays: cr > 0, or 0 where nothing is seen or the scale is 0)
        if (cr == 0.f) top = 0.f;
        const bool lift = top > m + 8.f;
        if (__any_sync(0xffffffffu, lift)) {
          const float up = lift ? top : m;
          const float alpha = m == -INFINITY ? (j == 0 ? 1.f : 0.f) : ex2(m - up);
          l *= alpha;
          m = up;
          if (j > 0) {
            wait(&o_done[i], (done[i] + j - 1) & 1);
            if (dead) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              uint32_t u[32];
              tmem_load32(t_o + 32 * c, u);
              tmem_load_wait();
#pragma unroll
              for (int k = 0; k < 32; ++k) u[k] = __float_as_uint(__uint_as_float(u[k]) * alpha);
              tmem_store32(t_o + 32 * c, u);
            }
            tmem_store_wait();
          }
        }
        const float minus = m == -INFINITY ? 0.f : -m;
        const uint64_t c2 = two(cr, cr), m2 = two(minus, minus);
        uint64_t sum = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t u[32], w[16];
          tmem_load32(t_s + 32 * c, u);
          tmem_load_wait();
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            float a, b;
            apart(fma2(two(__uint_as_float(u[k]), __uint_as_float(u[k + 1])), c2, m2), a, b);
            a = ex2(a), b = ex2(b);
            if (cut) {
              if (j * kTile + 32 * c + k >= limit) a = 0.f;
              if (j * kTile + 32 * c + k + 1 >= limit) b = 0.f;
            }
            sum = add2(sum, two(a, b));
            w[k / 2] = pack_f16(a, b);
          }
          tmem_store16(t_s + 16 * c, w);
        }
        float a, b;
        apart(sum, a, b);
        l += a + b;
        // a value row that is not finite entered as zeros: it makes NaN of the rows that see it
        const int st = (steps + j) % kStages;
        wait(&v_full[st], ((steps + j) / kStages) & 1);
        if (dead) break;
        const volatile uint32_t* bad = s_nan[st];
        const uint32_t x[4] = {bad[0], bad[1], bad[2], bad[3]};
        if (x[0] | x[1] | x[2] | x[3]) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int seen = limit - (j * kTile + 32 * c);
            const uint32_t mask = seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1u;
            if (x[c] & mask) l = __uint_as_float(0x7fffffffu);
          }
        }
        tmem_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[i]);
      }
      if (n[i] > 0) {
        wait(&o_done[i], (done[i] + n[i] - 1) & 1);
        tc_fence_after();
        if (!dead) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          uint16_t* dst = p.out + (it.q0 + (int64_t)token) * p.out_stride + col;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t u[32];
            tmem_load32(t_o + 32 * c, u);
            tmem_load_wait();
            if (there) {
#pragma unroll
              for (int k = 0; k < 32; k += 8) {
                uint32_t w[4];
#pragma unroll
                for (int x = 0; x < 4; ++x)
                  w[x] = pack_bf16(__uint_as_float(u[k + 2 * x]) * inv, __uint_as_float(u[k + 2 * x + 1]) * inv);
                *reinterpret_cast<uint4*>(dst + 32 * c + k) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          }
        }
        tc_fence_before();
      }
    } else if (warp < (kRowThreads + kFillThreads) / 32) {
      // -------------------------------------------------------------- keys and values
      const int f = tid - kRowThreads;
      const int32_t* table = p.table + (int64_t)it.b * p.width;
      auto block_of = [&](int key) -> const uint8_t* {  // null behind the last key
        if (key >= it.len) return nullptr;
        const int at = key >> shift, page = at < p.width ? table[at] : -1;
        if (page < 0 || page >= p.cache.pages) {
          set_status(p.status, kStatusBadIndex);
          return nullptr;
        }
        return p.cache.data + ((int64_t)page * heads + it.h) * block;
      };
      const int k_key = f & (kTile - 1), k_half = f >> 7;             // a key, half of its channels
      const int v_group = (f & 7) + 8 * (f >> 7), v_word = (f >> 3) & 15;  // eight keys, eight channels
      constexpr int KQ = D / 64;                                      // 16-byte pieces of half a key
      const int page_keys = 1 << shift;
      const bool v_there = D == 128 || v_word < 8;
      uint4 kc[KQ], vp[2];
      uint32_t kp, vc[8];
      auto load_k = [&](int j) {
        const int key = j * kTile + k_key;
        const uint8_t* bl = block_of(key);
        const int in = key & (page_keys - 1);
        kp = 0;
#pragma unroll
        for (int x = 0; x < KQ; ++x) kc[x] = make_uint4(0, 0, 0, 0);
        if (bl) {
#pragma unroll
          for (int x = 0; x < KQ; ++x)
            kc[x] = __ldg(reinterpret_cast<const uint4*>(bl + in * (D / 2) + k_half * (D / 4)) + x);
          kp = __ldg(reinterpret_cast<const uint32_t*>(bl + kv4_key_params<D>(shift)) + in);
        }
      };
      auto load_v = [&](int j) {
        const int key = j * kTile + 8 * v_group;
        const uint8_t* bl = block_of(key);
        const int in = key & (page_keys - 1);
        vp[0] = vp[1] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int x = 0; x < 8; ++x) vc[x] = 0;
        if (bl && v_there) {
#pragma unroll
          for (int x = 0; x < 8; ++x)
            vc[x] = __ldg(reinterpret_cast<const uint32_t*>(bl + kv4_value_codes<D>(shift) + (in + x) * (D / 2)) + v_word);
          const uint4* src = reinterpret_cast<const uint4*>(bl + kv4_value_params<D>(shift) + in * 4);
          vp[0] = __ldg(src), vp[1] = __ldg(src + 1);
        }
      };
      load_k(0);
      load_v(0);
      for (int j = 0; j < n_all; ++j) {
        const int st = (steps + j) % kStages;
        const uint32_t ph = ((steps + j) / kStages) & 1;
        wait(&k_empty[st], ph ^ 1);
        if (dead) break;
        {
          const uint32_t s = __byte_perm(kp, kp, 0x1010), m = __byte_perm(kp, kp, 0x3232);
          uint8_t* dst = s_k + st * L::kQ + k_key * 128;
#pragma unroll
          for (int x = 0; x < KQ; ++x) {
            const uint32_t w[4] = {kc[x].x, kc[x].y, kc[x].z, kc[x].w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int c = k_half * (D / 16) + 4 * x + y;  // eight channels
              const uint32_t h = w[y] >> 8;
              *reinterpret_cast<uint4*>(dst + (c >> 3) * kPanel + (((c & 7) ^ (k_key & 7)) << 4)) =
                  make_uint4(value_lo(w[y], s, m), value_hi(w[y], s, m), value_lo(h, s, m), value_hi(h, s, m));
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&k_full[st]);
        if (j + 1 < n_all) load_k(j + 1);  // (the next step's, while this one's values are expanded)
        wait(&v_empty[st], ph ^ 1);
        if (dead) break;
        {
          uint32_t par[8] = {vp[0].x, vp[0].y, vp[0].z, vp[0].w, vp[1].x, vp[1].y, vp[1].z, vp[1].w};
          uint32_t nan = 0;
          const int left = it.len - (j * kTile + 8 * v_group);  // keys of the eight that were written
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            if (x >= left) par[x] = 0;
            if ((par[x] & 0x7c00u) == 0x7c00u || (par[x] & 0x7c000000u) == 0x7c000000u) {
              par[x] = 0;
              nan |= 1u << x;
            }
          }
          // 32 keys a word: the four lanes' bytes side by side (every word of channels says the same)
          uint32_t word = nan << (8 * (v_group & 3));
          word |= __shfl_xor_sync(0xffffffffu, word, 1);
          word |= __shfl_xor_sync(0xffffffffu, word, 2);
          if (v_word == 0 && (v_group & 3) == 0) s_nan[st][v_group >> 2] = word;
          if (v_there) {
            uint32_t s[4], m[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              s[x] = __byte_perm(par[2 * x], par[2 * x + 1], 0x5410);
              m[x] = __byte_perm(par[2 * x], par[2 * x + 1], 0x7632);
            }
            uint8_t* dst = s_v + st * L::kV + (v_group >> 3) * (D * 128) + v_word * 8 * 128;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t w[4];
#pragma unroll
              for (int x = 0; x < 4; ++x) w[x] = __byte_perm(vc[2 * x], vc[2 * x + 1], half ? 0x7632 : 0x5410);
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                const int c = 4 * half + 2 * z;  // channel of the eight
                uint32_t lo[4], hi[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  const uint32_t y = z ? w[x] >> 8 : w[x];
                  lo[x] = value_lo(y, s[x], m[x]);
                  hi[x] = value_hi(y, s[x], m[x]);
                }
                *reinterpret_cast<uint4*>(dst + c * 128 + (((v_group & 7) ^ c) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                *reinterpret_cast<uint4*>(dst + (c + 1) * 128 + (((v_group & 7) ^ (c + 1)) << 4)) =
                    make_uint4(hi[0], hi[1], hi[2], hi[3]);
              }
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&v_full[st]);
        if (j + 1 < n_all) load_v(j + 1);
      }
    } else {
      // -------------------------------------------------------------- the products
      if (lane == 0) {
        Item next;
        do fetch(next);
        while (next.rows < 0);
        s_item[(round + 1) & 1] = next;
      }
      __syncwarp();
      const uint32_t a_q = smem_u32(s_q), a_k = smem_u32(s_k), a_v = smem_u32(s_v);
      auto scores = [&](int i, int j) {  // S_i = Q_i . K_j^T
        const int st = (steps + j) % kStages;
        wait(&k_full[st], ((steps + j) / kStages) & 1);
        tc_fence_after();
        if (!dead && elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = (kk >> 2) * kPanel + (kk & 3) * 32;
            mma_ss(tmem + i * kTile, smem_desc_sw128(a_q + i * L::kQ + off), smem_desc_sw128(a_k + st * L::kQ + off),
                   idesc_f16(kTile, kTile), kk > 0 ? 1u : 0u);
          }
          mma_commit(&s_full[i]);
        }
        __syncwarp();
      };
      wait(&q_full, round & 1);
      for (int i = 0; i < 2; ++i)
        if (n[i] > 0) scores(i, 0);
      if (!dead && elect_one()) mma_commit(&k_empty[steps % kStages]);
      __syncwarp();
      for (int j = 0; j < n_all && !dead; ++j) {
        const int st = (steps + j) % kStages;
        for (int i = 0; i < 2; ++i) {
          if (j < n[i]) {
            wait(&v_full[st], ((steps + j) / kStages) & 1);
            wait(&p_full[i], (done[i] + j) & 1);
            tc_fence_after();
            if (!dead && elect_one()) {
#pragma unroll
              for (int kk = 0; kk < kTile / 16; ++kk) {
                const uint32_t off = (kk >> 2) * (D * 128) + (kk & 3) * 32;
                mma_ts(tmem + 2 * kTile + i * D, tmem + i * kTile + kk * 8, smem_desc_sw128(a_v + st * L::kV + off),
                       idesc_f16(kTile, D), (j > 0 || kk > 0) ? 1u : 0u);
              }
              mma_commit(&o_done[i]);
            }
            __syncwarp();
          }
          if (j + 1 < n[i]) scores(i, j + 1);
        }
        if (!dead && elect_one()) {
          mma_commit(&v_empty[st]);
          if (j + 1 < n_all) mma_commit(&k_empty[(steps + j + 1) % kStages]);
        }
        __syncwarp();
      }
    }
    if (dead) s_dead = 1;
    steps += n_all;
    done[0] += n[0];
    done[1] += n[1];
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (s_dead) break;
  }
  if (warp == kRowThreads / 32 && !s_dead) {  // the products' last arrivals on this CTA's barriers
    for (uint32_t x = steps > kStages ? steps - kStages : 0; x < steps; ++x) {
      mbar_wait(&k_empty[x % kStages], (x / kStages) & 1, p.timeout_ns);
      mbar_wait(&v_empty[x % kStages], (x / kStages) & 1, p.timeout_ns);
    }
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

template <int D>
sp_status launch(const AttendParams& p, int sms, cudaStream_t stream) {
  static std::atomic<int> set[kMaxDevices] = {};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
    cudaGetLastError();
    return SP_ERR_CUDA;
  }
  const int ok = kept_or_looked_up(set[dev], [] {
    if (cudaFuncSetAttribute(attend_rows_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)Smem<D>::kTotal) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    return 1;
  });
  if (!ok) return SP_ERR_CUDA;
  return launch_pdl(attend_rows_kernel<D>, dim3((unsigned)sms), kThreads, Smem<D>::kTotal, 1, stream, p);
}

}  // namespace

sp_status launch_attend_rows(const AttendParams& p, int head_dim, cudaStream_t stream) {
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  return head_dim == 64 ? launch<64>(p, sms, stream) : launch<128>(p, sms, stream);
}

}  // namespace sp
