// sp_rope.cu -- per-head norms of queries and keys, the position rotation and the write of keys and
// values into the 4-bit cache, in one pass; and the cached rows back (include/sp_serve.h).
//
// Every byte is touched once, so the pass is bound by memory: a head of D channels is a row of D / 16
// lanes with twice 16 bytes each, half a head apart, so that a channel and the one it usually turns with
// are in one lane, and norm and the row's extremes are few shuffles.  A warp takes one token and several
// heads of one kind (queries, keys or values), so that the angles are loaded once per warp.
//
// Measured: 4096 tokens, 32 heads of queries, keys and values of 128 into the cache (152 MB) 31.8 us, 4.8 TB/s, with
// 61 % of the issue slots taken; 513 tokens with norms, 32 and 8 heads, 4.3 us; one token 1.9 us.
#include <algorithm>
#include <climits>

#include "sp_attend.cuh"
#include "sp_lookup.h"

namespace sp {
namespace {

constexpr int kRopeThreads = 128;

struct RopeParams {
  const uint16_t *q, *k, *v;
  int64_t qs, ks, vs;
  uint16_t *q_out, *k_out;
  Kv4 cache;
  const int64_t* slots;
  const int32_t* positions;
  const float* cos_sin;
  int64_t rows;
  const uint16_t *qw, *kw;
  float eps;
  int32_t tokens, heads, kv_heads;
  int32_t rot;
  int32_t iters;           // rows of GW heads per warp
  int32_t uq, uk, units;   // warps per token: of queries, of keys, in all
  int32_t* status;
};

__device__ __forceinline__ void unpack8(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ float min3_nan(float a, float b, float c) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// The row's codes (two times eight per lane) and its parameter, as the header defines them.
template <int LH>
__device__ __forceinline__ uint2 quantize(const float (&x)[2][8], __half2* param) {
  float lo = min3_nan(x[0][0], x[0][1], x[0][2]), hi = max3_nan(x[0][0], x[0][1], x[0][2]);
#pragma unroll
  for (int i = 3; i < 15; i += 2) {
    lo = min3_nan(lo, x[i >> 3][i & 7], x[(i + 1) >> 3][(i + 1) & 7]);
    hi = max3_nan(hi, x[i >> 3][i & 7], x[(i + 1) >> 3][(i + 1) & 7]);
  }
  lo = min3_nan(lo, lo, x[1][7]), hi = max3_nan(hi, hi, x[1][7]);
#pragma unroll
  for (int d = 1; d < LH; d <<= 1) {
    const float lo2 = __shfl_xor_sync(0xffffffffu, lo, d), hi2 = __shfl_xor_sync(0xffffffffu, hi, d);
    lo = min3_nan(lo, lo, lo2), hi = max3_nan(hi, hi, hi2);
  }
  const bool ok = finite(lo) && finite(hi);
  lo = fminf(fmaxf(lo, -kKvMost), kKvMost), hi = fminf(fmaxf(hi, -kKvMost), kKvMost);
  const __half m = __float2half_rn(lo);
  const __half s = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), (float)(1.0 / 15.0)));
  *param = ok ? __halves2half2(s, m) : __halves2half2(__ushort_as_half(0), __ushort_as_half(0x7fff));
  const float sf = __half2float(s), mf = __half2float(m);
  if (!ok || !(sf > 0.f)) return make_uint2(0, 0);
  const float inv = __frcp_rn(sf);
  const uint64_t inv2 = two(inv, inv), m2 = two(-mf, -mf), magic2 = two(12582912.f, 12582912.f);
  uint32_t w[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    uint32_t n[8];  // a code in the low byte: 1.5 * 2^23 + n rounds to whole numbers, ties to even
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float a, b;
      apart(mul2(add2(two(x[y][i], x[y][i + 1]), m2), inv2), a, b);
      a = fminf(fmaxf(a, 0.f), 15.f), b = fminf(fmaxf(b, 0.f), 15.f);
      apart(add2(two(a, b), magic2), a, b);
      n[i] = __float_as_uint(a), n[i + 1] = __float_as_uint(b);
    }
    const uint32_t even = __byte_perm(__byte_perm(n[0], n[2], 0x0040), __byte_perm(n[4], n[6], 0x0040), 0x5410);
    const uint32_t odd = __byte_perm(__byte_perm(n[1], n[3], 0x0040), __byte_perm(n[5], n[7], 0x0040), 0x5410);
    w[y] = even + odd * 16u;
  }
  return make_uint2(w[0], w[1]);
}

// How the channels turn: each with the one half a head further on, which the same lane holds; with
// one rot / 2 further on; with its neighbour.
enum : int { kTurnHalf = 0, kTurnShort = 1, kTurnPairs = 2 };

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// D channels; TURN: as above; CACHE: keys and values go to the cache.  Eight CTAs per SM (64 registers)
// keep more rows on their way than six: 4096 tokens of 32 + 2 x 32 heads and their rows read back 50 us
// against 54.
template <int D, int TURN, bool CACHE>
__global__ void __launch_bounds__(kRopeThreads, TURN == kTurnShort ? 4 : 8) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int LH = D / 16, GW = 32 / LH;  // lanes of a head, heads of a warp
  constexpr int S = TURN == kTurnShort ? 2 : 1;  // sets of angles
  const int lane = threadIdx.x & 31, gl = lane % LH, gi = lane / LH;
  const int64_t u = (int64_t)blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
  const int token = (int)(u / p.units);
  if (token >= p.tokens) return;
  int r = (int)(u - (int64_t)token * p.units);
  const int kind = r < p.uq ? 0 : r < p.uq + p.uk ? 1 : 2;  // queries, keys, values
  r -= kind == 0 ? 0 : kind == 1 ? p.uq : p.uq + p.uk;
  const int heads = kind == 0 ? p.heads : p.kv_heads;
  const int h0 = r * p.iters * GW + gi, h1 = min(heads, (r + 1) * p.iters * GW);
  pdl_wait();
  const uint16_t* src = kind == 0 ? p.q + token * p.qs : kind == 1 ? p.k + token * p.ks : p.v + token * p.vs;
  const int d0 = gl * 8;  // the lane's channels: eight from here on, and from D / 2 + here on

  float cs[S][8], sn[S][8];
  if (kind < 2) {
    int64_t pos = p.positions[token];
    if (pos < 0 || pos >= p.rows) {
      set_status(p.status, kStatusBadIndex);
      pos = 0;
    }
    const float* t = p.cos_sin + pos * p.rot;
    const int half = p.rot / 2;
    if constexpr (TURN == kTurnHalf) {
      load8(t + d0, cs[0]);
      load8(t + half + d0, sn[0]);
    } else if constexpr (TURN == kTurnShort) {
      // sn has the sign of the other channel's product
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int d = d0 + y * (D / 2), at = d < half ? d : d - half;
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[y][i] = 1.f, sn[y][i] = 0.f;
        if (d < p.rot) {
          load8(t + at, cs[y]);
          load8(t + half + at, sn[y]);
          if (d < half)
#pragma unroll
            for (int i = 0; i < 8; ++i) sn[y][i] = -sn[y][i];
        }
      }
    } else {  // four angles for each eight channels
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int d = d0 + y * (D / 2);
        float4 c = make_float4(1.f, 1.f, 1.f, 1.f), s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (d < p.rot) {
          c = *reinterpret_cast<const float4*>(t + d / 2);
          s = *reinterpret_cast<const float4*>(t + half + d / 2);
        }
        cs[0][4 * y] = c.x, cs[0][4 * y + 1] = c.y, cs[0][4 * y + 2] = c.z, cs[0][4 * y + 3] = c.w;
        sn[0][4 * y] = s.x, sn[0][4 * y + 1] = s.y, sn[0][4 * y + 2] = s.z, sn[0][4 * y + 3] = s.w;
      }
    }
  }
  const uint16_t* wp = kind == 0 ? p.qw : kind == 1 ? p.kw : nullptr;

  uint8_t* codes = nullptr;  // the token's rows of the first head
  __half2* params = nullptr;
  const int64_t block = kv4_block_bytes<D>(CACHE ? p.cache.shift : 0);
  if constexpr (CACHE) {
    if (kind > 0) {
      const int64_t slot = p.slots[token];
      const int sh = p.cache.shift;
      if (slot >= p.cache.pages << sh) set_status(p.status, kStatusBadIndex);
      if (slot >= 0 && slot < p.cache.pages << sh) {
        const int in = (int)(slot & ((1 << sh) - 1));
        uint8_t* b = p.cache.data + (slot >> sh) * p.cache.heads * block;
        codes = b + (kind == 1 ? 0 : kv4_value_codes<D>(sh)) + in * (D / 2) + gl * 4;
        params = reinterpret_cast<__half2*>(b + (kind == 1 ? kv4_key_params<D>(sh) : kv4_value_params<D>(sh))) + in;
      }
    }
  }

  constexpr int kBatch = 2;  // rows in flight per lane
#pragma unroll 1
  for (int it = 0; it < p.iters; it += kBatch) {
    uint4 in[kBatch][2];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + (it + j) * GW;
      in[j][0] = in[j][1] = make_uint4(0, 0, 0, 0);
      if (it + j < p.iters && h < h1) {
        in[j][0] = *reinterpret_cast<const uint4*>(src + (int64_t)h * D + d0);
        in[j][1] = *reinterpret_cast<const uint4*>(src + (int64_t)h * D + D / 2 + d0);
      }
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + (it + j) * GW;
      if (it + j >= p.iters || h - gi >= h1) break;  // the same in the whole warp
      float x[2][8];
      unpack8(in[j][0], x[0]);
      unpack8(in[j][1], x[1]);
      if (wp) {
        float s[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          s[y] = __fadd_rn(__fadd_rn(__fadd_rn(__fmul_rn(x[y][0], x[y][0]), __fmul_rn(x[y][1], x[y][1])),
                                     __fadd_rn(__fmul_rn(x[y][2], x[y][2]), __fmul_rn(x[y][3], x[y][3]))),
                           __fadd_rn(__fadd_rn(__fmul_rn(x[y][4], x[y][4]), __fmul_rn(x[y][5], x[y][5])),
                                     __fadd_rn(__fmul_rn(x[y][6], x[y][6]), __fmul_rn(x[y][7], x[y][7]))));
#pragma unroll
          for (int d = 1; d < LH; d <<= 1) s[y] = __fadd_rn(s[y], __shfl_xor_sync(0xffffffffu, s[y], d));
        }
        const float rs = __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(__fadd_rn(s[0], s[1]), 1.f / D), p.eps)));
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          float w[8];
          unpack8(__ldg(reinterpret_cast<const uint4*>(wp + y * (D / 2) + d0)), w);
#pragma unroll
          for (int i = 0; i < 8; i += 2)
            apart(mul2(mul2(two(x[y][i], x[y][i + 1]), two(rs, rs)), two(w[i], w[i + 1])), x[y][i], x[y][i + 1]);
        }
      }
      if (kind < 2) {
        // a * cos - b * sin and b * cos + a * sin, unpacked: a packed product and sum would become one
        // fused operation.  The sign of a product or of a sum of rounded products changes no bit of it.
        if constexpr (TURN == kTurnHalf) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float a = x[0][i], b = x[1][i];
            x[0][i] = __fsub_rn(__fmul_rn(a, cs[0][i]), __fmul_rn(b, sn[0][i]));
            x[1][i] = __fadd_rn(__fmul_rn(b, cs[0][i]), __fmul_rn(a, sn[0][i]));
          }
        } else if constexpr (TURN == kTurnShort) {
          // chunk c of eight channels turns with c + rot / 16 or c - rot / 16, in the lane c % LH
          const int hc = p.rot / 16;
          float o[2][8];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int c = gl + y * LH, pc = c >= 2 * hc ? c : c < hc ? c + hc : c - hc;
            const int from = gi * LH + pc % LH;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float a = __shfl_sync(0xffffffffu, x[0][i], from), b = __shfl_sync(0xffffffffu, x[1][i], from);
              o[y][i] = pc < LH ? a : b;
            }
          }
#pragma unroll
          for (int y = 0; y < 2; ++y)
            if (d0 + y * (D / 2) < p.rot)
#pragma unroll
              for (int i = 0; i < 8; ++i)
                x[y][i] = __fadd_rn(__fmul_rn(x[y][i], cs[y][i]), __fmul_rn(o[y][i], sn[y][i]));
        } else {
#pragma unroll
          for (int y = 0; y < 2; ++y)
            if (d0 + y * (D / 2) < p.rot)
#pragma unroll
              for (int i = 0; i < 8; i += 2) {
                const float a = x[y][i], b = x[y][i + 1], c = cs[0][4 * y + i / 2], s = sn[0][4 * y + i / 2];
                x[y][i] = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
                x[y][i + 1] = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
              }
        }
      }
      const bool there = h < h1;
      if (CACHE && kind > 0) {
        __half2 par;
        const uint2 n = quantize<LH>(x, &par);
        if (there && codes) {
          *reinterpret_cast<uint32_t*>(codes + h * block) = n.x;
          *reinterpret_cast<uint32_t*>(codes + h * block + D / 4) = n.y;
          if (gl == 0) *reinterpret_cast<__half2*>(reinterpret_cast<uint8_t*>(params) + h * block) = par;
        }
      } else if (there) {
        uint16_t* dst = (kind == 0 ? p.q_out + ((int64_t)token * p.heads + h) * D : p.k_out + ((int64_t)token * p.kv_heads + h) * D) + d0;
        *reinterpret_cast<uint4*>(dst) = pack8(x[0]);
        *reinterpret_cast<uint4*>(dst + D / 2) = pack8(x[1]);
      }
    }
  }
}

// Rows of the cache as bf16: D / 8 lanes per (slot, head); a warp takes a slot and `per` of its heads, four loads
// in flight.  Bound by memory, three quarters of the bytes its output's: 4096 slots of 32 heads of 128 (85 MB)
// 15.6 us, 5.5 TB/s; a thread per row and piece of the whole grid, with a division each, took 17.
constexpr int kReadThreads = 256;
template <int D>
__global__ void __launch_bounds__(kReadThreads) read_kernel(Kv4 c, const int64_t* __restrict__ slots, int64_t n,
                                                            uint4* __restrict__ k_out, uint4* __restrict__ v_out, int per,
                                                            int32_t* status) {
  constexpr int LH = D / 8, A = 32 / LH;  // lanes of a head, heads side by side
  pdl_wait();
  const int64_t i = blockIdx.x * (int64_t)(kReadThreads / 32) + (threadIdx.x >> 5);
  if (i >= n) return;
  const int lane = threadIdx.x & 31, gl = lane % LH;
  const int h1 = min(((int)blockIdx.y + 1) * per, c.heads);
  const int64_t slot = slots[i];
  const bool there = slot >= 0 && slot < c.pages << c.shift;
  if (slot >= 0 && !there) set_status(status, kStatusBadIndex);
  const int in = (int)(slot & ((1 << c.shift) - 1));
  const int64_t block = kv4_block_bytes<D>(c.shift);
  const uint8_t* b = c.data + (there ? (slot >> c.shift) * c.heads * block : 0);
#pragma unroll 4
  for (int h = (int)blockIdx.y * per + lane / LH; h < h1; h += A) {
    uint32_t code[2] = {0, 0};
    __half2 par[2] = {__half2half2(__ushort_as_half(0)), __half2half2(__ushort_as_half(0))};
    if (there) {
      const uint8_t* x = b + h * block;
      code[0] = *reinterpret_cast<const uint32_t*>(x + in * (D / 2) + gl * 4);
      code[1] = *reinterpret_cast<const uint32_t*>(x + kv4_value_codes<D>(c.shift) + in * (D / 2) + gl * 4);
      par[0] = *(reinterpret_cast<const __half2*>(x + kv4_key_params<D>(c.shift)) + in);
      par[1] = *(reinterpret_cast<const __half2*>(x + kv4_value_params<D>(c.shift)) + in);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float s = __low2float(par[w]), m = __high2float(par[w]);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = fmaf(s, (float)((code[w] >> (4 * j)) & 15u), m);  // s * n is exact
      (w ? v_out : k_out)[(i * c.heads + h) * LH + gl] = pack8(x);
    }
  }
}

}  // namespace

int current_sms() {
  static std::atomic<int> kept[64] = {};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return 0;
  }
  return kept_or_looked_up(kept[dev], [dev] {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    return n;
  });
}

}  // namespace sp

using namespace sp;

namespace {
sp_status check_cache(const sp_kv4* c) {
  if (!c || !c->data || !kv4_positive(c) || c->reserved != 0) return SP_ERR_INVALID_ARG;
  if (!kv4_supported(c)) return SP_ERR_UNSUPPORTED;
  return al16(c->data) ? SP_OK : SP_ERR_ALIGNMENT;
}

template <int D, bool CACHE>
sp_status launch_rope(const RopeParams& p, bool pairs, int64_t warps, cudaStream_t stream) {
  auto kern = pairs ? rope_kernel<D, kTurnPairs, CACHE>
                    : p.rot == D ? rope_kernel<D, kTurnHalf, CACHE> : rope_kernel<D, kTurnShort, CACHE>;
  const int64_t blocks = (warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
  return launch_pdl(kern, dim3((unsigned)blocks), kRopeThreads, 0, 1, stream, p);
}
}  // namespace

extern "C" {

sp_status sp_kv4_bytes(const sp_kv4* c, size_t* bytes) {
  if (!c || !bytes || !kv4_positive(c) || c->reserved != 0) return SP_ERR_INVALID_ARG;
  if (!kv4_supported(c)) return SP_ERR_UNSUPPORTED;
  *bytes = (size_t)c->pages * (size_t)c->kv_heads * (size_t)c->page_size * (size_t)(c->head_dim + 8);
  return SP_OK;
}

sp_status sp_qk_norm_rope(const sp_rope_args* a, void* stream) {
  if (!a || a->tokens < 0 || a->heads < 1 || a->kv_heads < 1 || a->rows < 1 || a->rot < 0 || a->rot > a->head_dim ||
      (a->pairs != 0 && a->pairs != 1))
    return SP_ERR_INVALID_ARG;
  if ((a->head_dim != 64 && a->head_dim != 128) || a->rot % 16 != 0) return SP_ERR_UNSUPPORTED;
  if (a->tokens == 0) return SP_OK;
  if ((a->cache != nullptr) != (a->slots != nullptr) || (a->cache != nullptr) != (a->v != nullptr) ||
      (a->cache != nullptr) != (a->k_out == nullptr))
    return SP_ERR_INVALID_ARG;
  if (a->cache) {
    const sp_status st = check_cache(a->cache);
    if (st != SP_OK) return st;
    if (a->cache->kv_heads != a->kv_heads || a->cache->head_dim != a->head_dim) return SP_ERR_INVALID_ARG;
  }
  if (!a->q || !a->k || !a->q_out || !a->positions || (!a->cos_sin && a->rot > 0)) return SP_ERR_INVALID_ARG;
  const int64_t dim = a->head_dim;
  if (a->q_stride < a->heads * dim || a->k_stride < a->kv_heads * dim || (a->v && a->v_stride < a->kv_heads * dim))
    return SP_ERR_INVALID_ARG;
  if (a->q_stride % 8 || a->k_stride % 8 || (a->v && a->v_stride % 8)) return SP_ERR_UNSUPPORTED;
  if (!al16(a->q) || !al16(a->k) || !al16(a->v) || !al16(a->q_out) || !al16(a->k_out) || !al16(a->cos_sin) ||
      !al16(a->q_weight) || !al16(a->k_weight))
    return SP_ERR_ALIGNMENT;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  RopeParams p = {};
  p.q = static_cast<const uint16_t*>(a->q);
  p.k = static_cast<const uint16_t*>(a->k);
  p.v = static_cast<const uint16_t*>(a->v);
  p.qs = a->q_stride;
  p.ks = a->k_stride;
  p.vs = a->v_stride;
  p.q_out = static_cast<uint16_t*>(a->q_out);
  p.k_out = static_cast<uint16_t*>(a->k_out);
  if (a->cache) p.cache = kv4_view(a->cache);
  p.slots = a->slots;
  p.positions = a->positions;
  p.cos_sin = a->cos_sin;
  p.rows = a->rows;
  p.qw = static_cast<const uint16_t*>(a->q_weight);
  p.kw = static_cast<const uint16_t*>(a->k_weight);
  p.eps = a->eps;
  p.tokens = a->tokens;
  p.heads = a->heads;
  p.kv_heads = a->kv_heads;
  p.rot = a->rot;
  p.status = device_status_ptr();
  // heads per warp: as many as still leave every SM its warps
  const int gw = 32 / ((int)dim / 16);
  const int64_t nq = (a->heads + gw - 1) / gw, nk = (a->kv_heads + gw - 1) / gw;
  const int64_t total = a->tokens * (nq + (a->cache ? 2 : 1) * nk);
  const int64_t iters = total / ((int64_t)sms * 48);
  p.iters = (int32_t)(iters < 1 ? 1 : iters > 8 ? 8 : iters);
  p.uq = (int32_t)((nq + p.iters - 1) / p.iters);
  p.uk = (int32_t)((nk + p.iters - 1) / p.iters);
  p.units = p.uq + (a->cache ? 2 : 1) * p.uk;
  const int64_t warps = (int64_t)a->tokens * p.units;
  if (warps / (kRopeThreads / 32) >= ((int64_t)1 << 31) - 1) return SP_ERR_UNSUPPORTED;
  cudaStream_t st = (cudaStream_t)stream;
  if (dim == 64)
    return a->cache ? launch_rope<64, true>(p, a->pairs != 0, warps, st) : launch_rope<64, false>(p, a->pairs != 0, warps, st);
  return a->cache ? launch_rope<128, true>(p, a->pairs != 0, warps, st) : launch_rope<128, false>(p, a->pairs != 0, warps, st);
}

sp_status sp_kv4_read(const sp_kv4* c, const int64_t* slots, int64_t n, void* k_out, void* v_out, void* stream) {
  const sp_status st = check_cache(c);
  if (st != SP_OK) return st;
  if (n < 0) return SP_ERR_INVALID_ARG;
  if (n == 0) return SP_OK;
  if (!slots || !k_out || !v_out) return SP_ERR_INVALID_ARG;
  if (!al16(k_out) || !al16(v_out)) return SP_ERR_ALIGNMENT;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  // heads of a warp: as many as still leave every SM its warps
  const int side = 256 / c->head_dim, all = (c->kv_heads + side - 1) / side;
  const int64_t parts = std::min<int64_t>(all, std::max<int64_t>(1, ((int64_t)sms * 64 + n - 1) / n));
  const int per = (int)((all + parts - 1) / parts) * side;
  const int64_t blocks = (n + kReadThreads / 32 - 1) / (kReadThreads / 32);
  if (blocks > INT_MAX) return SP_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks, (unsigned)((c->kv_heads + per - 1) / per));
  auto kern = c->head_dim == 64 ? read_kernel<64> : read_kernel<128>;
  return launch_pdl(kern, grid, kReadThreads, 0, 1, (cudaStream_t)stream, kv4_view(c), slots, n, static_cast<uint4*>(k_out),
                    static_cast<uint4*>(v_out), per, device_status_ptr());
}

}  // extern "C"
