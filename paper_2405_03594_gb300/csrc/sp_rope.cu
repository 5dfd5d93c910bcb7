// sp_rope.cu -- per-head norms of queries and keys, the position rotation and the write of keys and
// values into the 4-bit cache, in one pass; and the cached rows back (include/sp_serve.h).
//
// Every byte is touched once, so the pass is bound by memory: a head of D channels is a row of D / 8
// lanes with 16 bytes each, and norm, rotation and the row's extremes are shuffles among them.  A
// warp takes one token and several heads of one kind (queries, keys or values), so that the angles
// and the norm's weights are loaded once per warp and stay in registers.
#include "sp_kv4.cuh"
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
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// The row's codes (eight per lane) and its parameter, as the header defines them.
template <int LH>
__device__ __forceinline__ uint32_t quantize(const float (&x)[8], __half2* param) {
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) lo = min_nan(lo, x[i]), hi = max_nan(hi, x[i]);
#pragma unroll
  for (int d = 1; d < LH; d <<= 1) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, d));
  }
  if (!finite(lo) || !finite(hi)) {
    *param = __halves2half2(__ushort_as_half(0), __ushort_as_half(0x7fff));
    return 0;
  }
  const __half m = __float2half_rn(fminf(fmaxf(lo, -65504.f), 65504.f));
  const __half s = __float2half_rn(fminf(__fmul_rn(__fsub_rn(hi, lo), (float)(1.0 / 15.0)), 65504.f));
  *param = __halves2half2(s, m);
  const float sf = __half2float(s), mf = __half2float(m);
  if (!(sf > 0.f)) return 0;
  const float inv = __fdiv_rn(1.f, sf);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float n = fminf(fmaxf(rintf(__fmul_rn(__fsub_rn(x[i], mf), inv)), 0.f), 15.f);
    w |= (uint32_t)n << (4 * i);
  }
  return w;
}

// D channels; PAIRS: how channels pair up; CACHE: keys and values go to the cache.
template <int D, bool PAIRS, bool CACHE>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int LH = D / 8, GW = 32 / LH;  // lanes of a head, heads of a warp
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
  const int d0 = gl * 8;

  // angles of the lane's channels; sn has the sign of the other channel's product
  float cs[8], sn[8];
  const bool turns = kind < 2 && d0 < p.rot;
  if (turns) {
    int64_t pos = p.positions[token];
    if (pos < 0 || pos >= p.rows) {
      set_status(p.status, kStatusBadIndex);
      pos = 0;
    }
    const float* t = p.cos_sin + pos * p.rot;
    const int half = p.rot / 2;
    if constexpr (PAIRS) {
      const float4 c = *reinterpret_cast<const float4*>(t + d0 / 2), s = *reinterpret_cast<const float4*>(t + half + d0 / 2);
      const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) cs[2 * i] = cs[2 * i + 1] = cc[i], sn[2 * i] = -ss[i], sn[2 * i + 1] = ss[i];
    } else {
      const int a = d0 < half ? d0 : d0 - half;
      const float sign = d0 < half ? -1.f : 1.f;
      const float4 *c = reinterpret_cast<const float4*>(t + a), *s = reinterpret_cast<const float4*>(t + half + a);
      const float4 c0 = c[0], c1 = c[1], s0 = s[0], s1 = s[1];
      const float cc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
      const float ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i] = cc[i], sn[i] = sign * ss[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = 1.f, sn[i] = 0.f;
  }
  const uint16_t* wp = kind == 0 ? p.qw : kind == 1 ? p.kw : nullptr;
  float w[8];
  if (wp) unpack8(*reinterpret_cast<const uint4*>(wp + d0), w);
  // the lane that holds the other channels of this lane's pairs
  const int other = !turns || PAIRS ? lane : (d0 < p.rot / 2 ? lane + p.rot / 16 : lane - p.rot / 16);

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

  constexpr int kBatch = 4;  // loads in flight per lane
  for (int it = 0; it < p.iters; it += kBatch) {
    uint4 in[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + (it + j) * GW;
      in[j] = make_uint4(0, 0, 0, 0);
      if (it + j < p.iters && h < h1) in[j] = *reinterpret_cast<const uint4*>(src + (int64_t)h * D + d0);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + (it + j) * GW;
      if (it + j >= p.iters || h - gi >= h1) break;  // the same in the whole warp
      float x[8];
      unpack8(in[j], x);
      if (wp) {
        float s = __fadd_rn(__fadd_rn(__fadd_rn(__fmul_rn(x[0], x[0]), __fmul_rn(x[1], x[1])),
                                      __fadd_rn(__fmul_rn(x[2], x[2]), __fmul_rn(x[3], x[3]))),
                            __fadd_rn(__fadd_rn(__fmul_rn(x[4], x[4]), __fmul_rn(x[5], x[5])),
                                      __fadd_rn(__fmul_rn(x[6], x[6]), __fmul_rn(x[7], x[7]))));
#pragma unroll
        for (int d = 1; d < LH; d <<= 1) s = __fadd_rn(s, __shfl_xor_sync(0xffffffffu, s, d));
        const float rs = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fmul_rn(s, 1.f / D), p.eps)));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fmul_rn(__fmul_rn(x[i], rs), w[i]);
      }
      if (kind < 2) {
        // a * cos - b * sin and b * cos + a * sin: the sign of a product or a sum of rounded
        // products changes no bit of it
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = PAIRS ? x[i ^ 1] : __shfl_sync(0xffffffffu, x[i], other);
        if (turns) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __fadd_rn(__fmul_rn(x[i], cs[i]), __fmul_rn(y[i], sn[i]));
        }
      }
      const bool there = h < h1;
      if (kind == 0) {
        if (there)
          *reinterpret_cast<uint4*>(p.q_out + ((int64_t)token * p.heads + h) * D + d0) = pack8(x);
      } else if constexpr (CACHE) {
        __half2 par;
        const uint32_t n = quantize<LH>(x, &par);
        if (there && codes) {
          *reinterpret_cast<uint32_t*>(codes + h * block) = n;
          if (gl == 0) *reinterpret_cast<__half2*>(reinterpret_cast<uint8_t*>(params) + h * block) = par;
        }
      } else {
        if (there)
          *reinterpret_cast<uint4*>(p.k_out + ((int64_t)token * p.kv_heads + h) * D + d0) = pack8(x);
      }
    }
  }
}

// Rows of the cache as bf16: D / 8 lanes per (slot, head).
template <int D>
__global__ void __launch_bounds__(256) read_kernel(Kv4 c, const int64_t* __restrict__ slots, int64_t n,
                                                   uint4* __restrict__ k_out, uint4* __restrict__ v_out,
                                                   int32_t* status) {
  constexpr int LH = D / 8;
  pdl_wait();
  const int64_t rows = n * c.heads;
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < rows * LH; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / LH;
    const int gl = (int)(i % LH);
    const int64_t slot = slots[row / c.heads];
    const int h = (int)(row % c.heads);
    uint32_t code[2] = {0, 0};
    __half2 par[2] = {__half2half2(__ushort_as_half(0)), __half2half2(__ushort_as_half(0))};
    if (slot >= c.pages << c.shift) set_status(status, kStatusBadIndex);
    if (slot >= 0 && slot < c.pages << c.shift) {
      const int in = (int)(slot & ((1 << c.shift) - 1));
      const uint8_t* b = c.data + ((slot >> c.shift) * c.heads + h) * kv4_block_bytes<D>(c.shift);
      code[0] = *reinterpret_cast<const uint32_t*>(b + in * (D / 2) + gl * 4);
      code[1] = *reinterpret_cast<const uint32_t*>(b + kv4_value_codes<D>(c.shift) + in * (D / 2) + gl * 4);
      par[0] = *(reinterpret_cast<const __half2*>(b + kv4_key_params<D>(c.shift)) + in);
      par[1] = *(reinterpret_cast<const __half2*>(b + kv4_value_params<D>(c.shift)) + in);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float s = __low2float(par[w]), m = __high2float(par[w]);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = fmaf(s, (float)((code[w] >> (4 * j)) & 15u), m);  // s * n is exact
      (w ? v_out : k_out)[i] = pack8(x);
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

template <int D>
sp_status launch_rope(const RopeParams& p, bool pairs, bool cache, int64_t warps, cudaStream_t stream) {
  auto kern = cache ? (pairs ? rope_kernel<D, true, true> : rope_kernel<D, false, true>)
                    : (pairs ? rope_kernel<D, true, false> : rope_kernel<D, false, false>);
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
  const int gw = 32 / ((int)dim / 8);
  const int64_t nq = (a->heads + gw - 1) / gw, nk = (a->kv_heads + gw - 1) / gw;
  const int64_t total = a->tokens * (nq + (a->cache ? 2 : 1) * nk);
  const int64_t iters = total / ((int64_t)sms * 48);
  p.iters = (int32_t)(iters < 1 ? 1 : iters > 16 ? 16 : iters);
  p.uq = (int32_t)((nq + p.iters - 1) / p.iters);
  p.uk = (int32_t)((nk + p.iters - 1) / p.iters);
  p.units = p.uq + (a->cache ? 2 : 1) * p.uk;
  const int64_t warps = (int64_t)a->tokens * p.units;
  if (warps / (kRopeThreads / 32) >= ((int64_t)1 << 31) - 1) return SP_ERR_UNSUPPORTED;
  return dim == 64 ? launch_rope<64>(p, a->pairs != 0, a->cache != nullptr, warps, (cudaStream_t)stream)
                   : launch_rope<128>(p, a->pairs != 0, a->cache != nullptr, warps, (cudaStream_t)stream);
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
  const int64_t lanes = n * c->kv_heads * (c->head_dim / 8);
  const int64_t want = (lanes + 255) / 256, most = (int64_t)sms * 8;
  const dim3 grid((unsigned)(want < most ? want : most));
  auto kern = c->head_dim == 64 ? read_kernel<64> : read_kernel<128>;
  return launch_pdl(kern, grid, 256, 0, 1, (cudaStream_t)stream, kv4_view(c), slots, n, static_cast<uint4*>(k_out),
                    static_cast<uint4*>(v_out), device_status_ptr());
}

}  // extern "C"
