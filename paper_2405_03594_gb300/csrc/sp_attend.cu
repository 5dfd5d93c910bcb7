// sp_attend.cu -- attention over the cache held in 4 bits (include/sp_serve.h): single tokens and
// short runs of tokens of many requests.
//
// Mathematics.  With codes n, scale s and minimum m per key, and c = scale * log2(e):
//     log2 score   = c s_k (q . n) + c m_k sum(q)
//     out          = (sum_k (p_k s_k) (n - 8) + sum_k p_k (m_k + 8 s_k)) / sum_k p_k
// so the products run on the codes themselves, which bf16 holds exactly, and no value is rounded:
// the queries are bf16 already, and p_k s_k enters as the sum of two bf16 numbers.  The codes of
// the keys enter as 128 + n (a code's bits under the exponent of 128), and 128 s_k moves into m_k;
// over a long context that offset would swamp the fp32 sums of the values, which take n - 8.
//
// Layout.  A warp takes units of 32 keys.  Both products have the codes as the wide operand of
// m16n8k16 (keys, then channels, along M) and up to 8 NT query rows -- the heads that share the key
// head, times the new tokens -- along N.  The channels of a key, and the keys of a channel, may be
// taken in any order in a sum, so each lane's operand is the 16 consecutive bytes of a key (keys) or
// 8 of four keys (values) that it loads from global memory in one go: no shared memory, no shuffle.
// The scores' transposition between the products is movmatrix.
//
// Split.  The units of all requests, key heads and row tiles form one list, cut into equal ranges,
// one per CTA, whatever the lengths of the requests are; the warps of a CTA share each segment (the
// units of one request, head and row tile) and join their maxima and sums in shared memory.  A
// segment that several CTAs share is joined from the workspace, in their order, by the last of them.
#include <algorithm>

#include "sp_kv4.cuh"
#include "sp_lookup.h"

namespace sp {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kCtasPerSm = 3;
constexpr int kMinUnits = 2 * kWarps;  // units of a CTA, before more CTAs share the work
constexpr int kMaxDevices = 64;

struct AttendParams {
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;
  Kv4 cache;
  const int32_t *table, *lens, *cu_q, *work;
  int32_t requests, width, group;
  int32_t max_new;
  int64_t tokens;
  float scale_log2;
  float* part;  // [2 grid][8 NT] of (D sums, maximum, sum of weights, unused)
  int* cnt;     // [grid]
  int32_t* status;
};

__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// bf16 pair (128 + n_i, 128 + n_{i+4}) of the nibbles i and i + 4 of w
__device__ __forceinline__ uint32_t codes128(uint32_t w, int i) { return ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u; }
// bf16 pair (n - 8) of the same nibbles
__device__ __forceinline__ uint32_t codes8(uint32_t w, int i) {
  const uint32_t x = codes128(w, i);
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x43084308u));  // 136
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The codes and parameters of one unit, as a lane holds them.
template <int D>
struct UnitK {
  uint32_t w[2][2][D / 32];  // [16 keys][key g, g + 8][words: channels D/4 t ...]
  uint32_t par[2][2];
};
template <int D>
struct UnitV {
  uint32_t w[2][4][D / 64];  // [16 keys][keys 2t, 2t + 1, 2t + 8, 2t + 9][words: channels D/8 g ...]
  uint32_t par[2][2];        // of keys g, g + 8
};

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

// A segment: units [u0, u1) of `units` of one request, key head and row tile.
struct Segment {
  int b, h, rt;
  int units, u0, u1;
  int rows;       // query rows of the tile
  int row0;       // first of them among the request's
  int fresh, len;
};

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? kCtasPerSm : 2)
    attend_kernel(const __grid_constant__ AttendParams p) {
  constexpr int KW = D / 32, VW = D / 64;  // words of a lane: keys, values
  constexpr int MT = D / 16;               // channel tiles
  constexpr int R = 8 * NT;                // query rows
  extern __shared__ __align__(16) float smem[];  // [kWarps][R][D] sums, then [kWarps][R] (maximum, weights, offset)
  __shared__ int s_last;
  float* s_o = smem;
  float4* s_stat = reinterpret_cast<float4*>(smem + kWarps * R * D);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  pdl_wait();

  const int64_t total = (int64_t)p.work[p.requests] * p.cache.heads;
  const int64_t ctas = max((int64_t)1, min((int64_t)gridDim.x, total / kMinUnits));
  if (blockIdx.x >= ctas) return;
  const int64_t w0 = range_begin(blockIdx.x, total, ctas), w1 = range_begin(blockIdx.x + 1, total, ctas);
  const int shift = p.cache.shift;
  const int64_t block = kv4_block_bytes<D>(shift);

  int b = 0;
  if (w0 < w1) {  // the request of the first unit
    int lo = 0, hi = p.requests;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((int64_t)p.work[mid] * p.cache.heads <= w0) lo = mid;
      else hi = mid;
    }
    b = lo;
  }
  for (int64_t w = w0; w < w1;) {
    while (b + 1 < p.requests && (int64_t)p.work[b + 1] * p.cache.heads <= w) ++b;
    Segment s;
    s.b = b;
    s.len = p.lens[b];
    const int q0 = p.cu_q[b];
    s.fresh = p.cu_q[b + 1] - q0;
    const int64_t base = (int64_t)p.work[b] * p.cache.heads, next = (int64_t)p.work[b + 1] * p.cache.heads;
    s.units = (int)(((int64_t)s.len + kUnitKeys - 1) / kUnitKeys);
    // shares that do not belong to these lengths are passed over by every CTA alike
    const int64_t tiles = ((int64_t)s.fresh * p.group + kRowTile - 1) / kRowTile;
    if (w < base || next <= w || s.units <= 0 || tiles <= 0 || tiles * s.units * p.cache.heads != next - base) {
      if (tid == 0) set_status(p.status, kStatusBadIndex);
      if (next <= w) break;
      w = next;
      continue;
    }
    const int64_t idx = (w - base) / s.units;  // (row tile, key head)
    s.u0 = (int)((w - base) - idx * s.units);
    s.u1 = (int)min((int64_t)s.units, s.u0 + (w1 - w));
    s.h = (int)(idx % p.cache.heads);
    s.rt = (int)(idx / p.cache.heads);
    s.row0 = s.rt * kRowTile;
    s.rows = min(s.fresh * p.group - s.row0, kRowTile);
    if (s.fresh > p.max_new || q0 < 0 || q0 + (int64_t)s.fresh > p.tokens) {
      if (tid == 0) set_status(p.status, kStatusBadIndex);
      s.rows = 0;
    }
    const int rows = min(s.rows, R);
    const int64_t seg0 = w - s.u0;  // the segment's first unit in the list, with other CTAs' shares
    w += s.u1 - s.u0;

    // queries: operand registers, and sums over the channels
    uint32_t qf[NT][KW][4];
    float qsum[NT][2];
    int limit[NT][2];  // keys seen by query rows 2t, 2t + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 8 + g;
      float sum = 0.f;
      const int row = s.row0 + r;
      const uint16_t* src = p.q + (q0 + row / p.group) * p.q_stride + (int64_t)(s.h * p.group + row % p.group) * D + t * (D / 4);
#pragma unroll
      for (int i = 0; i < KW; ++i) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r < rows) u = *(reinterpret_cast<const uint4*>(src) + i);
        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += __uint_as_float(x[j] << 16) + __uint_as_float(x[j] & 0xffff0000u);
        qf[nt][i][0] = __byte_perm(u.x, u.z, 0x5410);  // channels 0, 4
        qf[nt][i][1] = __byte_perm(u.x, u.z, 0x7632);  // 1, 5
        qf[nt][i][2] = __byte_perm(u.y, u.w, 0x5410);  // 2, 6
        qf[nt][i][3] = __byte_perm(u.y, u.w, 0x7632);  // 3, 7
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        qsum[nt][c] = __shfl_sync(0xffffffffu, sum, 4 * (2 * t + c)) * p.scale_log2;
        const int rr = nt * 8 + 2 * t + c;
        limit[nt][c] = rr < rows ? s.len - s.fresh + (s.row0 + rr) / p.group + 1 : 0;
      }
    }
    const int most = rows > 0 ? s.len - s.fresh + (s.row0 + rows - 1) / p.group + 1 : 0;  // keys that any row sees

    float o[NT][MT][4];
    float mx[NT][2], l[NT][2], off[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
#pragma unroll
      for (int c = 0; c < 2; ++c) mx[nt][c] = -INFINITY, l[nt][c] = 0.f, off[nt][c] = 0.f;
    }

    const int u_end = min(s.u1, (most + kUnitKeys - 1) / kUnitKeys);
    const int32_t* table = p.table + (int64_t)s.b * p.width;
    // block of the 16 keys from k0 on; null behind the last key (or for a page that does not exist)
    auto block_of = [&](int k0) -> const uint8_t* {
      if (k0 >= most) return nullptr;
      const int page = (k0 >> shift) < p.width ? table[k0 >> shift] : -1;
      if (page < 0 || page >= p.cache.pages) {
        set_status(p.status, kStatusBadIndex);
        return nullptr;
      }
      return p.cache.data + ((int64_t)page * p.cache.heads + s.h) * block;
    };
    auto load_k = [&](UnitK<D>& k, int u) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k0 = u * kUnitKeys + 16 * i;
        const uint8_t* bl = block_of(k0);
        const int in = (k0 & ((1 << shift) - 1)) + g;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (bl) {
            load_words<KW>(k.w[i][j], bl + (in + 8 * j) * (D / 2) + t * (D / 8));
            k.par[i][j] = *(reinterpret_cast<const uint32_t*>(bl + kv4_key_params<D>(shift)) + in + 8 * j);
          } else {
#pragma unroll
            for (int x = 0; x < KW; ++x) k.w[i][j][x] = 0;
            k.par[i][j] = 0;
          }
        }
      }
    };
    auto load_v = [&](UnitV<D>& v, int u) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k0 = u * kUnitKeys + 16 * i;
        const uint8_t* bl = block_of(k0);
        const int in = k0 & ((1 << shift) - 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (bl) {
            load_words<VW>(v.w[i][j],
                           bl + kv4_value_codes<D>(shift) + (in + 2 * t + (j & 1) + 8 * (j >> 1)) * (D / 2) + g * (D / 16));
          } else {
#pragma unroll
            for (int x = 0; x < VW; ++x) v.w[i][j][x] = 0;
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
          v.par[i][j] = bl ? *(reinterpret_cast<const uint32_t*>(bl + kv4_value_params<D>(shift)) + in + g + 8 * j) : 0u;
      }
    };

    UnitK<D> kn;
    int u = s.u0 + warp;
    if (u < u_end) load_k(kn, u);
    for (; u < u_end; u += kWarps) {
      const UnitK<D> k = kn;
      UnitV<D> v;
      load_v(v, u);
      if (u + kWarps < u_end) load_k(kn, u + kWarps);

      float x[NT][2][4];  // scores: [16 keys][key g row 2t, row 2t + 1, key g + 8 ...]
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) x[nt][i][0] = x[nt][i][1] = x[nt][i][2] = x[nt][i][3] = 0.f;
#pragma unroll
        for (int j = 0; j < KW; ++j) {
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const uint32_t a0 = codes128(k.w[i][0][j], 2 * hh), a1 = codes128(k.w[i][1][j], 2 * hh);
            const uint32_t a2 = codes128(k.w[i][0][j], 2 * hh + 1), a3 = codes128(k.w[i][1][j], 2 * hh + 1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              mma_bf16(x[nt][i], a0, a1, a2, a3, qf[nt][j][2 * hh], qf[nt][j][2 * hh + 1]);
          }
        }
      }
      float ks[2][2], km[2][2], vs[2][2], vm[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 kp = __half22float2(*reinterpret_cast<const __half2*>(&k.par[i][j]));
          const float2 vp = __half22float2(*reinterpret_cast<const __half2*>(&v.par[i][j]));
          ks[i][j] = kp.x * p.scale_log2;
          km[i][j] = fmaf(-128.f, kp.x, kp.y);
          vs[i][j] = vp.x;
          vm[i][j] = fmaf(8.f, vp.x, vp.y);
        }
      uint32_t hi[NT][2][2], lo[NT][2][2];  // p s, transposed: rows g of the tile, keys 2t, 2t + 1 (+ 8)
      const int key = u * kUnitKeys + g;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        bool in[2][2][2];
        float top[2] = {mx[nt][0], mx[nt][1]};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              in[i][j][c] = key + 16 * i + 8 * j < limit[nt][c];
              float& y = x[nt][i][2 * j + c];
              y = in[i][j][c] ? fmaf(ks[i][j], y, km[i][j] * qsum[nt][c]) : -INFINITY;
              top[c] = fmaxf(top[c], y);
            }
        float alpha[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 4));
          top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 8));
          top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 16));
          const float safe = top[c] == -INFINITY ? 0.f : top[c];
          alpha[c] = exp2_approx(mx[nt][c] - safe);
          mx[nt][c] = top[c];
          top[c] = safe;
          l[nt][c] *= alpha[c];
          off[nt][c] *= alpha[c];
        }
        if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            o[nt][i][0] *= alpha[0], o[nt][i][1] *= alpha[1];
            o[nt][i][2] *= alpha[0], o[nt][i][3] *= alpha[1];
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float ps[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const float e = exp2_approx(x[nt][i][2 * j + c] - top[c]);
              l[nt][c] += e;
              // what a row does not see may hold anything, in its parameters too
              if (in[i][j][c]) off[nt][c] = fmaf(e, vm[i][j], off[nt][c]);
              ps[c] = in[i][j][c] ? e * vs[i][j] : 0.f;
            }
            const uint32_t h2 = pack_bf16(ps[0], ps[1]);
            const uint32_t l2 =
                pack_bf16(ps[0] - __uint_as_float(h2 << 16), ps[1] - __uint_as_float(h2 & 0xffff0000u));
            hi[nt][i][j] = transpose8x8(h2);
            lo[nt][i][j] = transpose8x8(l2);
          }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int y = 0; y < VW; ++y) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t sel = half ? 0x7632u : 0x5410u;
            const uint32_t w01 = __byte_perm(v.w[i][0][y], v.w[i][1][y], sel);
            const uint32_t w23 = __byte_perm(v.w[i][2][y], v.w[i][3][y], sel);
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const uint32_t a0 = codes8(w01, 2 * z), a1 = codes8(w01, 2 * z + 1);
              const uint32_t a2 = codes8(w23, 2 * z), a3 = codes8(w23, 2 * z + 1);
              const int mt = 4 * y + 2 * half + z;  // channels D/8 g + 2 mt (rows g), + 1 (rows g + 8)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_bf16(o[nt][mt], a0, a1, a2, a3, hi[nt][i][0], hi[nt][i][1]);
                mma_bf16(o[nt][mt], a0, a1, a2, a3, lo[nt][i][0], lo[nt][i][1]);
              }
            }
          }
        }
      }
    }

    // join the warps: sums to shared memory as (row, channel)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], d);
          off[nt][c] += __shfl_xor_sync(0xffffffffu, off[nt][c], d);
        }
        const int r = nt * 8 + 2 * t + c;
        float* dst = s_o + (warp * R + r) * D + g * (D / 8);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          *reinterpret_cast<float2*>(dst + 2 * mt) = make_float2(o[nt][mt][c] + off[nt][c], o[nt][mt][2 + c] + off[nt][c]);
        if (g == 0) s_stat[warp * R + r] = make_float4(mx[nt][c], l[nt][c], 0.f, 0.f);
      }
    }
    __syncthreads();
    const bool whole = s.u0 == 0 && s.u1 == s.units;
    // CTAs of the segment: the first of them counts the arrivals
    const int64_t first = whole ? blockIdx.x : owner_of(seg0, total, ctas);
    const int64_t last = whole ? blockIdx.x : owner_of(seg0 + s.units - 1, total, ctas);
    const int64_t slot = (int64_t)blockIdx.x * 2 + (s.u0 > 0 ? 0 : 1);
    constexpr int kPart = D + 4;
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) m = fmaxf(m, s_stat[k * R + r].x);
      const float safe = m == -INFINITY ? 0.f : m;
      float sum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float4 st = s_stat[k * R + r];
        const float f = exp2_approx(st.x - safe);
        const float4 a = *reinterpret_cast<const float4*>(s_o + (k * R + r) * D + d);
        sum = fmaf(st.y, f, sum);
        acc.x = fmaf(a.x, f, acc.x), acc.y = fmaf(a.y, f, acc.y);
        acc.z = fmaf(a.z, f, acc.z), acc.w = fmaf(a.w, f, acc.w);
      }
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int row = s.row0 + r;
        uint16_t* dst = p.out + (q0 + row / p.group) * p.out_stride + (int64_t)(s.h * p.group + row % p.group) * D + d;
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
      } else {
        float* dst = p.part + (slot * R + r) * kPart;
        __stcg(reinterpret_cast<float4*>(dst + d), acc);
        if (d == 0) __stcg(reinterpret_cast<float4*>(dst + D), make_float4(m, sum, 0.f, 0.f));
      }
    }
    if (!whole) {
      __threadfence();
      __syncthreads();
      if (tid == 0) s_last = atomicAdd(&p.cnt[first], 1) == (int)(last - first) ? 1 : 0;
      __syncthreads();
      if (s_last) {
        __threadfence();
        const int n = (int)(last - first) + 1;
        // a thread per (row, four channels): two passes over the parts, maxima first
        for (int i = tid; i < rows * (D / 4); i += kThreads) {
          const int r = i / (D / 4), d = i % (D / 4) * 4;
          auto part = [&](int k) { return p.part + (((first + k) * 2 + (k == 0 ? 1 : 0)) * R + r) * kPart; };
          float m = -INFINITY;
#pragma unroll 4
          for (int k = 0; k < n; ++k) m = fmaxf(m, __ldcg(part(k) + D));
          const float safe = m == -INFINITY ? 0.f : m;
          float sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int k = 0; k < n; ++k) {
            const float* src = part(k);
            const float2 st = __ldcg(reinterpret_cast<const float2*>(src + D));
            const float4 a = __ldcg(reinterpret_cast<const float4*>(src + d));
            const float f = exp2_approx(st.x - safe);
            sum = fmaf(st.y, f, sum);
            acc.x = fmaf(a.x, f, acc.x), acc.y = fmaf(a.y, f, acc.y);
            acc.z = fmaf(a.z, f, acc.z), acc.w = fmaf(a.w, f, acc.w);
          }
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          const int row = s.row0 + r;
          uint16_t* dst = p.out + (q0 + row / p.group) * p.out_stride + (int64_t)(s.h * p.group + row % p.group) * D + d;
          *reinterpret_cast<uint2*>(dst) =
              make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
        }
        if (tid == 0) atomicExch(&p.cnt[first], 0);
      }
    }
    __syncthreads();  // shared memory is free for the next segment
  }
}

template <int D, int NT>
constexpr size_t smem_bytes() {
  return (size_t)kWarps * 8 * NT * (D + 4) * sizeof(float);
}

// CTAs of a full grid; 0 if a lookup failed.
template <int D, int NT>
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
    if (cudaFuncSetAttribute(attend_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)smem_bytes<D, NT>()) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, attend_kernel<D, NT>, kThreads, smem_bytes<D, NT>()) !=
            cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    return n * sms;
  });
}

constexpr int kMaxCtasPerSm = 4;

size_t workspace_bytes(int head_dim, int sms) {
  const size_t ctas = (size_t)kMaxCtasPerSm * sms;
  return ws_counter_bytes(sms) + ctas * 2 * kRowTile * (size_t)(head_dim + 4) * sizeof(float);
}

template <int D, int NT>
sp_status launch(AttendParams p, cudaStream_t stream) {
  const int ctas = grid_of<D, NT>();
  if (ctas == 0) return SP_ERR_CUDA;
  return launch_pdl(attend_kernel<D, NT>, dim3((unsigned)std::min(ctas, kMaxCtasPerSm * current_sms())), kThreads,
                    smem_bytes<D, NT>(), 1, stream, p);
}

}  // namespace
}  // namespace sp

using namespace sp;

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
  p.max_new = a->max_new;
  p.tokens = a->tokens;
  p.scale_log2 = a->scale * 1.4426950408889634f;
  p.cnt = static_cast<int*>(workspace_dev);
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace_dev) + ws_counter_bytes(sms));
  p.status = device_status_ptr();
  const int64_t rows = std::min<int64_t>((int64_t)a->max_new * p.group, kRowTile);
  const int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  cudaStream_t s = (cudaStream_t)stream;
  if (d == 64) return nt == 1 ? launch<64, 1>(p, s) : nt == 2 ? launch<64, 2>(p, s) : launch<64, 4>(p, s);
  return nt == 1 ? launch<128, 1>(p, s) : nt == 2 ? launch<128, 2>(p, s) : launch<128, 4>(p, s);
}

}  // extern "C"
