// sp_fp8_few.cu -- y = x . W^T in e4m3 with a scale for each block of 128, for few tokens (include/sp_fp8.h).
//
// Bound by reading W once. A tile is 128 rows of W (the lanes of tensor memory) by MT tokens (its columns), so that
// W is the tensor cores' first operand and few tokens waste no time there. The blocks of a tile's rows are shared by the
// CTAs of a cluster, as many as fill the machine; each holds 80 kilobytes of W in flight (64 with tiles of 64 tokens), two of them on an SM, and
// their sums meet through the cluster's shared memory, in order. Nothing goes through global memory but
// W, x and y:
//   producer    W's tiles by TMA into a ring, asked into L2 before the launch before this one has ended; of quantised x its
//               tiles and scales too
//   quantisers  (where few_fused says so) four warps, x's blocks: a row's 128 entries held by 16 lanes, its codes
//               written to where the tensor cores read them (row r's 16-byte piece j lies at j ^ (r & 7)), its scale beside
//               them. Every tile does that again, so that more tokens are quantised once, by a launch before
//   products    a block's 128 columns in tensor memory, of a stage's own columns
//   epilogue    four warps, thread = row of W: the block's sums times sx * sw, added up in registers
//
// Measured, us and W's rate: 1 x 4096 x 4096 5.9 (2.8 TB/s: the launch, the first blocks' way in, the cluster's two barriers), 1 x 32000 x 4096
// 22.3 (5.9 TB/s), 16 x 32000 x 4096 23.8 with the launch that quantises (131.2 MB from memory), 64 x 32000 x 4096 26.9 (33.4 with one CTA of eight stages to an SM). With partial sums
// through the workspace and x quantised by a launch before, the first two took 13.7 and 28.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>

#include "sp_fp8.cuh"

namespace sp {
namespace {

constexpr int kTileN = 128;
constexpr uint32_t kWBytes = kTileN * 128;
// warps: epilogue 0-3, producer 4, products 5, quantisers 6-9
constexpr int kMostStages = 5;
constexpr int kFewCluster = 8;  // (few_cluster)
constexpr uint32_t kCtl = 512;

template <int MT, bool FUSED>
struct FewPlan {
  static constexpr int kThreads = FUSED ? 320 : 192;
  static constexpr int kStages = MT <= 32 ? 5 : 4;
  static constexpr uint32_t kTmem = MT == 16 ? 128 : 256;
  static constexpr uint32_t kStage = kWBytes + MT * 128;
  static constexpr uint32_t kScales = (kStages * MT * 4 + 511) / 512 * 512;
  static constexpr uint32_t kSmem = 1024 + kCtl + kScales + 512 + kStages * kStage;  // (1024: alignment)
};

struct FewParams {
  const float* w_scale;
  const uint16_t* x;
  const float* x_scale;
  uint16_t* y;
  int64_t x_stride, x_scale_stride, y_stride;
  int64_t n, k;
  int32_t m, blocks, cluster;
  int32_t wide;  // rows of x start at multiples of 16 bytes
  int* status;
  uint64_t timeout_ns;
  int32_t expire_cta, expire_warp, expire_block;  // in the variants of sp_test_expired_fp8
};

// kExpire: a variant for sp_test_expired_fp8, whose warp p.expire_warp of CTA p.expire_cta waits, before its block p.expire_block, for
// what never comes, and gives up.
template <int MT, bool FUSED, bool kExpire = false>
__global__ void __launch_bounds__(FewPlan<MT, FUSED>::kThreads, kFewCtas)
    fp8_few_kernel(const __grid_constant__ FewParams p, const __grid_constant__ CUtensorMap tmap_w,
                   const __grid_constant__ CUtensorMap tmap_x) {
  using P = FewPlan<MT, FUSED>;
  constexpr int S = P::kStages;
  extern __shared__ uint8_t smem_raw[];
  // the same offset in every CTA of the cluster: dynamic shared memory starts at one address
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* w_full = reinterpret_cast<uint64_t*>(smem);  // the copies have landed
  uint64_t* x_full = w_full + kMostStages;               // x's block is quantised
  uint64_t* done = x_full + kMostStages;                 // the block's sums are complete
  uint64_t* freed = done + kMostStages;                  // and taken out
  uint64_t* drain = freed + kMostStages;                 // no product is under way
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  uint64_t* never = drain + 2;                           // (kExpire) nothing completes it
  float* scales = reinterpret_cast<float*>(smem + kCtl);  // [S][MT]
  uint8_t* ring = smem + (kCtl + P::kScales + 1023) / 1024 * 1024;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = p.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t nt = blockIdx.x / p.cluster;
  const int b0 = (int)((int64_t)p.blocks * rank / p.cluster), b1 = (int)((int64_t)p.blocks * (rank + 1) / p.cluster);
  if (tid == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&w_full[s], 1);
      mbar_init(&x_full[s], 4);
      mbar_init(&done[s], 1);
      mbar_init(&freed[s], 4);
    }
    mbar_init(drain, 1);
    if constexpr (kExpire) mbar_init(never, 1);
    fence_barrier_init();
  }
  if (warp == 5) {
    tmem_alloc(tmem_slot, P::kTmem);
    tmem_relinquish();
  }
  if (warp == 4 && lane == 0) {
    prefetch_tmap(&tmap_w);
    if constexpr (!FUSED) prefetch_tmap(&tmap_x);
    for (int b = b0; b < min(b1, b0 + S); ++b) tma_prefetch_2d(&tmap_w, b * 128, (int)(nt * kTileN));
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // (once every CTA of this launch has its tensor memory: the next launch's may then wait for some of theirs)
  pdl_launch_dependents();

  if (warp == 4) {
    if (lane == 0) {
      // ---------------------------------------------------------- producer
      pdl_wait();
      int s = 0;
      uint32_t ph = 0;
      bool dead = false;
      int issued = 0;
      for (int b = b0; b < b1; ++b) {
        if (gives_up<kExpire>(p, b - b0, never) || !mbar_wait_short(&freed[s], ph ^ 1u, p.timeout_ns)) {
          dead = true;
          break;
        }
        uint8_t* st = ring + (size_t)s * P::kStage;
        if constexpr (FUSED) {
          mbar_arrive_expect_tx(&w_full[s], kWBytes);
        } else {
          const uint32_t sb = (uint32_t)imin64(MT, p.x_scale_stride) * 4;
          mbar_arrive_expect_tx(&w_full[s], P::kStage + sb);
          tma_load_2d(st + kWBytes, &tmap_x, b * 128, 0, &w_full[s]);
          bulk_g2s(scales + s * MT, p.x_scale + b * p.x_scale_stride, sb, &w_full[s]);
        }
        tma_load_2d(st, &tmap_w, b * 128, (int)(nt * kTileN), &w_full[s]);
        ++issued;
        if (++s == S) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (dead) set_status(p.status, kStatusTimeout);
      // the last copies, before the CTA's memory goes: whoever waited for them may have given up
      for (int i = max(0, issued - S); i < issued; ++i) mbar_wait(&w_full[i % S], (uint32_t)((i / S) & 1), p.timeout_ns);
    }
  } else if (warp == 5) {
    // ------------------------------------------------------------ products
    int s = 0;
    uint32_t ph = 0;
    for (int b = b0; b < b1; ++b) {
      bool ok = mbar_wait_short(&w_full[s], ph, p.timeout_ns);
      if constexpr (kExpire) ok = ok && !gives_up<kExpire>(p, b - b0, never);
      if constexpr (FUSED) ok = ok && mbar_wait_short(&x_full[s], ph, p.timeout_ns);
      if (!__all_sync(0xffffffffu, ok)) {
        if (lane == 0) set_status(p.status, kStatusTimeout);
        break;
      }
      tc_fence_after();
      const uint32_t w = smem_u32(ring + (size_t)s * P::kStage);
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          mma_fp8(tmem + (uint32_t)(s * MT), smem_desc_sw128(w + kk * 32u), smem_desc_sw128(w + kWBytes + kk * 32u),
                  idesc_e4m3(kTileN, MT), kk > 0 ? 1u : 0u);
        mma_commit(&done[s]);
      }
      __syncwarp();
      if (++s == S) {
        s = 0;
        ph ^= 1u;
      }
    }
    if (elect_one()) mma_commit(drain);
    __syncwarp();
    if (!mbar_wait_short(drain, 0, p.timeout_ns)) set_status(p.status, kStatusTimeout);
  } else if (warp >= 6) {
    // ------------------------------------------------------------ quantisers: units of two rows of a block, in turn
    pdl_wait();
    const int pairs = (p.m + 1) / 2, units = (b1 - b0) * pairs;
    const int l = lane & 15, hi = lane >> 4;
    auto ask = [&](int u) {
      const int b = b0 + u / pairs, r = u % pairs * 2 + hi;
      const int64_t c = (int64_t)b * kFp8Block + 8 * l;
      if (u >= units || r >= p.m || c >= p.k) return make_uint4(0, 0, 0, 0);
      const uint16_t* row = p.x + r * p.x_stride;
      return p.wide ? load8<true>(row, c, p.k) : load8<false>(row, c, p.k);
    };
    int s = 0, u = warp - 6;
    uint32_t ph = 0;
    uint4 next = ask(u);
    for (int b = b0; b < b1; ++b) {
      bool ok = mbar_wait_short(&freed[s], ph ^ 1u, p.timeout_ns);
      if constexpr (kExpire) ok = ok && !gives_up<kExpire>(p, b - b0, never);
      if (!__all_sync(0xffffffffu, ok)) {
        if (lane == 0) set_status(p.status, kStatusTimeout);
        break;
      }
      for (; u < (b - b0 + 1) * pairs; u += 4) {
        const uint4 v = next;
        next = ask(u + 4);
        const int r = u % pairs * 2 + hi;
        uint32_t a = largest_of(v);
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, d));
        const float sc = fp8_scale(a);
        const uint2 q = codes_of(v, __frcp_rn(sc));
        if (r < p.m) {
          uint8_t* row = ring + (size_t)s * P::kStage + kWBytes + r * 128;
          *reinterpret_cast<uint2*>(row + (((l >> 1) ^ (r & 7)) << 4) + ((l & 1) << 3)) = q;
          if (l == 0) scales[s * MT + r] = sc;
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&x_full[s]);
      if (++s == S) {
        s = 0;
        ph ^= 1u;
      }
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------ epilogue: thread = row of W
    const int64_t row = nt * kTileN + tid;
    const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
    const float* sw = p.w_scale + nt * p.blocks;
    uint64_t acc[MT / 2];
#pragma unroll
    for (int j = 0; j < MT / 2; ++j) acc[j] = 0;
    int s = 0;
    uint32_t ph = 0;
    bool dead = false;
    pdl_wait();  // y, and what this kernel shares with none, belong to the stream order
    float w = b0 < b1 ? __ldg(sw + b0) : 0.f;
    for (int b = b0; b < b1; ++b) {
      const float next = b + 1 < b1 ? __ldg(sw + b + 1) : 0.f;
      bool ok = mbar_wait_short(&done[s], ph, p.timeout_ns);
      if constexpr (kExpire) ok = ok && !gives_up<kExpire>(p, b - b0, never);
      ok = ok && mbar_wait_short(FUSED ? &x_full[s] : &w_full[s], ph, p.timeout_ns);  // (complete: for the scales)
      if (!__all_sync(0xffffffffu, ok)) {
        if (lane == 0) set_status(p.status, kStatusTimeout);
        dead = true;
        break;
      }
      tc_fence_after();
      const float4* sx = reinterpret_cast<const float4*>(scales + s * MT);
      const uint64_t w2 = two(w, w);
#pragma unroll
      for (int c = 0; c < MT; c += 16) {
        uint32_t d[16];
        tmem_load16(tmem + (uint32_t)(s * MT + c) + lane_base, d);
        float4 x4[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x4[j] = sx[c / 4 + j];
        tmem_load_wait();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          add_behind(acc[(c + 4 * j) / 2], d[4 * j], d[4 * j + 1], mul2(two(x4[j].x, x4[j].y), w2));
          add_behind(acc[(c + 4 * j) / 2 + 1], d[4 * j + 2], d[4 * j + 3], mul2(two(x4[j].z, x4[j].w), w2));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&freed[s]);
      w = next;
      if (++s == S) {
        s = 0;
        ph ^= 1u;
      }
    }
    if (p.cluster == 1) {
      uint16_t* yp = p.y + row;
#pragma unroll
      for (int j = 0; j < MT; j += 2) {
        float lo, hi;
        apart(acc[j / 2], lo, hi);
        if (row < p.n && j < p.m) yp[j * p.y_stride] = float_to_bf16_bits_rn(lo);
        if (row < p.n && j + 1 < p.m) yp[(j + 1) * p.y_stride] = float_to_bf16_bits_rn(hi);
      }
    } else {
      // (every product has read its stage: the ring is free, unless a wait has expired)
      float* part = reinterpret_cast<float*>(ring);  // [MT][kTileN]
      if (!dead) {
#pragma unroll
        for (int j = 0; j < MT; j += 2) {
          float lo, hi;
          apart(acc[j / 2], lo, hi);
          part[j * kTileN + tid] = lo, part[(j + 1) * kTileN + tid] = hi;
        }
      }
    }
  }
  tc_fence_before();
  if (p.cluster == 1) {
    __syncthreads();
  } else {
    __syncwarp();
    cluster_sync_all();
    if (warp < 4) {  // token j of the tile is this rank's where j % cluster is it: the ranks' sums in order
      const int64_t row = nt * kTileN + tid;
      const uint32_t at = smem_u32(ring) + (uint32_t)tid * 4;
      for (int j = rank; j < p.m; j += p.cluster) {
        float v[kFewCluster];
#pragma unroll
        for (int r = 0; r < kFewCluster; ++r)
          v[r] = r < p.cluster ? ld_cluster_f32(cluster_map(at + (uint32_t)(j * kTileN * 4), (uint32_t)r)) : 0.f;
        float sum = v[0];
#pragma unroll
        for (int r = 1; r < kFewCluster; ++r) sum += v[r];
        if (row < p.n) p.y[j * p.y_stride + row] = float_to_bf16_bits_rn(sum);
      }
    }
    __syncwarp();
    cluster_sync_all();  // the other CTAs have read this one's sums
  }
  if (warp == 5) {
    tc_fence_after();
    tmem_dealloc(tmem, P::kTmem);
  }
}

template <int MT, bool FUSED, bool kExpire = false>
sp_status launch(FewParams p, const CUtensorMap& map_w, const CUtensorMap& map_x, int sms, cudaStream_t stream) {
  using P = FewPlan<MT, FUSED>;
  if (cudaFuncSetAttribute(fp8_few_kernel<MT, FUSED, kExpire>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)P::kSmem) != cudaSuccess) {
    cudaGetLastError();
    return SP_ERR_CUDA;
  }
  const int64_t tiles = (p.n + kTileN - 1) / kTileN;
  p.cluster = few_cluster(p.m, p.n, p.blocks, sms);
  if (tiles * p.cluster > INT32_MAX) return SP_ERR_UNSUPPORTED;
  return launch_pdl(fp8_few_kernel<MT, FUSED, kExpire>, dim3((unsigned)(tiles * p.cluster)), P::kThreads, P::kSmem, p.cluster, stream, p,
                    map_w, map_x);
}

}  // namespace

sp_status launch_fp8_few(const sp_fp8_linear_args& a, const Fp8Rows* rows, const CUtensorMap& map_w, const CUtensorMap& map_x,
                         int sms, const Fp8Expire* expire, cudaStream_t stream) {
  FewParams p = {};
  p.w_scale = a.w_scale;
  p.x = static_cast<const uint16_t*>(a.x);
  p.x_scale = rows ? rows->scale : nullptr;
  p.y = static_cast<uint16_t*>(a.y);
  p.x_stride = a.x_stride;
  p.x_scale_stride = rows ? rows->scale_stride : 0;
  p.y_stride = a.y_stride;
  p.n = a.n;
  p.k = a.k;
  p.m = (int32_t)a.m;
  p.blocks = (int32_t)((a.k + kFp8Block - 1) / kFp8Block);
  p.wide = al16(a.x) && (a.m == 1 || a.x_stride % 8 == 0);
  p.status = device_status_ptr();
  p.timeout_ns = wait_timeout_ns();
  if (expire) {
    p.timeout_ns = expire->wait_ns;
    p.expire_cta = expire->cta, p.expire_warp = expire->warp, p.expire_block = expire->block;
    if (few_box(a.m) != 16) return SP_ERR_UNSUPPORTED;
    return rows ? launch<16, false, true>(p, map_w, map_x, sms, stream) : launch<16, true, true>(p, map_w, map_w, sms, stream);
  }
  if (!rows) return launch<16, true>(p, map_w, map_w, sms, stream);
  return few_box(a.m) == 16   ? launch<16, false>(p, map_w, map_x, sms, stream)
         : few_box(a.m) == 32 ? launch<32, false>(p, map_w, map_x, sms, stream)
                              : launch<64, false>(p, map_w, map_x, sms, stream);
}

}  // namespace sp
