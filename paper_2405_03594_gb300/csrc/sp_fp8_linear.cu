// sp_fp8_linear.cu -- y = x . W^T of weights and activations in e4m3 with a scale for each block of 128
// (include/sp_fp8.h).
//
// The tensor cores add up one block of 128 columns at a time, in tensor memory; the epilogue's threads take those sums
// out, multiply them by sx * sw, which changes from block to block, and add them up in registers. While they do, the next
// blocks' sums are made in other columns of tensor memory.
//
// fp8_pair_kernel (many tokens): pairs of SMs, 256 tokens (the lanes of tensor memory, 128 in each CTA) by NT rows of W. A
// thread's scale of a block is then one number, and a sum costs one FMA. A block's sums are read back from tensor
// memory by eight warps while the pair multiplies the next one.
//
// fp8_rows_kernel: a tile is 128 rows of W (the lanes of tensor memory) by MT tokens (its columns), so that few
// tokens waste no tensor time and a weight is read once. The tiles' blocks, all in a row, are cut into as many equal
// ranges as there are CTAs; a tile that is shared by several leaves its sums in the workspace, and the last CTA to
// arrive joins them in order.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "sp_fp8.cuh"
#include "sp_lookup.h"

namespace sp {
namespace {

constexpr int kMaxDevices = 64;
constexpr int kTileN = 128;               // rows of W in a tile
constexpr uint32_t kWBytes = kTileN * 128;  // of a block: 128 rows of 128 codes
constexpr int kMaxStages = 12;
constexpr int kAccs = 4;                  // sums of blocks in tensor memory at a time
constexpr uint32_t kCtl = 1024;

struct Fp8Params {
  const float *w_scale, *x_scale;
  uint16_t* y;
  int64_t y_stride, x_scale_stride;
  int64_t n, m;
  int32_t blocks;          // of 128 columns
  int32_t m_tiles;
  int64_t units;           // tiles * blocks
  int32_t stages;
  float* part;             // [2 grid][MT][kTileN]
  int* cnt;                // [grid]
  int* status;
  uint64_t timeout_ns;
};

template <int MT>
struct RowsPlan {
  static constexpr int kEpiWarps = MT >= 64 ? 8 : 4;
  static constexpr int kThreads = 128 + 32 * kEpiWarps;
  static constexpr int kColumns = MT * 4 / kEpiWarps;  // of a warp
  static constexpr uint32_t kTmem = MT * kAccs < 32 ? 32 : MT * kAccs;
  static constexpr uint32_t kStage = kWBytes + MT * 128;
  static constexpr uint32_t kScales = MT * 4;          // of a stage
  static constexpr uint32_t smem(int stages) { return 1024 + kCtl + (stages * kScales + 1023) / 1024 * 1024 + stages * kStage; }
};

template <int MT>
__global__ void __launch_bounds__(RowsPlan<MT>::kThreads, 1)
    fp8_rows_kernel(const __grid_constant__ Fp8Params p, const __grid_constant__ CUtensorMap tmap_w,
                    const __grid_constant__ CUtensorMap tmap_x) {
  using P = RowsPlan<MT>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem);
  uint64_t* empty = full + kMaxStages;     // the stage's products and scales are read
  uint64_t* d_full = empty + kMaxStages;   // a block's sums are complete
  uint64_t* d_empty = d_full + kAccs;      // they have been taken out
  uint64_t* drain = d_empty + kAccs;       // no product is under way
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* s_last = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* scales = reinterpret_cast<float*>(smem + kCtl);
  uint8_t* ring = smem + kCtl + (p.stages * P::kScales + 1023) / 1024 * 1024;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1 + P::kEpiWarps);
    }
    for (int b = 0; b < kAccs; ++b) {
      mbar_init(&d_full[b], 1);
      mbar_init(&d_empty[b], P::kEpiWarps);
    }
    mbar_init(drain, 1);
    fence_barrier_init();
  }
  if (warp == 2) {
    tmem_alloc(tmem_slot, P::kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int64_t G = gridDim.x, u0 = range_begin(blockIdx.x, p.units, G), u1 = range_begin(blockIdx.x + 1, p.units, G);

  if (warp == 0) {
    if (lane == 0) {
      // ---------------------------------------------------------- producer
      prefetch_tmap(&tmap_w);
      prefetch_tmap(&tmap_x);
      pdl_wait();
      int s = 0;
      uint32_t ph = 0;
      int64_t issued = 0;
      bool dead = false;
      for (int64_t u = u0; u < u1; ++u) {
        if (!mbar_wait_short(&empty[s], ph ^ 1u, p.timeout_ns)) {
          dead = true;
          break;
        }
        const int64_t tile = u / p.blocks, b = u % p.blocks, m0 = tile % p.m_tiles * MT, n0 = tile / p.m_tiles * kTileN;
        const uint32_t sb = (uint32_t)imin64(MT, p.x_scale_stride - m0) * 4;
        uint8_t* st = ring + (size_t)s * P::kStage;
        mbar_arrive_expect_tx(&full[s], P::kStage + sb);
        tma_load_2d(st, &tmap_w, (int)(b * 128), (int)n0, &full[s]);
        tma_load_2d(st + kWBytes, &tmap_x, (int)(b * 128), (int)m0, &full[s]);
        bulk_g2s(scales + s * MT, p.x_scale + b * p.x_scale_stride + m0, sb, &full[s]);
        ++issued;
        if (++s == p.stages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (dead) {  // the copies under way, before the CTA's memory goes
        set_status(p.status, kStatusTimeout);
        for (int64_t i = issued > p.stages ? issued - p.stages : 0; i < issued; ++i)
          mbar_wait_short(&full[i % p.stages], (uint32_t)((i / p.stages) & 1), p.timeout_ns);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ products
    int s = 0, a = 0;
    uint32_t ph = 0, aph = 0;
    for (int64_t u = u0; u < u1; ++u) {
      bool ok = mbar_wait_short(&d_empty[a], aph ^ 1u, p.timeout_ns);
      ok = ok && mbar_wait_short(&full[s], ph, p.timeout_ns);
      if (!__all_sync(0xffffffffu, ok)) {
        set_status(p.status, kStatusTimeout);
        break;
      }
      tc_fence_after();
      const uint32_t w = smem_u32(ring + (size_t)s * P::kStage);
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          mma_fp8(tmem + (uint32_t)(a * MT), smem_desc_sw128(w + kk * 32u), smem_desc_sw128(w + kWBytes + kk * 32u),
                  idesc_e4m3(kTileN, MT), kk > 0 ? 1u : 0u);
        mma_commit(&empty[s]);
        mma_commit(&d_full[a]);
      }
      __syncwarp();
      if (++s == p.stages) {
        s = 0;
        ph ^= 1u;
      }
      if (++a == kAccs) {
        a = 0;
        aph ^= 1u;
      }
    }
    if (elect_one()) mma_commit(drain);
    __syncwarp();
    if (!mbar_wait_short(drain, 0, p.timeout_ns)) set_status(p.status, kStatusTimeout);
  } else if (warp >= 4) {
    // ------------------------------------------------------------ epilogue: thread = row of W
    constexpr int C = P::kColumns;
    const int q = warp & 3, r = q * 32 + lane;
    const int col0 = (warp - 4) / 4 * C;
    const uint32_t lane_base = ((uint32_t)(q * 32) << 16) + (uint32_t)col0;
    const int epi_threads = P::kEpiWarps * 32;
    int s = 0, a = 0;
    uint32_t ph = 0, aph = 0;
    bool dead = false;
    pdl_wait();  // the scales and y belong to the stream order
    for (int64_t u = u0; u < u1;) {
      const int64_t tile = u / p.blocks, first = tile * p.blocks, end = imin64(first + p.blocks, u1);
      const int64_t m0 = tile % p.m_tiles * MT, nt = tile / p.m_tiles, row = nt * kTileN + r;
      const bool whole = u == first && end == first + p.blocks;
      uint64_t acc[C / 2];
#pragma unroll
      for (int j = 0; j < C / 2; ++j) acc[j] = 0;
      const float* sw = p.w_scale + nt * p.blocks;
      for (; u < end; ++u) {
        const float w = __ldg(sw + (u - first));
        if (!dead) {
          bool ok = mbar_wait_short(&d_full[a], aph, p.timeout_ns);
          ok = ok && mbar_wait_short(&full[s], ph, p.timeout_ns);  // (complete: the products have read the stage)
          if (!__all_sync(0xffffffffu, ok)) {
            if (lane == 0) set_status(p.status, kStatusTimeout);
            dead = true;
          }
        }
        if (!dead) {
          tc_fence_after();
          const float4* sx = reinterpret_cast<const float4*>(scales + s * MT + col0);
          const uint64_t w2 = two(w, w);
#pragma unroll
          for (int c = 0; c < C; c += 16) {
            uint32_t d[16];
            tmem_load16(tmem + (uint32_t)(a * MT + c) + lane_base, d);
            tmem_load_wait();
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
              const float4 x4 = sx[(c + j) / 4];
              acc[(c + j) / 2] = fma2(two(__uint_as_float(d[j]), __uint_as_float(d[j + 1])), mul2(two(x4.x, x4.y), w2), acc[(c + j) / 2]);
              acc[(c + j) / 2 + 1] = fma2(two(__uint_as_float(d[j + 2]), __uint_as_float(d[j + 3])), mul2(two(x4.z, x4.w), w2), acc[(c + j) / 2 + 1]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&d_empty[a]);
            mbar_arrive(&empty[s]);
          }
        }
        if (++s == p.stages) {
          s = 0;
          ph ^= 1u;
        }
        if (++a == kAccs) {
          a = 0;
          aph ^= 1u;
        }
      }
      float v[C];
#pragma unroll
      for (int j = 0; j < C / 2; ++j) apart(acc[j], v[2 * j], v[2 * j + 1]);
      if (!whole) {
        const int64_t c_first = owner_of(first, p.units, G), c_last = owner_of(first + p.blocks - 1, p.units, G);
        auto slot = [&](int64_t c) { return p.part + ((2 * c + (range_begin(c, p.units, G) >= first ? 0 : 1)) * MT + col0) * kTileN + r; };
        float* mine = slot(blockIdx.x);
#pragma unroll
        for (int j = 0; j < C; ++j) __stcg(mine + j * kTileN, v[j]);
        __threadfence();
        named_bar_sync(1, epi_threads);
        if (tid == 128) *s_last = atomicAdd(p.cnt + c_first, 1) == (int)(c_last - c_first) ? 1 : 0;
        named_bar_sync(1, epi_threads);
        const bool last = *s_last;
        named_bar_sync(1, epi_threads);  // (it is written again)
        if (!last) continue;
        __threadfence();
#pragma unroll
        for (int j = 0; j < C; ++j) v[j] = 0.f;
        for (int64_t c = c_first; c <= c_last; ++c) {
          const float* src = slot(c);
#pragma unroll
          for (int j = 0; j < C; ++j) v[j] += __ldcg(src + j * kTileN);
        }
        if (tid == 128) atomicExch(p.cnt + c_first, 0);
      }
      if (row < p.n) {
        uint16_t* yp = p.y + (m0 + col0) * p.y_stride + row;
        const int nv = (int)imin64(C, p.m - m0 - col0);
#pragma unroll
        for (int j = 0; j < C; ++j)
          if (j < nv) yp[j * p.y_stride] = float_to_bf16_bits_rn(v[j]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, P::kTmem);
  }
}

// ------------------------------------------------------------------ many tokens
constexpr int kPairTokens = 256;  // of a tile: 128 in each CTA
constexpr uint32_t kXBytes = 128 * 128;
constexpr uint32_t kStageBytes = 32 * 128;  // of y on its way out: 32 rows of 64 columns, a warp
constexpr int kPairEpi = 8;           // epilogue warps
constexpr int kPairThreads = 128 + 32 * kPairEpi;

template <int NT>  // rows of W in a tile
struct PairPlan {
  static constexpr int kAccs = NT == 256 ? 2 : 4;    // sums of blocks in tensor memory at a time
  static constexpr uint32_t kTmem = NT * kAccs;
  static constexpr uint32_t kStage = kXBytes + NT / 2 * 128;
  static constexpr uint32_t kStaging = kPairEpi * 2 * kStageBytes;
  static constexpr int kFit = (int)((227 * 1024 - 1024 - kCtl - kStaging) / kStage);
  static constexpr int kStages = kFit / kAccs * kAccs;  // so that a stage's block always has the same columns
  static constexpr uint32_t kSmem = 1024 + kCtl + kStages * kStage + kStaging;
};

struct PairParams {
  const float *w_scale, *x_scale;
  uint16_t* y;
  int64_t y_stride, x_scale_stride;
  int64_t n, m;
  int32_t blocks;
  int32_t m_tiles;
  int64_t tiles;
  int32_t y_tma;  // rows of y start at multiples of 16 bytes
  int* status;
  uint64_t timeout_ns;
};

template <int NT>
__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2, 1, 1)
    fp8_pair_kernel(const __grid_constant__ PairParams p, const __grid_constant__ CUtensorMap tmap_w,
                    const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_y) {
  using P = PairPlan<NT>;
  extern __shared__ uint8_t smem_raw[];
  // the same offset in both CTAs of the pair: dynamic shared memory starts at one address
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem);  // leader's: both CTAs' copies of a stage landed
  uint64_t* done = full + kMaxStages;                  // each CTA's: a stage's products are done, its sums complete
  uint64_t* d_empty = done + kMaxStages;               // leader's: both CTAs have taken the sums out
  uint64_t* drain = d_empty + 4;                       // leader's: no product is under way
  uint64_t* never = drain + 1;                         // nothing completes it
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(never + 1);
  uint8_t* ring = smem + kCtl;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (tid == 0) {
    for (int s = 0; s < P::kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&done[s], 1);
    }
    for (int b = 0; b < P::kAccs; ++b) mbar_init(&d_empty[b], 2 * kPairEpi);  // of both CTAs
    mbar_init(drain, 1);
    mbar_init(never, 1);
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc2(tmem_slot, P::kTmem);
    tmem_relinquish2();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the peer's barriers are initialised
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp < 4) {
    registers_down<40>();
    if (warp == 0 && lane == 0) {
      // ---------------------------------------------------------- producer (both CTAs)
      prefetch_tmap(&tmap_w);
      prefetch_tmap(&tmap_x);
      pdl_wait();
      int s = 0;
      uint32_t ph = 0;
      bool dead = false;
      const uint32_t full0 = cluster_map(smem_u32(full), 0);
      for (int64_t i = pair; i < p.tiles && !dead; i += pairs) {
        const int m0 = (int)(i % p.m_tiles * kPairTokens + rank * 128), n0 = (int)(i / p.m_tiles * NT + rank * (NT / 2));
        for (int b = 0; b < p.blocks; ++b) {
          if (!mbar_wait_short(&done[s], ph ^ 1u, p.timeout_ns)) {
            dead = true;
            break;
          }
          uint8_t* st = ring + (size_t)s * P::kStage;
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * P::kStage);
          tma_load_2d_pair(st, &tmap_x, b * 128, m0, full0 + 8u * s);
          tma_load_2d_pair(st + kXBytes, &tmap_w, b * 128, n0, full0 + 8u * s);
          if (++s == P::kStages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      // the products' last arrivals on this CTA's barriers, before it may exit
      for (int j = 0; j < P::kStages && !dead; ++j) {
        dead = !mbar_wait_short(&done[s], ph ^ 1u, p.timeout_ns);
        if (++s == P::kStages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (dead) {  // the copies under way get the time of another wait to land before the CTA's memory goes
        set_status(p.status, kStatusTimeout);
        mbar_wait(never, 0, p.timeout_ns);
      }
    } else if (warp == 1 && rank == 0) {
      // ---------------------------------------------------------- products (leader)
      constexpr uint32_t idesc = idesc_e4m3(kPairTokens, NT);
      int s = 0;
      uint32_t ph = 0, aph = 0;
      bool dead = false;
      for (int64_t i = pair; i < p.tiles && !dead; i += pairs) {
        for (int b = 0; b < p.blocks; ++b) {
          const int a = s % P::kAccs;
          bool ok = mbar_wait_short(&full[s], ph, p.timeout_ns);
          ok = ok && mbar_wait_short(&d_empty[a], aph ^ 1u, p.timeout_ns);
          if (!__all_sync(0xffffffffu, ok)) {
            if (lane == 0) set_status(p.status, kStatusTimeout);
            dead = true;
            break;
          }
          tc_fence_after();
          const uint32_t x = smem_u32(ring + (size_t)s * P::kStage);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_fp8_pair(tmem + (uint32_t)(a * NT), smem_desc_sw128(x + kk * 32u), smem_desc_sw128(x + kXBytes + kk * 32u),
                           idesc, kk > 0 ? 1u : 0u);
            mma_commit2(&done[s]);
          }
          __syncwarp();
          if (a == P::kAccs - 1) aph ^= 1u;
          if (++s == P::kStages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (elect_one()) mma_commit2(drain);
      __syncwarp();
      if (!mbar_wait_short(drain, 0, p.timeout_ns)) set_status(p.status, kStatusTimeout);
    }
  } else {
    // ------------------------------------------------------------ epilogue: thread = token, some of the columns
    registers_up<232>();
    constexpr int C = NT * 4 / kPairEpi;
    const int q = warp & 3, part = (warp - 4) >> 2;
    const uint32_t lane_base = ((uint32_t)(q * 32) << 16) + (uint32_t)(part * C);
    const uint32_t d_empty0 = cluster_map(smem_u32(d_empty), 0);
    uint8_t* staging = ring + P::kStages * P::kStage + (warp - 4) * 2 * kStageBytes;
    int s = 0;
    uint32_t ph = 0;
    bool dead = false, ready = false;
    pdl_wait();  // the scales and y belong to the stream order
    // the scales of four blocks are asked for while the four before them are worked on
    const float *px = nullptr, *pw = nullptr;
    float xs[4], ws[4];
    auto ask = [&](int b, int j) {
      const int64_t c = min(b + j, p.blocks - 1);
      xs[j] = __ldg(px + c * p.x_scale_stride), ws[j] = __ldg(pw + c);
    };
    auto ask_first = [&](int64_t i) {  // of tile i
      const int64_t token = i % p.m_tiles * kPairTokens + rank * 128 + q * 32 + lane, n0 = i / p.m_tiles * NT + part * C;
      const bool there = token < p.m && n0 < p.n;
      px = p.x_scale + (there ? token : 0);
      pw = p.w_scale + (there ? n0 / kFp8Block * p.blocks : 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) ask(0, j);
    };
    if (pair < p.tiles) ask_first(pair);
    for (int64_t i = pair; i < p.tiles; i += pairs) {
      const int64_t m0 = i % p.m_tiles * kPairTokens + rank * 128 + q * 32, n0 = i / p.m_tiles * NT + part * C;
      float acc[C];
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] = 0.f;
      auto block = [&](float sc) {
        if (!__all_sync(0xffffffffu, ready)) {
          // (behind a wait that has expired nothing waits, and what is read is worth nothing)
          if (!dead && !__all_sync(0xffffffffu, mbar_wait_short(&done[s], ph, p.timeout_ns))) {
            if (lane == 0) set_status(p.status, kStatusTimeout);
            dead = true;
          }
        }
        tc_fence_after();
        const int a = s % P::kAccs;
        const uint32_t at = tmem + (uint32_t)(a * NT) + lane_base;
        // a chunk is loaded while the one before it is added up
        uint32_t d[2][32];
        tmem_load32(at, d[0]);
#pragma unroll
        for (int c = 0; c < C; c += 32) {
          const int now = (c / 32) & 1;
          tmem_load_wait();
          if (c + 32 < C) {
            tmem_load32(at + c + 32, d[now ^ 1]);
          } else {  // the buffer is read; a look at the next block's barrier, whose answer comes while the last chunk is added
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(d_empty0 + 8u * a);
            if (++s == P::kStages) {
              s = 0;
              ph ^= 1u;
            }
            ready = mbar_test(&done[s], ph);
          }
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            if constexpr (NT == 128) {
              fma2_behind(acc[c + j], acc[c + j + 1], d[now][j], d[now][j + 1], sc);
            } else {
              fma_behind(acc[c + j], d[now][j], sc);
              fma_behind(acc[c + j + 1], d[now][j + 1], sc);
            }
          }
        }
      };
#pragma unroll 1
      for (int b = 0; b < p.blocks; b += 4) {
        float sc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sc[j] = xs[j] * ws[j];
          ask(b + 4, j);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (b + j < p.blocks) block(sc[j]);
      }
      if (i + pairs < p.tiles) ask_first(i + pairs);
      // the warp's 32 rows, 64 columns at a time, by way of shared memory: 16-byte piece j of row r lies at
      // j ^ (r & 7), so that neither the writes nor the copies out meet in a bank
#pragma unroll
      for (int c = 0; c < C; c += 64) {
        uint8_t* st = staging + (c / 64 & 1) * kStageBytes;
        if (p.y_tma && lane == 0) bulk_wait_read<1>();  // the copy that last read it is done
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *reinterpret_cast<uint4*>(st + lane * 128 + ((j ^ (lane & 7)) << 4)) =
              make_uint4(pack_bf16(acc[c + 8 * j], acc[c + 8 * j + 1]), pack_bf16(acc[c + 8 * j + 2], acc[c + 8 * j + 3]),
                         pack_bf16(acc[c + 8 * j + 4], acc[c + 8 * j + 5]), pack_bf16(acc[c + 8 * j + 6], acc[c + 8 * j + 7]));
        if (p.y_tma) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0 && n0 + c < p.n && m0 < p.m) {
            tma_store_2d(&tmap_y, st, (int)(n0 + c), (int)m0);
          }
          if (lane == 0) bulk_commit();
        } else {
          __syncwarp();
          const int rows = (int)imin64(32, p.m - m0);
          for (int r = 0; r < rows; ++r) {
            uint16_t* yp = p.y + (m0 + r) * p.y_stride + n0 + c;
#pragma unroll
            for (int k = 0; k < 64; k += 32) {
              const int j = (k + lane) >> 3;
              const uint16_t v = *reinterpret_cast<const uint16_t*>(st + r * 128 + ((j ^ (r & 7)) << 4) + ((lane & 7) << 1));
              if (n0 + c + k + lane < p.n) yp[k + lane] = v;
            }
          }
          __syncwarp();
        }
      }
    }
    if (p.y_tma && lane == 0) bulk_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // no arrive or copy of the peer is still to come
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc2(tmem, P::kTmem);
  }
}

// ------------------------------------------------------------------ host side
constexpr int64_t kMost = (int64_t)1 << 30;
constexpr uint32_t kMostSmem = 227 * 1024;

size_t round256(size_t b) { return (b + 255) / 256 * 256; }
int64_t code_stride(int64_t k) { return (k + 15) / 16 * 16; }
int64_t scale_stride(int64_t m) { return (m + 3) / 4 * 4; }
int tokens_of(int64_t m) { return m <= 16 ? 16 : m <= 32 ? 32 : m <= 64 ? 64 : 128; }

struct Workspace {
  size_t codes, scale, part, bytes;
};
Workspace workspace_for(int64_t m, int64_t k, int sms) {
  Workspace w;
  w.codes = ws_counter_bytes(sms);
  w.scale = w.codes + round256((size_t)m * code_stride(k));
  w.part = w.scale + round256((size_t)((k + kFp8Block - 1) / kFp8Block) * scale_stride(m) * 4);
  w.bytes = w.part + (m <= kFewTokens ? 0 : (size_t)2 * sms * tokens_of(m) * kTileN * 4);
  return w;
}

sp_status code_map(CUtensorMap* map, PFN_cuTensorMapEncodeTiled_v12000 encode, const void* codes, int64_t rows,
                   int64_t k, int64_t stride, int box_rows) {
  const cuuint64_t dim[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, estride[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dim, strides, box, estride,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? SP_OK
             : SP_ERR_CUDA;
}

// Rows of W in a tile of fp8_pair_kernel, or 0: fp8_rows_kernel, by their times in clocks. A pair takes 890 for a block of 256
// columns and 570 for one of 128, and some 3500 around a tile; fp8_rows_kernel 1300 for a block of 128 tokens, and 15000
// where tiles are shared. Measured, rows / 128 / 256, us: 128 x 4096 x 4096 22.3 / 17.2 / 22.9, 256 x 22016 x 4096 63.7 / 41.1 / 39.9,
// 256 x 4096 x 11008 38.0 / 39.6 / 47.3, 4096 x 22016 x 4096 714 / 362 / 305.
int pair_columns(int64_t m, int64_t n, int64_t blocks, int sms) {
  if (m <= 64) return 0;
  const int64_t pairs = sms / 2, m_tiles = (m + kPairTokens - 1) / kPairTokens;
  auto waves = [&](int nt) { return (double)((m_tiles * ((n + nt - 1) / nt) + pairs - 1) / pairs); };
  const double wide = waves(256) * (890.0 * blocks + 3500), narrow = waves(128) * (570.0 * blocks + 3500);
  const double units = (double)((m + 127) / 128 * ((n + kTileN - 1) / kTileN)) * blocks / sms;
  const double rows = 1300.0 * std::ceil(units) + 15000;
  if (rows < wide && rows < narrow) return 0;
  return wide <= narrow ? 256 : 128;
}

template <int MT>
sp_status launch_rows(Fp8Params p, const CUtensorMap& map_w, const CUtensorMap& map_x, int sms, cudaStream_t stream) {
  using P = RowsPlan<MT>;
  p.m_tiles = (int32_t)((p.m + MT - 1) / MT);
  p.units = (p.n + kTileN - 1) / kTileN * p.m_tiles * p.blocks;
  int stages = kMaxStages;
  while (P::smem(stages) > kMostSmem) --stages;
  p.stages = stages;
  const int grid = (int)std::min<int64_t>(sms, p.units);
  if (cudaFuncSetAttribute(fp8_rows_kernel<MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)P::smem(stages)) != cudaSuccess) {
    cudaGetLastError();
    return SP_ERR_CUDA;
  }
  return launch_pdl(fp8_rows_kernel<MT>, dim3((unsigned)grid), P::kThreads, P::smem(stages), 1, stream, p, map_w, map_x);
}

// CTA pairs of fp8_pair_kernel that the device, which is current, holds at once; 0: none, or the lookup failed.
template <int NT>
int resident_pairs(int dev) {
  static std::atomic<int> pairs[kMaxDevices] = {};
  if (dev < 0 || dev >= kMaxDevices) return 0;
  return kept_or_looked_up(pairs[dev], [] {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = PairPlan<NT>::kSmem;
    int c = 0;
    if (cudaFuncSetAttribute(fp8_pair_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairPlan<NT>::kSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&c, fp8_pair_kernel<NT>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      c = 0;
    }
    return c;
  });
}

// SP_ERR_UNSUPPORTED, with nothing launched, where the device holds no pair.
template <int NT>
sp_status launch_pair(const Fp8Params& f, PFN_cuTensorMapEncodeTiled_v12000 encode, const CUtensorMap& map_w, const CUtensorMap& map_x, int sms, cudaStream_t stream) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return SP_ERR_CUDA;
  }
  const int pairs = std::min(resident_pairs<NT>(dev), sms / 2);
  if (pairs < 1) return SP_ERR_UNSUPPORTED;
  PairParams p = {};
  p.w_scale = f.w_scale;
  p.x_scale = f.x_scale;
  p.x_scale_stride = f.x_scale_stride;
  p.y = f.y;
  p.y_stride = f.y_stride;
  p.n = f.n;
  p.m = f.m;
  p.blocks = f.blocks;
  p.m_tiles = (int32_t)((f.m + kPairTokens - 1) / kPairTokens);
  p.tiles = (f.n + NT - 1) / NT * p.m_tiles;
  p.y_tma = al16(f.y) && (f.y_stride % 8 == 0 || f.m == 1);
  CUtensorMap map_y = {};
  if (p.y_tma) {
    const cuuint64_t dim[2] = {(cuuint64_t)f.n, (cuuint64_t)f.m}, strides[1] = {(cuuint64_t)(f.y_stride + 7) / 8 * 16};
    const cuuint32_t box[2] = {64, 32}, estride[2] = {1, 1};
    if (encode(&map_y, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, f.y, dim, strides, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return SP_ERR_CUDA;
  }
  p.status = f.status;
  p.timeout_ns = f.timeout_ns;
  return launch_pdl(fp8_pair_kernel<NT>, dim3((unsigned)(2 * std::min<int64_t>(pairs, p.tiles))), kPairThreads, PairPlan<NT>::kSmem, 1,
                    stream, p, map_w, map_x, map_y);
}

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" sp_status sp_fp8_workspace_size(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  if (!bytes || m < 0 || n < 1 || k < 1) return SP_ERR_INVALID_ARG;
  if (m > kMost || n > kMost || k > kMost) return SP_ERR_UNSUPPORTED;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  *bytes = m == 0 || few_fused(m, n, k, sms) ? 0 : workspace_for(m, k, sms).bytes;
  return SP_OK;
}

extern "C" sp_status sp_fp8_linear(const sp_fp8_linear_args* a, void* ws, size_t ws_bytes, void* stream_) {
  if (!a || a->m < 0 || a->n < 1 || a->k < 1 || a->w_stride < a->k || !a->w || !a->w_scale || (a->x && a->xq))
    return SP_ERR_INVALID_ARG;
  if (a->m > 0 && (!a->y || a->y_stride < a->n || (!a->x && !a->xq))) return SP_ERR_INVALID_ARG;
  if ((a->x && a->x_stride < a->k) || (a->xq && (!a->x_scale || a->xq_stride < a->k || a->x_scale_stride < a->m)))
    return SP_ERR_INVALID_ARG;
  if (a->m > kMost || a->n > kMost || a->k > kMost || a->w_stride % 16 || (a->xq && (a->xq_stride % 16 || a->x_scale_stride % 4)))
    return SP_ERR_UNSUPPORTED;
  if (!al16(a->w) || !al16(a->xq) || !al16(ws) || (a->xq && !al16(a->x_scale)) || reinterpret_cast<uintptr_t>(a->w_scale) % 4 ||
      reinterpret_cast<uintptr_t>(a->x) % 2 || reinterpret_cast<uintptr_t>(a->y) % 2)
    return SP_ERR_ALIGNMENT;
  if (a->m == 0) return SP_OK;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  cudaStream_t stream = (cudaStream_t)stream_;
  PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
  sp_status st = tensor_map_encoder(&encode);
  if (st != SP_OK) return st;
  CUtensorMap map_w, map_x;
  if (a->x && few_fused(a->m, a->n, a->k, sms)) {
    st = code_map(&map_w, encode, a->w, a->n, a->k, a->w_stride, kTileN);
    return st != SP_OK ? st : launch_fp8_few(*a, nullptr, map_w, map_w, sms, stream);
  }
  const Workspace w = workspace_for(a->m, a->k, sms);
  if ((a->x || a->m > kFewTokens) && (!ws || ws_bytes < w.bytes)) return SP_ERR_WORKSPACE;
  uint8_t* base = static_cast<uint8_t*>(ws);

  Fp8Rows rows = {static_cast<const uint8_t*>(a->xq), a->x_scale, a->xq_stride, a->x_scale_stride};
  if (a->x) {
    rows = {base + w.codes, reinterpret_cast<const float*>(base + w.scale), code_stride(a->k), scale_stride(a->m)};
    st = launch_fp8_quantize_rows(static_cast<const uint16_t*>(a->x), a->x_stride, a->m, a->k, base + w.codes, rows.stride,
                                  reinterpret_cast<float*>(base + w.scale), rows.scale_stride, stream);
    if (st != SP_OK) return st;
  }
  if (a->m <= kFewTokens) {
    if ((st = code_map(&map_w, encode, a->w, a->n, a->k, a->w_stride, kTileN)) != SP_OK ||
        (st = code_map(&map_x, encode, rows.codes, a->m, a->k, rows.stride, few_box(a->m))) != SP_OK)
      return st;
    return launch_fp8_few(*a, &rows, map_w, map_x, sms, stream);
  }
  const int mt = tokens_of(a->m), nt = pair_columns(a->m, a->n, (a->k + kFp8Block - 1) / kFp8Block, sms);
  if ((st = code_map(&map_w, encode, a->w, a->n, a->k, a->w_stride, nt ? nt / 2 : kTileN)) != SP_OK ||
      (st = code_map(&map_x, encode, rows.codes, a->m, a->k, rows.stride, nt ? 128 : mt)) != SP_OK)
    return st;
  Fp8Params p = {};
  p.w_scale = a->w_scale;
  p.x_scale = rows.scale;
  p.x_scale_stride = rows.scale_stride;
  p.y = static_cast<uint16_t*>(a->y);
  p.y_stride = a->y_stride;
  p.n = a->n;
  p.m = a->m;
  p.blocks = (int32_t)((a->k + kFp8Block - 1) / kFp8Block);
  p.part = reinterpret_cast<float*>(base + w.part);
  p.cnt = static_cast<int*>(ws);
  p.status = device_status_ptr();
  p.timeout_ns = wait_timeout_ns();
  if (nt) {
    st = nt == 256 ? launch_pair<256>(p, encode, map_w, map_x, sms, stream)
                   : launch_pair<128>(p, encode, map_w, map_x, sms, stream);
    if (st != SP_ERR_UNSUPPORTED) return st;
    if ((st = code_map(&map_w, encode, a->w, a->n, a->k, a->w_stride, kTileN)) != SP_OK) return st;  // the device holds no pair
  }
  switch (mt) {
    case 16: return launch_rows<16>(p, map_w, map_x, sms, stream);
    case 32: return launch_rows<32>(p, map_w, map_x, sms, stream);
    case 64: return launch_rows<64>(p, map_w, map_x, sms, stream);
    default: return launch_rows<128>(p, map_w, map_x, sms, stream);
  }
}
