// sp_fp8_linear.cu -- y = x . W^T of weights and activations in e4m3 with a scale for each block of 128
// (include/sp_fp8.h): the call, and the kernel for many tokens.
//
// The tensor cores add up one block of 128 columns at a time, in tensor memory; the epilogue's threads take those sums
// out, multiply them by sx * sw, which changes from block to block, and add them up in registers. While they do, the next
// blocks' sums are made in other columns of tensor memory.
//
// fp8_pair_kernel: pairs of SMs (cta_group::2), a tile of 256 tokens (the lanes of tensor memory, 128 in each CTA) by NT rows of
// W. A thread's scale of a block is then one number, and a sum costs one FMA. What a block costs, 4096 x 22016 x 4096 with NT = 256,
// in clocks of the SM (a block's products alone: 512): copies 590, copies and products 680, copies and the epilogue 720,
// all together 890, in tiles that cost 3500 more (16 waves of tiles of 16, 32, 64 blocks: 138, 248, 468 us at 2070 MHz): 300 us, 2.46 PFLOP/s,
// of which 15 are the nineteenth wave of 8 tiles. The products and the epilogue meet at tensor memory,
// which both read, and the epilogue's eight warps hold as many sums as their registers take, so that they work on one block at a time.
// One commit a block, which frees the copies' stage and hands over the sums: with one for each it is 311 us. The scales of four
// blocks are under way in registers of their own, and rows go out through shared memory: 396 us at first, which waited for
// every block's scales.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>

#include "sp_fp8.cuh"
#include "sp_lookup.h"

namespace sp {
namespace {

constexpr int kMaxDevices = 64;
constexpr int kMaxStages = 8;
constexpr uint32_t kCtl = 1024;

constexpr int kPairTokens = 256;  // of a tile: 128 in each CTA
constexpr uint32_t kXBytes = 128 * 128;
constexpr uint32_t kStageBytes = 32 * 128;  // of y on its way out: 32 rows of 64 columns, a warp
constexpr int kPairEpi = 8;           // epilogue warps
constexpr int kPairThreads = 128 + 32 * kPairEpi;

template <int NT>  // rows of W in a tile
struct PairPlan {
  static constexpr int kColumns = NT * 4 / kPairEpi;              // of a warp
  static constexpr int kOut = kColumns % 64 == 0 ? 64 : 32;       // of them go out at a time
  static constexpr int kAccs = NT == 128 ? 4 : 2;    // sums of blocks in tensor memory at a time
  static constexpr uint32_t kTmem = 512;
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
  int64_t items;         // tiles, or their shares
  int32_t split;         // shares of a tile (of its blocks)
  int32_t y_tma;         // rows of y start and end at multiples of 16 bytes
  float* part;           // sums of the shares [items][2 CTAs][NT][128]
  int* cnt;              // their arrivals [tiles][2 CTAs]
  int* status;
  uint64_t timeout_ns;
  int32_t expire_cta, expire_warp, expire_block;  // in the variants of sp_test_expired_fp8
};

// Item i: its tile's place, and blocks [b0, b1).
struct PairItem {
  int64_t m_tile, n_tile;
  int b0, b1;
};
template <bool SPLIT>
__device__ __forceinline__ PairItem item_at(const PairParams& p, int64_t i) {
  if (!SPLIT) return {i % p.m_tiles, i / p.m_tiles, 0, p.blocks};
  const int64_t tile = i / p.split, part = i % p.split;
  return {tile % p.m_tiles, tile / p.m_tiles, (int)(part * p.blocks / p.split), (int)((part + 1) * p.blocks / p.split)};
}

// kExpire: a variant for sp_test_expired_fp8, whose warp p.expire_warp of CTA p.expire_cta waits, before its block p.expire_block, for
// what never comes, and gives up.
template <int NT, bool SPLIT, bool kExpire = false>
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
  volatile int* s_last = reinterpret_cast<volatile int*>(tmem_slot + 1);
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
  int count = 0;  // (kExpire) of the warp's blocks

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
      for (int64_t i = pair; i < p.items && !dead; i += pairs) {
        const PairItem it = item_at<SPLIT>(p, i);
        const int m0 = (int)(it.m_tile * kPairTokens + rank * 128), n0 = (int)(it.n_tile * NT + rank * (NT / 2));
        for (int b = it.b0; b < it.b1; ++b) {
          if (gives_up<kExpire>(p, count++, never) || !mbar_wait_short(&done[s], ph ^ 1u, p.timeout_ns)) {
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
      for (int64_t i = pair; i < p.items && !dead; i += pairs) {
        const PairItem it = item_at<SPLIT>(p, i);
        for (int b = it.b0; b < it.b1; ++b) {
          const int a = s % P::kAccs;
          bool ok = mbar_wait_short(&full[s], ph, p.timeout_ns);
          ok = ok && mbar_wait_short(&d_empty[a], aph ^ 1u, p.timeout_ns) && !gives_up<kExpire>(p, count++, never);
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
    constexpr int C = P::kColumns, O = P::kOut;
    constexpr bool kTwo = NT == 192;  // a warp's columns may lie in two of W's blocks (32 of them never do)
    const int q = warp & 3, part = (warp - 4) >> 2;
    const uint32_t lane_base = ((uint32_t)(q * 32) << 16) + (uint32_t)(part * C);
    const uint32_t d_empty0 = cluster_map(smem_u32(d_empty), 0);
    uint8_t* staging = ring + P::kStages * P::kStage + (warp - 4) * 2 * kStageBytes;
    int s = 0, turn = 0;
    uint32_t ph = 0;
    bool dead = false, ready = false;
    pdl_wait();  // the scales and y belong to the stream order
    // the scales of four blocks are asked for while the four before them are worked on
    const float *px = nullptr, *pw = nullptr, *pw2 = nullptr;
    float xs[4], ws[4], ws2[4];
    int b1 = 0;
    auto ask = [&](int b, int j) {
      const int64_t c = min(b + j, b1 - 1);
      xs[j] = __ldg(px + c * p.x_scale_stride), ws[j] = __ldg(pw + c);
      if constexpr (kTwo) ws2[j] = __ldg(pw2 + c);
    };
    auto ask_first = [&](int64_t i) {  // of item i
      const PairItem it = item_at<SPLIT>(p, i);
      b1 = it.b1;
      const int64_t token = it.m_tile * kPairTokens + rank * 128 + q * 32 + lane, n0 = it.n_tile * NT + part * C;
      const bool there = token < p.m && n0 < p.n;
      px = p.x_scale + (there ? token : 0);
      pw = p.w_scale + (there ? n0 / kFp8Block * p.blocks : 0);
      if constexpr (kTwo) pw2 = p.w_scale + (there ? imin64(n0 + C - 1, p.n - 1) / kFp8Block * p.blocks : 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) ask(it.b0, j);
    };
    if (pair < p.items) ask_first(pair);
    for (int64_t i = pair; i < p.items; i += pairs) {
      const PairItem it = item_at<SPLIT>(p, i);
      const int64_t m0 = it.m_tile * kPairTokens + rank * 128 + q * 32, n0 = it.n_tile * NT + part * C;
      float acc[C];
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] = 0.f;
      const int turn_at = kTwo ? (int)(kFp8Block - n0 % kFp8Block) : C;  // the first column of the second block
      auto block = [&](float sc1, float sc2) {
        if constexpr (kExpire) {
          if (!__all_sync(0xffffffffu, !gives_up<kExpire>(p, count++, never))) {
            if (lane == 0) set_status(p.status, kStatusTimeout);
            dead = true;
          }
        }
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
          const float sc = kTwo && c >= turn_at ? sc2 : sc1;
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            if constexpr (NT != 256) {
              fma2_behind(acc[c + j], acc[c + j + 1], d[now][j], d[now][j + 1], sc);
            } else {
              fma_behind(acc[c + j], d[now][j], sc);
              fma_behind(acc[c + j + 1], d[now][j + 1], sc);
            }
          }
        }
      };
#pragma unroll 1
      for (int b = it.b0; b < it.b1; b += 4) {
        float sc[4], sc2[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sc[j] = xs[j] * ws[j];
          sc2[j] = kTwo ? xs[j] * ws2[j] : 0.f;
          ask(b + 4, j);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (b + j < it.b1) block(sc[j], sc2[j]);
      }
      if (i + pairs < p.items) ask_first(i + pairs);
      // O columns of the warp's 32 rows, by way of shared memory, laid out as TMA swizzles them, so that neither the writes nor the
      // copies out meet in a bank: 16-byte piece j of a row r of 128 bytes lies at j ^ (r & 7), of 64 bytes at j ^ (r / 2 & 3)
      constexpr int kPieces = O / 8;
      auto place = [&](int r, int j) { return r * (2 * O) + ((O == 64 ? j ^ (r & 7) : j ^ (r >> 1 & 3)) << 4); };
      auto store = [&](int c, const float* v) {
        uint8_t* st = staging + turn * kStageBytes;
        turn ^= 1;  // (the two buffers in turn, over all tiles: the copy before the last one is waited for)
        if (p.y_tma && lane == 0) bulk_wait_read<1>();  // the copy that last read it is done
        __syncwarp();
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
          *reinterpret_cast<uint4*>(st + place(lane, j)) =
              make_uint4(pack_bf16(v[8 * j], v[8 * j + 1]), pack_bf16(v[8 * j + 2], v[8 * j + 3]),
                         pack_bf16(v[8 * j + 4], v[8 * j + 5]), pack_bf16(v[8 * j + 6], v[8 * j + 7]));
        if (p.y_tma) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0 && n0 + c < p.n && m0 < p.m) tma_store_2d(&tmap_y, st, (int)(n0 + c), (int)m0);
          if (lane == 0) bulk_commit();
        } else {
          __syncwarp();
          const int rows = (int)imin64(32, p.m - m0);
          uint16_t* yp = p.y + m0 * p.y_stride + n0 + c + lane;
#pragma unroll 1
          for (int r0 = 0; r0 < rows; r0 += 8) {
#pragma unroll
            for (int r = r0; r < r0 + 8; ++r) {
#pragma unroll
              for (int k = 0; k < O; k += 32) {
                const uint16_t u = *reinterpret_cast<const uint16_t*>(st + place(r, (k + lane) >> 3) + ((lane & 7) << 1));
                if (r < rows && n0 + c + k + lane < p.n) yp[r * p.y_stride + k] = u;
              }
            }
          }
          __syncwarp();
        }
      };
      if (!SPLIT) {
#pragma unroll
        for (int c = 0; c < C; c += O) store(c, acc + c);
      } else {
        const int64_t rest = i / p.split;
        auto share = [&](int64_t k) { return p.part + ((k * 2 + rank) * NT + part * C) * 128 + q * 32 + lane; };
        float* mine = share(i);
#pragma unroll
        for (int j = 0; j < C; ++j) __stcg(mine + j * 128, acc[j]);
        __threadfence();
        named_bar_sync(1, kPairEpi * 32);
        if (tid == 128) *s_last = atomicAdd(p.cnt + rest * 2 + rank, 1) == p.split - 1 ? 1 : 0;
        named_bar_sync(1, kPairEpi * 32);
        const bool last = *s_last;
        named_bar_sync(1, kPairEpi * 32);  // (it is written again)
        if (last) {  // of the tile's shares to arrive: it adds up all of them, in order
          __threadfence();
#pragma unroll 1
          for (int c = 0; c < C; c += O) {
            float v[O];
#pragma unroll
            for (int j = 0; j < O; ++j) v[j] = 0.f;
            for (int k = 0; k < p.split; ++k) {
              const float* src = share(rest * p.split + k) + c * 128;
              float u[O];
#pragma unroll
              for (int j = 0; j < O; ++j) u[j] = __ldcg(src + j * 128);
#pragma unroll
              for (int j = 0; j < O; ++j) v[j] += u[j];
            }
            store(c, v);
          }
          if (tid == 128) atomicExch(p.cnt + rest * 2 + rank, 0);
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

size_t round256(size_t b) { return (b + 255) / 256 * 256; }
int64_t code_stride(int64_t k) { return (k + 15) / 16 * 16; }
int64_t scale_stride(int64_t m) { return (m + 3) / 4 * 4; }

struct Workspace {
  size_t codes, scale, part, bytes;
};
Workspace workspace_for(int64_t m, int64_t k, int sms) {
  Workspace w;
  w.codes = ws_counter_bytes(sms);
  w.scale = w.codes + round256((size_t)m * code_stride(k));
  w.part = w.scale + round256((size_t)((k + kFp8Block - 1) / kFp8Block) * scale_stride(m) * 4);
  // sums of shares: of each pair 256 tokens by up to 256 columns
  w.bytes = w.part + (m <= kFewTokens ? 0 : (size_t)(sms / 2) * kPairTokens * 256 * 4);
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

// The work of fp8_pair_kernel on `pairs` pairs, and its time in clocks: 890 for a block of 256 columns, 750 for one of 192 and 570 for one of 128,
// and some 3500 around a tile. Where tiles are fewer than the pairs they are shared by the blocks of their columns, at 4000
// and some for each share, if that is less. Measured, us, with shares / without: 128 x 4096 x 11008 (NT = 128, two) 26.5 / 38.3; tiles left
// by whole waves in a launch of shares behind them: 512 x 12288 x 4096 52 / 38, so those are not shared. The three widths, 128 / 192 / 256, us:
// 100 x 3000 x 4096 15.1 / 19.3 / 21.4, 512 x 12288 x 4096 39.5 / 34.8 / 36.8, 4096 x 22016 x 4096 367 / 364 / 301.
struct PairWork {
  int64_t tiles;
  int split;
  double clocks;
};
PairWork pair_work(int nt, int64_t m, int64_t n, int64_t blocks, int64_t pairs) {
  const double block = nt == 256 ? 890 : nt == 192 ? 750 : 570, share = nt == 128 ? 1000 : 2500;
  PairWork w = {(m + kPairTokens - 1) / kPairTokens * ((n + nt - 1) / nt), 1, 0};
  double best = block * blocks;
  for (int s = 2; s <= pairs / w.tiles && s <= blocks / 4; ++s) {
    const double c = block * ((blocks + s - 1) / s) + 4000 + share * s;
    if (c < best) best = c, w.split = s;
  }
  w.clocks = (double)((w.tiles + pairs - 1) / pairs) * (best + 3500);
  return w;
}

// Rows of W in a tile: where the time is less.
int pair_rows(int64_t m, int64_t n, int64_t k, int sms) {
  auto clocks = [&](int nt) { return pair_work(nt, m, n, (k + kFp8Block - 1) / kFp8Block, sms / 2).clocks; };
  return clocks(256) <= clocks(192) && clocks(256) <= clocks(128) ? 256 : clocks(192) <= clocks(128) ? 192 : 128;
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
    if (cudaFuncSetAttribute(fp8_pair_kernel<NT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairPlan<NT>::kSmem) != cudaSuccess ||
        cudaFuncSetAttribute(fp8_pair_kernel<NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairPlan<NT>::kSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&c, fp8_pair_kernel<NT, true>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      c = 0;
    }
    return c;
  });
}

// SP_ERR_UNSUPPORTED where the device holds no pair (x has been quantised into the workspace by then).  Registers: the epilogue's
// sums leave few; with shared tiles of 256 columns 164 bytes of a thread's others are kept in memory, with the rest 28 or 48.
template <int NT>
sp_status launch_pair(const sp_fp8_linear_args& a, const Fp8Rows& rows, void* ws, float* part, int sms,
                      PFN_cuTensorMapEncodeTiled_v12000 encode, const Fp8Expire* expire, cudaStream_t stream) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return SP_ERR_CUDA;
  }
  const int pairs = std::min(resident_pairs<NT>(dev), sms / 2);
  if (pairs < 1) return SP_ERR_UNSUPPORTED;
  CUtensorMap map_w, map_x, map_y = {};
  sp_status st = code_map(&map_w, encode, a.w, a.n, a.k, a.w_stride, NT / 2);
  if (st == SP_OK) st = code_map(&map_x, encode, rows.codes, a.m, a.k, rows.stride, 128);
  if (st != SP_OK) return st;
  PairParams p = {};
  p.w_scale = a.w_scale;
  p.x_scale = rows.scale;
  p.x_scale_stride = rows.scale_stride;
  p.y = static_cast<uint16_t*>(a.y);
  p.y_stride = a.y_stride;
  p.n = a.n;
  p.m = a.m;
  p.blocks = (int32_t)((a.k + kFp8Block - 1) / kFp8Block);
  p.m_tiles = (int32_t)((a.m + kPairTokens - 1) / kPairTokens);
  const PairWork w = pair_work(NT, a.m, a.n, p.blocks, pairs);
  p.split = w.split;
  p.items = w.tiles * w.split;
  p.part = part;
  p.cnt = static_cast<int*>(ws);
  // (a bulk store writes whole pieces of 16 bytes: a row that ended inside one would have up to seven columns beside it written)
  p.y_tma = al16(a.y) && a.y_stride % 8 == 0 && a.n % 8 == 0;
  if (p.y_tma) {
    const cuuint64_t dim[2] = {(cuuint64_t)a.n, (cuuint64_t)a.m}, strides[1] = {(cuuint64_t)a.y_stride * 2};
    const cuuint32_t box[2] = {(cuuint32_t)PairPlan<NT>::kOut, 32}, estride[2] = {1, 1};
    if (encode(&map_y, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, a.y, dim, strides, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE,
               PairPlan<NT>::kOut == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return SP_ERR_CUDA;
  }
  p.status = device_status_ptr();
  p.timeout_ns = wait_timeout_ns();
  auto kern = w.split > 1 ? fp8_pair_kernel<NT, true> : fp8_pair_kernel<NT, false>;
  if (NT == 128 && expire) {
    p.timeout_ns = expire->wait_ns;
    p.expire_cta = expire->cta, p.expire_warp = expire->warp, p.expire_block = expire->block;
    kern = w.split > 1 ? fp8_pair_kernel<128, true, true> : fp8_pair_kernel<128, false, true>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairPlan<NT>::kSmem) != cudaSuccess) {
      cudaGetLastError();
      return SP_ERR_CUDA;
    }
  }
  return launch_pdl(kern,
                    dim3((unsigned)(2 * std::min<int64_t>(pairs, p.items))), kPairThreads, PairPlan<NT>::kSmem, 1, stream, p, map_w, map_x, map_y);
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

namespace {

sp_status linear(const sp_fp8_linear_args* a, void* ws, size_t ws_bytes, const Fp8Expire* expire, void* stream_) {
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
  const int nt = a->m <= kFewTokens ? 0 : pair_rows(a->m, a->n, a->k, sms);
  if (expire && (a->m <= kFewTokens ? few_box(a->m) != 16 : nt != 128)) return SP_ERR_UNSUPPORTED;
  cudaStream_t stream = (cudaStream_t)stream_;
  PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
  sp_status st = tensor_map_encoder(&encode);
  if (st != SP_OK) return st;
  CUtensorMap map_w, map_x;
  if (a->m <= kFewTokens && (st = code_map(&map_w, encode, a->w, a->n, a->k, a->w_stride, kFp8Block)) != SP_OK) return st;
  if (a->x && few_fused(a->m, a->n, a->k, sms)) return launch_fp8_few(*a, nullptr, map_w, map_w, sms, expire, stream);
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
    st = code_map(&map_x, encode, rows.codes, a->m, a->k, rows.stride, few_box(a->m));
    return st != SP_OK ? st : launch_fp8_few(*a, &rows, map_w, map_x, sms, expire, stream);
  }
  float* part = reinterpret_cast<float*>(base + w.part);
  return nt == 256   ? launch_pair<256>(*a, rows, ws, part, sms, encode, nullptr, stream)
         : nt == 192 ? launch_pair<192>(*a, rows, ws, part, sms, encode, nullptr, stream)
                     : launch_pair<128>(*a, rows, ws, part, sms, encode, expire, stream);
}

}  // namespace

extern "C" sp_status sp_fp8_linear(const sp_fp8_linear_args* a, void* ws, size_t ws_bytes, void* stream) {
  return linear(a, ws, ws_bytes, nullptr, stream);
}

extern "C" sp_status sp_test_expired_fp8(const sp_fp8_linear_args* a, void* ws, size_t ws_bytes, int32_t cta, int32_t warp,
                                         int32_t block, uint32_t wait_ms, void* stream) {
  if (cta < 0 || warp < 0 || block < 0 || wait_ms < 1 || wait_ms > 10000) return SP_ERR_INVALID_ARG;
  const Fp8Expire e = {cta, warp, block, (uint64_t)wait_ms * 1000000ull};
  return linear(a, ws, ws_bytes, &e, stream);
}
