// sp_fp8_linear.cu -- y = x . W^T of weights and activations in e4m3 with a scale for each block of 128
// (include/sp_fp8.h).
//
// The tensor cores add up one block of 128 columns at a time, in tensor memory; the epilogue's threads take those sums
// out, multiply them by sx * sw, which changes from block to block, and add them up in registers. While they do, the next
// blocks' sums are made in other columns of tensor memory.
//
// fp8_rows_kernel: a tile is 128 rows of W (the lanes of tensor memory) by MT tokens (its columns), so that few
// tokens waste no tensor time and a weight is read once. The tiles' blocks, all in a row, are cut into as many equal
// ranges as there are CTAs; a tile that is shared by several leaves its sums in the workspace, and the last CTA to
// arrive joins them in order.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cstring>

#include "sp_fp8.cuh"

namespace sp {
namespace {

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
        if (!mbar_wait(&empty[s], ph ^ 1u, p.timeout_ns)) {
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
          mbar_wait(&full[i % p.stages], (uint32_t)((i / p.stages) & 1), p.timeout_ns);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ products
    int s = 0, a = 0;
    uint32_t ph = 0, aph = 0;
    for (int64_t u = u0; u < u1; ++u) {
      bool ok = mbar_wait(&d_empty[a], aph ^ 1u, p.timeout_ns);
      ok = ok && mbar_wait(&full[s], ph, p.timeout_ns);
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
    if (!mbar_wait(drain, 0, p.timeout_ns)) set_status(p.status, kStatusTimeout);
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
          bool ok = mbar_wait(&d_full[a], aph, p.timeout_ns);
          ok = ok && mbar_wait(&full[s], ph, p.timeout_ns);  // (complete: the products have read the stage)
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
  w.bytes = w.part + (size_t)2 * sms * tokens_of(m) * kTileN * 4;
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

}  // namespace
}  // namespace sp

using namespace sp;

extern "C" sp_status sp_fp8_workspace_size(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  if (!bytes || m < 0 || n < 1 || k < 1) return SP_ERR_INVALID_ARG;
  if (m > kMost || n > kMost || k > kMost) return SP_ERR_UNSUPPORTED;
  const int sms = current_sms();
  if (sms == 0) return SP_ERR_CUDA;
  *bytes = m == 0 ? 0 : workspace_for(m, k, sms).bytes;
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
  const Workspace w = workspace_for(a->m, a->k, sms);
  if (!ws || ws_bytes < w.bytes) return SP_ERR_WORKSPACE;
  uint8_t* base = static_cast<uint8_t*>(ws);
  cudaStream_t stream = (cudaStream_t)stream_;
  PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
  sp_status st = tensor_map_encoder(&encode);
  if (st != SP_OK) return st;

  Fp8Rows rows = {static_cast<const uint8_t*>(a->xq), a->x_scale, a->xq_stride, a->x_scale_stride};
  if (a->x) {
    rows = {base + w.codes, reinterpret_cast<const float*>(base + w.scale), code_stride(a->k), scale_stride(a->m)};
    st = launch_fp8_quantize_rows(static_cast<const uint16_t*>(a->x), a->x_stride, a->m, a->k, base + w.codes, rows.stride,
                                  reinterpret_cast<float*>(base + w.scale), rows.scale_stride, stream);
    if (st != SP_OK) return st;
  }
  const int mt = tokens_of(a->m);
  CUtensorMap map_w, map_x;
  if ((st = code_map(&map_w, encode, a->w, a->n, a->k, a->w_stride, kTileN)) != SP_OK ||
      (st = code_map(&map_x, encode, rows.codes, a->m, a->k, rows.stride, mt)) != SP_OK)
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
  switch (mt) {
    case 16: return launch_rows<16>(p, map_w, map_x, sms, stream);
    case 32: return launch_rows<32>(p, map_w, map_x, sms, stream);
    case 64: return launch_rows<64>(p, map_w, map_x, sms, stream);
    default: return launch_rows<128>(p, map_w, map_x, sms, stream);
  }
}
