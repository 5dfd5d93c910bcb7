// sp_kv4.cuh -- the layout of a cache held in 4 bits (include/sp_serve.h), and the launch helper of
// the serving kernels.
#pragma once

#include <cuda_fp16.h>

#include "../../include/sp_serve.h"
#include "sp_internal.cuh"

namespace sp {

constexpr int kStatusBadIndex = 3;  // device status, behind kStatusBadFormat: an index that a kernel left out

constexpr float kKvMost = 32768.f;  // largest magnitude that the cache holds
constexpr int kMaxGroup = 64;       // query heads per key head
constexpr int kUnitKeys = 32;       // keys of one step of attend_kernel
constexpr int kRowTile = 32;        // query rows (token, head of the group) of its widest form
// Query rows of a request from which attend_rows_kernel takes it: every request that attend_kernel would
// need a second row tile for.  32 heads over 8 of 128, 12 new tokens (48 rows), attend_kernel / attend_rows_kernel,
// us: 16 requests behind 1000 tokens 44 / 30, behind 8000 209 / 149; one request 21 / 26 and 36 / 43, alone with its 12
// tokens 11 / 16: what one request loses is less than what several gain, and the host, which launches both kernels or one, sees no lengths.
constexpr int kManyRows = 33;
constexpr int kPairRows = 256;      // query rows of one of its items
constexpr int kSetupUnits = 2;      // what a segment costs beside its units, in units (64 requests of 100 to
                                    // 16384 tokens: 57.9 us at 0, 52.5 at 1, 49.9 at 2, 50.0 at 3, 50.6 at 4)

struct Kv4 {
  uint8_t* data;
  int64_t pages;
  int32_t shift;  // page_size = 1 << shift
  int32_t heads;
};

// (the buffer's bytes, and so every slot and offset, are 63-bit numbers; of a positive cache)
inline bool kv4_supported(const sp_kv4* c) {
  return (c->page_size == 16 || c->page_size == 32 || c->page_size == 64 || c->page_size == 128) &&
         (c->head_dim == 64 || c->head_dim == 128) &&
         c->pages <= INT64_MAX / ((int64_t)c->page_size * (c->head_dim + 8)) / c->kv_heads;
}
inline bool kv4_positive(const sp_kv4* c) { return c->pages > 0 && c->kv_heads > 0; }
inline int page_shift(int page_size) { return __builtin_ctz((unsigned)page_size); }
inline Kv4 kv4_view(const sp_kv4* c) {
  return {static_cast<uint8_t*>(c->data), c->pages, page_shift(c->page_size), c->kv_heads};
}

// Offsets inside a block of P = 1 << shift tokens.
template <int D>
__host__ __device__ constexpr int64_t kv4_block_bytes(int shift) { return (int64_t)(D + 8) << shift; }
template <int D>
__host__ __device__ constexpr int kv4_value_codes(int shift) { return (D / 2) << shift; }
template <int D>
__host__ __device__ constexpr int kv4_key_params(int shift) { return D << shift; }
template <int D>
__host__ __device__ constexpr int kv4_value_params(int shift) { return (D + 4) << shift; }

inline bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// SMs of the current device, looked up once per device; 0 if that failed.
int current_sms();

// A launch under programmatic dependent launch, as the stack's kernels: every kernel starts with
// griddepcontrol.wait.
template <typename... Params, typename... Args>
sp_status launch_pdl(void (*kern)(Params...), dim3 grid, int block, size_t smem, int cluster, cudaStream_t stream,
                     Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kern, args...) != cudaSuccess) {
    cudaGetLastError();
    return SP_ERR_CUDA;
  }
  return SP_OK;
}

}  // namespace sp
