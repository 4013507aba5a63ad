// What the products of quantized tokens with quantized weights share: tiles of channels by tokens, plain or grouped by
// expert, their order, and the tensor maps of codes and outputs.
//
// `P`, the parameters of a product, has M, row0, all_rows, groups, offsets, status and tiles_n.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "common.cuh"

namespace luqdev {

constexpr int kBand = 8;                  // token tiles that walk the channels together

__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ uint32_t cluster_nctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// Arrival at a barrier of the cluster's leader that orders no memory: what it reports is that this warp's
// accumulators are in registers (a releasing arrival at cluster scope waits for all earlier stores: 2000 cycles a tile)
__device__ __forceinline__ void mbar_arrive_leader(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// meets the other CTAs without waiting for this one's stores to global memory
__device__ __forceinline__ void cluster_sync_relaxed() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int ld_shared_cluster(uint32_t cluster_addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
  return v;
}
template <int CHUNK>
__device__ __forceinline__ void load_chunk(uint32_t taddr, uint32_t (&r)[CHUNK]) {
  if constexpr (CHUNK == 32) tmem_ld_32x32(taddr, r);
  else tmem_ld_32x16(taddr, r);
}

// Row ranges of the groups among this launch's rows and the running count of their token tiles, by one warp.  Offsets
// are taken as their running maximum clamped to [0, all_rows]: whatever they hold, every row belongs to one group at
// most and no address leaves the tensors; offsets that had to be changed raise LUQ_STATUS_OFFSETS.
template <class P>
__device__ __forceinline__ void find_groups(const P& p, int tile_rows, int* hi, int* first_tile, bool report) {
  const int lane = threadIdx.x & 31;
  const int M = static_cast<int>(p.M);
  int carry = 0;
  bool bad = false;
  for (int e0 = 0; e0 <= p.groups; e0 += 32) {
    const int e = e0 + lane;
    const int raw = e <= p.groups ? *(p.offsets + e) : 0;
    int v = min(max(raw, 0), p.all_rows);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xFFFFFFFFu, v, o);
      if (lane >= o) v = max(v, up);
    }
    v = max(v, carry);
    if (e <= p.groups) { hi[e] = min(max(v - p.row0, 0), M); bad |= v != raw; }
    carry = __shfl_sync(0xFFFFFFFFu, v, 31);
  }
  if (report && __any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(p.status, LUQ_STATUS_OFFSETS);
  __syncwarp();
  carry = 0;
  for (int e0 = 0; e0 < p.groups; e0 += 32) {
    const int e = e0 + lane;
    int v = e < p.groups ? (hi[e + 1] - hi[e] + tile_rows - 1) / tile_rows : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xFFFFFFFFu, v, o);
      if (lane >= o) v += up;
    }
    v += carry;
    if (e < p.groups) first_tile[e + 1] = v;
    carry = __shfl_sync(0xFFFFFFFFu, v, 31);
  }
  if (lane == 0) first_tile[0] = 0;
  __syncwarp();
}

struct Unit {
  int group, row0, rows, ch0;
  int in_group;               // row0 counted from the group's first row
};
// The tiles of one CTA (or cluster), in order.  Tiles walk the channels in bands of kBand token tiles, tokens
// fastest: what runs together shares both operands' tiles in L2.  Every role and every epilogue warp walks for
// itself, so a step has no division but in the last band.  (There are less than 2^31 tiles: they would need more
// outputs than memory holds.)
struct Walk {
  int u, step, units, band, in_band, per_band, token_tiles;
  template <class P>
  __device__ __forceinline__ Walk(const P& p, int tiles, int first, int by)
      : u(first), step(by), units(tiles * p.tiles_n), band(first / (kBand * p.tiles_n)), per_band(kBand * p.tiles_n), token_tiles(tiles) {
    in_band = first - band * per_band;
  }
  __device__ __forceinline__ bool more() const { return u < units; }
  __device__ __forceinline__ void next() {
    u += step;
    in_band += step;
    while (in_band >= per_band) { in_band -= per_band; ++band; }
  }
  template <class P>
  __device__ __forceinline__ Unit unit(const P& p, int tile_rows, int tile_ch, const int* hi, const int* first_tile) const {
    const int width = min(kBand, token_tiles - band * kBand);
    const int c = width == kBand ? in_band / kBand : in_band / width;
    const int j = band * kBand + in_band - c * width;
    if (p.offsets == nullptr) {
      const int row0 = j * tile_rows;
      return Unit{0, row0, min(tile_rows, static_cast<int>(p.M) - row0), c * tile_ch, row0};
    }
    int lo = 0, up = p.groups;                     // the last group whose first tile is <= j
    while (up - lo > 1) {
      const int mid = (lo + up) >> 1;
      if (first_tile[mid] <= j) lo = mid; else up = mid;
    }
    Unit v;
    v.group = lo;
    v.in_group = (j - first_tile[lo]) * tile_rows;
    v.row0 = hi[lo] + v.in_group;
    v.rows = min(tile_rows, hi[lo + 1] - v.row0);
    v.ch0 = c * tile_ch;
    return v;
  }
};

__device__ __forceinline__ void store_z(void* z, long long at, float v, bool bf16) {
  if (bf16) static_cast<__nv_bfloat16*>(z)[at] = __float2bfloat16_rn(v);
  else static_cast<float*>(z)[at] = v;
}
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// codes as [planes][rows][cols] bytes, boxes of box_rows x 128 bytes, 128-byte swizzle; what lies beyond the
// extents reads as zero
inline int encode_codes(void* fn, CUtensorMap* map, const void* ptr, int64_t cols, int64_t rows, int64_t ld, int64_t planes,
                 int64_t plane_stride, int box_rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(planes)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld), static_cast<cuuint64_t>(plane_stride)};
  const cuuint32_t box[3] = {128, static_cast<cuuint32_t>(box_rows), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return reinterpret_cast<EncodeTiledFn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, planes > 0 ? 3 : 2, const_cast<void*>(ptr),
                                             dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS;
}
// output [rows x cols], boxes of 32 x 32 elements as they lie in memory
inline int encode_z(void* fn, CUtensorMap* map, void* ptr, int64_t cols, int64_t rows, int64_t ld, bool bf16) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * (bf16 ? 2 : 4)};
  const cuuint32_t box[2] = {32, 32};
  const cuuint32_t estr[2] = {1, 1};
  return reinterpret_cast<EncodeTiledFn>(fn)(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2,
                                             ptr, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS;
}

}  // namespace luqdev
