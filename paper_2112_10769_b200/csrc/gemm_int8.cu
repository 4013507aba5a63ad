// int8 products with a scale for each token and each output channel, plain or grouped by expert (sm_100a).
//
//   Z[t, n] = sx[t] sw[e, n] sum_k X[t, k] W[e, n, k] + bias[e, n]      e = the expert (group) of row t
//
// X: int8 codes of the tokens [M x K], W: int8 codes [groups x N x K], both with rows that start at
// multiples of 16 bytes; the rows of a group follow one another, offsets[e] .. offsets[e+1], and the sizes
// are known on the device only.  Integer sums are exact (int32 accumulators, K <= 131071).
//
// The weights are the MMA's A operand (128 channels = the lanes of tensor memory) and the tokens its B operand:
// B's extent is an instruction field that may be any multiple of 16, so a tile costs what its tokens need -
// a group's last, partial tile and a handful of tokens of a model that answers alike.
//
// One persistent CTA per SM, warp-specialised:
//   warp 0     TMA producer: 128 x 128 bytes of W and the tile's token rows x 128 bytes, 128-byte swizzle
//   warp 1     one thread issues tcgen05.mma kind::i8; owns the tensor-memory allocation (two accumulators)
//   warps 2-5  epilogue: tcgen05.ld -> scales, bias -> staged 32 x 32 boxes -> TMA store; token rows
//              that share a box with another group's, and outputs TMA cannot address, are stored directly
// All waits are bounded; on expiry the CTA flags LUQ_STATUS_TIMEOUT, drains its copies, frees its
// tensor memory and returns.
#include <cuda.h>
#include <cuda_bf16.h>

#include "common.cuh"

namespace {

using namespace luqdev;

constexpr int kCh = 128;                  // output channels per tile (tensor-memory lanes)
constexpr int kBk = 128;                  // contraction elements per stage
constexpr int kSlab = kCh * kBk;          // bytes of W per stage
constexpr int kThreads = 192;
constexpr int kFirstEpiWarp = 2;
constexpr int kBox = 32 * 32 * 4;         // one 32 x 32 fp32 store box (half of it for bf16)
constexpr int kBand = 8;                  // token tiles that walk the channels together

struct Int8Params {
  const float* sx;
  const float* sw;
  const float* bias;        // may be null
  const int* offsets;       // may be null: one group, all rows
  void* z;
  long long ld_z;
  unsigned int* status;
  long long M, N;
  int groups;
  int num_kb;
  int tiles_n;              // channel tiles
  int out_bf16;
  int z_tma;                // the output can be addressed by TMA
  long long tma_cols;       // a store copy writes whole 16-byte pieces: boxes up to this column end on one
};

template <int BT>
struct Cfg {
  static constexpr int x_bytes = BT * kBk;
  static constexpr int stage_bytes = kSlab + x_bytes;
  static constexpr int stages = BT == 256 ? 3 : BT == 128 ? 5 : BT == 64 ? 7 : BT == 32 ? 8 : 9;
  static constexpr int chunk = BT < 32 ? BT : 32;                 // tokens per epilogue step
  static constexpr int tmem_cols = 2 * BT;
  static constexpr int staging = stages * stage_bytes;            // 4 warps x 2 boxes
  static constexpr int token_scales = staging + 4 * 2 * kBox;     // 4 warps x 32 floats
  static constexpr int barriers = token_scales + 4 * 128;
  static constexpr int num_barriers = 2 * stages + 4;
  static constexpr int tmem_slot = barriers + 8 * num_barriers;
  static constexpr int abort_flag = tmem_slot + 4;
  static constexpr int groups = abort_flag + 4;                   // group ends, then tile prefix: 2 x (groups + 1) ints
  static int smem_bytes(int n_groups) { return groups + 8 * (n_groups + 1) + 1024; }
};

__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
template <int CHUNK>
__device__ __forceinline__ void load_chunk(uint32_t taddr, uint32_t (&r)[CHUNK]) {
  if constexpr (CHUNK == 32) tmem_ld_32x32(taddr, r);
  else tmem_ld_32x16(taddr, r);
}

// Row ranges of the groups and the running count of their token tiles, by one warp.  Offsets are taken
// as their running maximum clamped to [0, M]: whatever they hold, every row belongs to one group at most and no
// address leaves the tensors; offsets that had to be changed raise LUQ_STATUS_OFFSETS.
__device__ __forceinline__ void find_groups(const Int8Params& p, int tile_rows, int* hi, int* first_tile, bool report) {
  const int lane = threadIdx.x & 31;
  const int M = static_cast<int>(p.M);
  if (p.offsets == nullptr) {
    if (lane == 0) {
      hi[0] = 0; hi[1] = M;
      first_tile[0] = 0; first_tile[1] = (M + tile_rows - 1) / tile_rows;
    }
    __syncwarp();
    return;
  }
  int carry = 0;
  bool bad = false;
  for (int e0 = 0; e0 <= p.groups; e0 += 32) {
    const int e = e0 + lane;
    const int raw = e <= p.groups ? __ldg(p.offsets + e) : 0;
    int v = min(max(raw, 0), M);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xFFFFFFFFu, v, o);
      if (lane >= o) v = max(v, up);
    }
    v = max(v, carry);
    if (e <= p.groups) { hi[e] = v; bad |= v != raw; }
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
};
// Units walk the channel tiles in bands of kBand token tiles, tokens fastest: what runs together shares
// both operands' tiles in L2.
__device__ __forceinline__ Unit find_unit(long long u, const Int8Params& p, int tile_rows, const int* hi, const int* first_tile) {
  const int token_tiles = first_tile[p.groups];
  const long long per_band = static_cast<long long>(kBand) * p.tiles_n;
  const int band = static_cast<int>(u / per_band);
  const int in_band = static_cast<int>(u - band * per_band);
  const int width = min(kBand, token_tiles - band * kBand);
  const int c = in_band / width;
  const int j = band * kBand + (in_band - c * width);
  int lo = 0, up = p.groups;                       // the last group whose first tile is <= j
  while (up - lo > 1) {
    const int mid = (lo + up) >> 1;
    if (first_tile[mid] <= j) lo = mid; else up = mid;
  }
  Unit v;
  v.group = lo;
  v.row0 = hi[lo] + (j - first_tile[lo]) * tile_rows;
  v.rows = min(tile_rows, hi[lo + 1] - v.row0);
  v.ch0 = c * kCh;
  return v;
}

template <int BT>
__global__ void __launch_bounds__(kThreads, 1)
int8_gemm_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x,
                 const __grid_constant__ CUtensorMap tm_z, const Int8Params p) {
  using C = Cfg<BT>;
  constexpr int ES = C::stages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* const gen = smem_raw + (base - raw);

  const uint32_t bar0 = base + C::barriers;
  auto full = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty = [&](uint32_t s) { return bar0 + 8u * (ES + s); };
  auto acc_full = [&](uint32_t b) { return bar0 + 8u * (2 * ES + b); };
  auto acc_empty = [&](uint32_t b) { return bar0 + 8u * (2 * ES + 2 + b); };
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + C::tmem_slot);
  volatile uint32_t* const abort_flag = reinterpret_cast<volatile uint32_t*>(gen + C::abort_flag);
  int* const hi = reinterpret_cast<int*>(gen + C::groups);
  int* const first_tile = hi + p.groups + 1;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < ES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), 4); }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async();
    tma_prefetch_desc(&tm_w); tma_prefetch_desc(&tm_x);
    if (p.z_tma) tma_prefetch_desc(&tm_z);
  }
  if (warp == 1) {
    tmem_alloc(base + C::tmem_slot, C::tmem_cols);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_trigger();
  if (warp == kFirstEpiWarp) find_groups(p, BT, hi, first_tile, blockIdx.x == 0);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const long long units = static_cast<long long>(first_tile[p.groups]) * p.tiles_n;

  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    if (lane == 0) {
      uint32_t issued = 0, stage = 0, phase = 0;
      bool ok = true;
      for (long long u = blockIdx.x; ok && u < units; u += gridDim.x) {
        const Unit v = find_unit(u, p, BT, hi, first_tile);
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (!mbar_wait(empty(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t dst = base + stage * C::stage_bytes;
          mbar_arrive_expect_tx(full(stage), C::stage_bytes);
          tma_load_3d(dst, &tm_w, full(stage), kb * kBk, v.ch0, v.group);
          tma_load_2d(dst + kSlab, &tm_x, full(stage), kb * kBk, v.row0);
          ++issued;
          if (++stage == static_cast<uint32_t>(ES)) { stage = 0; phase ^= 1u; }
        }
      }
      // every copy must have landed before the CTA may exit
      for (int s = 0; s < ES; ++s)
        if (issued > static_cast<uint32_t>(s)) mbar_wait(full(s), ((issued - 1 - s) / ES) & 1u, abort_flag);
    }
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issuer
    if (lane == 0) {
      // S32 accumulator, signed 8-bit A and B, both K-major, M = 128; N per tile
      constexpr uint32_t idesc0 = (2u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kCh >> 4) << 24);
      const uint64_t da0 = umma_desc_sw128(base, 16, 1024), db0 = umma_desc_sw128(base + kSlab, 16, 1024);
      constexpr uint64_t kStageStep = C::stage_bytes >> 4;
      uint32_t stage = 0, phase = 0, it = 0;
      bool ok = true;
      for (long long u = blockIdx.x; ok && u < units; u += gridDim.x, ++it) {
        const Unit v = find_unit(u, p, BT, hi, first_tile);
        const uint32_t idesc = idesc0 | (static_cast<uint32_t>((v.rows + 15) / 16 * 2) << 17);
        const uint32_t buf = it & 1u;
        if (!mbar_wait(acc_empty(buf), ((it >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t tmem_d = tmem_base + buf * BT;
        uint32_t accumulate = 0;
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (!mbar_wait(full(stage), phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t da = da0 + stage * kStageStep, db = db0 + stage * kStageStep;
#pragma unroll
          for (int kk = 0; kk < kBk / 32; ++kk) {
            tc_mma<1>(tmem_d, da + kk * 2, db + kk * 2, idesc, accumulate);
            accumulate = 1;
          }
          tc_commit(empty(stage));
          if (++stage == static_cast<uint32_t>(ES)) { stage = 0; phase ^= 1u; }
        }
        if (ok) tc_commit(acc_full(buf));
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3;                      // tensor-memory lanes this warp may read
    const uint32_t stage0 = base + C::staging + (warp - kFirstEpiWarp) * 2 * kBox;
    uint8_t* const stage0_gen = gen + C::staging + (warp - kFirstEpiWarp) * 2 * kBox;
    float* const scales = reinterpret_cast<float*>(gen + C::token_scales + (warp - kFirstEpiWarp) * 128);
    uint32_t it = 0, box_it = 0;
    for (long long u = blockIdx.x; u < units; u += gridDim.x, ++it) {
      const Unit v = find_unit(u, p, BT, hi, first_tile);
      const int ch_first = v.ch0 + quarter * 32;
      const int ch = ch_first + lane;
      const bool ch_in = ch < p.N;
      const long long wi = static_cast<long long>(v.group) * p.N + ch;
      const float sw = ch_in ? __ldg(p.sw + wi) : 0.0f;
      const float bias = ch_in && p.bias ? __ldg(p.bias + wi) : 0.0f;
      const uint32_t buf = it & 1u;
      if (!mbar_wait(acc_full(buf), (it >> 1) & 1u, abort_flag)) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + buf * BT;
      if (ch_first < p.N) {                            // warp-uniform
#pragma unroll 1
        for (int c0 = 0; c0 < v.rows; c0 += C::chunk) {
          const int left = v.rows - c0;                // token rows of this step that exist
          uint32_t r[C::chunk];
          load_chunk<C::chunk>(taddr + c0, r);
          __syncwarp();                                // the previous step's scales have been read
          scales[lane] = lane < left ? __ldg(p.sx + v.row0 + c0 + lane) : 0.0f;
          __syncwarp();
          tmem_ld_wait();
          auto value = [&](int i, float s) { return fmaf(static_cast<float>(static_cast<int>(r[i])) * sw, s, bias); };
          if (C::chunk == 32 && p.z_tma && left >= 32 && (ch_first + 32 <= p.N || p.tma_cols == p.N)) {
            const uint32_t b = box_it & 1u;
            ++box_it;
            if (lane == 0) bulk_wait_read<1>();        // the store that last read this box is done
            __syncwarp();
            uint8_t* const box = stage0_gen + b * kBox;
#pragma unroll
            for (int i = 0; i < C::chunk; i += 4) {
              const float4 s4 = *reinterpret_cast<const float4*>(scales + i);
              const float s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float z = value(i + j, s[j]);
                uint8_t* const at = box + (p.out_bf16 ? (i + j) * 64 + lane * 2 : (i + j) * 128 + lane * 4);
                if (smem_in(at, gen, C::staging, C::token_scales, 4, p.status)) {
                  if (p.out_bf16) *reinterpret_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(z);
                  else *reinterpret_cast<float*>(at) = z;
                }
              }
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
              tma_store_2d(&tm_z, stage0 + b * kBox, ch_first, v.row0 + c0);
              bulk_commit();
            }
          } else if (ch_in) {
            const long long z0 = (static_cast<long long>(v.row0) + c0) * p.ld_z + ch;
#pragma unroll
            for (int i = 0; i < C::chunk; ++i) {
              if (i < left) {
                const float z = value(i, scales[i]);
                const long long at = z0 + i * p.ld_z;
                if (p.out_bf16) static_cast<__nv_bfloat16*>(p.z)[at] = __float2bfloat16_rn(z);
                else static_cast<float*>(p.z)[at] = z;
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(acc_empty(buf));
    }
    if (lane == 0) bulk_wait<0>();   // all stores of this warp are complete before the CTA exits
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, LUQ_STATUS_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::tmem_cols);
  }
}

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// int8 codes as [planes][rows][cols], boxes of box_rows x 128 bytes, 128-byte swizzle; what lies beyond the
// extents reads as zero
int encode_codes(void* fn, CUtensorMap* map, const int8_t* ptr, int64_t cols, int64_t rows, int64_t ld, int64_t planes,
                 int64_t plane_stride, int box_rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(planes)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld), static_cast<cuuint64_t>(plane_stride)};
  const cuuint32_t box[3] = {kBk, static_cast<cuuint32_t>(box_rows), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return reinterpret_cast<EncodeTiledFn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, planes > 0 ? 3 : 2, const_cast<int8_t*>(ptr),
                                             dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS;
}
// output [rows x cols], boxes of 32 x 32 elements as they lie in memory
int encode_z(void* fn, CUtensorMap* map, void* ptr, int64_t cols, int64_t rows, int64_t ld, bool bf16) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * (bf16 ? 2 : 4)};
  const cuuint32_t box[2] = {32, 32};
  const cuuint32_t estr[2] = {1, 1};
  return reinterpret_cast<EncodeTiledFn>(fn)(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2,
                                             ptr, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS;
}

template <int BT>
int launch(luq_ctx* ctx, const luq_int8_args& a, const Int8Params& p, const CUtensorMap& tw, const CUtensorMap& tz,
           cudaStream_t st) {
  CUtensorMap tx;
  if (encode_codes(ctx->encode_tiled, &tx, a.x_codes, a.K, a.M, a.ld_x, 0, 0, BT)) return LUQ_ERR_CUDA;
  auto kernel = int8_gemm_kernel<BT>;
  const int smem = Cfg<BT>::smem_bytes(p.groups);
  const cudaError_t attr = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (attr != cudaSuccess) return static_cast<int>(attr);
  // token tiles: at most one partial tile per group that has rows
  const long long partial = p.groups < a.M ? p.groups : a.M;
  const long long most = (a.M / BT + partial) * p.tiles_n;
  const int sms = (ctx->sm_limit > 0 && ctx->sm_limit < ctx->sm_count) ? ctx->sm_limit : ctx->sm_count;
  const int grid = static_cast<int>(most < sms ? most : sms);
  const cudaError_t e = luq_launch_kernel(kernel, grid, kThreads, static_cast<size_t>(smem), st, LUQ_LAUNCH_EARLY, 1, tw, tx, tz, p);
  if (e == cudaSuccess) ctx->launches += 1;
  return static_cast<int>(e);
}

}  // namespace

int luq_launch_gemm_int8(luq_ctx* ctx, const luq_int8_args& a, cudaStream_t st) {
  Int8Params p{};
  p.sx = a.sx; p.sw = a.sw; p.bias = a.bias; p.offsets = a.offsets; p.z = a.z; p.ld_z = a.ld_z; p.status = ctx->d_status;
  p.M = a.M; p.N = a.N; p.groups = a.groups; p.out_bf16 = a.out_bf16;
  p.num_kb = static_cast<int>((a.K + kBk - 1) / kBk);
  p.tiles_n = static_cast<int>((a.N + kCh - 1) / kCh);
  const int64_t esize = a.out_bf16 ? 2 : 4;
  p.z_tma = (reinterpret_cast<uintptr_t>(a.z) & 15u) == 0 && (a.ld_z * esize) % 16 == 0;
  p.tma_cols = a.N / (16 / esize) * (16 / esize);
  CUtensorMap tw, tz;
  if (encode_codes(ctx->encode_tiled, &tw, a.w_codes, a.K, a.N, a.ld_w, a.groups, a.w_stride, kCh)) return LUQ_ERR_CUDA;
  if (p.z_tma) {
    if (encode_z(ctx->encode_tiled, &tz, a.z, a.N, a.M, a.ld_z, a.out_bf16 != 0)) return LUQ_ERR_CUDA;
  } else {
    tz = tw;                                          // not used
  }
  // tokens a group has on average decide the tile: one tile holds them where it can
  const long long mean_rows = (a.M + a.groups - 1) / a.groups;
  if (mean_rows <= 16) return launch<16>(ctx, a, p, tw, tz, st);
  if (mean_rows <= 32) return launch<32>(ctx, a, p, tw, tz, st);
  if (mean_rows <= 64) return launch<64>(ctx, a, p, tw, tz, st);
  if (mean_rows <= 512) return launch<128>(ctx, a, p, tw, tz, st);
  return launch<256>(ctx, a, p, tw, tz, st);
}
