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
//   warp 0     TMA producer of W, 128 x 128 bytes per stage, 128-byte swizzle
//   warp 1     one thread issues tcgen05.mma kind::i8; owns the tensor-memory allocation (two accumulators)
//   warp 2     TMA producer of the tile's token rows x 128 bytes
//   warps 3..  epilogue: tcgen05.ld -> scales, bias -> staged 32 x 32 boxes -> TMA store; token rows
//              that share a box with another group's, and outputs TMA cannot address, are stored directly
// All waits are bounded; on expiry the CTA flags LUQ_STATUS_TIMEOUT, drains its copies, frees its
// tensor memory and returns.
//
// What bounds it: many tokens, the L2's delivery of operands next to the tensor cores (16384x4096x4096 175 us, 3.1 POP/s;
// 8192x4096x1024 32.8 us, 2.1 POP/s: a tile's epilogue, beside the next tile's contraction, takes longer than its eight stages); few tokens, the
// weights' bytes (32 tokens over 64 experts of 2048x1024 14.2 us) or, for one layer, the latency of a launch and one
// trip through memory (5 tokens, 4096x4096 6.0 us).
#include <cuda.h>
#include <cuda_bf16.h>

#include <climits>

#include "common.cuh"

namespace {

using namespace luqdev;

constexpr int kCh = 128;                  // output channels per tile (tensor-memory lanes)
constexpr int kBk = 128;                  // contraction elements per stage
constexpr int kSlab = kCh * kBk;          // bytes of W per stage
constexpr int kXWarp = 2;
constexpr int kFirstEpiWarp = 3;
constexpr int kWarpStaging = 32 * 32 * 4; // a warp's store boxes: one of 32 x 32 fp32, or two of bf16
constexpr int kMaxSplit = 8;              // CTAs that share a tile's contraction (a portable cluster)
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
  int row0, all_rows;       // these M rows are row0 .. of the rows that the offsets count
  int groups;
  int num_kb;
  int tiles_n;              // channel tiles
  int early;                // everything but the tokens' codes and scales was there before the preceding kernel
  int z_tma;                // the output can be addressed by TMA
  long long tma_cols;       // a store copy writes whole 16-byte pieces: boxes up to this column end on one
#ifdef LUQ_DEBUG
  int slack;                // LUQ_OPT_CHECK_SLACK
#endif
};
#ifdef LUQ_DEBUG
#define LUQ_CHECKED_N(p) ((p).N - (p).slack)
#else
#define LUQ_CHECKED_N(p) ((p).N)
#endif

// One tile: kCh channels (twice that on a CTA pair) by up to BT tokens.  The epilogue's warps come in groups of
// four (one per quarter of the lanes, 32 channels each); a group takes `span` tokens of the tile.
template <int BT, bool PAIR>
struct Cfg {
  static constexpr int epi_warps = BT <= 32 ? 4 : 8;
  static constexpr int span = BT / (epi_warps / 4);
  static constexpr int threads = 32 * (kFirstEpiWarp + epi_warps);
  static constexpr int x_rows = PAIR ? BT / 2 : BT;               // token rows this CTA holds of a tile
  static constexpr int part_rows = BT < 32 ? BT : 32;             // token rows per copy of a tile that is not full
  static constexpr int stage_bytes = kSlab + x_rows * kBk;
  static constexpr int per_sm = BT <= 32 ? 2 : 1;
  static constexpr int stages = BT == 16 ? 5 : BT == 32 ? 4 : BT == 64 ? 7 : 5;
  static constexpr int chunk = BT < 32 ? BT : 32;                 // tokens per epilogue step
  static constexpr int tmem_cols = 2 * BT;
  static constexpr int staging = stages * stage_bytes;            // store boxes
  static constexpr int token_scales = staging + (BT == 16 ? 0 : epi_warps * kWarpStaging);      // two tiles' scales
  // a split's partial tile lies where the stages were, which its contraction is done with
  static_assert(BT * kCh * 4 <= stages * stage_bytes, "a partial tile has to fit the stages");
  static constexpr int barriers = token_scales + 2 * BT * 4;
  static constexpr int num_barriers = 2 * stages + 4;
  static constexpr int tmem_slot = barriers + 8 * num_barriers;
  static constexpr int abort_flag = tmem_slot + 4;
  static constexpr int groups = abort_flag + 4;                   // group ends, then tile prefix: 2 x (groups + 1) ints
  static constexpr int smem_bytes(int n_groups) { return groups + 8 * (n_groups + 1) + 1024; }
  static_assert(groups + 8 * (LUQ_MAX_GROUPS + 1) + 1024 <= 232448, "exceeds the 227 KB of shared memory a CTA may use");
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
__device__ __forceinline__ void find_groups(const Int8Params& p, int tile_rows, int* hi, int* first_tile, bool report) {
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
};
// The tiles of one CTA (or cluster), in order.  Tiles walk the channels in bands of kBand token tiles, tokens
// fastest: what runs together shares both operands' tiles in L2.  Every role and every epilogue warp walks for
// itself, so a step has no division but in the last band.  (There are less than 2^31 tiles: they would need more
// outputs than memory holds.)
struct Walk {
  int u, step, units, band, in_band, per_band, token_tiles;
  __device__ __forceinline__ Walk(const Int8Params& p, int tiles, int first, int by)
      : u(first), step(by), units(tiles * p.tiles_n), band(first / (kBand * p.tiles_n)), per_band(kBand * p.tiles_n), token_tiles(tiles) {
    in_band = first - band * per_band;
  }
  __device__ __forceinline__ bool more() const { return u < units; }
  __device__ __forceinline__ void next() {
    u += step;
    in_band += step;
    while (in_band >= per_band) { in_band -= per_band; ++band; }
  }
  __device__ __forceinline__ Unit unit(const Int8Params& p, int tile_rows, int tile_ch, const int* hi, const int* first_tile) const {
    const int width = min(kBand, token_tiles - band * kBand);
    const int c = width == kBand ? in_band / kBand : in_band / width;
    const int j = band * kBand + in_band - c * width;
    if (p.offsets == nullptr) {
      const int row0 = j * tile_rows;
      return Unit{0, row0, min(tile_rows, static_cast<int>(p.M) - row0), c * tile_ch};
    }
    int lo = 0, up = p.groups;                     // the last group whose first tile is <= j
    while (up - lo > 1) {
      const int mid = (lo + up) >> 1;
      if (first_tile[mid] <= j) lo = mid; else up = mid;
    }
    Unit v;
    v.group = lo;
    v.row0 = hi[lo] + (j - first_tile[lo]) * tile_rows;
    v.rows = min(tile_rows, hi[lo + 1] - v.row0);
    v.ch0 = c * tile_ch;
    return v;
  }
};

__device__ __forceinline__ void store_z(void* z, long long at, float v, bool bf16) {
  if (bf16) static_cast<__nv_bfloat16*>(z)[at] = __float2bfloat16_rn(v);
  else static_cast<float*>(z)[at] = v;
}
// is [row, ch] an output?  (always true outside the checking build)
__device__ __forceinline__ bool z_in(const Int8Params& p, long long row, int ch) {
  (void)p; (void)row; (void)ch;
  return LUQ_IN_BOUNDS(row >= 0 && row < p.M && ch >= 0 && ch < LUQ_CHECKED_N(p), p.status);
}
// two products and two sums of neighbouring tokens: z = (acc * sw) * s + bias
__device__ __forceinline__ float2 scale2(uint32_t a0, uint32_t a1, float2 sw, float2 s, float2 bias) {
  const float2 acc = make_float2(static_cast<float>(static_cast<int>(a0)), static_cast<float>(static_cast<int>(a1)));
  return __ffma2_rn(__fmul2_rn(acc, sw), s, bias);
}

// Takes a tile's accumulators out of tensor memory, scales them and writes them: this warp's quarter of the
// lanes (32 channels) and its group's span of tokens, in steps of 32.
// A full step goes through a staged box [token][channel] and a copy; a step that holds rows of another
// group, or an output the copies cannot address, is written element by element (32 channels in a row).
// One fence serves all boxes a warp has (two of bf16, one of fp32).
template <typename C, bool BF16>
__device__ __forceinline__ void write_tile(const Int8Params& p, const void* tm_z, const Unit& v, float sw, float bias,
                                           uint32_t taddr, uint32_t tmem_base, int warp_e, int lane, uint32_t staging,
                                           uint8_t* gen, const float* scales) {
  constexpr int CH = C::chunk, kSteps = C::span / CH, kPair = kSteps < 2 ? kSteps : 2;
  constexpr int kBoxes = BF16 ? 2 : 1, kBoxBytes = kWarpStaging / kBoxes;
  const int quarter = (warp_e + kFirstEpiWarp) & 3;
  const int ch_first = v.ch0 + quarter * 32, ch = ch_first + lane;
  const int c_first = (warp_e >> 2) * C::span;
  if (ch_first >= p.N || c_first >= v.rows) return;    // warp-uniform
  const bool boxes = CH == 32 && p.z_tma && (ch_first + 32 <= p.N || p.tma_cols == p.N);
  const float2 sw2 = make_float2(sw, sw), bias2 = make_float2(bias, bias);
  const uint32_t slot = static_cast<uint32_t>(warp_e) * kWarpStaging;
  uint8_t* const box0 = gen + C::staging + slot;

  int staged = 0, first_staged = c_first;
  auto flush = [&]() {                                 // hands the staged boxes to the copy engine
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
      for (int i = 0; i < staged; ++i)
        if (z_in(p, v.row0 + first_staged + 32 * i + 31, min(ch_first + 31, static_cast<int>(p.N) - 1)))
          tma_store_2d(tm_z, staging + slot + i * kBoxBytes, ch_first, v.row0 + first_staged + 32 * i);
      bulk_commit();
    }
    staged = 0;
  };
#pragma unroll 1
  for (int pair = 0; pair < kSteps && c_first + pair * CH < v.rows; pair += kPair) {
    uint32_t r[kPair][CH];
#pragma unroll
    for (int i = 0; i < kPair; ++i)
      if (c_first + (pair + i) * CH < v.rows &&
          tmem_in(taddr + c_first + (pair + i) * CH, tmem_base, C::tmem_cols, p.status, CH)) load_chunk<CH>(taddr + c_first + (pair + i) * CH, r[i]);
    tmem_ld_wait();
#pragma unroll
    for (int step = 0; step < kPair; ++step) {
      const int c0 = c_first + (pair + step) * CH, left = v.rows - c0;
      if (boxes && left >= 32) {
        if (staged == 0) {                               // (first of its pair) the stores that last read this warp's boxes are done
          if (lane == 0) bulk_wait_read<0>();
          __syncwarp();
        }
        if (staged == 0) first_staged = c0;
        uint8_t* const box = box0 + staged * kBoxBytes;
        ++staged;
        // all scales first: between the stores below every load would wait for the last store
        float4 s_step[CH / 4];
#pragma unroll
        for (int i = 0; i < CH / 4; ++i) s_step[i] = reinterpret_cast<const float4*>(scales + c0)[i];
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
          const float4 s4 = s_step[i / 4];
          const float2 z[2] = {scale2(r[step][i], r[step][i + 1], sw2, make_float2(s4.x, s4.y), bias2),
                               scale2(r[step][i + 2], r[step][i + 3], sw2, make_float2(s4.z, s4.w), bias2)};
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if constexpr (BF16) {
              // a lane has one channel of two tokens, a word is two channels of one: neighbours swap halves, the
              // even lane keeps the first token's word, the odd lane the second's
              const __nv_bfloat162 h = __floats2bfloat162_rn(z[j].x, z[j].y);
              const uint32_t own = *reinterpret_cast<const uint32_t*>(&h);
              const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, own, 1);
              const uint32_t word = __byte_perm(own, other, lane & 1 ? 0x3276 : 0x5410);
              uint8_t* const at = box + (i + 2 * j + (lane & 1)) * 64 + (lane >> 1) * 4;
              if (smem_in(at, gen, C::staging, C::token_scales, 4, p.status)) *reinterpret_cast<uint32_t*>(at) = word;
            } else {
              uint8_t* const at = box + (i + 2 * j) * 128 + lane * 4;
              if (smem_in(at, gen, C::staging, C::token_scales, 132, p.status)) {
                *reinterpret_cast<float*>(at) = z[j].x;
                *reinterpret_cast<float*>(at + 128) = z[j].y;
              }
            }
          }
        }
        if (staged == kBoxes) flush();
      } else if (left > 0 && ch < p.N) {
        const long long z0 = (static_cast<long long>(v.row0) + c0) * p.ld_z + ch;
#pragma unroll
        for (int i = 0; i < CH; i += 2) {
          if (i < left) {
            const float2 z = scale2(r[step][i], r[step][i + 1], sw2, make_float2(scales[c0 + i], scales[c0 + i + 1]), bias2);
            if (z_in(p, v.row0 + c0 + i, ch)) store_z(p.z, z0 + i * p.ld_z, z.x, BF16);
            if (i + 1 < left && z_in(p, v.row0 + c0 + i + 1, ch)) store_z(p.z, z0 + (i + 1) * p.ld_z, z.y, BF16);
          }
        }
      }
    }
    if (staged) flush();
  }
}

// Adds a channel's partial sums of Q CTAs (of fewer, if the cluster has fewer) for every stride-th token and
// writes the results; sixteen loads from the other CTAs are on their way at once.
template <int Q>
__device__ __forceinline__ void join(const Int8Params& p, const Unit& v, uint32_t column, uint32_t end, int first_token, int stride, int ch,
                                     float sw, float bias, const float* scales, bool bf16) {
  constexpr int U = 16 / Q;
  const int cluster = static_cast<int>(cluster_nctarank());
  for (int t0 = first_token; t0 < v.rows; t0 += U * stride) {
    int part[U][Q];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int q = 0; q < Q; ++q)
        part[u][q] = q < cluster && t0 + u * stride < v.rows &&
                             LUQ_IN_BOUNDS(t0 >= 0 && column + (t0 + u * stride) * kCh * 4 + 4 <= end, p.status) ? ld_shared_cluster(mapa_shared(column + (t0 + u * stride) * kCh * 4, q)) : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * stride;
      int sum = 0;
#pragma unroll
      for (int q = 0; q < Q; ++q) sum += part[u][q];
      if (t < v.rows && z_in(p, v.row0 + t, ch))
        store_z(p.z, (static_cast<long long>(v.row0) + t) * p.ld_z + ch, fmaf(static_cast<float>(sum) * sw, scales[t], bias), bf16);
    }
  }
}

// SPLIT: the CTAs of a cluster share a tile and take a share of its contraction each (few tokens: too few tiles
// for the SMs); partial tiles meet through distributed shared memory, as integers, in any order exact.
// PAIR: the two CTAs of a cluster compute a tile of 256 channels together (cta_group::2), each fetches half of
// the tokens' rows.
template <int BT, bool PAIR, bool SPLIT, bool BF16>
__global__ void __launch_bounds__((Cfg<BT, PAIR>::threads), (Cfg<BT, PAIR>::per_sm))
int8_gemm_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x,
                 const __grid_constant__ CUtensorMap tm_x_part, const __grid_constant__ CUtensorMap tm_z, const Int8Params p) {
  static_assert(!(PAIR && SPLIT), "one use of the cluster at a time");
  using C = Cfg<BT, PAIR>;
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
  const uint32_t rank = PAIR || SPLIT ? cluster_ctarank() : 0u;
  const uint32_t cluster = PAIR ? 2u : (SPLIT ? cluster_nctarank() : 1u);
  // this CTA's share of a tile's contraction
  const int kb_first = SPLIT ? static_cast<int>(static_cast<long long>(p.num_kb) * rank / cluster) : 0;
  const int kb_end = SPLIT ? static_cast<int>(static_cast<long long>(p.num_kb) * (rank + 1) / cluster) : p.num_kb;
  const int by = static_cast<int>(gridDim.x / cluster), first = static_cast<int>(blockIdx.x / cluster);
  auto unit_of = [&](const Walk& w) { return w.unit(p, BT, PAIR ? 2 * kCh : kCh, hi, first_tile); };
  // copies of the tokens that a tile takes (one for a full tile: a quarter of the size is a quarter slower), and
  // the bytes of a stage of this CTA
  auto token_parts = [&](const Unit& v) {
    return ((PAIR ? (v.rows + 31) / 32 * 16 : v.rows) + C::part_rows - 1) / C::part_rows;
  };
  // the weights of a stage; counts the bytes of its tokens too
  auto w_copy = [&](const Unit& v, int kb, uint32_t s) {
    const uint32_t bytes = kSlab + token_parts(v) * C::part_rows * kBk;
    const uint32_t dst = base + s * C::stage_bytes;
    if constexpr (PAIR) {
      if (rank == 0) mbar_arrive_expect_tx(full(s), 2 * bytes);        // both CTAs' bytes
      tma_pair_load_3d(dst, &tm_w, mapa_shared(full(s), 0), kb * kBk, v.ch0 + static_cast<int>(rank) * kCh, v.group);
    } else {
      mbar_arrive_expect_tx(full(s), bytes);
      tma_load_3d(dst, &tm_w, full(s), kb * kBk, v.ch0, v.group);
    }
  };

  // (Loads in this file are plain ones: a load marked as read-only may be moved ahead of the wait for the kernel
  // that writes what it reads.)
  // Weights, offsets and channel scales may be read before the preceding kernel has ended when that kernel is
  // this call's own quantizer (which started after all earlier ones had ended); its codes and scales may not
  if (threadIdx.x == 0) {
    // on a pair the leader's barriers count both CTAs
    for (int s = 0; s < ES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), (PAIR ? 2 : 1) * C::epi_warps); }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async();
    tma_prefetch_desc(&tm_w); tma_prefetch_desc(&tm_x);
    if (C::part_rows < C::x_rows) tma_prefetch_desc(&tm_x_part);
    if (p.z_tma) tma_prefetch_desc(&tm_z);
  }
  if (warp == 1) {
    if constexpr (PAIR) { tmem_alloc_pair(base + C::tmem_slot, C::tmem_cols); tmem_relinquish_pair(); }
    else { tmem_alloc(base + C::tmem_slot, C::tmem_cols); tmem_relinquish(); }
  }
  if (!p.early) pdl_wait();
  pdl_trigger();
  if (warp == kFirstEpiWarp && p.offsets) find_groups(p, BT, hi, first_tile, blockIdx.x == 0);
  tc_fence_before();
  __syncwarp();
  if constexpr (PAIR) cluster_sync_all();              // both CTAs' barriers are set up
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // the tiles of this cluster: every (number of clusters)-th
  Walk walk(p, p.offsets ? first_tile[p.groups] : static_cast<int>((p.M + BT - 1) / BT), first, by);
  const bool idle = !walk.more();

  // ---- the roles, a unit at a time; state lives across units ----
  uint32_t stage = 0, phase = 0, issued = 0, it = 0;
  bool ok = true, waited = !p.early;

  // one thread fetches the weights, another the tokens (two threads pull more than one)
  auto produce = [&](const Unit& v, bool tokens) {
    // token rows of this CTA: all of the tile's, or on a pair its half of the instruction's extent
    const int x_row0 = v.row0 + (PAIR ? static_cast<int>(rank) * ((v.rows + 31) / 32 * 16) : 0);
    const int parts = token_parts(v);
    const bool whole = parts * C::part_rows == C::x_rows;
    for (int kb = kb_first; kb < kb_end; ++kb) {
      if (!mbar_wait(empty(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
      if (!tokens) {
        w_copy(v, kb, stage);
      } else {
        const uint32_t dst = base + stage * C::stage_bytes + kSlab;
        const uint32_t bar = PAIR ? mapa_shared(full(stage), 0) : full(stage);
        if (whole) {
          if constexpr (PAIR) tma_pair_load_2d(dst, &tm_x, bar, kb * kBk, x_row0);
          else tma_load_2d(dst, &tm_x, bar, kb * kBk, x_row0);
        } else {
          for (int b = 0; b < parts; ++b) {
            const int off = b * C::part_rows;
            if constexpr (PAIR) tma_pair_load_2d(dst + off * kBk, &tm_x_part, bar, kb * kBk, x_row0 + off);
            else tma_load_2d(dst + off * kBk, &tm_x_part, bar, kb * kBk, x_row0 + off);
          }
        }
      }
      ++issued;
      if (++stage == static_cast<uint32_t>(ES)) { stage = 0; phase ^= 1u; }
    }
  };
  auto drain = [&]() {                                 // every copy must have landed before the CTA may exit
    if (PAIR && rank != 0) return;                     // the leader's barriers count both CTAs' copies
    for (int s = 0; s < ES; ++s)
      if (issued > static_cast<uint32_t>(s)) {
        if constexpr (PAIR) mbar_wait_cluster(full(s), ((issued - 1 - s) / ES) & 1u, abort_flag);
        else mbar_wait(full(s), ((issued - 1 - s) / ES) & 1u, abort_flag);
      }
  };
  auto multiply = [&](const Unit& v) {                 // one thread (of the leader)
    // S32 accumulator, signed 8-bit A and B, both K-major; N covers the tile's tokens
    const uint32_t n8 = PAIR ? (v.rows + 31) / 32 * 4 : (v.rows + 15) / 16 * 2;
    const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (n8 << 17) | (static_cast<uint32_t>((PAIR ? 2 : 1) * kCh >> 4) << 24);
    const uint64_t da0 = umma_desc_sw128(base, 16, 1024), db0 = umma_desc_sw128(base + kSlab, 16, 1024);
    constexpr uint64_t kStageStep = C::stage_bytes >> 4;
    const uint32_t buf = it & 1u;
    const bool free = PAIR ? mbar_wait_cluster(acc_empty(buf), ((it >> 1) & 1u) ^ 1u, abort_flag)
                           : mbar_wait(acc_empty(buf), ((it >> 1) & 1u) ^ 1u, abort_flag);
    if (!free) { ok = false; return; }
    tc_fence_after();
    const uint32_t tmem_d = tmem_base + buf * BT;
    uint32_t accumulate = 0;
    for (int kb = kb_first; kb < kb_end; ++kb) {
      const bool there = PAIR ? mbar_wait_cluster(full(stage), phase, abort_flag) : mbar_wait(full(stage), phase, abort_flag);
      if (!there) { ok = false; return; }
      tc_fence_after();
      const uint64_t da = da0 + stage * kStageStep, db = db0 + stage * kStageStep;
#pragma unroll
      for (int kk = 0; kk < kBk / 32; ++kk) {
        if constexpr (PAIR) tc_mma_pair<1>(tmem_d, da + kk * 2, db + kk * 2, idesc, accumulate);
        else tc_mma<1>(tmem_d, da + kk * 2, db + kk * 2, idesc, accumulate);
        accumulate = 1;
      }
      if constexpr (PAIR) tc_commit_pair(empty(stage));
      else tc_commit(empty(stage));
      if (++stage == static_cast<uint32_t>(ES)) { stage = 0; phase ^= 1u; }
    }
    if constexpr (PAIR) tc_commit_pair(acc_full(buf));
    else tc_commit(acc_full(buf));
  };

  const int warp_e = warp - kFirstEpiWarp;
  const uint32_t lane_base = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  auto scales_of = [&](uint32_t i) { return reinterpret_cast<float*>(gen + C::token_scales) + (i & 1u) * BT; };
  // What a tile's epilogue needs from global memory, one tile ahead: this thread's token scale (the warps share
  // them through shared memory) and its channel's scale and bias.
  float s_ahead = 0.0f, sw_ahead = 0.0f, bias_ahead = 0.0f;
  auto look_ahead = [&](const Unit& v) {
    const int ch = v.ch0 + (warp & 3) * 32 + lane;
    const bool ch_in = ch < p.N;
    const long long wi = static_cast<long long>(v.group) * p.N + ch;
    (void)LUQ_IN_BOUNDS(v.group >= 0 && v.group < p.groups && v.row0 >= 0 && v.row0 + v.rows <= p.M && v.rows <= BT, p.status);
    sw_ahead = ch_in ? *(p.sw + wi) : 0.0f;
    bias_ahead = ch_in && p.bias ? *(p.bias + wi) : 0.0f;
    if (!waited) { pdl_wait(); waited = true; }
    const int t = threadIdx.x - 32 * kFirstEpiWarp;
    if (t < v.rows) s_ahead = *(p.sx + v.row0 + t);
  };
  // the tile two before has been written by all warps once this one meets them here
  auto share_scales = [&]() {
    const int t = threadIdx.x - 32 * kFirstEpiWarp;
    if (t < BT) scales_of(it)[t] = s_ahead;
    asm volatile("bar.sync 1, %0;" ::"n"(32 * C::epi_warps) : "memory");
  };
  static_assert(32 * C::epi_warps >= BT, "a thread fetches one token's scale");

  if constexpr (!SPLIT) {
    if (warp == 0 || warp == kXWarp) {
      if (lane == 0) {
        if (warp == kXWarp && !waited) pdl_wait();
        for (; ok && walk.more(); walk.next()) produce(unit_of(walk), warp == kXWarp);
        if (warp == 0) drain();
      }
    } else if (warp == 1) {
      if (lane == 0 && rank == 0)
        for (; ok && walk.more(); walk.next(), ++it) multiply(unit_of(walk));
    } else {
      Unit next{};
      auto ahead = [&]() {
        next = unit_of(walk);
        if (PAIR) next.ch0 += static_cast<int>(rank) * kCh;
        look_ahead(next);
      };
      if (walk.more()) ahead();
      while (walk.more()) {
        const Unit v = next;
        const float sw = sw_ahead, bias = bias_ahead;
        share_scales();
        walk.next();
        if (walk.more()) ahead();
        const uint32_t buf = it & 1u;
        // after a wait that ran out the loop goes on without touching the tile: the warps keep meeting
        ok = ok && mbar_wait(acc_full(buf), (it >> 1) & 1u, abort_flag);
        if (ok) {
          tc_fence_after();
          write_tile<C, BF16>(p, &tm_z, v, sw, bias, lane_base + buf * BT, tmem_base, warp_e, lane, base + C::staging, gen, scales_of(it));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) mbar_arrive_leader(mapa_shared(acc_empty(buf), 0));
          else mbar_arrive(acc_empty(buf));
        }
        ++it;
      }
      if (lane == 0) bulk_wait<0>();   // all stores of this warp are complete before the CTA exits
    }
  } else {
    int* const partial = reinterpret_cast<int*>(gen);      // [token][channel], in place of the stages
    for (; walk.more(); walk.next(), ++it) {
      const Unit v = unit_of(walk);
      if (warp == 0 || warp == kXWarp) {
        if (lane == 0 && ok) {
          if (warp == kXWarp && !waited) { pdl_wait(); waited = true; }
          produce(v, warp == kXWarp);
        }
      } else if (warp == 1) {
        if (lane == 0 && ok) multiply(v);
      } else {
        look_ahead(v);
        share_scales();
        const uint32_t buf = it & 1u;
        ok = ok && mbar_wait(acc_full(buf), (it >> 1) & 1u, abort_flag);
        tc_fence_after();
        for (int c = (warp_e >> 2) * C::chunk; ok && c < v.rows; c += C::epi_warps / 4 * C::chunk) {
          uint32_t r[C::chunk];
          if (!tmem_in(lane_base + buf * BT + c, tmem_base, C::tmem_cols, p.status, C::chunk)) continue;
          load_chunk<C::chunk>(lane_base + buf * BT + c, r);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < C::chunk; ++i)
            if (smem_in(partial + (c + i) * kCh + (warp & 3) * 32 + lane, gen, 0, C::staging, 4, p.status))
              partial[(c + i) * kCh + (warp & 3) * 32 + lane] = static_cast<int>(r[i]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acc_empty(buf));
      }
      __syncwarp();
      cluster_sync_all();              // every CTA's partial tile is there
      if (warp >= kFirstEpiWarp) {
        // a token's 128 channels at a time, tokens dealt out over the CTAs
        const int ch = v.ch0 + (warp & 3) * 32 + lane;
        const int first_token = static_cast<int>(rank) + (warp_e >> 2) * static_cast<int>(cluster);
        const int stride = static_cast<int>(cluster) * (C::epi_warps / 4);
        const uint32_t column = smem_u32(partial + (warp & 3) * 32 + lane);
        if (ch < p.N) {                // every load below is used, and so has ended, before the meeting after it
          if (cluster <= 2) join<2>(p, v, column, base + C::staging, first_token, stride, ch, sw_ahead, bias_ahead, scales_of(it), BF16);
          else if (cluster <= 4) join<4>(p, v, column, base + C::staging, first_token, stride, ch, sw_ahead, bias_ahead, scales_of(it), BF16);
          else join<8>(p, v, column, base + C::staging, first_token, stride, ch, sw_ahead, bias_ahead, scales_of(it), BF16);
        }
        fence_proxy_async();           // the next tile's copies come after these reads
      }
      __syncwarp();
      cluster_sync_relaxed();          // and has been read by all
    }
    if (warp == 0 && lane == 0) drain();
  }

  // a CTA without tiles has waited for nothing yet: what comes after this kernel relies on the preceding one
  // having ended too
  if (p.early && idle) pdl_wait();
  tc_fence_before();
  __syncwarp();
  if constexpr (PAIR) cluster_sync_all();              // neither CTA leaves while the other's copies or arrivals need it
  else __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, LUQ_STATUS_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    if constexpr (PAIR) tmem_dealloc_pair(tmem_base, C::tmem_cols);
    else tmem_dealloc(tmem_base, C::tmem_cols);
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

template <int BT, bool PAIR, bool SPLIT, bool BF16>
int launch(luq_ctx* ctx, const luq_int8_args& a, const Int8Params& p, long long units, int cluster,
           const CUtensorMap& tz, cudaStream_t st) {
  using C = Cfg<BT, PAIR>;
  CUtensorMap tw, tx, tx_part;
  if (encode_codes(ctx->encode_tiled, &tw, a.w_codes, a.K, a.N, a.ld_w, a.groups, a.w_stride, kCh)) return LUQ_ERR_CUDA;
  if (encode_codes(ctx->encode_tiled, &tx, a.x_codes, a.K, a.M, a.ld_x, 0, 0, C::x_rows)) return LUQ_ERR_CUDA;
  if (C::part_rows == C::x_rows) tx_part = tx;
  else if (encode_codes(ctx->encode_tiled, &tx_part, a.x_codes, a.K, a.M, a.ld_x, 0, 0, C::part_rows)) return LUQ_ERR_CUDA;
  auto kernel = int8_gemm_kernel<BT, PAIR, SPLIT, BF16>;
  static luq_once_per_device allowed;
  const cudaError_t attr = allowed([&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem_bytes(LUQ_MAX_GROUPS));
  }, ctx->device);
  if (attr != cudaSuccess) return static_cast<int>(attr);
  const int sms = (ctx->sm_limit > 0 && ctx->sm_limit < ctx->sm_count) ? ctx->sm_limit : ctx->sm_count;
  const long long most = sms * C::per_sm / cluster > 0 ? sms * C::per_sm / cluster : 1;
  const int grid = static_cast<int>(units < most ? units : most) * cluster;
  const cudaError_t e = luq_launch_kernel(kernel, grid, C::threads, static_cast<size_t>(C::smem_bytes(p.groups)), st,
                                          LUQ_LAUNCH_EARLY, static_cast<unsigned>(cluster), tw, tx, tx_part, tz, p);
  if (e == cudaSuccess) ctx->launches += 1;
  return static_cast<int>(e);
}
template <int BT, bool PAIR, bool SPLIT>
int launch_out(luq_ctx* ctx, const luq_int8_args& a, const Int8Params& p, long long units, int cluster,
               const CUtensorMap& tz, cudaStream_t st) {
  return a.out_bf16 ? launch<BT, PAIR, SPLIT, true>(ctx, a, p, units, cluster, tz, st)
                    : launch<BT, PAIR, SPLIT, false>(ctx, a, p, units, cluster, tz, st);
}

// How long the product takes with each tile, in hundredths of a microsecond past the launch: rounds over the SMs
// x (stages x the time of one + what a tile costs at its ends).  The rates were fitted to 22 products of 40 to
// 13097 tokens, each timed with every tile and split; of 26 others the choice was the best or within 10% of it.
// What a stage takes is its share of the L2 (24 to 32 KB at 75-85 KB a microsecond and SM), not of the tensor cores.  A
// split pays its meeting and the sums over the other CTAs' memory; it is taken in a single round only.  Product
// alone: 2443x576x4096 14.7 us with 128-token tiles in one round, 24.0 with 64-token tiles in two, 17.2 with pairs;
// 1313x2340x3033 15.3 with pairs, 21.7 with 128; 142x384x3904 7.0 with 32-token tiles split in four, 12.3 unsplit.
struct Choice { int tokens, split; };
template <class Units>
Choice choose_tile(int sms, int num_kb, long long mean_rows, Units units) {
  struct Tile { int tokens, channels, ctas, stage, ends, meeting; };        // ctas: that one tile occupies
  constexpr Tile tiles[] = {{256, 2 * kCh, 2, 43, 150, 0}, {128, kCh, 1, 38, 50, 210}, {64, kCh, 1, 30, 50, 140}, {32, kCh, 1, 27, 40, 120}};
  Choice best{64, 1};
  long long best_time = LLONG_MAX;
  for (const Tile& t : tiles) {
    if (t.tokens == 256 && (sms < 2 || mean_rows <= 128)) continue;
    const long long n = units(t.tokens, t.channels);
    for (int split = 1; split <= kMaxSplit; split *= 2) {
      // clusters of four and eight do not fill the SMs: a group of SMs that share clusters has 16 to 20
      const long long slots = split > 2 ? sms - sms / 8 : sms;
      if (split > 1 && (t.tokens == 256 || n * split > slots || split > num_kb)) break;
      const long long rounds = (n + sms / t.ctas - 1) / (sms / t.ctas);
      const long long time = rounds * ((num_kb + split - 1) / split * t.stage + t.ends) + (split > 1 ? t.meeting : 0);
      if (time < best_time) { best_time = time; best = {t.tokens, split}; }
    }
  }
  return best;
}

}  // namespace

int luq_launch_gemm_int8(luq_ctx* ctx, const luq_int8_args& a, bool early, cudaStream_t st) {
  Int8Params p{};
  p.sx = a.sx; p.sw = a.sw; p.bias = a.bias; p.offsets = a.offsets; p.z = a.z; p.ld_z = a.ld_z; p.status = ctx->d_status;
  p.M = a.M; p.N = a.N; p.groups = a.groups; p.early = early;
  p.row0 = static_cast<int>(a.row0); p.all_rows = static_cast<int>(a.all_rows);
#ifdef LUQ_DEBUG
  p.slack = ctx->check_slack;
#endif
  p.num_kb = static_cast<int>((a.K + kBk - 1) / kBk);
  const int64_t esize = a.out_bf16 ? 2 : 4;
  p.z_tma = (reinterpret_cast<uintptr_t>(a.z) & 15u) == 0 && (a.ld_z * esize) % 16 == 0;
  p.tma_cols = a.N / (16 / esize) * (16 / esize);
  CUtensorMap tz{};                                   // not used where copies cannot address the output
  if (p.z_tma && encode_z(ctx->encode_tiled, &tz, a.z, a.N, a.M, a.ld_z, a.out_bf16 != 0)) return LUQ_ERR_CUDA;
  // most tiles there can be: at most one partial token tile per group that has rows
  const long long used = p.groups < a.M ? p.groups : a.M;
  auto units = [&](int tile_rows, int tile_ch) {
    p.tiles_n = static_cast<int>((a.N + tile_ch - 1) / tile_ch);
    return (p.groups == 1 ? (a.M + tile_rows - 1) / tile_rows : a.M / tile_rows + used) * p.tiles_n;
  };
  const int sms = (ctx->sm_limit > 0 && ctx->sm_limit < ctx->sm_count) ? ctx->sm_limit : ctx->sm_count;
  const long long mean_rows = (a.M + used - 1) / used;
  // The tile is the one that the model below expects to end first.  Up to 32 tokens a group, two small CTAs share
  // an SM (64 experts of 32 rows 16.8 -> 16.1 us, 8 experts of one row 15.7 -> 12.6 us, 60 experts of 17 rows 19.4 us
  // with 64-token tiles -> 18.1 us) and the contraction is split as far as it goes (one token, 4096x1024: 5.0 us).
  if (mean_rows > 32) {
    const Choice best = choose_tile(sms, p.num_kb, mean_rows, units);
    const long long n = units(best.tokens, best.tokens == 256 ? 2 * kCh : kCh);
    if (best.tokens == 256) return launch_out<256, true, false>(ctx, a, p, n, 2, tz, st);
    if (best.tokens == 128)
      return best.split > 1 ? launch_out<128, false, true>(ctx, a, p, n, best.split, tz, st) : launch_out<128, false, false>(ctx, a, p, n, 1, tz, st);
    if (best.tokens == 64)
      return best.split > 1 ? launch_out<64, false, true>(ctx, a, p, n, best.split, tz, st) : launch_out<64, false, false>(ctx, a, p, n, 1, tz, st);
    return best.split > 1 ? launch_out<32, false, true>(ctx, a, p, n, best.split, tz, st) : launch_out<32, false, false>(ctx, a, p, n, 1, tz, st);
  }
  const bool few = mean_rows <= 16;
  const long long n = units(few ? 16 : 32, kCh);
  int split = 1;
  while (split < kMaxSplit && n * split * 2 <= sms && split * 2 <= p.num_kb) split *= 2;
  if (few) return split > 1 ? launch_out<16, false, true>(ctx, a, p, n, split, tz, st) : launch_out<16, false, false>(ctx, a, p, n, 1, tz, st);
  return split > 1 ? launch_out<32, false, true>(ctx, a, p, n, split, tz, st) : launch_out<32, false, false>(ctx, a, p, n, 1, tz, st);
}
