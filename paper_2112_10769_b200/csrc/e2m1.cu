// Quantizer of rows (tokens, or the output channels of a weight) to 4-bit floating point with a scale for each block of a row
// (sm_100a).  Numbers are e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, packed two to a byte, the earlier one in the
// lower half.  Every operation below is rounded to binary32, to nearest.
//
//   blocks of 16   g = max|row| / 2688       s = e4m3(max|block| / (6 g))              q = e2m1(x * (1 / (s g)))
//   blocks of 32                             s = 2^(floor(log2 max|block|) - 2)        q = e2m1(x / s)
//
// 2688 = 6 * 448: the row's largest block gets the largest e4m3 number, its largest element the largest e2m1 number.  A block
// that is less than 2^-10 of the row's scale has a zero scale and zero numbers.
//
// Warps that share a row walk over rows; a thread holds chunks of 16 neighbouring elements in registers, so x is read once; the row's
// maximum meets in shared memory.  Block scales leave in the tiles that the
// tensor cores copy (128 rows x 4 blocks, row r, block b at 16 (r mod 32) + 4 (r / 32) + b): the threads of four blocks put
// their bytes together and one stores the word.
#include <cuda_bf16.h>

#include "common.cuh"

namespace {

using namespace luqdev;

constexpr int kChunk = 16;                 // elements of a thread
constexpr int kScaleTile = 512;

struct RowsParams {
  const void* x;
  long long rows, ld_x;
  int cols;
  long long plane_rows;
  const int* offsets;       // may be null
  int groups;
  const int* position;      // may be null
  int copies;
  long long out_rows;
  uint8_t* codes;
  long long ld_codes;
  uint8_t* tiles;
  float* scale;             // blocks of 16
  int k_tiles;
  unsigned int* status;
  bool vec;                 // rows of x start at multiples of 16 bytes
};

// The words of a thread's 16 elements, zeros beyond the row's end.  Where they do not lie in whole aligned pieces of 16 bytes they
// are put together from the pieces that hold an element of theirs.
template <typename T> constexpr int kWords = kChunk * static_cast<int>(sizeof(T)) / 4;
template <typename T>
__device__ __forceinline__ void load_chunk16(const T* row, int c0, int cols, bool vec, uint32_t (&w)[kWords<T>]) {
  constexpr int W = kWords<T>;
  if (vec && c0 + kChunk <= cols) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const uint4 u = reinterpret_cast<const uint4*>(row + c0)[i];
      w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
    }
    return;
  }
  if (c0 >= cols) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0u;
    return;
  }
  const uintptr_t at = reinterpret_cast<uintptr_t>(row + c0), end = reinterpret_cast<uintptr_t>(row + min(c0 + kChunk, cols));
  const uintptr_t low = at & ~static_cast<uintptr_t>(15);
  const int shift = static_cast<int>(at & 15u);
  uint32_t v[W + 4];
#pragma unroll
  for (int i = 0; i <= W / 4; ++i) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (low + 16 * i < end) u = *reinterpret_cast<const uint4*>(low + 16 * i);
    v[4 * i] = u.x; v[4 * i + 1] = u.y; v[4 * i + 2] = u.z; v[4 * i + 3] = u.w;
  }
  if (shift & 8) {
#pragma unroll
    for (int i = 0; i < W + 2; ++i) v[i] = v[i + 2];
  }
  if (shift & 4) {
#pragma unroll
    for (int i = 0; i < W + 1; ++i) v[i] = v[i + 1];
  }
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = sizeof(T) == 4 ? v[i] : __funnelshift_r(v[i], v[i + 1], 8 * (shift & 2));
  if (c0 + kChunk > cols) {
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
      if (c0 + i >= cols) {
        if constexpr (sizeof(T) == 4) w[i] = 0u;
        else w[i / 2] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
      }
  }
}
// the largest pattern of |x|, as a binary32 one: of numbers the largest, Inf above every number, NaN above Inf
template <typename T>
__device__ __forceinline__ uint32_t top_of(const uint32_t (&w)[kWords<T>]) {
  uint32_t t = 0;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < kWords<T>; ++i) t = max(t, w[i] & 0x7FFFFFFFu);
    return t;
  } else {
#pragma unroll
    for (int i = 0; i < kWords<T>; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(t) : "r"(w[i] & 0x7FFF7FFFu));
    return max(t << 16, t & 0xFFFF0000u);
  }
}
template <typename T>
__device__ __forceinline__ float2 pair_of(const uint32_t (&w)[kWords<T>], int i) {
  if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  else return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
// eight numbers from pairs `first` .. `first` + 3, the first in the lowest four bits
template <typename T>
__device__ __forceinline__ uint32_t pack8(const uint32_t (&w)[kWords<T>], int first, float f) {
  float2 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __fmul2_rn(pair_of<T>(w, first + i), make_float2(f, f));
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0].x), "f"(v[0].y), "f"(v[1].x), "f"(v[1].y), "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y));
  return r;
}
// the e4m3 number nearest to v >= 0 (at most 448), and its value
__device__ __forceinline__ uint32_t to_e4m3(float v, float& value) {
  uint16_t b;
  uint32_t h;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(0.0f), "f"(v));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(b));
  asm("{\n\t.reg .f16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.f32.f16 %0, lo;\n\t}" : "=f"(value) : "r"(h));
  return b & 0xFFu;
}

// What a row's elements are made of: the row's scale and six times it (blocks of 16), and whether it has numbers at all
struct RowScale {
  float g, six;
  bool dead;             // Inf or NaN, or nothing to scale by: zero codes
};
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  RowScale s;
  s.dead = top >= 0x7F800000u || top < 0x0D800000u;                 // 2^-100
  s.g = s.dead ? (top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : 0.0f) : __fdiv_rn(__uint_as_float(top), 2688.0f);
  s.six = __fmul_rn(s.g, 6.0f);
  return s;
}
// a block's scale byte and the factor of its elements
template <int BLOCK>
__device__ __forceinline__ uint32_t block_scale(uint32_t top, const RowScale& row, float& factor) {
  if constexpr (BLOCK == 16) {
    factor = 0.0f;
    if (row.dead) return 0u;
    float s;
    const uint32_t byte = to_e4m3(__fdiv_rn(__uint_as_float(top), row.six), s);
    if (s > 0.0f) factor = __frcp_rn(__fmul_rn(s, row.g));
    return byte;
  } else {
    if (top >= 0x7F800000u) { factor = 0.0f; return 255u; }
    const uint32_t byte = max(static_cast<int>(top >> 23) - 2, 0);
    factor = __uint_as_float((254u - byte) << 23);
    return byte;
  }
}

// The group of a row and the row's number in it, by a whole warp; false: the row belongs to none.  Whatever the offsets
// hold, start / 128 + group + in_group / 128 is below out_rows / 128 + groups.
__device__ __forceinline__ bool group_of(const RowsParams& p, int row, int& tile_row, int& in_tile) {
  const int lane = threadIdx.x & 31;
  int before = 0;                              // offsets 1 .. groups that are at most `row`
  for (int e0 = 1; e0 <= p.groups; e0 += 32) {
    const int e = e0 + lane;
    before += __popc(__ballot_sync(0xFFFFFFFFu, e <= p.groups && *(p.offsets + e) <= row));
  }
  if (before >= p.groups) return false;
  const int start = max(*(p.offsets + before), 0);
  if (start > row) return false;
  tile_row = start / 128 + before + (row - start) / 128;
  in_tile = (row - start) % 128;
  return true;
}

// Where a thread's chunk lies in every row: nothing here depends on the row.
template <int BLOCK>
struct Place {
  int bytes;             // of its codes that belong to the row, 8 at most
  long long code, tile;  // offsets of its codes, and of the word of four blocks' scales (negative: another thread stores it)
  int shift;             // its scale's place in that word
  __device__ __forceinline__ Place(const RowsParams& p, int chunk) {
    constexpr int kThreads4 = BLOCK == 16 ? 4 : 8;          // (blocks of 32 are two threads)
    const int lane = threadIdx.x & 31, kt = chunk / kThreads4;
    code = chunk * (kChunk / 2);
    bytes = min(max((p.cols + 1) / 2 - chunk * (kChunk / 2), 0), 8);
    tile = (lane & (kThreads4 - 1)) == 0 && kt < p.k_tiles ? static_cast<long long>(kt) * kScaleTile : -1;
    shift = 8 * (BLOCK == 16 ? lane & 3 : (lane >> 1) & 3);
  }
};
// the scales' bytes of four blocks in one word
template <int BLOCK>
__device__ __forceinline__ uint32_t scale_word(uint32_t byte, int shift) {
  uint32_t word = byte << shift;
  word |= __shfl_xor_sync(0xFFFFFFFFu, word, BLOCK == 16 ? 1 : 4);
  return word | __shfl_xor_sync(0xFFFFFFFFu, word, 2);
}
__device__ __forceinline__ long long tile_offset(const RowsParams& p, int tile_row, int in_tile) {
  return static_cast<long long>(tile_row) * (p.k_tiles * static_cast<long long>(kScaleTile)) + (in_tile & 31) * 16 + (in_tile >> 5) * 4;
}
template <int BLOCK>
__device__ __forceinline__ void store_chunk(const RowsParams& p, const Place<BLOCK>& at, int out_row, long long tiles_from, bool tiled, uint2 codes,
                                            uint32_t word) {
  if (!LUQ_IN_BOUNDS(out_row >= 0 && out_row < p.out_rows, p.status)) return;
  if (tiled && at.tile >= 0) *reinterpret_cast<uint32_t*>(p.tiles + tiles_from + at.tile) = word;
  uint8_t* const to = p.codes + out_row * p.ld_codes + at.code;
  if (at.bytes == 8) {
    *reinterpret_cast<uint2*>(to) = codes;
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < at.bytes) to[i] = static_cast<uint8_t>((i < 4 ? codes.x : codes.y) >> (8 * (i & 3)));
  }
}

// A chunk in registers -> its codes and scale byte
template <typename T, int BLOCK>
__device__ __forceinline__ void quantize_chunk(const uint32_t (&w)[kWords<T>], uint32_t top, const RowScale& row, uint2& codes, uint32_t& byte) {
  float f;
  byte = block_scale<BLOCK>(top, row, f);
  // (a factor of zero would leave NaN where there is Inf)
  codes = f > 0.0f ? make_uint2(pack8<T>(w, 0, f), pack8<T>(w, 4, f)) : make_uint2(0u, 0u);
}

// LANES lanes (kBlockRow: a block, of any number of warps) share a row; blocks walk over rows.  CHUNKS chunks of a thread, every
// LANES-th of the row; CHUNKS = 0: any width, chunks are read again for the second pass (from L2).  PLAN: rows go where offsets and
// positions say.
constexpr int kBlockRow = 0;
template <typename T, int BLOCK, int LANES, int CHUNKS, bool PLAN>
__global__ void __launch_bounds__(LANES == kBlockRow ? 1024 : 128) e2m1_rows_kernel(const RowsParams p) {
  static_assert(!PLAN || LANES == kBlockRow || LANES == 32, "a plan is read by whole warps");
  constexpr int kHeld = CHUNKS > 0 ? CHUNKS : 1;
  __shared__ uint32_t box[2][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lanes = LANES == kBlockRow ? static_cast<int>(blockDim.x) : LANES, per_block = LANES == kBlockRow ? 1 : 128 / (LANES == kBlockRow ? 1 : LANES);
  const int t = LANES == kBlockRow ? static_cast<int>(threadIdx.x) : static_cast<int>(threadIdx.x) % (LANES == kBlockRow ? 1 : LANES);
  const int chunks = p.k_tiles * (4 * BLOCK / kChunk);        // with the padding of the last tile of scales
  const int rows = static_cast<int>(p.rows), step = static_cast<int>(gridDim.x) * per_block;
  const long long plane_tiles = (p.plane_rows + 127) / 128;
  pdl_wait();
  pdl_trigger();
  int turn = 0;
  for (int first = static_cast<int>(blockIdx.x) * per_block; first < rows; first += step, turn ^= 1) {
    const int r = first + (LANES == kBlockRow ? 0 : static_cast<int>(threadIdx.x) / (LANES == kBlockRow ? 1 : LANES));
    const bool there = r < rows;
    if (LANES == 32 && !there) break;                          // (a whole warp; nothing meets)
    const T* const x = static_cast<const T*>(p.x) + (there ? r : 0) * p.ld_x;
    uint32_t w[kHeld][kWords<T>], top[kHeld] = {}, row_top = 0;
    if constexpr (CHUNKS > 0) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) load_chunk16(x, (t + i * lanes) * kChunk, p.cols, p.vec, w[i]);
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) { top[i] = top_of<T>(w[i]); row_top = max(row_top, top[i]); }
    } else {
      for (int c = t; c * kChunk < p.cols; c += lanes) {
        load_chunk16(x, c * kChunk, p.cols, p.vec, w[0]);
        row_top = max(row_top, top_of<T>(w[0]));
      }
    }
    if constexpr (LANES == kBlockRow || LANES == 32) {
      row_top = __reduce_max_sync(0xFFFFFFFFu, row_top);
    } else {
#pragma unroll
      for (int o = LANES / 2; o; o >>= 1) row_top = max(row_top, __shfl_xor_sync(0xFFFFFFFFu, row_top, o));
    }
    if (LANES == kBlockRow && BLOCK == 16) {                   // (blocks of 32 need no maximum of the row: each warp reports its own)
      if (lane == 0) box[turn][warp] = row_top;
      __syncthreads();                                         // (the box of the row before has been read by all: two are enough)
      row_top = __reduce_max_sync(0xFFFFFFFFu, lane * 32 < lanes ? box[turn][lane] : 0u);
    }
    RowScale row{};
    if constexpr (BLOCK == 16) row = row_scale(row_top);
    if (row_top >= 0x7F800000u || (BLOCK == 16 && row_top < 0x0D800000u && row_top > 0)) {
      if ((LANES == kBlockRow ? lane : t) == 0 && there) atomicOr(p.status, row_top >= 0x7F800000u ? LUQ_STATUS_NONFINITE : LUQ_STATUS_RANGE);
    }
    // calls f(row to write, offset of its scales' words, have they a place) for every place that the row goes to
    auto places = [&](auto f) {
      if constexpr (!PLAN) {
        if (!there) return;
        if (p.plane_rows == p.rows) {
          f(r, tile_offset(p, r / 128, r % 128), true);
        } else {
          const int plane = r / static_cast<int>(p.plane_rows), in_plane = r - plane * static_cast<int>(p.plane_rows);
          f(r, tile_offset(p, static_cast<int>(plane * plane_tiles) + in_plane / 128, in_plane % 128), true);
        }
      } else {
        for (int j = 0; j < p.copies; ++j) {
          const int to = p.position ? *(p.position + static_cast<long long>(r) * p.copies + j) : r;
          if (to < 0 || to >= p.out_rows) continue;            // warp-uniform
          int tile_row = 0, in_tile = 0;
          const bool tiled = group_of(p, to, tile_row, in_tile);
          f(to, tile_offset(p, tile_row, in_tile), tiled);
        }
      }
    };
    auto finish = [&](const uint32_t (&v)[kWords<T>], uint32_t b, int c, uint2& codes) {        // codes, and the scales' word
      uint32_t byte;
      if (BLOCK == 32) b = max(b, __shfl_xor_sync(0xFFFFFFFFu, b, 1));
      quantize_chunk<T, BLOCK>(v, b, row, codes, byte);
      return scale_word<BLOCK>(c < chunks ? byte : 0u, Place<BLOCK>(p, c).shift);
    };
    if constexpr (CHUNKS > 0) {
      uint2 codes[kHeld];
      uint32_t word[kHeld];
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) word[i] = finish(w[i], top[i], t + i * lanes, codes[i]);
      places([&](int to, long long tiles_from, bool tiled) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) store_chunk<BLOCK>(p, Place<BLOCK>(p, t + i * lanes), to, tiles_from, tiled, codes[i], word[i]);
      });
    } else {
      for (int c = t; c - lane < chunks; c += lanes) {
        load_chunk16(x, c * kChunk, p.cols, p.vec, w[0]);
        uint2 codes;
        const uint32_t word = finish(w[0], top_of<T>(w[0]), c, codes);
        const Place<BLOCK> at(p, c);
        places([&](int to, long long tiles_from, bool tiled) { store_chunk<BLOCK>(p, at, to, tiles_from, tiled, codes, word); });
      }
    }
    if (BLOCK == 16 && t == 0 && there) {
      if constexpr (PLAN) {
        for (int j = 0; j < p.copies; ++j) {
          const int to = p.position ? *(p.position + static_cast<long long>(r) * p.copies + j) : r;
          if (to >= 0 && to < p.out_rows) p.scale[to] = row.g;
        }
      } else {
        p.scale[r] = row.g;
      }
    }
  }
}

template <typename T, int BLOCK, int LANES, int CHUNKS, bool PLAN>
int launch(luq_ctx* ctx, const RowsParams& p, int threads, cudaStream_t st) {
  const int per_block = LANES == kBlockRow ? 1 : 128 / (LANES == kBlockRow ? 1 : LANES);
  // bf16: as many blocks as may be resident at once, which walk (16384 x 4096, blocks of 32: 27.8 us, 29.2 with a block for every
  // row); fp32: a block for every row (44.8 us, walking 49.3)
  const long long blocks = (p.rows + per_block - 1) / per_block, most = sizeof(T) == 2 ? static_cast<long long>(ctx->sm_count) * (2048 / threads) : blocks;
  const cudaError_t e = luq_launch_kernel(e2m1_rows_kernel<T, BLOCK, LANES, CHUNKS, PLAN>, static_cast<int>(blocks < most ? blocks : most), threads, 0,
                                          st, LUQ_LAUNCH_EARLY, 1, p);
  if (e == cudaSuccess) ctx->launches += 1;
  return static_cast<int>(e);
}
// Narrow rows share a warp.  A thread takes two chunks where there are rows enough to fill the card (the steps that a row costs are
// shared: 16384 x 4096 bf16, blocks of 16: 33 us, with one chunk 44, with four 43), one where a few rows' latency counts.
template <typename T, int BLOCK, bool PLAN>
int launch_width(luq_ctx* ctx, const RowsParams& p, cudaStream_t st) {
  const int chunks = p.k_tiles * (4 * BLOCK / kChunk);
  if constexpr (!PLAN) {
    if (chunks <= 8) return launch<T, BLOCK, 8, 1, PLAN>(ctx, p, 128, st);
    if (chunks <= 16) return launch<T, BLOCK, 16, 1, PLAN>(ctx, p, 128, st);
  }
  if (chunks <= 32) return launch<T, BLOCK, 32, 1, PLAN>(ctx, p, 128, st);
  const bool many = p.rows >= 4ll * ctx->sm_count;
  if (chunks <= 64 && many) return launch<T, BLOCK, 32, 2, PLAN>(ctx, p, 128, st);
  if (chunks <= 1024 && !many) return launch<T, BLOCK, kBlockRow, 1, PLAN>(ctx, p, (chunks + 31) / 32 * 32, st);
  if (chunks <= 2048) return launch<T, BLOCK, kBlockRow, 2, PLAN>(ctx, p, (chunks + 63) / 64 * 32, st);
  return launch<T, BLOCK, kBlockRow, 0, PLAN>(ctx, p, 1024, st);
}
template <typename T, int BLOCK>
int launch_plan(luq_ctx* ctx, const RowsParams& p, cudaStream_t st) {
  return p.offsets ? launch_width<T, BLOCK, true>(ctx, p, st) : launch_width<T, BLOCK, false>(ctx, p, st);
}

}  // namespace

int luq_launch_e2m1_rows(luq_ctx* ctx, const luq_e2m1_rows_args& a, cudaStream_t st) {
  RowsParams p{};
  p.x = a.x; p.rows = a.rows; p.ld_x = a.ld_x; p.cols = static_cast<int>(a.cols);
  p.plane_rows = a.plane_rows; p.offsets = a.offsets; p.groups = a.groups; p.position = a.position; p.copies = a.copies;
  p.out_rows = a.out_rows; p.codes = a.codes; p.ld_codes = a.ld_codes; p.tiles = a.tiles; p.scale = a.scale;
  p.k_tiles = static_cast<int>(luq_e2m1_k_tiles(a.cols, a.block));
  p.status = ctx->d_status;
  p.vec = (reinterpret_cast<uintptr_t>(a.x) & 15u) == 0 && (a.rows <= 1 || a.ld_x * (a.dtype == LUQ_BF16 ? 2 : 4) % 16 == 0);
  if (a.dtype == LUQ_BF16) return a.block == 16 ? launch_plan<__nv_bfloat16, 16>(ctx, p, st) : launch_plan<__nv_bfloat16, 32>(ctx, p, st);
  return a.block == 16 ? launch_plan<float, 16>(ctx, p, st) : launch_plan<float, 32>(ctx, p, st);
}
