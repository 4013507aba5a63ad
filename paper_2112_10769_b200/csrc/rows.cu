// Row-wise operators (sm_100a): layer norm forward and backward, and the quantizer that gives every row
// (token) an int8 scale of its own, alone or on the result of the layer norm.
//
//   mean = 1/C sum_c x_c        var = 1/C sum_c (x_c - mean)^2        rstd = (var + eps)^-1/2
//   y_c  = (x_c - mean) rstd gamma_c + beta_c
//   backward, with xhat = (x - mean) rstd and g = dy gamma:
//   dx_c = rstd (g_c - 1/C sum g - xhat_c 1/C sum g xhat)   dgamma_c = sum_r dy xhat   dbeta_c = sum_r dy
//   int8: scale = max_c |v_c| / 127, q_c = rint(v_c * fl32(127 / max)), ties to even
//
// All statistics and sums are binary32 and summed in a fixed order (no atomics on sums), so a call
// repeats bit for bit.  The mean is corrected once by the sum of the centred values, and values are centred with
// both parts: a row whose mean is far above its spread loses nothing beyond the input's own rounding.
#include <cuda_bf16.h>

#include "common.cuh"

namespace {

using namespace luqdev;

constexpr int kNorm = 0, kNormInt8 = 1, kInt8 = 2;   // what a row kernel makes of a row

struct RowParams {
  const void* x;
  long long rows, ld_x;
  int cols;
  const float* gamma;    // may be null: ones
  const float* beta;     // may be null: zeros
  float eps;
  void* y;               // kNorm
  long long ld_y;
  float* mean;           // kNorm, may be null
  float* rstd;           // kNorm, may be null
  int8_t* codes;         // the int8 modes
  long long ld_codes;
  float* scale;
  unsigned int* status;
};

__device__ __forceinline__ float load1(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// sums of two values over the block, in every thread; `box` holds two floats per warp
__device__ __forceinline__ float2 block_sum2(float a, float b, float2* box) {
  a = warp_sum(a);
  b = warp_sum(b);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  __syncthreads();                       // the box's previous contents have been read
  if (lane == 0) box[warp] = make_float2(a, b);
  __syncthreads();
  const float2 v = lane < warps ? box[lane] : make_float2(0.0f, 0.0f);
  return make_float2(warp_sum(v.x), warp_sum(v.y));
}
__device__ __forceinline__ unsigned int block_max(unsigned int v, unsigned int* box) {
  v = __reduce_max_sync(0xFFFFFFFFu, v);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  __syncthreads();
  if (lane == 0) box[warp] = v;
  __syncthreads();
  return __reduce_max_sync(0xFFFFFFFFu, lane < warps ? box[lane] : 0u);
}

// shift: what the centred values' mean says the first mean is off by, and 1/std.  Below the spread the
// first sum is the more exact one (the rounding of the centred values outweighs what it lost), above it the correction
// is (a mean 1e4 times the spread: 1e-3 of the spread without it).
__device__ __forceinline__ void finish_stats(float d1, float d2, float eps, float mean0, float& shift, float& rstd) {
  const float var = fmaxf(d2 - d1 * d1, 0.0f);
  shift = mean0 * mean0 > var ? d1 : 0.0f;
  rstd = rsqrtf(var + eps);
}

// Factor and scale of a row with the maximum |v| whose bit pattern is `top` (NaN patterns are above
// Inf's, Inf's above every number's).  Inf/NaN: zero codes and a NaN scale, so that what is made of the row is NaN
// and of the others is not; a maximum below 2^-100 (127 / max would overflow): zero codes, zero scale.
__device__ __forceinline__ float row_factor(unsigned int top, float& scale, unsigned int& flags) {
  const float m = __uint_as_float(top);
  if (top >= 0x7F800000u) { scale = __uint_as_float(0x7FC00000u); flags = LUQ_STATUS_NONFINITE; return 0.0f; }
  if (m < 0x1p-100f) { scale = 0.0f; flags = top ? LUQ_STATUS_RANGE : 0u; return 0.0f; }
  scale = __fdiv_rn(m, 127.0f);
  flags = 0u;
  return __fdiv_rn(127.0f, m);
}
__device__ __forceinline__ int quantize1(float v, float factor) {
  // a zero factor also serves rows that hold Inf or NaN: their products are not looked at
  return factor == 0.0f ? 0 : __float2int_rn(__fmul_rn(v, factor));
}

// Any width, any alignment: one block per row, the row is read again for every pass (from L2).  Serves the
// rows that do not fit a block's registers (above 16384 elements).
template <typename T, int MODE>
__global__ void __launch_bounds__(512) row_loop_kernel(const RowParams p) {
  __shared__ float2 box[32];
  pdl_wait();
  pdl_trigger();
  const int C = p.cols;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* const x = static_cast<const T*>(p.x) + r * p.ld_x;
    float mean0 = 0.0f, shift = 0.0f, rstd = 1.0f;
    if (MODE != kInt8) {
      float s = 0.0f;
      for (int c = threadIdx.x; c < C; c += blockDim.x) s += load1(x + c);
      mean0 = block_sum2(s, 0.0f, box).x / C;
      float s1 = 0.0f, s2 = 0.0f;
      for (int c = threadIdx.x; c < C; c += blockDim.x) {
        const float d = load1(x + c) - mean0;
        s1 += d;
        s2 = fmaf(d, d, s2);
      }
      const float2 t = block_sum2(s1, s2, box);
      finish_stats(t.x / C, t.y / C, p.eps, mean0, shift, rstd);
    }
    auto value = [&](int c) {
      float v = load1(x + c);
      if (MODE != kInt8) {
        v = ((v - mean0) - shift) * rstd;
        v = fmaf(v, p.gamma ? __ldg(p.gamma + c) : 1.0f, p.beta ? __ldg(p.beta + c) : 0.0f);
      }
      return v;
    };
    if (MODE == kNorm) {
      T* const y = static_cast<T*>(p.y) + r * p.ld_y;
      for (int c = threadIdx.x; c < C; c += blockDim.x) store1(y + c, value(c));
      if (threadIdx.x == 0) {
        if (p.mean) p.mean[r] = mean0 + shift;
        if (p.rstd) p.rstd[r] = rstd;
      }
    } else {
      unsigned int top = 0u;
      for (int c = threadIdx.x; c < C; c += blockDim.x) top = max(top, __float_as_uint(value(c)) & 0x7FFFFFFFu);
      top = block_max(top, reinterpret_cast<unsigned int*>(box));
      float scale;
      unsigned int flags;
      const float factor = row_factor(top, scale, flags);
      int8_t* const q = p.codes + r * p.ld_codes;
      for (int c = threadIdx.x; c < C; c += blockDim.x) q[c] = static_cast<int8_t>(quantize1(value(c), factor));
      if (threadIdx.x == 0) {
        p.scale[r] = scale;
        if (flags) atomicOr(p.status, flags);
      }
    }
  }
}

// ---- rows held in registers ----------------------------------------------------------------------------
// A thread holds EPT elements of a row in pieces of 16 bytes, piece j at (thread + j * threads) * V: one pass
// over memory.  Where rows do not start at multiples of 16 bytes (VEC false) a warp moves the same 512 bytes
// element by element, coalesced, through 512 bytes of shared memory: every element has the same owner, so
// sums are made in the same order and results do not depend on strides and alignment.

template <typename T>
struct Piece {
  static constexpr int V = 16 / static_cast<int>(sizeof(T));
};
__device__ __forceinline__ void unpack(const uint4& w, const float*, float* v) {
  v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ void unpack(const uint4& w, const __nv_bfloat16*, float* v) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ uint4 pack(const float* v, const float*) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float* v, const __nv_bfloat16*) {
  return make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}
__device__ __forceinline__ float zero_of(const float*) { return 0.0f; }
__device__ __forceinline__ __nv_bfloat16 zero_of(const __nv_bfloat16*) { return __float2bfloat16_rn(0.0f); }

// elements c .. c + V - 1 of a row of `cols`, zero beyond its end; `wbuf`: the warp's 32 x 16 bytes (VEC false).
// All lanes of a warp call it, with consecutive pieces.
template <typename T, bool VEC>
__device__ __forceinline__ void load_piece(const T* row, int c, int cols, uint4* wbuf, float* v) {
  constexpr int V = Piece<T>::V;
  if constexpr (VEC) {
    if (c + V <= cols) {
      unpack(__ldg(reinterpret_cast<const uint4*>(row + c)), row, v);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = c + i < cols ? load1(row + c + i) : 0.0f;
    }
  } else {
    const int lane = threadIdx.x & 31, c0 = c - lane * V;
    T* const b = reinterpret_cast<T*>(wbuf);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * 32 + lane;
      b[e] = c0 + e < cols ? row[c0 + e] : zero_of(row);
    }
    __syncwarp();
    unpack(wbuf[lane], row, v);
    __syncwarp();
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_piece(T* row, int c, int cols, uint4* wbuf, const float* v) {
  constexpr int V = Piece<T>::V;
  if constexpr (VEC) {
    if (c + V <= cols) {
      *reinterpret_cast<uint4*>(row + c) = pack(v, row);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < cols) store1(row + c + i, v[i]);
    }
  } else {
    const int lane = threadIdx.x & 31, c0 = c - lane * V;
    const T* const b = reinterpret_cast<const T*>(wbuf);
    wbuf[lane] = pack(v, row);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * 32 + lane;
      if (c0 + e < cols) row[c0 + e] = b[e];
    }
    __syncwarp();
  }
}
// V parameters, `other` where there are none
template <int V, bool VEC>
__device__ __forceinline__ void load_params(const float* g, int c, int cols, float other, float* v) {
  if (g == nullptr) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = other;
  } else if (VEC && c + V <= cols) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(g + c + i));
      v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = c + i < cols ? __ldg(g + c + i) : 0.0f;
  }
}

// sums and maxima over the threads of a row: a warp (WARP), or the block
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float* box) {
  v = warp_sum(v);
  if (WARP) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) box[warp] = v;
  __syncthreads();
  return warp_sum(lane < warps ? box[lane] : 0.0f);
}
template <bool WARP>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* box) {
  a = warp_sum(a);
  b = warp_sum(b);
  if (WARP) return make_float2(a, b);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) box[warp] = make_float2(a, b);
  __syncthreads();
  const float2 v = lane < warps ? box[lane] : make_float2(0.0f, 0.0f);
  return make_float2(warp_sum(v.x), warp_sum(v.y));
}
template <bool WARP>
__device__ __forceinline__ unsigned int row_max(unsigned int v, unsigned int* box) {
  v = __reduce_max_sync(0xFFFFFFFFu, v);
  if (WARP) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) box[warp] = v;
  __syncthreads();
  return __reduce_max_sync(0xFFFFFFFFu, lane < warps ? box[lane] : 0u);
}

template <typename T, int MODE, int EPT, bool VEC, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 512) row_kernel(const RowParams p) {
  constexpr int V = Piece<T>::V, VPT = EPT / V;
  // one box per reduction of a row, so that a row costs one barrier per reduction; the next row's first write to
  // a box comes after a later barrier than the last read of it
  __shared__ float sum_box[16];
  __shared__ float2 sum2_box[16];
  __shared__ unsigned int max_box[2][16];
  __shared__ uint4 move[VEC ? 1 : (WARP ? 8 : 16)][32];
  uint4* const wbuf = move[VEC ? 0 : threadIdx.x >> 5];
  pdl_wait();
  pdl_trigger();
  const int C = p.cols;
  const int G = WARP ? 32 : static_cast<int>(blockDim.x);
  const int tid = WARP ? static_cast<int>(threadIdx.x & 31) : static_cast<int>(threadIdx.x);
  const long long first = WARP ? static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  const long long step = WARP ? static_cast<long long>(gridDim.x) * (blockDim.x >> 5) : gridDim.x;
  const float inv_c = 1.0f / C;
  int parity = 0;
  for (long long r = first; r < p.rows; r += step, parity ^= 1) {
    const T* const x = static_cast<const T*>(p.x) + r * p.ld_x;
    float v[EPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) load_piece<T, VEC>(x, (tid + j * G) * V, C, wbuf, v + j * V);
    if (MODE != kInt8) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) s += v[i];
      const float mean0 = row_sum<WARP>(s, sum_box) * inv_c;
      float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int left = C - (tid + j * G) * V;          // elements of this piece that exist
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = i < left ? v[j * V + i] - mean0 : 0.0f;
          v[j * V + i] = d;
          s1 += d;
          s2 = fmaf(d, d, s2);
        }
      }
      const float2 t = row_sum2<WARP>(s1, s2, sum2_box);
      float shift, rstd;
      finish_stats(t.x * inv_c, t.y * inv_c, p.eps, mean0, shift, rstd);
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (tid + j * G) * V;
        float w[V], b[V];
        load_params<V, VEC>(p.gamma, c, C, 1.0f, w);
        load_params<V, VEC>(p.beta, c, C, 0.0f, b);
#pragma unroll
        for (int i = 0; i < V; ++i) v[j * V + i] = fmaf((v[j * V + i] - shift) * rstd, w[i], b[i]);
        if (MODE == kNorm) store_piece<T, VEC>(static_cast<T*>(p.y) + r * p.ld_y, c, C, wbuf, v + j * V);
      }
      if (MODE == kNorm && tid == 0) {
        if (p.mean) p.mean[r] = mean0 + shift;
        if (p.rstd) p.rstd[r] = rstd;
      }
    }
    if (MODE != kNorm) {
      unsigned int top = 0u;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int left = C - (tid + j * G) * V;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < left) top = max(top, __float_as_uint(v[j * V + i]) & 0x7FFFFFFFu);
      }
      // (without the norm this is the only reduction of a row: two boxes in turn)
      top = row_max<WARP>(top, max_box[parity]);
      float scale;
      unsigned int flags;
      const float factor = row_factor(top, scale, flags);
      int8_t* const q = p.codes + r * p.ld_codes;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (tid + j * G) * V;
        uint32_t word[V / 4];                       // codes' rows always start at multiples of 16 bytes
#pragma unroll
        for (int i = 0; i < V; i += 4) {
          const uint32_t a = static_cast<uint32_t>(quantize1(v[j * V + i], factor)) & 0xFFu;
          const uint32_t b = static_cast<uint32_t>(quantize1(v[j * V + i + 1], factor)) & 0xFFu;
          const uint32_t d = static_cast<uint32_t>(quantize1(v[j * V + i + 2], factor)) & 0xFFu;
          const uint32_t e = static_cast<uint32_t>(quantize1(v[j * V + i + 3], factor)) & 0xFFu;
          word[i / 4] = a | (b << 8) | (d << 16) | (e << 24);
        }
        if (c + V <= C) {
          if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(word[0], word[1]);
          else *reinterpret_cast<uint32_t*>(q + c) = word[0];
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (c + i < C) q[c + i] = static_cast<int8_t>(word[i / 4] >> (8 * (i & 3)));
        }
      }
      if (tid == 0) {
        p.scale[r] = scale;
        if (flags) atomicOr(p.status, flags);
      }
    }
  }
}

struct NormBwdParams {
  const void* dy;
  const void* x;
  long long rows, ld_dy, ld_x, ld_dx;
  int cols;
  const float* gamma;    // may be null: ones
  const float* mean;
  const float* rstd;
  void* dx;              // may be null
  float2* row_means;     // workspace: mean of g and of g xhat, per row
  float* partial;        // workspace: [chunks][2][cols] partial dgamma / dbeta
  int chunks;
  long long rows_per_chunk;
};

// mean_c(g) and mean_c(g xhat) of every row
template <typename T>
__global__ void __launch_bounds__(512) norm_bwd_means_kernel(const NormBwdParams p) {
  __shared__ float2 box[32];
  pdl_wait();
  pdl_trigger();
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* const x = static_cast<const T*>(p.x) + r * p.ld_x;
    const T* const dy = static_cast<const T*>(p.dy) + r * p.ld_dy;
    const float mean = __ldg(p.mean + r), rstd = __ldg(p.rstd + r);
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      const float g = load1(dy + c) * (p.gamma ? __ldg(p.gamma + c) : 1.0f);
      s1 += g;
      s2 = fmaf(g, (load1(x + c) - mean) * rstd, s2);
    }
    const float2 t = block_sum2(s1, s2, box);
    if (threadIdx.x == 0) p.row_means[r] = make_float2(t.x / p.cols, t.y / p.cols);
  }
}

// dx and the partial column sums of one chunk of rows (blockIdx.y) and 256 columns (blockIdx.x)
template <typename T>
__global__ void __launch_bounds__(256) norm_bwd_columns_kernel(const NormBwdParams p) {
  pdl_wait();
  pdl_trigger();
  const long long column_tiles = (p.cols + 255) / 256;
  const long long c64 = (blockIdx.x % column_tiles) * 256 + threadIdx.x;
  const long long chunk = blockIdx.x / column_tiles;
  if (c64 >= p.cols) return;
  const int c = static_cast<int>(c64);
  const float w = p.gamma ? __ldg(p.gamma + c) : 1.0f;
  const long long r0 = chunk * p.rows_per_chunk;
  const long long r1 = r0 + p.rows_per_chunk < p.rows ? r0 + p.rows_per_chunk : p.rows;
  float dgamma = 0.0f, dbeta = 0.0f;
  for (long long r = r0; r < r1; ++r) {
    const float mean = __ldg(p.mean + r), rstd = __ldg(p.rstd + r);
    const float dy = load1(static_cast<const T*>(p.dy) + r * p.ld_dy + c);
    const float xhat = (load1(static_cast<const T*>(p.x) + r * p.ld_x + c) - mean) * rstd;
    dgamma = fmaf(dy, xhat, dgamma);
    dbeta += dy;
    if (p.dx) {
      const float2 m = p.row_means[r];
      store1(static_cast<T*>(p.dx) + r * p.ld_dx + c, rstd * (fmaf(-xhat, m.y, dy * w) - m.x));
    }
  }
  p.partial[(2 * chunk) * p.cols + c] = dgamma;
  p.partial[(2 * chunk + 1) * p.cols + c] = dbeta;
}

// Rows in registers: a block is several groups of G threads, a group takes every gridDim.x * groups-th row
// and keeps its columns' sums of dgamma and dbeta in registers over all of them; at the end the block adds its
// groups' sums (in order, through shared memory) into one row of partial sums.  One pass over x and dy; the
// next row's pieces are loaded before this row's reduction waits.
template <typename T, int EPT, bool VEC>
__global__ void __launch_bounds__(1024) norm_bwd_kernel(const NormBwdParams p, int G) {
  constexpr int V = Piece<T>::V, VPT = EPT / V;
  __shared__ float2 box[2][32];
  __shared__ uint4 move[VEC ? 1 : 32][32];
  extern __shared__ float sums[];                    // [2][cols], only with more than one group
  pdl_wait();
  pdl_trigger();
  const int C = p.cols;
  const int groups = blockDim.x / G, group = threadIdx.x / G, tid = threadIdx.x - group * G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int warps = G >> 5, first_warp = group * warps;
  uint4* const wbuf = move[VEC ? 0 : warp];
  const long long step = static_cast<long long>(gridDim.x) * groups;
  const float inv_c = 1.0f / C;
  float dgamma[EPT], dbeta[EPT], w[EPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) load_params<V, VEC>(p.gamma, (tid + j * G) * V, C, 1.0f, w + j * V);
#pragma unroll
  for (int i = 0; i < EPT; ++i) dgamma[i] = dbeta[i] = 0.0f;
  long long r = static_cast<long long>(blockIdx.x) * groups + group;
  int parity = 0;
  for (; r < p.rows; r += step, parity ^= 1) {
    const float mean = __ldg(p.mean + r), rstd = __ldg(p.rstd + r);
    float x[EPT], dy[EPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      load_piece<T, VEC>(static_cast<const T*>(p.x) + r * p.ld_x, (tid + j * G) * V, C, wbuf, x + j * V);
      load_piece<T, VEC>(static_cast<const T*>(p.dy) + r * p.ld_dy, (tid + j * G) * V, C, wbuf, dy + j * V);
    }
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {                  // beyond the row's end dy is zero: nothing is added
      x[i] = (x[i] - mean) * rstd;
      dgamma[i] = fmaf(dy[i], x[i], dgamma[i]);
      dbeta[i] += dy[i];
      dy[i] *= w[i];
      s1 += dy[i];
      s2 = fmaf(dy[i], x[i], s2);
    }
    if (p.dx) {
      s1 = warp_sum(s1);
      s2 = warp_sum(s2);
      if (warps > 1) {
        // the two boxes in turn: one barrier per row
        if (lane == 0) box[parity][warp] = make_float2(s1, s2);
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(G) : "memory");
        const float2 t = lane < warps ? box[parity][first_warp + lane] : make_float2(0.0f, 0.0f);
        s1 = warp_sum(t.x);
        s2 = warp_sum(t.y);
      }
      s1 *= inv_c;
      s2 *= inv_c;
#pragma unroll
      for (int i = 0; i < EPT; ++i) dy[i] = rstd * (fmaf(-x[i], s2, dy[i]) - s1);
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        store_piece<T, VEC>(static_cast<T*>(p.dx) + r * p.ld_dx, (tid + j * G) * V, C, wbuf, dy + j * V);
    }
  }
  if (p.partial == nullptr) return;
  float* const out = p.partial + 2ll * blockIdx.x * C;
  for (int g = 0; g < groups; ++g) {
    if (group == g) {
      float* const to = g == groups - 1 ? out : sums;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int c = (tid + j * G) * V + i;
          if (c < C) {
            to[c] = g ? sums[c] + dgamma[j * V + i] : dgamma[j * V + i];
            to[C + c] = g ? sums[C + c] + dbeta[j * V + i] : dbeta[j * V + i];
          }
        }
      }
    }
    if (groups > 1) __syncthreads();
  }
}

// adds the chunks' partial sums in a fixed order: 32 columns by 8 strands per block
__global__ void __launch_bounds__(256) norm_bwd_reduce_kernel(const float* __restrict__ partial, int chunks, int cols,
                                                              float* dgamma, float* dbeta) {
  __shared__ float box[8][33];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
  const long long total = 2ll * cols;
  const long long j = static_cast<long long>(blockIdx.x) * 32 + lane;    // column of [dgamma | dbeta]
  float s = 0.0f;
  if (j < total)
    for (int k = strand; k < chunks; k += 8) s += partial[k * total + j];
  box[strand][lane] = s;
  __syncthreads();
  if (strand == 0 && j < total) {
#pragma unroll
    for (int k = 1; k < 8; ++k) s += box[k][lane];
    if (j < cols) { if (dgamma) dgamma[j] = s; }
    else if (dbeta) dbeta[j - cols] = s;
  }
}

bool aligned(const void* p, long long ld, int size) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * size) % 16 == 0;
}

template <typename T, int MODE, int EPT, bool VEC, bool WARP>
cudaError_t launch_row(luq_ctx* ctx, const RowParams& p, int block, long long blocks, cudaStream_t st) {
  // enough blocks to fill the SMs, each walking its rows
  const long long cap = static_cast<long long>(ctx->sm_count) * (2048 / block);
  return luq_launch_kernel(row_kernel<T, MODE, EPT, VEC, WARP>, static_cast<int>(blocks < cap ? blocks : cap), block, 0, st,
                           LUQ_LAUNCH_EARLY, 1, p);
}

template <typename T, int MODE, bool VEC>
cudaError_t launch_row_width(luq_ctx* ctx, const RowParams& p, cudaStream_t st) {
  const int C = p.cols;
  const int warps = p.rows >= 8ll * ctx->sm_count ? 8 : 1;           // rows per block while every SM has some
  const long long blocks = (p.rows + warps - 1) / warps;
  if (C <= 256) return launch_row<T, MODE, 8, VEC, true>(ctx, p, 32 * warps, blocks, st);
  if (C <= 1024) return launch_row<T, MODE, 32, VEC, true>(ctx, p, 32 * warps, blocks, st);
  if (C <= 4096) return launch_row<T, MODE, 8, VEC, false>(ctx, p, (C + 255) / 256 * 32, p.rows, st);
  if (C <= 8192) return launch_row<T, MODE, 16, VEC, false>(ctx, p, (C + 511) / 512 * 32, p.rows, st);
  return launch_row<T, MODE, 32, VEC, false>(ctx, p, (C + 1023) / 1024 * 32, p.rows, st);
}

template <typename T, int MODE>
int launch_rows(luq_ctx* ctx, const RowParams& p, cudaStream_t st) {
  cudaError_t e;
  if (p.cols > 16384) {
    const long long cap = 4ll * ctx->sm_count;
    e = luq_launch_kernel(row_loop_kernel<T, MODE>, static_cast<int>(p.rows < cap ? p.rows : cap), 512, 0, st, LUQ_LAUNCH_EARLY, 1, p);
  } else {
    const bool vec = aligned(p.x, p.ld_x, sizeof(T)) && aligned(p.gamma, 0, 4) && aligned(p.beta, 0, 4) &&
                     (MODE != kNorm || aligned(p.y, p.ld_y, sizeof(T)));
    e = vec ? launch_row_width<T, MODE, true>(ctx, p, st) : launch_row_width<T, MODE, false>(ctx, p, st);
  }
  if (e == cudaSuccess) ctx->launches += 1;
  return static_cast<int>(e);
}

template <typename T, bool VEC>
cudaError_t launch_norm_bwd_rows(const NormBwdParams& p, int G, int block, int grid, cudaStream_t st) {
  const size_t smem = block > G ? 2 * sizeof(float) * static_cast<size_t>(p.cols) : 0;
  return luq_launch_kernel(norm_bwd_kernel<T, 8, VEC>, grid, block, smem, st, LUQ_LAUNCH_EARLY, 1, p, G);
}

template <typename T>
int launch_norm_bwd(luq_ctx* ctx, NormBwdParams p, float* dgamma, float* dbeta, cudaStream_t st) {
  const size_t per_chunk = 2 * sizeof(float) * static_cast<size_t>(p.cols);
  cudaError_t e = cudaSuccess;
  if (p.cols <= 8192) {
    // eight elements of a row per thread; groups of threads that share a block while there are rows for them
    const int G = (p.cols + 255) / 256 * 32;
    int groups = G <= 256 ? 512 / G : 1;
    while (groups > 1 && static_cast<long long>(groups) * ctx->sm_count > 2 * p.rows) groups >>= 1;
    const int block = G * groups;
    long long blocks = static_cast<long long>(ctx->sm_count) * (block > 512 ? 1 : 1024 / block);
    if (blocks * groups > p.rows) blocks = (p.rows + groups - 1) / groups;
    p.partial = dgamma || dbeta ? ctx->d_workspace : nullptr;
    p.chunks = static_cast<int>(blocks);
    const bool vec = aligned(p.x, p.ld_x, sizeof(T)) && aligned(p.dy, p.ld_dy, sizeof(T)) && aligned(p.dx, p.ld_dx, sizeof(T)) &&
                     aligned(p.gamma, 0, 4);
    e = vec ? launch_norm_bwd_rows<T, true>(p, G, block, p.chunks, st) : launch_norm_bwd_rows<T, false>(p, G, block, p.chunks, st);
  } else {
    // workspace: two floats per row, then the chunks' partial sums
    const size_t means = ((static_cast<size_t>(p.rows) * sizeof(float2) + 255) / 256) * 256;
    if (means + per_chunk > ctx->workspace_bytes) return LUQ_ERR_WORKSPACE;
    p.row_means = reinterpret_cast<float2*>(ctx->d_workspace);
    p.partial = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(ctx->d_workspace) + means);
    const long long column_tiles = (p.cols + 255) / 256;
    long long chunks = (8ll * ctx->sm_count + column_tiles - 1) / column_tiles;
    const long long room = static_cast<long long>((ctx->workspace_bytes - means) / per_chunk);
    if (chunks > room) chunks = room;
    if (chunks > p.rows) chunks = p.rows;
    p.rows_per_chunk = (p.rows + chunks - 1) / chunks;
    p.chunks = static_cast<int>((p.rows + p.rows_per_chunk - 1) / p.rows_per_chunk);
    if (p.dx) {
      const long long cap = 4ll * ctx->sm_count;
      e = luq_launch_kernel(norm_bwd_means_kernel<T>, static_cast<int>(p.rows < cap ? p.rows : cap), 512, 0, st,
                            LUQ_LAUNCH_EARLY, 1, p);
      if (e != cudaSuccess) return static_cast<int>(e);
      ctx->launches += 1;
    }
    e = luq_launch_kernel(norm_bwd_columns_kernel<T>, static_cast<int>(column_tiles * p.chunks), 256, 0, st, LUQ_LAUNCH_EARLY, 1, p);
  }
  if (e != cudaSuccess) return static_cast<int>(e);
  ctx->launches += 1;
  if (dgamma || dbeta) {
    e = luq_launch_kernel(norm_bwd_reduce_kernel, static_cast<int>((2ll * p.cols + 31) / 32), 256, 0, st, LUQ_LAUNCH_EARLY, 1,
                          p.partial, p.chunks, p.cols, dgamma, dbeta);
    if (e == cudaSuccess) ctx->launches += 1;
  }
  return static_cast<int>(e);
}

}  // namespace

int luq_launch_layer_norm(luq_ctx* ctx, const void* d_x, int dtype, int64_t rows, int cols, int64_t ld_x,
                          const float* d_gamma, const float* d_beta, float eps, void* d_y, int64_t ld_y, float* d_mean,
                          float* d_rstd, cudaStream_t st) {
  RowParams p{};
  p.x = d_x; p.rows = rows; p.ld_x = ld_x; p.cols = cols; p.gamma = d_gamma; p.beta = d_beta; p.eps = eps;
  p.y = d_y; p.ld_y = ld_y; p.mean = d_mean; p.rstd = d_rstd; p.status = ctx->d_status;
  return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16, kNorm>(ctx, p, st) : launch_rows<float, kNorm>(ctx, p, st);
}

int luq_launch_int8_rows(luq_ctx* ctx, const void* d_x, int dtype, int64_t rows, int cols, int64_t ld_x, bool norm,
                         const float* d_gamma, const float* d_beta, float eps, int8_t* d_codes, int64_t ld_codes,
                         float* d_scale, cudaStream_t st) {
  RowParams p{};
  p.x = d_x; p.rows = rows; p.ld_x = ld_x; p.cols = cols; p.gamma = d_gamma; p.beta = d_beta; p.eps = eps;
  p.codes = d_codes; p.ld_codes = ld_codes; p.scale = d_scale; p.status = ctx->d_status;
  if (norm) return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16, kNormInt8>(ctx, p, st) : launch_rows<float, kNormInt8>(ctx, p, st);
  return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16, kInt8>(ctx, p, st) : launch_rows<float, kInt8>(ctx, p, st);
}

int luq_launch_layer_norm_bwd(luq_ctx* ctx, const void* d_dy, int64_t ld_dy, const void* d_x, int64_t ld_x, int dtype,
                              int64_t rows, int cols, const float* d_gamma, const float* d_mean, const float* d_rstd,
                              void* d_dx, int64_t ld_dx, float* d_dgamma, float* d_dbeta, cudaStream_t st) {
  NormBwdParams p{};
  p.dy = d_dy; p.x = d_x; p.rows = rows; p.cols = cols; p.ld_dy = ld_dy; p.ld_x = ld_x; p.ld_dx = ld_dx;
  p.gamma = d_gamma; p.mean = d_mean; p.rstd = d_rstd; p.dx = d_dx;
  return dtype == LUQ_BF16 ? launch_norm_bwd<__nv_bfloat16>(ctx, p, d_dgamma, d_dbeta, st)
                           : launch_norm_bwd<float>(ctx, p, d_dgamma, d_dbeta, st);
}
