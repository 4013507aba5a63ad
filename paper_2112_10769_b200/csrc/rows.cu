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
// rows that do not fit a block's registers.
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
      shift = t.x / C;
      rstd = rsqrtf(fmaxf(t.y / C - shift * shift, 0.0f) + p.eps);
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

template <typename T>
int launch_rows(luq_ctx* ctx, const RowParams& p, int mode, cudaStream_t st) {
  const long long cap = 16ll * ctx->sm_count;
  const int grid = static_cast<int>(p.rows < cap ? p.rows : cap);
  const int block = p.cols >= 512 ? 512 : ((p.cols + 31) / 32) * 32;
  cudaError_t e;
  if (mode == kNorm) e = luq_launch_kernel(row_loop_kernel<T, kNorm>, grid, block, 0, st, LUQ_LAUNCH_EARLY, 1, p);
  else if (mode == kNormInt8) e = luq_launch_kernel(row_loop_kernel<T, kNormInt8>, grid, block, 0, st, LUQ_LAUNCH_EARLY, 1, p);
  else e = luq_launch_kernel(row_loop_kernel<T, kInt8>, grid, block, 0, st, LUQ_LAUNCH_EARLY, 1, p);
  if (e == cudaSuccess) ctx->launches += 1;
  return static_cast<int>(e);
}

template <typename T>
int launch_norm_bwd(luq_ctx* ctx, NormBwdParams p, float* dgamma, float* dbeta, cudaStream_t st) {
  // workspace: two floats per row, then the chunks' partial sums
  const size_t means = ((static_cast<size_t>(p.rows) * sizeof(float2) + 255) / 256) * 256;
  const size_t per_chunk = 2 * sizeof(float) * static_cast<size_t>(p.cols);
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
  cudaError_t e = cudaSuccess;
  if (p.dx) {
    const long long cap = 16ll * ctx->sm_count;
    const int block = p.cols >= 512 ? 512 : ((p.cols + 31) / 32) * 32;
    e = luq_launch_kernel(norm_bwd_means_kernel<T>, static_cast<int>(p.rows < cap ? p.rows : cap), block, 0, st,
                          LUQ_LAUNCH_EARLY, 1, p);
    if (e != cudaSuccess) return static_cast<int>(e);
    ctx->launches += 1;
  }
  e = luq_launch_kernel(norm_bwd_columns_kernel<T>, static_cast<int>(column_tiles * p.chunks), 256, 0, st, LUQ_LAUNCH_EARLY, 1, p);
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
  return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16>(ctx, p, kNorm, st) : launch_rows<float>(ctx, p, kNorm, st);
}

int luq_launch_int8_rows(luq_ctx* ctx, const void* d_x, int dtype, int64_t rows, int cols, int64_t ld_x, bool norm,
                         const float* d_gamma, const float* d_beta, float eps, int8_t* d_codes, int64_t ld_codes,
                         float* d_scale, cudaStream_t st) {
  RowParams p{};
  p.x = d_x; p.rows = rows; p.ld_x = ld_x; p.cols = cols; p.gamma = d_gamma; p.beta = d_beta; p.eps = eps;
  p.codes = d_codes; p.ld_codes = ld_codes; p.scale = d_scale; p.status = ctx->d_status;
  const int mode = norm ? kNormInt8 : kInt8;
  return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16>(ctx, p, mode, st) : launch_rows<float>(ctx, p, mode, st);
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
