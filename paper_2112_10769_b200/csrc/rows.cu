// Row-wise operators (sm_100a): layer norm forward and backward, and the quantizer that gives every row
// (token) an int8 scale of its own, alone or on the result of the layer norm.
//
//   mean = 1/C sum_c x_c        var = 1/C sum_c (x_c - mean)^2        rstd = (var + eps)^-1/2
//   y_c  = (x_c - mean) rstd gamma_c + beta_c
//   backward, with xhat = (x - mean) rstd and g = dy gamma:
//   dx_c = rstd (g_c - 1/C sum g - xhat_c 1/C sum g xhat)   dgamma_c = sum_r dy xhat   dbeta_c = sum_r dy
//   int8: scale = max_c |v_c| / 127, q_c = rint(v_c * fl32(127 * fl32(1 / max))), ties to even
//
// All statistics and sums are binary32 and summed in a fixed order (no atomics on sums), so a call
// repeats bit for bit.  The mean is corrected once by the sum of the centred values, and values are centred with
// both parts: a row whose mean is far above its spread loses nothing beyond the input's own rounding.
#include <cuda_bf16.h>

#include "common.cuh"

namespace {

using namespace luqdev;

constexpr int kNorm = 0, kNormInt8 = 1, kInt8 = 2;   // what a row kernel makes of a row

// Checking build: where the checks take a row to end, and the shared memory of the launch.
#ifdef LUQ_DEBUG
#define LUQ_CHECKED_COLS(p) ((p).cols - (p).slack)
__device__ __forceinline__ int dynamic_smem() {
  int n;
  asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(n));
  return n;
}
#else
#define LUQ_CHECKED_COLS(p) ((p).cols)
#endif

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
  bool vec_params, vec_y;   // gamma and beta, and the rows of y, are 16-byte aligned
#ifdef LUQ_DEBUG
  int slack;                // LUQ_OPT_CHECK_SLACK
#endif
};

__device__ __forceinline__ float load1(const float* p) { return *(p); }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load1_any(const float* p) { return *p; }              // shared or global memory
__device__ __forceinline__ float load1_any(const __nv_bfloat16* p) { return __bfloat162float(*p); }
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
  float var;                                             // at least zero; NaN, of a row with Inf or NaN, stays NaN
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(var) : "f"(d2 - d1 * d1));
  shift = mean0 * mean0 > var ? d1 : 0.0f;
  rstd = rsqrtf(var + eps);
}

// What a row whose maximum |v| has the bit pattern `top` is multiplied with (NaN patterns are above Inf's, Inf's
// above every number's).  Zero: all codes are zero - a row of zeros; a row with Inf or NaN, which gets a NaN
// scale, so that what is made of it is NaN and of the others is not; a maximum below 2^-100, where 127 / max could
// overflow, which gets a zero scale.
__device__ __forceinline__ float row_factor(unsigned int top) {
  return top >= 0x7F800000u || top < 0x0D800000u ? 0.0f : __fmul_rn(127.0f, __frcp_rn(__uint_as_float(top)));
}
__device__ __forceinline__ void store_scale(unsigned int top, float* scale, unsigned int* status) {
  const bool bad = top >= 0x7F800000u, tiny = top < 0x0D800000u;   // 2^-100
  *scale = bad ? __uint_as_float(0x7FC00000u) : tiny ? 0.0f : __fdiv_rn(__uint_as_float(top), 127.0f);
  if (bad || (tiny && top)) atomicOr(status, bad ? LUQ_STATUS_NONFINITE : LUQ_STATUS_RANGE);
}
// max(a, |b|), NaN if either is
__device__ __forceinline__ float max_abs(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
  return r;
}
// rint(v * factor) in the low byte: the sum's last mantissa bit is worth 1, so it is rounded to the nearest whole
// number, ties to even, and holds it in two's complement (|v * factor| <= 127)
__device__ __forceinline__ uint32_t quantize1(float v, float factor) {
  return __float_as_uint(__fadd_rn(__fmul_rn(v, factor), 12582912.0f));
}

// Any width, any alignment: one block per row, the row is read again for every pass (from L2).  Serves the
// rows that do not fit a block's registers (above 16384 elements).  Element by element in every pass: 2048 x 32768 bf16
// norm 266 us, to codes 354, codes alone 189 (1.0, 0.8 and 1.1 TB/s of what has to move).
template <typename T, int MODE>
__global__ void __launch_bounds__(512) row_loop_kernel(const RowParams p) {
  __shared__ float2 box[32];
  pdl_wait();
  pdl_trigger();
  const int C = p.cols;
  // (every address below is a row's start and c < C)
  auto in_row = [&](int c) { (void)c; return LUQ_IN_BOUNDS(c >= 0 && c < LUQ_CHECKED_COLS(p), p.status); };
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
        v = fmaf(v, p.gamma ? *(p.gamma + c) : 1.0f, p.beta ? *(p.beta + c) : 0.0f);
      }
      return v;
    };
    if (MODE == kNorm) {
      T* const y = static_cast<T*>(p.y) + r * p.ld_y;
      for (int c = threadIdx.x; c < C; c += blockDim.x)
        if (in_row(c)) store1(y + c, value(c));
      if (threadIdx.x == 0) {
        if (p.mean) p.mean[r] = mean0 + shift;
        if (p.rstd) p.rstd[r] = rstd;
      }
    } else {
      unsigned int top = 0u;
      for (int c = threadIdx.x; c < C; c += blockDim.x) top = max(top, __float_as_uint(value(c)) & 0x7FFFFFFFu);
      top = block_max(top, reinterpret_cast<unsigned int*>(box));
      const float factor = row_factor(top);
      int8_t* const q = p.codes + r * p.ld_codes;
      for (int c = threadIdx.x; c < C; c += blockDim.x)
        if (in_row(c)) q[c] = factor == 0.0f ? 0 : static_cast<int8_t>(quantize1(value(c), factor));
      if (threadIdx.x == 0) store_scale(top, p.scale + r, p.status);
    }
  }
}

// ---- rows held in registers ----------------------------------------------------------------------------
// A group of G threads takes a row: G = 1 .. 32 lanes of a warp (NARROW, rows up to 512 elements: several rows per
// warp), or several warps.  A thread holds EPT elements in pieces of 16 bytes, piece j at (thread + j * G) * V, so
// a row is read once; 16 of them share what a row costs beside its elements (reductions, divisions, loop).
// How the pieces get there:
//   kRing    many wide rows: every group has a ring of whole rows in shared memory, filled by bulk copies several
//            rows ahead - what an SM can stream is the bytes it has in flight, and registers hold too few.  Rows
//            that start inside a 16-byte piece are copied with the pieces around them and shifted into place, and
//            take this way however few they are (890 x 7161 norm: bf16 17 us, fp32 30; fetched element by element
//            54 and 60)
//   kDirect  16-byte loads into registers, one row ahead
//   kBounce  the same for narrow rows that do not start at multiples of 16 bytes: element by element, coalesced,
//            and through shared memory to their owners in the same warp
// An element has the same owner in all three, and sums are made in the same order: results do not depend on
// strides, alignment or the number of rows.
constexpr int kRing = 0, kDirect = 1, kBounce = 2;

template <typename T>
struct Piece {
  static constexpr int V = 16 / static_cast<int>(sizeof(T));
};
// pieces per thread that pass through a warp's shared memory together (16 elements: 2 KB of fp32, 1 KB of bf16)
template <typename T>
constexpr int kBouncePieces = 16 / Piece<T>::V;
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

// What a row consists of: kFull, every thread has EPT elements; kWhole, whole pieces; kRagged, anything.  The first
// two also mean that all tensors are there and aligned.
constexpr int kRagged = 0, kWhole = 1, kFull = 2;
template <typename T>
int fit_of(int cols, int full) { return cols == full ? kFull : cols % Piece<T>::V == 0 ? kWhole : kRagged; }
// do all elements of the piece at c exist?
template <int FIT, int V>
__device__ __forceinline__ bool piece_exists(int c, int cols) {
  return FIT == kFull || (FIT == kWhole ? c < cols : c + V <= cols);
}

// V parameters, `other` where there are none, zero beyond the row's end; `vec`: 16-byte aligned
template <int V, int FIT>
__device__ __forceinline__ void load_params(const float* g, bool vec, int c, int cols, float other, float* v, int limit, unsigned int* status) {
  if (FIT == kRagged && g == nullptr) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = other;
  } else if (piece_exists<FIT, V>(c, cols) && (FIT != kRagged || vec)) {
    if (!LUQ_IN_BOUNDS(c >= 0 && c + V <= limit, status)) return;
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 f = *(reinterpret_cast<const float4*>(g + c + i));
      v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = c + i < cols && LUQ_IN_BOUNDS(c + i < limit, status) ? *(g + c + i) : 0.0f;
  }
}

// A group, its barrier, and sums and maxima over its threads, with the result in all of them.  `box` has slots for
// each warp of the group; consecutive reductions of a group use different boxes, so each costs one barrier.
template <bool NARROW>
struct Group {
  int index, tid, G, warps;
  __device__ __forceinline__ explicit Group(int threads) : G(threads) {
    index = threadIdx.x / G;
    tid = threadIdx.x - index * G;
    warps = NARROW ? 1 : G >> 5;
  }
  __device__ __forceinline__ void sync() const {
    if (NARROW) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + index), "r"(G) : "memory");
  }
  __device__ __forceinline__ int sub() const { return NARROW ? (threadIdx.x & 31) / G : 0; }   // row within the warp
  __device__ __forceinline__ float sum(float v, float* box) const {
    if constexpr (NARROW) {
      for (int o = G >> 1; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
      return v;
    }
    const int lane = threadIdx.x & 31;
    v = warp_sum(v);
    if (lane == 0) box[tid >> 5] = v;
    sync();
    v = (lane & 15) < warps ? box[lane & 15] : 0.0f;
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
  }
  // two sums; over whole warps for the price of one: after the first exchange the lower half of the lanes carries
  // a, the upper b
  __device__ __forceinline__ float2 sum2(float a, float b, float* box) const {
    if constexpr (NARROW) {
      for (int o = G >> 1; o; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
      }
      return make_float2(a, b);
    }
    const int lane = threadIdx.x & 31;
    const bool upper = lane & 16;
    float v = (upper ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, upper ? a : b, 16);
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((lane & 15) == 0) box[2 * (tid >> 5) + (lane >> 4)] = v;
    sync();
    v = (lane & 15) < warps ? box[2 * (lane & 15) + (lane >> 4)] : 0.0f;
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    const float other = __shfl_xor_sync(0xFFFFFFFFu, v, 16);
    return upper ? make_float2(other, v) : make_float2(v, other);
  }
  __device__ __forceinline__ unsigned int max(unsigned int v, unsigned int* box) const {
    if constexpr (NARROW) {
      for (int o = G >> 1; o; o >>= 1) {
        const unsigned int w = __shfl_xor_sync(0xFFFFFFFFu, v, o);
        v = v > w ? v : w;
      }
      return v;
    }
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    const int lane = threadIdx.x & 31;
    if (lane == 0) box[tid >> 5] = v;
    sync();
    return __reduce_max_sync(0xFFFFFFFFu, lane < warps ? box[lane] : 0u);
  }
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar) : "memory");
}

// The rows of one to two tensors on their way into a group's registers.
//   start(r)   before the first row, after the wait for the preceding kernel
//   take(r, v) row r's elements, zero beyond its end; rows come in the order first, first + step, ...
//   release(r) kRing: once every thread of the group has taken row r (a barrier lies between or, of one warp, is made), the stage is
//              filled again
// kRing waits are bounded; when one runs out the group goes on without writing anything (ok() is false), so that
// its barriers still meet, and finish() waits for the copies under way and raises the status.
template <typename T, int TENSORS, int EPT, int LOAD, int FIT, bool NARROW>
struct Rows {
  static constexpr int V = Piece<T>::V, VPT = EPT / V;
  const T* base[2];
  long long ld[2];
  long long rows, step;
  int cols, tid, G;
  // kRing
  uint32_t bars = 0, data = 0, phase = 0;
  uint8_t* held = nullptr;
  int depth = 0, row_bytes = 0, stage = 0, issued = 0;
  volatile uint32_t* abort_flag = nullptr;
  bool fine = true;
  // kDirect, kBounce: the next row, as it lies in memory or element by element
  uint4 raw[TENSORS][LOAD == kDirect ? VPT : 1];
  T single[TENSORS][LOAD == kBounce ? EPT : 1];
  uint4* wbuf = nullptr;
  // for the checks: where rows end
  int limit;
  unsigned int* status;

  static int ring_row_bytes(int cols) { return (cols * static_cast<int>(sizeof(T)) + 32 + 127) / 128 * 128; }
  // shared memory of a block's rings: [groups][depth] barriers, the abort word, then [groups][depth][TENSORS] rows
  static int ring_head(int groups, int depth) { return (groups * depth * 8 + 4 + 127) / 128 * 128; }
  static int ring_bytes(int groups, int depth, int cols) {
    return ring_head(groups, depth) + groups * depth * TENSORS * ring_row_bytes(cols);
  }

  __device__ __forceinline__ void init_ring(uint8_t* smem, int groups, int group, int n) {   // all threads; a barrier follows
    depth = n;
    row_bytes = (cols * static_cast<int>(sizeof(T)) + 32 + 127) / 128 * 128;
    const int head = (groups * depth * 8 + 4 + 127) / 128 * 128;
    bars = smem_u32(smem) + group * depth * 8;
    abort_flag = reinterpret_cast<volatile uint32_t*>(smem + groups * depth * 8);
    held = smem + head + group * depth * TENSORS * row_bytes;
    (void)LUQ_IN_BOUNDS(head + groups * depth * TENSORS * row_bytes <= dynamic_smem(), status);
    data = smem_u32(held);
    if (tid == 0)
      for (int s = 0; s < depth; ++s) mbar_init(bars + 8 * s, 1);
    if (threadIdx.x == 0) *abort_flag = 0;
    fence_barrier_init();
  }
  // A row's bytes lie at (address & 15) in its stage.  Rows at the tensor's ends are copied without the pieces that
  // reach beyond it (await() fetches what they hold).
  __device__ __forceinline__ void fill(int s, long long r) {
    const int bytes = cols * static_cast<int>(sizeof(T));
    uint32_t total = 0, lo[TENSORS], n[TENSORS];
#pragma unroll
    for (int t = 0; t < TENSORS; ++t) {
      const uint32_t m = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base[t] + r * ld[t]) & 15u);
      lo[t] = r == 0 && m ? 16u : 0u;
      n[t] = (r + 1 < rows ? (m + bytes + 15u) & ~15u : (m + bytes) & ~15u) - lo[t];
      // inside the tensor, and inside the stage
      if (!LUQ_IN_BOUNDS((r > 0 || lo[t] >= m) && r >= 0 && r < rows && lo[t] + n[t] <= static_cast<uint32_t>(row_bytes) && s < depth &&
                         r * ld[t] * static_cast<long long>(sizeof(T)) - m + lo[t] + n[t] <=
                             ((rows - 1) * ld[t] + limit) * static_cast<long long>(sizeof(T)), status)) n[t] = 0u;
      total += n[t];
    }
    mbar_arrive_expect_tx(bars + 8 * s, total);
#pragma unroll
    for (int t = 0; t < TENSORS; ++t) {
      if (!LUQ_IN_BOUNDS(n[t] != 0u, status)) continue;
      const uintptr_t from = reinterpret_cast<uintptr_t>(base[t] + r * ld[t]) & ~static_cast<uintptr_t>(15);
      bulk_load(data + (s * TENSORS + t) * row_bytes + lo[t], reinterpret_cast<const void*>(from + lo[t]), n[t], bars + 8 * s);
    }
    ++issued;
  }
  // elements c .. c + V - 1 of tensor t's row in the present stage, m = the row's address & 15
  template <bool ALIGNED>
  __device__ __forceinline__ void ring_piece(int t, uint32_t m, int c, float* v) const {
    if (!LUQ_IN_BOUNDS(c >= 0 && c < cols && c / V * 16 + (ALIGNED ? 16 : 32) <= row_bytes && stage < depth, status)) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = 0.0f;
      return;
    }
    const uint4* const q = reinterpret_cast<const uint4*>(held + (stage * TENSORS + t) * row_bytes) + c / V;
    const uint4 a = q[0];
    if (ALIGNED) { unpack(a, base[0], v); return; }
    const uint4 b = q[1];
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (m & 8) {
#pragma unroll
      for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (m & 4) {
#pragma unroll
      for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (m & 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    unpack(make_uint4(w[0], w[1], w[2], w[3]), base[0], v);
  }
  __device__ __forceinline__ uint32_t skew(int t, long long r) const {
    return FIT != kRagged ? 0u : static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base[t] + r * ld[t]) & 15u);
  }
  // Waits for row r's stage.  In the tensor's first and last row the elements in the pieces that reach beyond it were
  // not copied: a lane each puts them there.
  __device__ __forceinline__ void await(const Group<NARROW>& g, long long r) {
    fine = fine && mbar_wait(bars + 8 * stage, phase, abort_flag);
    if (FIT != kRagged || (r != 0 && r + 1 != rows)) return;
    if (tid < V) {
#pragma unroll
      for (int t = 0; t < TENSORS; ++t) {
        const T* const row = base[t] + r * ld[t];
        const int m = static_cast<int>(skew(t, r)) / static_cast<int>(sizeof(T)), tail = (m + cols) % V;
        T* const to = reinterpret_cast<T*>(held + (stage * TENSORS + t) * row_bytes) + m;
        auto patch = [&](int c) {
          if (LUQ_IN_BOUNDS(c >= 0 && c < limit && (m + c + 1) * static_cast<int>(sizeof(T)) <= row_bytes, status)) to[c] = row[c];
        };
        if (r == 0 && m && tid < V - m && tid < cols) patch(tid);
        if (r + 1 == rows && tid < tail && tid < cols) patch(cols - 1 - tid);
      }
      fence_proxy_async();               // before the stage's next copy
    }
    g.sync();
  }
  __device__ __forceinline__ void fetch(long long r) {
#pragma unroll
    for (int t = 0; t < TENSORS; ++t) {
      const T* const row = base[t] + r * ld[t];
      if constexpr (LOAD == kDirect) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
          const int c = (tid + j * G) * V;
          raw[t][j] = make_uint4(0u, 0u, 0u, 0u);
          if (r < rows) {
            if (piece_exists<FIT, V>(c, cols)) {
              if (LUQ_IN_BOUNDS(c >= 0 && c + V <= limit && r >= 0, status)) raw[t][j] = *(reinterpret_cast<const uint4*>(row + c));
            } else if (FIT == kRagged) {
              float v[V];
#pragma unroll
              for (int i = 0; i < V; ++i) v[i] = c + i < cols && LUQ_IN_BOUNDS(c + i < limit, status) ? load1(row + c + i) : 0.0f;
              raw[t][j] = pack(v, row);                // exact: the values are of type T
            }
          }
        }
      } else if constexpr (LOAD == kBounce) {
        const int width = NARROW ? G : 32, l = threadIdx.x & (width - 1);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
          const int c0 = (tid - l + j * G) * V;          // the lanes' common range of elements
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int c = c0 + i * width + l;
            single[t][j * V + i] = r < rows && c < cols && LUQ_IN_BOUNDS(c >= 0 && c < limit && r >= 0, status) ? row[c] : zero_of(row);
          }
        }
      }
    }
  }
  __device__ __forceinline__ void start(long long first) {
    if constexpr (LOAD == kRing) {
      if (tid < depth && first + tid * step < rows) fill(tid, first + tid * step);
      issued = 0;
      while (issued < depth && first + issued * step < rows) ++issued;
    } else {
      fetch(first);
    }
  }
  // (in a narrow group's warp, r may lie beyond the rows)
  __device__ __forceinline__ void take(const Group<NARROW>& g, long long r, float (*v)[EPT]) {
    if constexpr (LOAD == kRing) {
      await(g, r);
#pragma unroll
      for (int t = 0; t < TENSORS; ++t) {
        const uint32_t m = skew(t, r);
        // (aligned rows apart: a test for each piece would keep the next one's load waiting)
        if (m == 0) {
#pragma unroll
          for (int j = 0; j < VPT; ++j)
            if (FIT == kFull || (tid + j * G) * V < cols) ring_piece<true>(t, 0u, (tid + j * G) * V, v[t] + j * V);
        } else {
#pragma unroll
          for (int j = 0; j < VPT; ++j)
            if ((tid + j * G) * V < cols) ring_piece<false>(t, m, (tid + j * G) * V, v[t] + j * V);
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
          const int c = (tid + j * G) * V;
          if (!piece_exists<FIT, V>(c, cols)) {
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (FIT != kRagged || c + i >= cols) v[t][j * V + i] = 0.0f;
          }
        }
      }
    } else if constexpr (LOAD == kDirect) {
#pragma unroll
      for (int t = 0; t < TENSORS; ++t)
#pragma unroll
        for (int j = 0; j < VPT; ++j) unpack(raw[t][j], base[0], v[t] + j * V);
      fetch(r + step);
    } else {
      const int lane = threadIdx.x & 31, width = NARROW ? G : 32, l = lane & (width - 1);
      T* const b = reinterpret_cast<T*>(wbuf) + (lane - l) * V;
#pragma unroll
      for (int t = 0; t < TENSORS; ++t) {
#pragma unroll
        for (int j0 = 0; j0 < VPT; j0 += kBouncePieces<T>) {
#pragma unroll
          for (int j = 0; j < kBouncePieces<T>; ++j)
            if (j0 + j < VPT) {
#pragma unroll
              for (int i = 0; i < V; ++i)
                if (LUQ_IN_BOUNDS((lane - l) * V + i * width + l < 32 * V, status)) b[j * 32 * V + i * width + l] = single[t][(j0 + j) * V + i];
            }
          __syncwarp();
#pragma unroll
          for (int j = 0; j < kBouncePieces<T>; ++j)
            if (j0 + j < VPT) unpack(wbuf[j * 32 + lane], base[0], v[t] + (j0 + j) * V);
          __syncwarp();
        }
      }
      fetch(r + step);
    }
  }
  __device__ __forceinline__ void release(long long r) {
    if constexpr (LOAD == kRing) {
      // (a wide group's reductions have a barrier; the shuffles of a warp's order no memory)
      if constexpr (NARROW) __syncwarp();
      const long long next = r + depth * step;
      if (tid == 0 && next < rows) fill(stage, next);
      if (++stage == depth) { stage = 0; phase ^= 1u; }
    }
  }
  __device__ __forceinline__ bool ok() const { return LOAD != kRing || fine; }
  __device__ __forceinline__ void finish(unsigned int* status) const {
    if constexpr (LOAD == kRing) {
      if (tid != 0 || !*abort_flag) return;
      for (int s = 0; s < depth; ++s)
        if (issued > s) mbar_wait(bars + 8 * s, ((issued - 1 - s) / depth) & 1u, abort_flag);
      atomicOr(status, LUQ_STATUS_TIMEOUT);
    }
  }
};

// writes a thread's elements of a row; `vec`: the row starts at a multiple of 16 bytes (else through the warp's
// shared memory, as kBounce reads)
template <typename T, int EPT, int FIT, bool NARROW>
__device__ __forceinline__ void store_row(T* row, bool exists, bool vec, int tid, int G, int cols, uint4* wbuf, const float* v, int limit,
                                          unsigned int* status) {
  constexpr int V = Piece<T>::V, VPT = EPT / V;
  if (FIT != kRagged || vec) {
    if (!exists) return;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = (tid + j * G) * V;
      if (piece_exists<FIT, V>(c, cols)) {
        if (LUQ_IN_BOUNDS(c >= 0 && c + V <= limit, status)) *reinterpret_cast<uint4*>(row + c) = pack(v + j * V, row);
      } else if (FIT == kRagged) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (c + i < cols && LUQ_IN_BOUNDS(c + i < limit, status)) store1(row + c + i, v[j * V + i]);
      }
    }
  } else {
    constexpr int P = VPT < kBouncePieces<T> ? VPT : kBouncePieces<T>;
    const int lane = threadIdx.x & 31, width = NARROW ? G : 32, l = lane & (width - 1);
    const T* const b = reinterpret_cast<const T*>(wbuf) + (lane - l) * V;
#pragma unroll
    for (int j0 = 0; j0 < VPT; j0 += P) {
#pragma unroll
      for (int j = 0; j < P; ++j)
        if (j0 + j < VPT) wbuf[j * 32 + lane] = pack(v + (j0 + j) * V, row);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < P; ++j) {
        if (j0 + j >= VPT) continue;
        const int c0 = (tid - l + (j0 + j) * G) * V + l;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (exists && c0 + i * width < cols && LUQ_IN_BOUNDS(c0 >= 0 && c0 + i * width < limit && (lane - l) * V + i * width + l < 32 * V, status))
            row[c0 + i * width] = b[j * 32 * V + i * width + l];
      }
      __syncwarp();
    }
  }
}

// Threads of a row kernel's block (at most), and blocks that share an SM, which leaves a thread 80 or 128 registers.  A
// third of the instances spill under that: most a few words, the norms of 32 fp32 elements a thread by 16-byte loads (few
// rows of widths above 1024) the most, 156 bytes for full rows, 372 for whole pieces, 784 for ragged ones.
template <int EPT>
constexpr int kRowThreads = EPT == 32 ? 512 : 256;
template <int MODE, int EPT, int LOAD, int FIT>
constexpr int kRowBlocks = EPT == 32 ? 1
                           : MODE == kInt8 || (EPT == 16 && (FIT != kRagged || (MODE == kNormInt8 && LOAD == kRing))) ? 3 : 2;

// What bounds it: many rows, HBM (16384 x 4096 bf16 norm 46 us, 5.8 TB/s; 8192 x 1024 fp32 13.1 us, 5.1 TB/s); rows
// that do not fill their threads or are narrow, the instructions per element; few rows, the latency of one row (1.9 us).
// FIT, norm of 16384 x 4096 bf16: 46 us with kFull, 58 with kWhole; of 41582 x 704 bf16: 31 with kWhole, 45 with kRagged.
template <typename T, int MODE, int EPT, int LOAD, int FIT, bool NARROW>
__global__ void __launch_bounds__((kRowThreads<EPT>), (kRowBlocks<MODE, EPT, LOAD, FIT>))
row_kernel(const RowParams p, int threads_per_row, int ring_depth) {
  constexpr int V = Piece<T>::V, VPT = EPT / V;
  // one box per reduction of a row; without the norm a row has one reduction only and uses two in turn
  __shared__ float sum_box[16];
  __shared__ float sum2_box[32];
  __shared__ unsigned int max_box[2][16];
  constexpr bool MOVES = FIT == kRagged && (MODE == kNorm || LOAD == kBounce);
  __shared__ uint4 move[MOVES ? kRowThreads<EPT> / 32 : 1][MOVES ? 32 * kBouncePieces<T> : 1];
  extern __shared__ __align__(128) uint8_t ring_smem[];
  const Group<NARROW> g(threads_per_row);
  const int groups = blockDim.x / g.G, slot = g.index * g.warps, tid = g.tid, G = g.G, C = p.cols;
  uint4* const wbuf = move[MOVES ? threadIdx.x >> 5 : 0];
  Rows<T, 1, EPT, LOAD, FIT, NARROW> in;
  in.base[0] = static_cast<const T*>(p.x); in.ld[0] = p.ld_x; in.rows = p.rows; in.cols = C; in.tid = tid; in.G = G;
  in.step = static_cast<long long>(gridDim.x) * groups;
  in.wbuf = wbuf;
  in.limit = LUQ_CHECKED_COLS(p);
  in.status = p.status;
  if constexpr (LOAD == kRing) {
    in.init_ring(ring_smem, groups, g.index, ring_depth);
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  const long long first = static_cast<long long>(blockIdx.x) * groups + g.index;
  in.start(first);
  // the columns' parameters stay in registers (read again for every row they cost more of L1 than the row itself:
  // 76 us instead of 53 us for 16384 rows of 4096 bf16)
  float w[MODE == kInt8 ? 1 : EPT], b[MODE == kInt8 ? 1 : EPT];
  if constexpr (MODE != kInt8) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      load_params<V, FIT>(p.gamma, p.vec_params, (tid + j * G) * V, C, 1.0f, w + j * V, LUQ_CHECKED_COLS(p), p.status);
      load_params<V, FIT>(p.beta, p.vec_params, (tid + j * G) * V, C, 0.0f, b + j * V, LUQ_CHECKED_COLS(p), p.status);
    }
  }
  const float inv_c = 1.0f / C;
  int parity = 0;
  for (long long r = first; r - g.sub() < p.rows; r += in.step, parity ^= 1) {
    float row[1][EPT];
    in.take(g, r, row);
    float (&v)[EPT] = row[0];
    const bool exists = in.ok() && (!NARROW || r < p.rows);
    if (MODE != kInt8) {
      // four strands of additions: a single one would be as long as the loads
      float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < EPT; ++i) s[i & 3] += v[i];
      const float mean0 = g.sum((s[0] + s[1]) + (s[2] + s[3]), sum_box + slot) * inv_c;
      in.release(r);
      float s1[2] = {0.0f, 0.0f}, s2[2] = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (tid + j * G) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) v[j * V + i] -= FIT == kWhole && c >= C ? 0.0f : mean0;
        if (FIT == kRagged && c + V > C) {                        // elements that do not exist
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (c + i >= C) v[j * V + i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s1[i & 1] += v[j * V + i];
          s2[i & 1] = fmaf(v[j * V + i], v[j * V + i], s2[i & 1]);
        }
      }
      const float2 t = g.sum2(s1[0] + s1[1], s2[0] + s2[1], sum2_box + 2 * slot);
      float shift, rstd;
      finish_stats(t.x * inv_c, t.y * inv_c, p.eps, mean0, shift, rstd);
      const float minus = -shift * rstd;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (tid + j * G) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) v[j * V + i] = fmaf(fmaf(v[j * V + i], rstd, minus), w[j * V + i], b[j * V + i]);
        // (a full row piece by piece: its stores leave while the next piece is computed)
        if (MODE == kNorm && FIT != kRagged && exists && piece_exists<FIT, V>(c, C) && LUQ_IN_BOUNDS(c + V <= LUQ_CHECKED_COLS(p) && r < p.rows, p.status))
          *reinterpret_cast<uint4*>(static_cast<T*>(p.y) + r * p.ld_y + c) = pack(v + j * V, static_cast<const T*>(nullptr));
        if (MODE != kNorm && FIT == kRagged && c + V > C) {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (c + i >= C) v[j * V + i] = 0.0f;
        }
      }
      if (MODE == kNorm && FIT == kRagged) store_row<T, EPT, FIT, NARROW>(static_cast<T*>(p.y) + r * p.ld_y, exists, p.vec_y, tid, G, C, wbuf, v,
                                                                                  LUQ_CHECKED_COLS(p), p.status);
      if (MODE == kNorm && tid == 0 && exists) {
        if (p.mean) p.mean[r] = mean0 + shift;
        if (p.rstd) p.rstd[r] = rstd;
      }
    }
    if (MODE != kNorm) {
      float m[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < EPT; ++i) m[i & 1] = max_abs(m[i & 1], v[i]);
      const unsigned int top = g.max(__float_as_uint(max_abs(m[0], m[1])), max_box[parity] + slot);
      if (MODE == kInt8) in.release(r);
      const float factor = row_factor(top);
      int8_t* const q = p.codes + r * p.ld_codes;
      if (factor == 0.0f) {                              // products with Inf and NaN are not looked at
#pragma unroll
        for (int i = 0; i < EPT; ++i) v[i] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (tid + j * G) * V;
        uint32_t word[V / 4];                            // codes' rows always start at multiples of 16 bytes
#pragma unroll
        for (int i = 0; i < V; i += 4)
          word[i / 4] = __byte_perm(__byte_perm(quantize1(v[j * V + i], factor), quantize1(v[j * V + i + 1], factor), 0x0040),
                                    __byte_perm(quantize1(v[j * V + i + 2], factor), quantize1(v[j * V + i + 3], factor), 0x0040),
                                    0x5410);
        if (!exists) continue;
        if (piece_exists<FIT, V>(c, C)) {
          if (!LUQ_IN_BOUNDS(c >= 0 && c + V <= LUQ_CHECKED_COLS(p) && r < p.rows, p.status)) continue;
          if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(word[0], word[1]);
          else *reinterpret_cast<uint32_t*>(q + c) = word[0];
        } else if (FIT == kRagged) {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (c + i < C && LUQ_IN_BOUNDS(c + i < LUQ_CHECKED_COLS(p) && r < p.rows, p.status)) q[c + i] = static_cast<int8_t>(word[i / 4] >> (8 * (i & 3)));
        }
      }
      if (tid == 0 && exists) store_scale(top, p.scale + r, p.status);
    }
  }
  in.finish(p.status);
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
  float* dgamma;         // the results (may be null), written directly by a grid of one block
  float* dbeta;
  int chunks;
  long long rows_per_chunk;
  unsigned int* status;
  bool vec_gamma, vec_dx;
#ifdef LUQ_DEBUG
  int slack;
#endif
};

// mean_c(g) and mean_c(g xhat) of every row (wider than 16384 elements: with the kernel below and the sum of the chunks
// 2048 x 32768 bf16 410 us, 1.0 TB/s)
template <typename T>
__global__ void __launch_bounds__(512) norm_bwd_means_kernel(const NormBwdParams p) {
  __shared__ float2 box[32];
  pdl_wait();
  pdl_trigger();
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* const x = static_cast<const T*>(p.x) + r * p.ld_x;
    const T* const dy = static_cast<const T*>(p.dy) + r * p.ld_dy;
    const float mean = *(p.mean + r), rstd = *(p.rstd + r);
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      const float g = load1(dy + c) * (p.gamma ? *(p.gamma + c) : 1.0f);
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
  const float w = p.gamma ? *(p.gamma + c) : 1.0f;
  const long long r0 = chunk * p.rows_per_chunk;
  const long long r1 = r0 + p.rows_per_chunk < p.rows ? r0 + p.rows_per_chunk : p.rows;
  float dgamma = 0.0f, dbeta = 0.0f;
  for (long long r = r0; r < r1; ++r) {
    const float mean = *(p.mean + r), rstd = *(p.rstd + r);
    const float dy = load1(static_cast<const T*>(p.dy) + r * p.ld_dy + c);
    const float xhat = (load1(static_cast<const T*>(p.x) + r * p.ld_x + c) - mean) * rstd;
    dgamma = fmaf(dy, xhat, dgamma);
    dbeta += dy;
    if (p.dx && LUQ_IN_BOUNDS(c >= 0 && c < LUQ_CHECKED_COLS(p) && r < p.rows, p.status)) {
      const float2 m = p.row_means[r];
      store1(static_cast<T*>(p.dx) + r * p.ld_dx + c, rstd * (fmaf(-xhat, m.y, dy * w) - m.x));
    }
  }
  if (!LUQ_IN_BOUNDS(chunk >= 0 && chunk < p.chunks, p.status)) return;
  p.partial[(2 * chunk) * p.cols + c] = dgamma;
  p.partial[(2 * chunk + 1) * p.cols + c] = dbeta;
}

// Threads of a block (at most): narrow rows that are fetched element by element need more than the 128 registers of
// 512 threads - what they spill waits for its load (1032 x 187 fp32 19.8 us with 512 threads, 8.4 with 384; 65536 x 128
// fp32 29.8 -> 21.6, bf16, which spills little, 15.5 -> 15.4).
constexpr int bwd_threads(bool narrow) { return narrow ? 384 : 512; }
// Rows in registers: a group takes every gridDim.x * groups-th row and keeps its columns' sums of dgamma and
// dbeta in registers over all of them; at the end the block adds its groups' sums (in order) into one row of partial
// sums.  One pass over x and dy.  Rows wider than 8192 elements (EPT 32: 64 sums a thread leave no room for the row)
// stay in the ring's stage and are read from there twice.  16384 x 4096 bf16 72 us (5.6 TB/s, HBM); 4099 x 771 fp32 of
// pitch 776 16.3 us, the latency of four rows a group and the second kernel's 2.7 us.
template <typename T, int EPT, int LOAD, int FIT, bool NARROW>
__global__ void __launch_bounds__(bwd_threads(NARROW)) norm_bwd_kernel(const NormBwdParams p, int threads_per_row, int ring_depth) {
  constexpr int V = Piece<T>::V, VPT = EPT / V;
  constexpr bool TWICE = EPT == 32;
  static_assert(!TWICE || LOAD == kRing, "a row that is read twice stays in the ring");
  __shared__ float box[2][32];
  __shared__ uint4 move[FIT != kRagged ? 1 : 16][FIT != kRagged ? 1 : 32 * kBouncePieces<T>];
  extern __shared__ __align__(128) uint8_t ring_smem[];   // the ring; at the end [groups][2][cols] sums
  const Group<NARROW> g(threads_per_row);
  const int groups = blockDim.x / g.G, group = g.index, slot = g.index * g.warps, tid = g.tid, G = g.G, C = p.cols;
  uint4* const wbuf = move[FIT != kRagged ? 0 : threadIdx.x >> 5];
  Rows<T, 2, TWICE ? V : EPT, LOAD, FIT, NARROW> in;
  in.base[0] = static_cast<const T*>(p.x); in.ld[0] = p.ld_x;
  in.base[1] = static_cast<const T*>(p.dy); in.ld[1] = p.ld_dy;
  in.rows = p.rows; in.cols = C; in.tid = tid; in.G = G; in.wbuf = wbuf;
  in.limit = LUQ_CHECKED_COLS(p);
  in.status = p.status;
  in.step = static_cast<long long>(gridDim.x) * groups;
  if constexpr (LOAD == kRing) {
    in.init_ring(ring_smem, groups, group, ring_depth);
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  const long long first = static_cast<long long>(blockIdx.x) * groups + group, step = in.step;
  const float inv_c = 1.0f / C;
  float mean = 0.0f, rstd = 0.0f;
  if (first < p.rows) { mean = *(p.mean + first); rstd = *(p.rstd + first); }
  float dgamma[EPT], dbeta[EPT], w[TWICE ? 1 : EPT];
  if constexpr (!TWICE) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) load_params<V, FIT>(p.gamma, p.vec_gamma, (tid + j * G) * V, C, 1.0f, w + j * V, LUQ_CHECKED_COLS(p), p.status);
  }
#pragma unroll
  for (int i = 0; i < EPT; ++i) dgamma[i] = dbeta[i] = 0.0f;
  in.start(first);
  int parity = 0;
  for (long long r = first; r - g.sub() < p.rows; r += step, parity ^= 1) {
    // the next row's mean and 1/std are on their way while this row is worked on
    const long long after = r + step;
    float next_mean = 0.0f, next_rstd = 0.0f;
    if (after < p.rows) { next_mean = *(p.mean + after); next_rstd = *(p.rstd + after); }
    float s1[2] = {0.0f, 0.0f}, s2[2] = {0.0f, 0.0f};
    // beyond a row's end dy is zero: nothing is added
    auto gather = [&](float& x, float& dy, float weight, float& dg, float& db, int i) {
      x = (x - mean) * rstd;
      dg = fmaf(dy, x, dg);
      db += dy;
      dy *= weight;
      s1[i & 1] += dy;
      s2[i & 1] = fmaf(dy, x, s2[i & 1]);
    };
    T* const dx = static_cast<T*>(p.dx) + r * p.ld_dx;
    if constexpr (!TWICE) {
      float row[2][EPT];
      in.take(g, r, row);
      float (&x)[EPT] = row[0], (&dy)[EPT] = row[1];
#pragma unroll
      for (int i = 0; i < EPT; ++i) gather(x[i], dy[i], w[i], dgamma[i], dbeta[i], i);
      if (p.dx) {
        const float2 t = g.sum2(s1[0] + s1[1], s2[0] + s2[1], box[parity] + 2 * slot);   // two boxes in turn: one barrier per row
        in.release(r);
        const bool exists = in.ok() && (!NARROW || r < p.rows);
        const float m1 = -t.x * inv_c * rstd, m2 = t.y * inv_c;
#pragma unroll
        for (int i = 0; i < EPT; ++i) dy[i] = fmaf(fmaf(-x[i], m2, dy[i]), rstd, m1);
        store_row<T, EPT, FIT, NARROW>(dx, exists, p.vec_dx, tid, G, C, wbuf, dy, LUQ_CHECKED_COLS(p), p.status);
      } else if constexpr (LOAD == kRing) {
        g.sync();                                      // everyone has read the stage
        in.release(r);
      }
    } else {
      in.await(g, r);
      auto piece = [&](int t, int c, float* v) {
        if (FIT == kFull || c < C) {
          if (in.skew(t, r) == 0) in.template ring_piece<true>(t, 0u, c, v);
          else in.template ring_piece<false>(t, in.skew(t, r), c, v);
        }
        if (!piece_exists<FIT, V>(c, C)) {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (FIT != kRagged || c + i >= C) v[i] = 0.0f;
        }
      };
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (tid + j * G) * V;
        float x[V], dy[V], weight[V];
        piece(0, c, x);
        piece(1, c, dy);
        load_params<V, FIT>(p.gamma, p.vec_gamma, c, C, 1.0f, weight, LUQ_CHECKED_COLS(p), p.status);
#pragma unroll
        for (int i = 0; i < V; ++i) gather(x[i], dy[i], weight[i], dgamma[j * V + i], dbeta[j * V + i], i);
      }
      const float2 t = g.sum2(s1[0] + s1[1], s2[0] + s2[1], box[parity] + 2 * slot);
      const float m1 = -t.x * inv_c * rstd, m2 = t.y * inv_c;
      if (p.dx) {
#pragma unroll 1
        for (int j = 0; j < VPT; ++j) {
          const int c = (tid + j * G) * V;
          float x[V], dy[V], weight[V];
          piece(0, c, x);
          piece(1, c, dy);
          load_params<V, FIT>(p.gamma, p.vec_gamma, c, C, 1.0f, weight, LUQ_CHECKED_COLS(p), p.status);
#pragma unroll
          for (int i = 0; i < V; ++i) dy[i] = fmaf(fmaf(-((x[i] - mean) * rstd), m2, dy[i] * weight[i]), rstd, m1);
          store_row<T, V, FIT, NARROW>(dx + j * G * V, in.ok(), p.vec_dx, tid, G, C - j * G * V, wbuf, dy,
                                    LUQ_CHECKED_COLS(p) - j * G * V, p.status);
        }
      }
      g.sync();                                        // everyone has read the stage
      in.release(r);
    }
    mean = next_mean;
    rstd = next_rstd;
  }
  in.finish(p.status);
  if (!p.dgamma && !p.dbeta) return;
  float* const out = p.partial + 2ll * blockIdx.x * C;
  // a narrow warp's rows first, then the block's warps (or groups) in order, each thread a column
  if constexpr (NARROW) {
    for (int o = G; o < 32; o <<= 1) {
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        dgamma[i] += __shfl_xor_sync(0xFFFFFFFFu, dgamma[i], o);
        dbeta[i] += __shfl_xor_sync(0xFFFFFFFFu, dbeta[i], o);
      }
    }
  }
  const int turns = NARROW ? blockDim.x >> 5 : groups, mine = NARROW ? threadIdx.x >> 5 : group;
  // (one block: these are the results)
  float* const out_gamma = gridDim.x == 1 ? p.dgamma : out;
  float* const out_beta = gridDim.x == 1 ? p.dbeta : out + C;
  float* const sums = reinterpret_cast<float*>(ring_smem);
  const int Cp = (C + 3) & ~3;                         // a row of sums in shared memory
  __syncthreads();                                     // the ring is done with
  if (g.sub() == 0) {
    float* const to = sums + 2 * mine * Cp;
#pragma unroll
    for (int i = 0; i < EPT; i += 4) {
      const int c = (tid + i / V * G) * V + i % V;
      if (c < Cp && LUQ_IN_BOUNDS(c >= 0 && ((2 * mine + 1) * Cp + c + 4) * 4 <= dynamic_smem() && mine < turns, p.status)) {
        *reinterpret_cast<float4*>(to + c) = make_float4(dgamma[i], dgamma[i + 1], dgamma[i + 2], dgamma[i + 3]);
        *reinterpret_cast<float4*>(to + Cp + c) = make_float4(dbeta[i], dbeta[i + 1], dbeta[i + 2], dbeta[i + 3]);
      }
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < C; c += blockDim.x) {
    if (!LUQ_IN_BOUNDS(((2 * turns - 1) * Cp + c + 1) * 4 <= dynamic_smem() && c < LUQ_CHECKED_COLS(p) && blockIdx.x < p.chunks, p.status)) continue;
    float sg = sums[c], sb = sums[Cp + c];
    for (int k = 1; k < turns; ++k) {
      sg += sums[2 * k * Cp + c];
      sb += sums[(2 * k + 1) * Cp + c];
    }
    if (out_gamma) out_gamma[c] = sg;
    if (out_beta) out_beta[c] = sb;
  }
}

// adds the chunks' partial sums in a fixed order: 32 columns by 32 strands per block, five loads in flight each (a
// chunk for every SM then takes one trip)
__global__ void __launch_bounds__(1024) norm_bwd_reduce_kernel(const float* partial, int chunks, int cols,
                                                               float* dgamma, float* dbeta) {
  constexpr int U = 5;
  __shared__ float box[32][33];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
  const long long total = 2ll * cols;
  const long long j = static_cast<long long>(blockIdx.x) * 32 + lane;    // column of [dgamma | dbeta]
  float s = 0.0f;
  if (j < total) {
    for (int k = strand; k < chunks; k += 32 * U) {
      float v[U];
#pragma unroll
      for (int i = 0; i < U; ++i) v[i] = k + 32 * i < chunks ? __ldcg(partial + (k + 32ll * i) * total + j) : 0.0f;
#pragma unroll
      for (int i = 0; i < U; ++i) s += v[i];
    }
  }
  box[strand][lane] = s;
  __syncthreads();
  if (strand == 0 && j < total) {
#pragma unroll
    for (int k = 1; k < 32; ++k) s += box[k][lane];
    if (j < cols) { if (dgamma) dgamma[j] = s; }
    else if (dbeta) dbeta[j - cols] = s;
  }
}

bool aligned(const void* p, long long ld, int size) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * size) % 16 == 0;
}

constexpr int kRingBytes = 66 * 1024;      // of a block of the forward kernels: two or three blocks share an SM
constexpr int kRingBytesAlone = 190 * 1024;

template <typename K>
cudaError_t allow_smem(K kernel, luq_once_per_device& once, int device) {
  return once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 192 * 1024); }, device);
}
// stages of a ring: as many as fit, eight at most, two if two do fit an SM (one row of x and dy may be 128 KB)
int ring_depth_for(int groups, int stage_bytes, int budget) {
  int d = budget / (groups * (stage_bytes + 8));
  if (d < 2) d = 2 * groups * (stage_bytes + 8) <= kRingBytesAlone ? 2 : 1;
  return d > 8 ? 8 : d;
}
// threads of a row: a power of two of lanes up to a warp, whole warps beyond
int threads_of_row(int cols, int ept) {
  if (cols <= 32 * ept) {
    int g = 1;
    while (g * ept < cols) g <<= 1;
    return g;
  }
  return (cols + 32 * ept - 1) / (32 * ept) * 32;
}

template <typename T, int MODE, int EPT, int LOAD, bool NARROW>
cudaError_t launch_row(luq_ctx* ctx, const RowParams& p, bool vec, cudaStream_t st) {
  const int G = threads_of_row(p.cols, EPT);
  // groups share a block while every SM has some; a block has whole warps
  int groups = (G > 256 ? 512 : 256) / G;
  while (groups > 1 && G * groups > 32 && p.rows < static_cast<long long>(groups) * ctx->sm_count) groups >>= 1;
  const int fit = LOAD == kBounce || !vec || (MODE != kInt8 && !(p.gamma && p.beta)) ? kRagged : fit_of<T>(p.cols, G * EPT);
  int per_sm = fit == kRagged ? kRowBlocks<MODE, EPT, LOAD, kRagged> : kRowBlocks<MODE, EPT, LOAD, kWhole>;
  if (kRowThreads<EPT> == 512 && G <= 256) per_sm = 2;
  const int row_bytes = Rows<T, 1, EPT, LOAD, kRagged, NARROW>::ring_row_bytes(p.cols);
  const int depth = LOAD == kRing ? ring_depth_for(groups, row_bytes, per_sm > 1 ? kRingBytes : kRingBytesAlone) : 0;
  const size_t smem = LOAD == kRing ? static_cast<size_t>(Rows<T, 1, EPT, LOAD, kRagged, NARROW>::ring_bytes(groups, depth, p.cols)) : 0;
  auto kernel = row_kernel<T, MODE, EPT, LOAD, kRagged, NARROW>;
  // (narrow rows of 16 elements a thread take the ring where they are unaligned only)
  if constexpr (LOAD == kDirect || (LOAD == kRing && !(NARROW && EPT == 16))) {
    if (fit == kWhole) kernel = row_kernel<T, MODE, EPT, LOAD, kWhole, NARROW>;
    if (fit == kFull) kernel = row_kernel<T, MODE, EPT, LOAD, kFull, NARROW>;
  }
  if (LOAD == kRing) {
    static luq_once_per_device once[3];
    const cudaError_t e = allow_smem(kernel, once[fit], ctx->device);
    if (e != cudaSuccess) return e;
  }
  const long long blocks = (p.rows + groups - 1) / groups;
  const long long cap = static_cast<long long>(ctx->sm_count) * per_sm *
                        (LOAD == kRing ? 1 : (G > 256 ? 512 : 256) / (G * groups));
  return luq_launch_kernel(kernel, static_cast<int>(blocks < cap ? blocks : cap), G * groups, smem, st, LUQ_LAUNCH_EARLY, 1, p, G, depth);
}

template <typename T, int MODE, int EPT, bool NARROW>
cudaError_t launch_row_from(luq_ctx* ctx, const RowParams& p, bool vec_x, bool vec, bool ring, cudaStream_t st) {
  if (ring || (!NARROW && !vec_x)) return launch_row<T, MODE, EPT, kRing, NARROW>(ctx, p, vec, st);
  if constexpr (NARROW && EPT == 16)                     // (with 24 all unaligned ones take the ring)
    if (!vec_x) return launch_row<T, MODE, EPT, kBounce, NARROW>(ctx, p, vec, st);
  return launch_row<T, MODE, EPT, kDirect, NARROW>(ctx, p, vec, st);
}
template <typename T, int MODE, int EPT>
cudaError_t launch_row_load(luq_ctx* ctx, const RowParams& p, bool vec_x, bool vec, bool many, cudaStream_t st) {
  if constexpr (EPT == 32) return launch_row_from<T, MODE, EPT, false>(ctx, p, vec_x, vec, many, st);   // above 1024 columns only
  else if (p.cols > 32 * EPT) return launch_row_from<T, MODE, EPT, false>(ctx, p, vec_x, vec, many, st);
  // rows of up to a warp: the ring's copies are small, and pay for rows that fill it and are unaligned only (20000 x
  // 301 fp32 44 -> 24 us, norm backward 78 -> 38; aligned, 20000 x 320 bf16 backward: 17 us, 23 from the ring)
  else return launch_row_from<T, MODE, EPT, true>(ctx, p, vec_x, vec, (many && p.cols > 512) || (!vec_x && p.cols > 16 * EPT), st);
}

// Elements per thread by the width alone (what a row becomes must not depend on where it lies).  What counts is the
// share of a block's 256 x elements that a row's groups use, and how much of a row's fixed cost an element bears
// (16 -> chosen, norm / norm to int8 / int8, us):
//   32  whole multiples of 1024 that fit 24 no better: 16384x4096 bf16 57 -> 46 / 70 -> 57 / 37; to int8 also widths that
//       it fits as well as the others: 5223x3830 bf16 35 -> 33 / 21 -> 19.  Unaligned norms it costs dear (10000x1311
//       fp32 32 -> 61 / 36 -> 44 / 21 -> 23)
//   24  where it fits better: 41582x704 bf16 41 -> 32 / 48 -> 40 / 26 -> 22, 10000x1311 bf16 27 -> 23 / 32 -> 26 / 19 -> 15,
//       5000x6144 bf16 (32) 26.7 -> 25.4 / 31.5 -> 30.8 / 21 -> 18; norms of odd widths of up to a warp stay at 16
//       (60000x700 bf16: 84, 24: 124)
int elements_per_thread(int mode, int cols) {
  if (cols <= 512) return 16;
  if (cols > 8192) return 32;
  auto fit = [&](int ept) {
    const int G = threads_of_row(cols, ept);
    return G > 256 ? 0.0f : static_cast<float>(cols) / (G * ept) * (G * (256 / G)) / 256.0f;
  };
  const float f16 = fit(16), f24 = fit(24), f32 = fit(32);
  if (cols > 1024 && f32 >= f24 && (cols % 1024 == 0 || (cols > 2048 && mode != kNorm && f32 >= f16))) return 32;
  if (f24 >= f16 && f24 > 0.0f && (mode != kNorm || cols % 8 == 0 || cols > 768)) return 24;
  return f16 > 0.0f ? 16 : 32;
}

template <typename T, int MODE>
int launch_rows(luq_ctx* ctx, RowParams p, cudaStream_t st) {
  cudaError_t e;
  p.vec_params = aligned(p.gamma, 0, 4) && aligned(p.beta, 0, 4);
  p.vec_y = MODE != kNorm || aligned(p.y, p.ld_y, sizeof(T));
  const bool vec_x = aligned(p.x, p.ld_x, sizeof(T)), vec = vec_x && p.vec_params && p.vec_y;
  // the ring pays where every group has several rows
  const bool many = p.rows >= 8ll * ctx->sm_count;
  if (p.cols > 16384) {
    const long long cap = 4ll * ctx->sm_count;
    e = luq_launch_kernel(row_loop_kernel<T, MODE>, static_cast<int>(p.rows < cap ? p.rows : cap), 512, 0, st, LUQ_LAUNCH_EARLY, 1, p);
  } else {
    switch (elements_per_thread(MODE, p.cols)) {
      case 16: e = launch_row_load<T, MODE, 16>(ctx, p, vec_x, vec, many, st); break;
      case 24: e = launch_row_load<T, MODE, 24>(ctx, p, vec_x, vec, many, st); break;
      default: e = launch_row_load<T, MODE, 32>(ctx, p, vec_x, vec, many, st);
    }
  }
  if (e == cudaSuccess) ctx->launches += 1;
  return static_cast<int>(e);
}

template <typename T, int EPT, int LOAD, bool NARROW>
cudaError_t launch_norm_bwd_rows(int device, const NormBwdParams& p, bool vec, int G, int block, int grid, cudaStream_t st) {
  const int groups = block / G;
  using R = Rows<T, 2, 16, LOAD, kRagged, NARROW>;
  const int depth = LOAD == kRing ? ring_depth_for(groups, 2 * R::ring_row_bytes(p.cols), kRingBytesAlone) : 0;
  const int turns = NARROW ? block / 32 : groups;
  const size_t sums = 2 * sizeof(float) * static_cast<size_t>((p.cols + 3) & ~3) * turns;
  const size_t ring = LOAD == kRing ? static_cast<size_t>(R::ring_bytes(groups, depth, p.cols)) : 0;
  const int fit = LOAD == kBounce || !vec || !p.gamma ? kRagged : fit_of<T>(p.cols, EPT == 16 ? G * EPT : 0);
  constexpr int least = LOAD == kDirect && !NARROW ? kWhole : kRagged;     // (such rows take the ring)
  auto kernel = norm_bwd_kernel<T, EPT, LOAD, least, NARROW>;
  if constexpr (LOAD == kDirect || (LOAD == kRing && !NARROW)) {           // (narrow rows take the ring where they are unaligned only)
    if (fit == kWhole) kernel = norm_bwd_kernel<T, EPT, LOAD, kWhole, NARROW>;
    if constexpr (EPT == 16)
      if (fit == kFull) kernel = norm_bwd_kernel<T, EPT, LOAD, kFull, NARROW>;
  }
  static luq_once_per_device once[3];
  const cudaError_t e = allow_smem(kernel, once[fit], device);
  if (e != cudaSuccess) return e;
  return luq_launch_kernel(kernel, grid, block, LOAD == kRing && ring > sums ? ring : sums, st, LUQ_LAUNCH_EARLY, 1, p, G, depth);
}

template <typename T>
int launch_norm_bwd(luq_ctx* ctx, NormBwdParams p, float* dgamma, float* dbeta, cudaStream_t st) {
  const size_t per_chunk = 2 * sizeof(float) * static_cast<size_t>(p.cols);
  cudaError_t e = cudaSuccess;
  luq_call_workspace workspace(ctx, st);
  p.vec_gamma = aligned(p.gamma, 0, 4);
  p.dgamma = dgamma;
  p.dbeta = dbeta;
  bool reduced = false;
  p.vec_dx = aligned(p.dx, p.ld_dx, sizeof(T));
  const bool vec_in = aligned(p.x, p.ld_x, sizeof(T)) && aligned(p.dy, p.ld_dy, sizeof(T)), vec = vec_in && p.vec_gamma && p.vec_dx;
  // a row of x and one of dy have to fit the ring
  if (p.cols <= 16384 && Rows<T, 2, 16, kRing, kRagged, false>::ring_bytes(1, 1, p.cols) <= 192 * 1024) {
    // as many sums of both kinds per thread as elements of a row; groups share a block while there are rows for them
    const int ept = p.cols > 8192 ? 32 : 16;
    const int G = threads_of_row(p.cols, ept);
    // (narrow rows: whole warps of them)
    int groups = 512 / G;
    if (p.cols <= 512) {
      const int per_warp = 32 / G;
      const long long warps = p.rows / (static_cast<long long>(per_warp) * ctx->sm_count);
      groups = per_warp * static_cast<int>(warps < 1 ? 1 : warps > bwd_threads(true) / 32 ? bwd_threads(true) / 32 : warps);
    } else {
      while (groups > 1 && static_cast<long long>(groups) * ctx->sm_count > p.rows) groups >>= 1;
    }
    const int block = G * groups;
    long long blocks = ctx->sm_count;
    if (blocks * groups > p.rows) blocks = (p.rows + groups - 1) / groups;
    p.chunks = static_cast<int>(blocks);
    reduced = blocks == 1;
    if ((dgamma || dbeta) && !reduced) {                 // (at most 16384 columns and a block for every SM: 20 MB)
      p.partial = static_cast<float*>(workspace.get(per_chunk * static_cast<size_t>(blocks)));
      if (!p.partial) return LUQ_ERR_WORKSPACE;
    }
    const bool ring = p.rows >= 2 * blocks * groups;
    const bool whole = vec && p.gamma && p.cols % Piece<T>::V == 0;
    if (ept == 32) e = launch_norm_bwd_rows<T, 32, kRing, false>(ctx->device, p, vec, G, block, p.chunks, st);
    else if (p.cols > 256 && p.cols <= 512 && !vec_in) e = launch_norm_bwd_rows<T, 16, kRing, true>(ctx->device, p, vec, G, block, p.chunks, st);
    else if (p.cols <= 512) e = vec_in ? launch_norm_bwd_rows<T, 16, kDirect, true>(ctx->device, p, vec, G, block, p.chunks, st)
                                       : launch_norm_bwd_rows<T, 16, kBounce, true>(ctx->device, p, vec, G, block, p.chunks, st);
    else if (ring || !whole) e = launch_norm_bwd_rows<T, 16, kRing, false>(ctx->device, p, vec, G, block, p.chunks, st);
    else e = launch_norm_bwd_rows<T, 16, kDirect, false>(ctx->device, p, vec, G, block, p.chunks, st);
  } else {
    // workspace: two floats per row, then the chunks' partial sums
    const size_t means = ((static_cast<size_t>(p.rows) * sizeof(float2) + 255) / 256) * 256;
    if (means + per_chunk > ctx->workspace_bytes) return LUQ_ERR_WORKSPACE;
    const long long column_tiles = (p.cols + 255) / 256;
    long long chunks = (8ll * ctx->sm_count + column_tiles - 1) / column_tiles;
    const long long room = static_cast<long long>((ctx->workspace_bytes - means) / per_chunk);
    if (chunks > room) chunks = room;
    if (chunks > p.rows) chunks = p.rows;
    p.rows_per_chunk = (p.rows + chunks - 1) / chunks;
    p.chunks = static_cast<int>((p.rows + p.rows_per_chunk - 1) / p.rows_per_chunk);
    uint8_t* const w = static_cast<uint8_t*>(workspace.get(means + per_chunk * static_cast<size_t>(p.chunks)));
    if (!w) return LUQ_ERR_WORKSPACE;
    p.row_means = reinterpret_cast<float2*>(w);
    p.partial = reinterpret_cast<float*>(w + means);
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
  if ((dgamma || dbeta) && !reduced) {
    e = luq_launch_kernel(norm_bwd_reduce_kernel, static_cast<int>((2ll * p.cols + 31) / 32), 1024, 0, st, LUQ_LAUNCH_EARLY, 1,
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
#ifdef LUQ_DEBUG
  p.slack = ctx->check_slack;
#endif
  return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16, kNorm>(ctx, p, st) : launch_rows<float, kNorm>(ctx, p, st);
}

int luq_launch_int8_rows(luq_ctx* ctx, const void* d_x, int dtype, int64_t rows, int cols, int64_t ld_x, bool norm,
                         const float* d_gamma, const float* d_beta, float eps, int8_t* d_codes, int64_t ld_codes,
                         float* d_scale, cudaStream_t st) {
  RowParams p{};
  p.x = d_x; p.rows = rows; p.ld_x = ld_x; p.cols = cols; p.gamma = d_gamma; p.beta = d_beta; p.eps = eps;
  p.codes = d_codes; p.ld_codes = ld_codes; p.scale = d_scale; p.status = ctx->d_status;
#ifdef LUQ_DEBUG
  p.slack = ctx->check_slack;
#endif
  if (norm) return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16, kNormInt8>(ctx, p, st) : launch_rows<float, kNormInt8>(ctx, p, st);
  return dtype == LUQ_BF16 ? launch_rows<__nv_bfloat16, kInt8>(ctx, p, st) : launch_rows<float, kInt8>(ctx, p, st);
}

int luq_launch_layer_norm_bwd(luq_ctx* ctx, const void* d_dy, int64_t ld_dy, const void* d_x, int64_t ld_x, int dtype,
                              int64_t rows, int cols, const float* d_gamma, const float* d_mean, const float* d_rstd,
                              void* d_dx, int64_t ld_dx, float* d_dgamma, float* d_dbeta, cudaStream_t st) {
  NormBwdParams p{};
  p.dy = d_dy; p.x = d_x; p.rows = rows; p.cols = cols; p.ld_dy = ld_dy; p.ld_x = ld_x; p.ld_dx = ld_dx;
  p.gamma = d_gamma; p.mean = d_mean; p.rstd = d_rstd; p.dx = d_dx; p.status = ctx->d_status;
#ifdef LUQ_DEBUG
  p.slack = ctx->check_slack;
#endif
  return dtype == LUQ_BF16 ? launch_norm_bwd<__nv_bfloat16>(ctx, p, d_dgamma, d_dbeta, st)
                           : launch_norm_bwd<float>(ctx, p, d_dgamma, d_dbeta, st);
}
