// A layer of experts around its products (sm_100a): which experts a token goes to and with what weights, the tokens' copies in
// the experts' order, the weighted sum of their results, and the gradients.
//
//   route         s = softmax(l) or sigmoid(l);  c = s + bias;  of G equal groups the H with the largest sums of their best c stay;
//                 the k largest c are chosen, ties to the lowest index;  w_j = scale s_j, or scale s_j / sum of the chosen s
//   order         position[t, j] = number of copies that come before copy j of token t: by expert, then by token and place
//   dispatch      out[position[t, j]] = x[t]
//   combine       out[t] = residual[t] + sum_j w[t, j] y[position[t, j]]
//
// Statistics and sums are binary32 in a fixed order; there are no atomics on sums: a call repeats bit for bit.
#include <cuda_bf16.h>

#include <climits>
#include <type_traits>

#include "common.cuh"

namespace {

using namespace luqdev;

constexpr uint32_t kFull = 0xFFFFFFFFu;

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

// ---- keys: whole numbers in the order of the values they stand for ------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);                        // (-0 is 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ unsigned long long key_of(double v) {
  const unsigned long long b = static_cast<unsigned long long>(__double_as_longlong(v + 0.0));
  return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double value_of(unsigned long long k) {
  return __longlong_as_double(static_cast<long long>(k >> 63 ? k & ~(1ull << 63) : ~k));
}
__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(kFull, k); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
  const uint32_t hi = __reduce_max_sync(kFull, static_cast<uint32_t>(k >> 32));
  const uint32_t lo = __reduce_max_sync(kFull, static_cast<uint32_t>(k >> 32) == hi ? static_cast<uint32_t>(k) : 0u);
  return static_cast<unsigned long long>(hi) << 32 | lo;
}
template <typename V> struct KeyOf;
template <> struct KeyOf<float> { using type = uint32_t; };
template <> struct KeyOf<double> { using type = unsigned long long; };

// ---- route ---------------------------------------------------------------------------------------------------------------
struct RouteParams {
  const void* logits;
  long long rows, ld;
  int experts, k;
  bool sigmoid;
  const float* bias;        // may be null
  int groups, top_groups, group_top;
  bool renormalize;
  float scale;
  int* chosen;
  float* weights;
  unsigned int* status;
};

__device__ __forceinline__ float minus_inf() { return __int_as_float(0xFF800000u); }
// scores in 32 and in 64 bits
__device__ __forceinline__ float sigmoid_of(float l) { return __fdividef(1.0f, 1.0f + expf(-l)); }
__device__ __forceinline__ double sigmoid_of(double l) { return 1.0 / (1.0 + exp(-l)); }

// Chooses: lane j gets the j-th expert (-1: none was left) and its logit.  Lane L holds the logits of experts L, L + 32, ...
// Values are of type V; with float the result is the exact one only if true is returned (no two values that decide lie closer
// than their error).
template <int VPL, typename V>
__device__ __forceinline__ bool choose(const RouteParams& p, const float (&l)[VPL], float row_max, int lane, int& mine, float& my_logit) {
  using Key = typename KeyOf<V>::type;
  const bool scored = p.bias || p.groups > 1;       // else the logits' order decides, which is exact
  V s[VPL];                                         // scores plus bias, or logits
  V err = 0;                                        // what a value may be off by
  if (!scored) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) s[i] = l[i];
  } else {
    V factor = 1;
    if (!p.sigmoid) {
      V sum = 0;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        if constexpr (std::is_same_v<V, float>) s[i] = expf(l[i] - row_max);
        else s[i] = exp(static_cast<double>(l[i]) - static_cast<double>(row_max));
        sum += s[i];
      }
      sum = warp_sum(sum);
      factor = V(1) / sum;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      if (p.sigmoid) s[i] = sigmoid_of(static_cast<V>(l[i]));
      else s[i] *= factor;
    }
    if constexpr (std::is_same_v<V, float>) {
      // Of scores up to s: sigmoid, the exponential's 2 ulp, a sum and a quotient (2 ulp): 6 half steps of 2^-24 s at most, s < 1.
      // Softmax: the difference of two logits is off by half a step of itself, which moves s by at most 0.37 2^-24 of the
      // row's largest; the exponential, VPL + 5 sums, quotient, product: VPL + 12 half steps.  The bias adds half a step of
      // the sum.  Twice that is taken.
      float largest = 0.0f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) largest = fmaxf(largest, s[i]);
      err = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(largest))) * (p.sigmoid ? 12.0f : 2.0f * (VPL + 13)) * 0x1p-24f;
    }
    float bias_top = 0.0f;
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = lane + 32 * i;
        if (e < p.experts) { const float b = *(p.bias + e); s[i] += static_cast<V>(b); bias_top = fmaxf(bias_top, fabsf(b) > 3e38f ? 0.0f : fabsf(b)); }
      }
    }
    if constexpr (std::is_same_v<V, float>) err += (1.0f + __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(bias_top)))) * 0x1p-24f;
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (lane + 32 * i >= p.experts || l[i] == minus_inf()) s[i] = minus_inf();
  }
  uint32_t gone = 0;                                // bit i: expert lane + 32 i cannot be chosen (any more)
  bool sure = true;
  // the best of the values for which `take` holds: its key and index
  auto best_of = [&](auto take, Key& key, int& index) {
    Key k = key_of(static_cast<V>(minus_inf()));
    int at = INT_MAX;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const Key ki = key_of(s[i]);
      if (take(i) && ki > k) { k = ki; at = lane + 32 * i; }
    }
    key = warp_max(k);
    index = static_cast<int>(__reduce_min_sync(kFull, static_cast<unsigned>(k == key ? at : INT_MAX)));
  };
  if (p.groups > 1) {
    // lane g keeps group g's value, its key
    const int size = p.experts / p.groups;
    V value = minus_inf();
    for (int g = 0; g < p.groups; ++g) {
      Key k1;
      int at;
      best_of([&](int i) { return (lane + 32 * i) / size == g; }, k1, at);
      V sum = value_of(k1);
      if (p.group_top == 2 && at != INT_MAX) {
        Key k2;
        int at2;
        best_of([&](int i) { return (lane + 32 * i) / size == g && lane + 32 * i != at; }, k2, at2);
        if (at2 != INT_MAX) sum += value_of(k2);
      }
      if (lane == g) value = sum;
    }
    uint32_t stay = 0;
    bool out = false;
    V last = 0;
    for (int h = 0; h <= p.top_groups && h < p.groups; ++h) {
      const Key k = lane < p.groups && !out ? key_of(value) : 0;
      const Key best = warp_max(k);
      const int g = static_cast<int>(__reduce_min_sync(kFull, static_cast<unsigned>(k == best && lane < p.groups && !out ? lane : INT_MAX)));
      const V v = value_of(best);
      if (h == p.top_groups) {
        // the first group that goes: is it clear of the last one that stays?
        if (std::is_same_v<V, float> && v > minus_inf() && !(last - v > 4 * err + (fabs(last) + 1) * V(0x1p-22f))) sure = false;
      } else {
        last = v;
        stay |= 1u << g;
        if (lane == g) out = true;
      }
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (!(stay >> min((lane + 32 * i) / size, 31) & 1)) gone |= 1u << i;
    if (!p.bias) {                                  // scores are in the order of the logits
#pragma unroll
      for (int i = 0; i < VPL; ++i) s[i] = l[i];
    }
  }
  mine = -1;
  my_logit = minus_inf();
  V before = 0;
  float before_logit = 0.0f, before_bias = 0.0f;
  for (int j = 0; j <= p.k; ++j) {
    if (j == p.k && !(std::is_same_v<V, float> && p.bias)) break;      // one more, to see how close it is
    Key key;
    int e;
    best_of([&](int i) { return !(gone >> i & 1); }, key, e);
    if (e == INT_MAX) break;
    float le = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (e >> 5 == i) le = l[i];
    le = __shfl_sync(kFull, le, e & 31);
    if (std::is_same_v<V, float> && p.bias) {
      const float be = *(p.bias + e);
      const V v = value_of(key);
      // (equal logits and biases have equal values, of which the lower index comes first)
      if (j > 0 && !(before - v > 2 * err) && !(le == before_logit && be == before_bias)) sure = false;
      before = v; before_logit = le; before_bias = be;
    }
    if (j < p.k) {
      if (lane == j) { mine = e; my_logit = le; }
      if (lane == (e & 31)) gone |= 1u << (e >> 5);
    }
  }
  return sure;
}

template <typename T, int VPL>
__global__ void __launch_bounds__(128) route_kernel(const RouteParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long r = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (r >= p.rows) return;
  const T* const row = static_cast<const T*>(p.logits) + r * p.ld;
  float l[VPL], top = minus_inf();
  bool bad = false;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int e = lane + 32 * i;
    l[i] = e < p.experts ? load1(row + e) : minus_inf();
    bad |= !(l[i] <= 3.402823466e38f);
    if (p.bias && e < p.experts) bad |= !(*(p.bias + e) <= 3.402823466e38f);
    top = fmaxf(top, l[i]);
  }
  top = value_of(warp_max(key_of(top)));
  int mine = -1;
  float logit = minus_inf(), w = 0.0f;
  if (__any_sync(kFull, bad)) {
    w = __int_as_float(0x7FC00000);
    if (lane == 0) atomicOr(p.status, LUQ_STATUS_NONFINITE);
  } else if (top > minus_inf()) {
    if (!choose<VPL, float>(p, l, top, lane, mine, logit)) choose<VPL, double>(p, l, top, lane, mine, logit);
    if (p.sigmoid) {
      w = mine >= 0 ? sigmoid_of(logit) : 0.0f;
    } else {
      // renormalised: relative to the largest chosen logit, so that they cannot all vanish
      const float shift = p.renormalize ? value_of(warp_max(key_of(mine >= 0 ? logit : minus_inf()))) : top;
      w = mine >= 0 ? expf(logit - shift) : 0.0f;
      if (!p.renormalize) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) sum += expf(l[i] - top);
        w /= warp_sum(sum);
      }
    }
    if (p.renormalize) {
      const float sum = warp_sum(w);
      w = sum > 0.0f ? w / sum : 0.0f;
    }
    w *= p.scale;
  }
  if (lane < p.k) {
    p.chosen[r * p.k + lane] = mine;
    p.weights[r * p.k + lane] = w;
  }
}

struct RouteBwdParams {
  const float* dweights;
  const void* logits;
  long long rows, ld;
  int experts, k;
  bool sigmoid, renormalize;
  float scale;
  const int* chosen;
  void* dlogits;
  long long ld_d;
};

// A warp has a row.  Renormalised scores and sigmoids have gradients at the chosen experts only; the softmax's other experts
// get -s_e sum_j s_j ds_j.
template <typename T>
__global__ void __launch_bounds__(128) route_bwd_kernel(const RouteBwdParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long r = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (r >= p.rows) return;
  const T* const row = static_cast<const T*>(p.logits) + r * p.ld;
  T* const out = static_cast<T*>(p.dlogits) + r * p.ld_d;
  int e = lane < p.k ? p.chosen[r * p.k + lane] : -1;
  if (e >= p.experts) e = -1;
  const float dw = e >= 0 ? p.dweights[r * p.k + lane] : 0.0f;
  const float l = e >= 0 ? load1(row + e) : minus_inf();
  const bool whole = !p.sigmoid && !p.renormalize;       // every logit has a gradient
  float top = minus_inf(), sum = 0.0f;
  if (whole) {
    for (int c = lane; c < p.experts; c += 32) top = fmaxf(top, load1(row + c));
    top = value_of(warp_max(key_of(top)));
    if (top > minus_inf())
      for (int c = lane; c < p.experts; c += 32) sum += expf(load1(row + c) - top);
    sum = warp_sum(sum);
  } else if (!p.sigmoid) {
    top = value_of(warp_max(key_of(l)));
  }
  float s = 0.0f;                                        // my score, or its share of the chosen ones' sum
  if (e >= 0 && l > minus_inf()) s = p.sigmoid ? sigmoid_of(l) : expf(l - top);
  if (whole && sum > 0.0f) s /= sum;
  float d = p.scale * dw;
  if (p.renormalize) {
    const float total = warp_sum(s);
    s = total > 0.0f ? s / total : 0.0f;
    d -= warp_sum(d * s);
  }
  const float along = whole ? warp_sum(s * d) : 0.0f;
  const float term = p.sigmoid ? d * s * (l > minus_inf() ? sigmoid_of(-l) : 0.0f) : s * d;
  // an expert that stands in several places gets the sum of theirs
  float mine = 0.0f;
  bool first = e >= 0;
  for (int j = 0; j < p.k; ++j) {
    const int ej = __shfl_sync(kFull, e, j);
    const float tj = __shfl_sync(kFull, term, j);
    if (ej == e) {
      mine += tj;
      first &= j >= lane;
    }
  }
  for (int c = lane; c < p.experts; c += 32) store1(out + c, whole && sum > 0.0f ? -along * (expf(load1(row + c) - top) / sum) : 0.0f);
  __syncwarp();
  if (first) store1(out + e, whole ? mine - s * along : mine);
}

// ---- order ---------------------------------------------------------------------------------------------------------------
// A stable counting sort.  A block has a segment of the assignments, a warp a run of it; runs are counted, the counts are
// summed over the runs before, and every run is walked once more, 32 assignments at a time: a lane's place is the number of
// lanes below it with the same expert.  More than one segment: a kernel counts them first.
struct OrderParams {
  const int* chosen;
  long long total;          // assignments
  int experts;
  long long segment;        // of a block; a multiple of 32 * kOrderWarps
  int* counts;              // [segments][experts], more than one segment
  int* position;
  int* offsets;
};
constexpr int kOrderWarps = 32;

// counts of a warp's run into `hist` (cleared)
__device__ __forceinline__ void count_run(const OrderParams& p, long long from, long long to, int* hist, int lane) {
  for (long long a = from; a < to; a += 32) {
    const int e = a + lane < to ? p.chosen[a + lane] : -1;
    const unsigned same = __match_any_sync(kFull, e);
    if (e >= 0 && e < p.experts && lane == __ffs(same) - 1) hist[e] += __popc(same);
    __syncwarp();
  }
}

__global__ void __launch_bounds__(32 * kOrderWarps) order_count_kernel(const OrderParams p) {
  extern __shared__ int hist[];                         // [warps][experts]
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kOrderWarps * p.experts; i += blockDim.x) hist[i] = 0;
  __syncthreads();
  const long long run = p.segment / kOrderWarps, from = blockIdx.x * p.segment + warp * run;
  count_run(p, from, min(from + run, p.total), hist + warp * p.experts, lane);
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
    int n = 0;
    for (int w = 0; w < kOrderWarps; ++w) n += hist[w * p.experts + e];
    p.counts[static_cast<long long>(blockIdx.x) * p.experts + e] = n;
  }
}

__global__ void __launch_bounds__(32 * kOrderWarps) order_kernel(const OrderParams p) {
  extern __shared__ int hist[];                         // [warps][experts]: counts, then the next position of each
  __shared__ int sums[kOrderWarps];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kOrderWarps * p.experts; i += blockDim.x) hist[i] = 0;
  __syncthreads();
  const long long run = p.segment / kOrderWarps, from = blockIdx.x * p.segment + warp * run, to = min(from + run, p.total);
  int* const own = hist + warp * p.experts;
  count_run(p, from, to, own, lane);
  __syncthreads();
  // a thread has an expert (there are at most as many): its copies before this block's segment, and in all segments
  const int e = threadIdx.x;
  int before = 0, all = 0;
  if (e < p.experts) {
    if (gridDim.x > 1) {
      for (unsigned b = 0; b < gridDim.x; ++b) {
        const int n = p.counts[static_cast<long long>(b) * p.experts + e];
        all += n;
        if (b < blockIdx.x) before += n;
      }
    } else {
      for (int w = 0; w < kOrderWarps; ++w) all += hist[w * p.experts + e];
    }
  }
  int start = all;                                      // sum over the experts up to this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(kFull, start, o);
    if (lane >= o) start += up;
  }
  if (lane == 31) sums[warp] = start;
  __syncthreads();
  for (int w = 0; w < warp; ++w) start += sums[w];
  if (e < p.experts) {
    if (blockIdx.x == 0) p.offsets[e + 1] = start;
    int next = start - all + before;
    for (int w = 0; w < kOrderWarps; ++w) {
      const int n = hist[w * p.experts + e];
      hist[w * p.experts + e] = next;
      next += n;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[0] = 0;
  __syncthreads();
  for (long long a = from; a < to; a += 32) {
    const int x = a + lane < to ? p.chosen[a + lane] : -1;
    const unsigned same = __match_any_sync(kFull, x);
    const bool valid = x >= 0 && x < p.experts;
    int at = -1;
    if (valid) at = own[x] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (valid && lane == __ffs(same) - 1) own[x] += __popc(same);
    __syncwarp();
    if (a + lane < to) p.position[a + lane] = at;
  }
}

// ---- dispatch and combine --------------------------------------------------------------------------------------------------
// Rows in pieces of 16 bytes where every row starts at a multiple of them, else element by element.  A warp has a token's
// segment of 32 pieces.
template <typename T, bool VEC>
struct Piece {
  static constexpr int n = VEC ? 16 / static_cast<int>(sizeof(T)) : 1;
  float v[n];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (!VEC) {
      v[0] = load1(p);
    } else if constexpr (sizeof(T) == 4) {
      const float4 f = *reinterpret_cast<const float4*>(p);
      v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    } else {
      const uint4 u = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (!VEC) {
      store1(p, v[0]);
    } else if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};

struct MoveParams {
  const void* x;            // dispatch: tokens; combine: results; combine_bwd: results
  long long ld_x;
  const void* more;         // combine: residual (may be null); combine_bwd: dout
  long long ld_more;
  const int* position;
  long long rows;           // tokens
  int k, cols, segments;
  long long copies;         // rows of the copies' tensor
  const float* weights;     // may be null: ones
  const int* offsets;       // dispatch, combine_bwd: rows from offsets[groups] on are zeroed
  int groups;
  void* out;
  long long ld_out;
  float* dweights;
  unsigned int* status;
};

__device__ __forceinline__ bool copy_in(const MoveParams& p, int to) { return to >= 0 && to < p.copies; }

// rows of the copies that no token has
template <typename T, bool VEC>
__device__ __forceinline__ void zero_rest(const MoveParams& p, long long warp, long long warps, int lane) {
  const int used = min(max(*(p.offsets + p.groups), 0), static_cast<int>(p.copies));
  Piece<T, VEC> zero;
#pragma unroll
  for (int i = 0; i < zero.n; ++i) zero.v[i] = 0.0f;
  for (long long r = used + warp; r < p.copies; r += warps)
    for (int c = lane * zero.n; c < p.cols; c += 32 * zero.n) zero.store(static_cast<T*>(p.out) + r * p.ld_out + c);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dispatch_kernel(const MoveParams p) {
  using P = Piece<T, VEC>;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long warp = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5), warps = static_cast<long long>(gridDim.x) * 8;
  for (long long i = warp; i < p.rows * p.segments; i += warps) {
    const long long t = i / p.segments;
    const int c = (static_cast<int>(i - t * p.segments) * 32 + lane) * P::n;
    const int* const to = p.position + t * p.k;
    if (c >= p.cols) continue;
    P v;
    v.load(static_cast<const T*>(p.x) + t * p.ld_x + c);
    for (int j = 0; j < p.k; ++j)
      if (copy_in(p, to[j])) v.store(static_cast<T*>(p.out) + to[j] * p.ld_out + c);
  }
  zero_rest<T, VEC>(p, warp, warps, lane);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) combine_kernel(const MoveParams p) {
  using P = Piece<T, VEC>;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long warp = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5), warps = static_cast<long long>(gridDim.x) * 8;
  for (long long i = warp; i < p.rows * p.segments; i += warps) {
    const long long t = i / p.segments;
    const int c = (static_cast<int>(i - t * p.segments) * 32 + lane) * P::n;
    if (c >= p.cols) continue;
    P sum;
    if (p.more) sum.load(static_cast<const T*>(p.more) + t * p.ld_more + c);
    else
#pragma unroll
      for (int q = 0; q < P::n; ++q) sum.v[q] = 0.0f;
    for (int j = 0; j < p.k; ++j) {
      const int at = p.position[t * p.k + j];
      const float w = p.weights ? p.weights[t * p.k + j] : 1.0f;
      P v;
#pragma unroll
      for (int q = 0; q < P::n; ++q) v.v[q] = 0.0f;
      if (copy_in(p, at)) v.load(static_cast<const T*>(p.x) + at * p.ld_x + c);
#pragma unroll
      for (int q = 0; q < P::n; ++q) sum.v[q] = fmaf(w, v.v[q], sum.v[q]);
    }
    sum.store(static_cast<T*>(p.out) + t * p.ld_out + c);
  }
}

// dy[position] = w dout, dw = dout . y[position]: a warp has a copy
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) combine_bwd_kernel(const MoveParams p) {
  using P = Piece<T, VEC>;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long warp = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5), warps = static_cast<long long>(gridDim.x) * 8;
  for (long long i = warp; i < p.rows * p.k; i += warps) {
    const int at = p.position[i];
    if (!copy_in(p, at)) {
      if (lane == 0 && p.dweights) p.dweights[i] = 0.0f;
      continue;
    }
    const long long t = i / p.k;
    const float w = p.weights ? p.weights[i] : 1.0f;
    float dot = 0.0f;
    for (int c = lane * P::n; c < p.cols; c += 32 * P::n) {
      P d, y;
      d.load(static_cast<const T*>(p.more) + t * p.ld_more + c);
      if (p.dweights) {
        y.load(static_cast<const T*>(p.x) + at * p.ld_x + c);
#pragma unroll
        for (int q = 0; q < P::n; ++q) dot = fmaf(d.v[q], y.v[q], dot);
      }
      if (p.out) {
#pragma unroll
        for (int q = 0; q < P::n; ++q) d.v[q] *= w;
        d.store(static_cast<T*>(p.out) + at * p.ld_out + c);
      }
    }
    dot = warp_sum(dot);
    if (lane == 0 && p.dweights) p.dweights[i] = dot;
  }
  if (p.out) zero_rest<T, VEC>(p, warp, warps, lane);
}

bool vec16(const void* p, long long ld, long long rows, int esize) {
  return !p || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld * esize % 16 == 0));
}
int blocks_of(const luq_ctx* ctx, long long warps) {
  const long long blocks = (warps + 7) / 8, most = ctx->sm_count * 32ll;
  return static_cast<int>(blocks < 1 ? 1 : blocks < most ? blocks : most);
}
int done(luq_ctx* ctx, cudaError_t e) {
  if (e == cudaSuccess) ctx->launches += 1;
  return static_cast<int>(e);
}

template <typename T, int VPL>
int launch_route(luq_ctx* ctx, const RouteParams& p, cudaStream_t st) {
  return done(ctx, luq_launch_kernel(route_kernel<T, VPL>, static_cast<int>((p.rows + 3) / 4), 128, 0, st, LUQ_LAUNCH_EARLY, 1, p));
}
template <typename T>
int launch_route_width(luq_ctx* ctx, const RouteParams& p, cudaStream_t st) {
  if (p.experts <= 32) return launch_route<T, 1>(ctx, p, st);
  if (p.experts <= 64) return launch_route<T, 2>(ctx, p, st);
  if (p.experts <= 128) return launch_route<T, 4>(ctx, p, st);
  if (p.experts <= 256) return launch_route<T, 8>(ctx, p, st);
  if (p.experts <= 512) return launch_route<T, 16>(ctx, p, st);
  return launch_route<T, 32>(ctx, p, st);
}

MoveParams move_params(const luq_ctx* ctx, const luq_move_args& a, bool& vec) {
  const int esize = a.dtype == LUQ_BF16 ? 2 : 4;
  MoveParams p{};
  p.x = a.x; p.ld_x = a.ld_x; p.more = a.more; p.ld_more = a.ld_more; p.position = a.position; p.rows = a.rows; p.k = a.k;
  p.cols = static_cast<int>(a.cols); p.copies = a.copies; p.weights = a.weights; p.offsets = a.offsets; p.groups = a.groups;
  p.out = a.out; p.ld_out = a.ld_out; p.dweights = a.dweights; p.status = ctx->d_status;
  // (row counts play no part: a row of one is as good as any)
  vec = a.cols * esize % 16 == 0 && vec16(a.x, a.ld_x, 2, esize) && vec16(a.more, a.ld_more, 2, esize) && vec16(a.out, a.ld_out, 2, esize);
  const int n = vec ? 16 / esize : 1;
  p.segments = static_cast<int>((a.cols + 32 * n - 1) / (32 * n));
  return p;
}
// chooses one of a kernel's four forms
#define LUQ_MOVE(kernel, warps)                                                                                               \
  (a.dtype == LUQ_BF16                                                                                                        \
       ? done(ctx, luq_launch_kernel(vec ? kernel<__nv_bfloat16, true> : kernel<__nv_bfloat16, false>, blocks_of(ctx, warps), 256, 0, st, LUQ_LAUNCH_EARLY, 1, p)) \
       : done(ctx, luq_launch_kernel(vec ? kernel<float, true> : kernel<float, false>, blocks_of(ctx, warps), 256, 0, st, LUQ_LAUNCH_EARLY, 1, p)))

}  // namespace

int luq_launch_route(luq_ctx* ctx, const luq_route_args& a, cudaStream_t st) {
  RouteParams p{a.logits, a.rows, a.ld, a.experts, a.k, a.sigmoid, a.bias, a.groups, a.top_groups, a.group_top, a.renormalize, a.scale,
                a.chosen, a.weights, ctx->d_status};
  return a.dtype == LUQ_BF16 ? launch_route_width<__nv_bfloat16>(ctx, p, st) : launch_route_width<float>(ctx, p, st);
}

int luq_launch_route_bwd(luq_ctx* ctx, const luq_route_args& a, const float* dweights, void* dlogits, int64_t ld_d, cudaStream_t st) {
  RouteBwdParams p{dweights, a.logits, a.rows, a.ld, a.experts, a.k, a.sigmoid, a.renormalize, a.scale, a.chosen, dlogits, ld_d};
  const int blocks = static_cast<int>((a.rows + 3) / 4);
  return done(ctx, luq_launch_kernel(a.dtype == LUQ_BF16 ? route_bwd_kernel<__nv_bfloat16> : route_bwd_kernel<float>, blocks, 128, 0, st,
                                     LUQ_LAUNCH_EARLY, 1, p));
}

// bytes of workspace that the order of `total` assignments needs
static int64_t order_segments(int64_t total, int64_t* segment) {
  constexpr int64_t kLeast = 32 * kOrderWarps * 4, kMost = 256;
  int64_t s = kLeast;
  if (total > kLeast * kMost) s = ((total + kMost - 1) / kMost + 32 * kOrderWarps - 1) / (32 * kOrderWarps) * (32 * kOrderWarps);
  *segment = s;
  return (total + s - 1) / s;
}
size_t luq_order_workspace(int64_t total, int experts) {
  int64_t segment;
  const int64_t n = order_segments(total, &segment);
  return n > 1 ? static_cast<size_t>(n) * experts * sizeof(int) : 0;
}
int luq_launch_order(luq_ctx* ctx, const int* chosen, int64_t total, int experts, int* position, int* offsets, int* counts, cudaStream_t st) {
  OrderParams p{chosen, total, experts, 0, counts, position, offsets};
  int64_t segment;
  const int blocks = total > 0 ? static_cast<int>(order_segments(total, &segment)) : 1;
  if (total == 0) segment = 32 * kOrderWarps;
  p.segment = segment;
  const size_t smem = static_cast<size_t>(kOrderWarps) * experts * sizeof(int);
  static luq_once_per_device allowed;
  const cudaError_t attr = allowed([&] {
    constexpr int most = kOrderWarps * LUQ_MAX_GROUPS * sizeof(int);
    const cudaError_t e = cudaFuncSetAttribute(order_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(order_count_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  }, ctx->device);
  if (attr != cudaSuccess) return static_cast<int>(attr);
  if (blocks > 1) {
    const int e = done(ctx, luq_launch_kernel(order_count_kernel, blocks, 32 * kOrderWarps, smem, st, LUQ_LAUNCH_EARLY, 1, p));
    if (e) return e;
  }
  return done(ctx, luq_launch_kernel(order_kernel, blocks, 32 * kOrderWarps, smem, st, LUQ_LAUNCH_EARLY, 1, p));
}

int luq_launch_dispatch(luq_ctx* ctx, const luq_move_args& a, cudaStream_t st) {
  bool vec;
  const MoveParams p = move_params(ctx, a, vec);
  return LUQ_MOVE(dispatch_kernel, p.rows * p.segments);
}
int luq_launch_combine(luq_ctx* ctx, const luq_move_args& a, cudaStream_t st) {
  bool vec;
  const MoveParams p = move_params(ctx, a, vec);
  return LUQ_MOVE(combine_kernel, p.rows * p.segments);
}
int luq_launch_combine_bwd(luq_ctx* ctx, const luq_move_args& a, cudaStream_t st) {
  bool vec;
  const MoveParams p = move_params(ctx, a, vec);
  return LUQ_MOVE(combine_bwd_kernel, p.rows * p.k);
}
