// The preference loss of paired sequences on the LM head's logits, forward and backward.
//
// A pair is one example of 2T rows, the preferred sequence's T rows and then the other's.  With log-probabilities
// l = sum over the unmasked tokens of log softmax(logits)[target] and those of a reference model r,
//   h = beta * ((l_c - r_c) - (l_r - r_r)),   loss = -(1 - e) log s(h) - e log s(-h),   s the logistic function,
// and the gradient at the logits of a row is c * (onehot(target) - softmax), where c = +-dloss/dh * beta: the G of the
// head in a clipped step.  A row's statistics are its maximum and the sum of its exponentials, kept together (the sum is
// rescaled when the maximum moves); logits are read for them and read again for the gradient, which needs both
// sequences' sums.  Rows whose target is masked are not read; their gradient is 0.
//
// Exponents are x log2 e - c and a row's sum is fp32; a token's log-probability is ((x_target log2 e - c) - log2(sum)) ln 2,
// without the cancellation of x - (c ln 2 + log(sum)); sequences are added up in 64 bits, since h is
// a small difference of long sums.
#include <algorithm>
#include <cmath>

#include "dp_common.cuh"

namespace dpg {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kPrefThreads = 512;

// 16 bytes of logits: eight bf16 or four fp32
template <typename T> struct Quad;
template <> struct Quad<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    __nv_bfloat162 h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
    uint4 q;
    memcpy(&q, h, 16);
    return q;
  }
  static __device__ __forceinline__ __nv_bfloat16 round(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Quad<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
  static __device__ __forceinline__ float round(float v) { return v; }
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sum of 2^(x log2 e - c) over the values seen so far, c = (their maximum) * log2 e as rounded; -inf and 0 of none.  With the
// rounded c as the reference everywhere its rounding cancels, and an exponent is one FMA.
struct Softmax {
  float c, s;
  static __device__ __forceinline__ float exponent(float x, float c) { return fmaf(x, kLog2e, c == -INFINITY ? 0.f : -c); }
  __device__ __forceinline__ void add(float x) {
    const float top = x * kLog2e;
    if (top > c) { s *= exp2_fast(c - top); c = top; }
    s += exp2_fast(exponent(x, c));
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&v)[N]) {
    float top = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, v[e]);
    top *= kLog2e;
    if (top > c) { s *= exp2_fast(c - top); c = top; }
    const float minus = c == -INFINITY ? 0.f : -c;
#pragma unroll
    for (int e = 0; e < N; ++e) s += exp2_fast(fmaf(v[e], kLog2e, minus));
  }
  __device__ __forceinline__ void join(float oc, float os) {
    const float top = fmaxf(c, oc);
    if (top == -INFINITY) { s += os; return; }       // nothing in either (or only NaN, which the sums carry)
    s = s * exp2_fast(c - top) + os * exp2_fast(oc - top);
    c = top;
  }
};

struct PrefParams {
  const void* logits; long long ldl;
  void* G; long long ldg;
  const int32_t* targets;
  const float* ref;
  float* loss; float* logp;
  float* row_logp; float* row_max; float* row_inv;     // [2BT] workspace
  float* coef;                                         // [2B]
  int* dev_status;
  int B, T, V;
  float beta, smoothing, scale;
};

// a row's target, or -1 where the row does not count
__device__ __forceinline__ int row_target(const PrefParams& P, long long row, bool report) {
  const int t = P.targets[row];
  if (t >= P.V) {
    if (report && P.dev_status) atomicOr(P.dev_status, DP_DEV_BAD_ID);
    return -1;
  }
  return t;
}

template <typename T>
__global__ void __launch_bounds__(kPrefThreads)
logit_stats_kernel(const PrefParams P) {
  constexpr int N = Quad<T>::N;
  __shared__ float sm[32], ss[32];
  const long long row = blockIdx.x;
  const int target = row_target(P, row, threadIdx.x == 0);
  if (target < 0) {
    if (threadIdx.x == 0) { P.row_logp[row] = 0.f; P.row_max[row] = 0.f; P.row_inv[row] = 0.f; }
    return;
  }
  const T* x = static_cast<const T*>(P.logits) + row * P.ldl;
  const int head = min(P.V, int(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
  const int quads = (P.V - head) / N;
  const uint4* xq = reinterpret_cast<const uint4*>(x + head);
  Softmax acc{-INFINITY, 0.f};
  for (int k = threadIdx.x; k < quads; k += blockDim.x) {
    float v[N];
    Quad<T>::unpack(xq[k], v);
    acc.add(v);
  }
  for (int k = threadIdx.x; k < head; k += blockDim.x) acc.add(to_f32(x[k]));
  for (int k = head + quads * N + threadIdx.x; k < P.V; k += blockDim.x) acc.add(to_f32(x[k]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    acc.join(__shfl_xor_sync(0xffffffffu, acc.c, o), __shfl_xor_sync(0xffffffffu, acc.s, o));
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) { sm[warp] = acc.c; ss[warp] = acc.s; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < int(blockDim.x >> 5); ++w) acc.join(sm[w], ss[w]);
    P.row_logp[row] = (Softmax::exponent(to_f32(x[target]), acc.c) - log2f(acc.s)) * kLn2;
    P.row_max[row] = acc.c;
    P.row_inv[row] = 1.f / acc.s;
  }
}

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }
__device__ __forceinline__ double logistic(double x) { return 1.0 / (1.0 + exp(-x)); }

// a pair's sequences summed, its loss and the factor of its rows
__global__ void __launch_bounds__(128)
pair_loss_kernel(const PrefParams P) {
  __shared__ double part[2][4];
  const int pair = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double l[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    double s = 0.0;
    const float* in = P.row_logp + (2LL * pair + q) * P.T;
    for (int t = threadIdx.x; t < P.T; t += 128) s += double(in[t]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) part[q][warp] = s;
  }
  __syncthreads();
  if (threadIdx.x) return;
#pragma unroll
  for (int q = 0; q < 2; ++q) l[q] = (part[q][0] + part[q][1]) + (part[q][2] + part[q][3]);
  const double rc = P.ref ? double(P.ref[2 * pair]) : 0.0, rr = P.ref ? double(P.ref[2 * pair + 1]) : 0.0;
  const double h = double(P.beta) * ((l[0] - rc) - (l[1] - rr)), e = double(P.smoothing);
  if (P.loss) P.loss[pair] = float((1.0 - e) * softplus(-h) + e * softplus(h));
  if (P.logp) { P.logp[2 * pair] = float(l[0]); P.logp[2 * pair + 1] = float(l[1]); }
  const double slope = double(P.scale) * double(P.beta) * (e * logistic(h) - (1.0 - e) * logistic(-h));
  P.coef[2 * pair] = float(slope);
  P.coef[2 * pair + 1] = float(-slope);
}

template <typename T>
__global__ void __launch_bounds__(kPrefThreads)
logit_gradient_kernel(const PrefParams P) {
  constexpr int N = Quad<T>::N;
  const long long row = blockIdx.x;
  const int target = row_target(P, row, false);
  const T* x = static_cast<const T*>(P.logits) + row * P.ldl;
  T* g = static_cast<T*>(P.G) + row * P.ldg;
  const float c = target < 0 ? 0.f : P.coef[row / P.T];
  const float m = P.row_max[row], f = c * P.row_inv[row];
  auto grad = [&](float v, int k) {
    const float e = f * exp2_fast(Softmax::exponent(v, m));
    return k == target ? c - e : -e;
  };
  // quads where reads and writes share their alignment, and the columns around them
  const int head = min(P.V, int(((16 - (reinterpret_cast<uintptr_t>(g) & 15)) & 15) / sizeof(T)));
  const bool aligned = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  const int quads = aligned || target < 0 ? (P.V - head) / N : 0;
  const uint4* xq = reinterpret_cast<const uint4*>(x + head);
  uint4* gq = reinterpret_cast<uint4*>(g + head);
  for (int k = threadIdx.x; k < quads; k += blockDim.x) {
    uint4 q = make_uint4(0u, 0u, 0u, 0u);
    if (target >= 0) {
      float v[N];
      Quad<T>::unpack(xq[k], v);
      const int c0 = head + k * N;
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = grad(v[e], c0 + e);
      q = Quad<T>::pack(v);
    }
    gq[k] = q;
  }
  for (int k = threadIdx.x; k < head; k += blockDim.x) g[k] = Quad<T>::round(target < 0 ? 0.f : grad(to_f32(x[k]), k));
  for (int k = head + quads * N + threadIdx.x; k < P.V; k += blockDim.x)
    g[k] = Quad<T>::round(target < 0 ? 0.f : grad(to_f32(x[k]), k));
}

template <typename T>
dp_status pref_launch(const PrefParams& P, cudaStream_t st) {
  const unsigned rows = 2u * unsigned(P.B) * unsigned(P.T);
  logit_stats_kernel<T><<<rows, kPrefThreads, 0, st>>>(P);
  DP_LAUNCH_OK();
  pair_loss_kernel<<<P.B, 128, 0, st>>>(P);
  DP_LAUNCH_OK();
  if (!P.G) return DP_OK;
  logit_gradient_kernel<T><<<rows, kPrefThreads, 0, st>>>(P);
  DP_LAUNCH_OK();
  return DP_OK;
}

}  // namespace

}  // namespace dpg

using namespace dpg;

extern "C" {

size_t dp_preference_loss_ws_bytes(int32_t B, int32_t T) {
  if (B <= 0 || T <= 0) return 0;
  return align_up((3 * 2 * size_t(B) * size_t(T) + 2 * size_t(B)) * sizeof(float), 256);
}

dp_status dp_preference_loss(const void* logits, int64_t ldl, dp_dtype dt, int32_t B, int32_t T, int32_t V, const int32_t* targets,
                             const float* ref_logp, float beta, float smoothing, float scale, float* loss, float* logp, void* G,
                             int64_t ldg, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) {
  if (!logits || !targets || B <= 0 || T <= 0 || V <= 0 || ldl < V || (G && ldg < V)) return DP_ERR_INVALID_ARG;
  if (!loss && !logp && !G) return DP_ERR_INVALID_ARG;
  if (dt != DP_F32 && dt != DP_BF16) return DP_ERR_INVALID_ARG;
  if (!std::isfinite(beta) || beta < 0.f || !(smoothing >= 0.f && smoothing <= 1.f) || !std::isfinite(scale)) return DP_ERR_INVALID_ARG;
  if (G == logits && ldg != ldl) return DP_ERR_INVALID_ARG;
  if (2LL * B * T > 0x7fffffffLL) return DP_ERR_UNSUPPORTED;
  const size_t es = dt == DP_F32 ? 4 : 2;
  if (!on_boundary(es, logits, G) || !on_boundary(4, targets, ref_logp, loss, logp)) return DP_ERR_ALIGNMENT;
  if (!ws || ws_bytes < dp_preference_loss_ws_bytes(B, T)) return DP_ERR_WORKSPACE;
  if (!on_boundary(4, ws)) return DP_ERR_ALIGNMENT;
  const size_t rows = 2 * size_t(B) * size_t(T);
  float* f = static_cast<float*>(ws);
  const PrefParams P{logits, ldl, G, ldg, targets, ref_logp, loss, logp, f, f + rows, f + 2 * rows, f + 3 * rows, dev_status,
                     B, T, V, beta, smoothing, scale};
  const cudaStream_t st = (cudaStream_t)stream;
  return dt == DP_F32 ? pref_launch<float>(P, st) : pref_launch<__nv_bfloat16>(P, st);
}

}  // extern "C"
