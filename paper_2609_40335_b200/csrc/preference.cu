// The preference loss of paired sequences on the LM head's logits, forward and backward.
//
// A pair is one example of 2T rows, the preferred sequence's T rows and then the other's.  With log-probabilities
// l = sum over the unmasked tokens of log softmax(logits)[target] and those of a reference model r,
//   h = beta * ((l_c - r_c) - (l_r - r_r)),   loss = -(1 - e) log s(h) - e log s(-h),   s the logistic function,
// and the gradient at the logits of a row is c * (onehot(target) - softmax), where c = +-dloss/dh * beta: the G of the
// head in a clipped step.  A row's statistics are its maximum and the sum of its exponentials, kept together (the sum is
// rescaled when the maximum moves).  The gradient needs both sequences' sums, so a row is read again for it; rows whose target is
// masked are not read, their gradient is 0.
//
// Two forms.  pair_kernel: a cluster of up to eight CTAs per pair, one launch, no workspace; the rows of a small call stay in the caches in
// between.  preference_kernel: persistent CTAs draw rows in order, statistics of later pairs alternating with gradients of earlier ones, so
// that a row's second reading comes soon enough after the first to find it in the L2: the call then reads logits once from memory and
// writes the gradient once.  The CTA that finishes a pair's last row adds up its sequences.
//
// Exponents are x log2 e - c and a row's sum is fp32; a token's log-probability is ((x_target log2 e - c) - log2(sum)) ln 2,
// without the cancellation of x - (c ln 2 + log(sum)); sequences are added up in 64 bits, since h is
// a small difference of long sums.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "dp_common.cuh"

namespace dpg {

namespace {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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
    float t[N];
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = exp2_fast(fmaf(v[e], kLog2e, minus));
#pragma unroll
    for (int w = N / 2; w > 0; w /= 2)
#pragma unroll
      for (int e = 0; e < w; ++e) t[e] += t[e + w];
    s += t[0];
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
  float* row_logp; float* row_c; float* row_inv;       // [2BT] workspace
  float* coef;                                         // [2B]
  uint32_t* ticket; uint32_t* done; uint32_t* ready;   // the next row to draw; rows finished and sums made, [B] each
  int* dev_status;
  int B, T, V;
  long long rows, lag;                                 // a gradient follows the statistics of `lag` rows later
  float beta, smoothing, scale;
  long long wait_limit;
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

// elements up to the next 16-byte boundary
template <typename T>
__device__ __forceinline__ int head_of(const T* x, int V) {
  return min(V, int(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
}

// This thread's share of a row's statistics, one thread of n.
template <typename T>
__device__ __forceinline__ Softmax scan_row(const T* x, int V, int tid, int n) {
  constexpr int N = Quad<T>::N, U = 4;
  const int head = head_of(x, V), quads = (V - head) / N;
  const uint4* xq = reinterpret_cast<const uint4*>(x + head);
  Softmax acc{-INFINITY, 0.f};
  int k = tid;
  for (; k + (U - 1) * n < quads; k += U * n) {
    uint4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) q[u] = xq[k + u * n];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[N];
      Quad<T>::unpack(q[u], v);
      acc.add(v);
    }
  }
  for (; k < quads; k += n) {
    float v[N];
    Quad<T>::unpack(xq[k], v);
    acc.add(v);
  }
  for (int c = tid; c < head; c += n) acc.add(to_f32(x[c]));
  for (int c = head + quads * N + tid; c < V; c += n) acc.add(to_f32(x[c]));
  return acc;
}

__device__ __forceinline__ Softmax warp_join(Softmax a) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float c = __shfl_xor_sync(0xffffffffu, a.c, o), s = __shfl_xor_sync(0xffffffffu, a.s, o);
    a.join(c, s);
  }
  return a;
}

__device__ __forceinline__ float token_logp(float x, const Softmax& a) { return (Softmax::exponent(x, a.c) - log2f(a.s)) * kLn2; }

// This thread's share of a row's gradient: f = c / (sum of exponentials).  target < 0: zeros.
template <typename T>
__device__ __forceinline__ void write_gradient(const T* x, T* g, int V, int target, float c, float row_c, float inv, int tid, int n) {
  constexpr int N = Quad<T>::N, U = 4;
  const float f = c * inv;
  auto grad = [&](float v, int k) {
    const float e = f * exp2_fast(Softmax::exponent(v, row_c));
    return k == target ? c - e : -e;
  };
  // quads where reads and writes share their alignment, and the columns around them
  const int head = head_of(g, V);
  const bool aligned = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  const int quads = aligned || target < 0 ? (V - head) / N : 0;
  const uint4* xq = reinterpret_cast<const uint4*>(x + head);
  uint4* gq = reinterpret_cast<uint4*>(g + head);
  // x and g may be one tensor: a thread has read what it writes
  auto one = [&](int k, const uint4& q) {
    float v[N];
    Quad<T>::unpack(q, v);
    const int at = head + k * N, hit = target - at;
    const float minus = row_c == -INFINITY ? 0.f : -row_c;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = -f * exp2_fast(fmaf(v[e], kLog2e, minus));
    if (hit >= 0 && hit < N) {
#pragma unroll
      for (int e = 0; e < N; ++e) if (e == hit) v[e] += c;
    }
    __stcs(gq + k, Quad<T>::pack(v));
  };
  if (target < 0) {
    for (int k = tid; k < quads; k += n) __stcs(gq + k, make_uint4(0u, 0u, 0u, 0u));
  } else {
    int k = tid;
    for (; k + (U - 1) * n < quads; k += U * n) {
      uint4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = __ldcs(xq + k + u * n);
#pragma unroll
      for (int u = 0; u < U; ++u) one(k + u * n, q[u]);
    }
    for (; k < quads; k += n) one(k, __ldcs(xq + k));
  }
  for (int k = tid; k < head; k += n) g[k] = Quad<T>::round(target < 0 ? 0.f : grad(to_f32(x[k]), k));
  for (int k = head + quads * N + tid; k < V; k += n) g[k] = Quad<T>::round(target < 0 ? 0.f : grad(to_f32(x[k]), k));
}

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }
__device__ __forceinline__ double logistic(double x) { return 1.0 / (1.0 + exp(-x)); }

// The factor of a pair's preferred rows (the others' is its negative); its loss and log-probabilities if `write`.
__device__ float pair_loss(const PrefParams& P, int pair, double lc, double lr, bool write) {
  const double rc = P.ref ? double(P.ref[2 * pair]) : 0.0, rr = P.ref ? double(P.ref[2 * pair + 1]) : 0.0;
  const double h = double(P.beta) * ((lc - rc) - (lr - rr)), e = double(P.smoothing);
  if (write) {
    if (P.loss) P.loss[pair] = float((1.0 - e) * softplus(-h) + e * softplus(h));
    if (P.logp) { P.logp[2 * pair] = float(lc); P.logp[2 * pair + 1] = float(lr); }
  }
  return float(double(P.scale) * double(P.beta) * (e * logistic(h) - (1.0 - e) * logistic(-h)));
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---- small calls: a cluster per pair ---------------------------------------------------------------

constexpr int kPairThreads = 512;
constexpr int kPairRows = 512;             // rows of a CTA, at most
constexpr int kWarpRow = 2048;             // vocabularies up to this: a warp per row, else the CTA

template <typename T>
__global__ void __launch_bounds__(kPairThreads)
pair_kernel(const PrefParams P) {
  __shared__ float row_c[kPairRows], row_inv[kPairRows], row_logp[kPairRows], sc[kPairThreads / 32], ss[kPairThreads / 32];
  __shared__ double part[2];
  __shared__ float factor;
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank(), pair = blockIdx.x / ctas;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r0 = 2 * P.T * rank / ctas, n = 2 * P.T * (rank + 1) / ctas - r0;
  const long long first = 2LL * P.T * pair + r0;
  const T* logits = static_cast<const T*>(P.logits);
  const bool by_warp = P.V <= kWarpRow;
  for (int r = by_warp ? warp : 0; r < n; r += by_warp ? kPairThreads / 32 : 1) {
    const T* x = logits + (first + r) * P.ldl;
    const int target = row_target(P, first + r, by_warp ? lane == 0 : tid == 0);
    Softmax a{-INFINITY, 0.f};
    if (target >= 0) a = warp_join(scan_row(x, P.V, by_warp ? lane : tid, by_warp ? 32 : kPairThreads));
    if (!by_warp) {
      if (lane == 0) { sc[warp] = a.c; ss[warp] = a.s; }
      __syncthreads();
      a = Softmax{sc[0], ss[0]};
      for (int w = 1; w < kPairThreads / 32; ++w) a.join(sc[w], ss[w]);
      __syncthreads();
    }
    if (by_warp ? lane == 0 : tid == 0) {
      row_c[r] = a.c;
      row_inv[r] = target < 0 ? 0.f : 1.f / a.s;
      row_logp[r] = target < 0 ? 0.f : token_logp(to_f32(x[target]), a);
    }
  }
  __syncthreads();
  if (warp < 2) {                                      // warp q: this CTA's rows of sequence q
    double s = 0.0;
    for (int r = lane; r < n; r += 32)
      if ((r0 + r >= P.T) == (warp == 1)) s += double(row_logp[r]);
    s = warp_sum(s);
    if (lane == 0) part[warp] = s;
  }
  cluster.sync();
  if (tid == 0) {
    double lc = 0.0, lr = 0.0;
    for (int k = 0; k < ctas; ++k) {
      const double* other = cluster.map_shared_rank(part, k);
      lc += other[0];
      lr += other[1];
    }
    factor = pair_loss(P, pair, lc, lr, rank == 0);
  }
  __syncthreads();
  if (P.G) {
    for (int r = by_warp ? warp : 0; r < n; r += by_warp ? kPairThreads / 32 : 1)
      write_gradient(logits + (first + r) * P.ldl, static_cast<T*>(P.G) + (first + r) * P.ldg, P.V, row_target(P, first + r, false),
                     r0 + r < P.T ? factor : -factor, row_c[r], row_inv[r], by_warp ? lane : tid, by_warp ? 32 : kPairThreads);
  }
  cluster.sync();                                      // no CTA leaves while its sums are read
}

// ---- large calls: rows in the order of their second reading -----------------------------------------

constexpr int kRowThreads = 512, kRowBlocks = 2;       // per CTA, per SM

// Which row the n-th draw is, and whether it is a gradient: `lag` statistics, then gradients and statistics in turn, then gradients.
struct Draw { long long row; bool gradient; };
__device__ __forceinline__ Draw draw_of(const PrefParams& P, long long n) {
  if (!P.G || n < P.lag) return {n, false};
  const long long u = n - P.lag, both = 2 * (P.rows - P.lag);
  if (u >= both) return {P.rows - P.lag + (u - both), true};
  return u & 1 ? Draw{P.lag + (u >> 1), false} : Draw{u >> 1, true};
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads, kRowBlocks)
preference_kernel(const PrefParams P) {
  __shared__ float sc[kRowThreads / 32], ss[kRowThreads / 32];
  __shared__ double part[2][kRowThreads / 32];
  __shared__ uint32_t next;
  __shared__ int last;
  __shared__ float factor;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long draws = P.G ? 2 * P.rows : P.rows;
  const int rows_of_pair = 2 * P.T;
  long long n = blockIdx.x;                            // the first draws are the CTAs' own, the counter goes on behind them
  while (n < draws) {
    // the row after this one is drawn now: it comes later in the order than all that this one waits for
    if (tid == 0) next = gridDim.x + atomicAdd(P.ticket, 1u);
    const Draw d = draw_of(P, n);
    const int pair = int(d.row / rows_of_pair), target = row_target(P, d.row, tid == 0 && !d.gradient);
    const T* x = static_cast<const T*>(P.logits) + d.row * P.ldl;
    if (!d.gradient) {
      Softmax a{-INFINITY, 0.f};
      if (target >= 0) {
        a = warp_join(scan_row(x, P.V, tid, kRowThreads));
        if (lane == 0) { sc[warp] = a.c; ss[warp] = a.s; }
      }
      __syncthreads();
      if (tid == 0) {
        if (target >= 0) {
          a = Softmax{sc[0], ss[0]};
          for (int w = 1; w < kRowThreads / 32; ++w) a.join(sc[w], ss[w]);
        }
        P.row_logp[d.row] = target < 0 ? 0.f : token_logp(to_f32(x[target]), a);
        P.row_c[d.row] = a.c;
        P.row_inv[d.row] = target < 0 ? 0.f : 1.f / a.s;
        __threadfence();                               // the row's values before the count
        last = atomicAdd(P.done + pair, 1u) == uint32_t(rows_of_pair - 1);
      }
      __syncthreads();
      if (last) {                                      // every row of the pair is there: its sums, in a fixed order
        __threadfence();
        const float* l = P.row_logp + (long long)pair * rows_of_pair;
        double s[2] = {0.0, 0.0};
        for (int t = tid; t < P.T; t += kRowThreads) { s[0] += double(__ldcg(l + t)); s[1] += double(__ldcg(l + P.T + t)); }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          s[q] = warp_sum(s[q]);
          if (lane == 0) part[q][warp] = s[q];
        }
        __syncthreads();
        if (tid == 0) {
          s[0] = s[1] = 0.0;
          for (int w = 0; w < kRowThreads / 32; ++w) { s[0] += part[0][w]; s[1] += part[1][w]; }
          const float c = pair_loss(P, pair, s[0], s[1], true);
          P.coef[2 * pair] = c;
          P.coef[2 * pair + 1] = -c;
          __threadfence();
          atomicExch(P.ready + pair, 1u);
        }
      }
    } else {
      if (tid == 0) {
        // rows that this one waits for were drawn before it, by CTAs that wait for nothing
        const long long t0 = clock64();
        bool ok = true;
        while (*reinterpret_cast<volatile uint32_t*>(P.ready + pair) == 0u) {
          if (clock64() - t0 > P.wait_limit) { ok = false; break; }
          __nanosleep(100);
        }
        if (!ok && P.dev_status) atomicOr(P.dev_status, DP_DEV_TIMEOUT);
        __threadfence();
        factor = __ldcg(P.coef + d.row / P.T);
      }
      __syncthreads();
      write_gradient(x, static_cast<T*>(P.G) + d.row * P.ldg, P.V, target, factor, __ldcg(P.row_c + d.row), __ldcg(P.row_inv + d.row), tid,
                     kRowThreads);
    }
    __syncthreads();
    n = next;
    __syncthreads();
  }
}

// Bytes of logits up to which a call takes the cluster form.
constexpr long long kSmallCall = 24LL << 20;

template <typename T>
dp_status pref_launch(PrefParams& P, cudaStream_t st) {
  const int ctas = std::min(8, 2 * P.T);
  if (2 * P.T <= kPairRows * ctas && P.rows * P.V * (long long)sizeof(T) <= kSmallCall) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(P.B) * unsigned(ctas));
    cfg.blockDim = dim3(kPairThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {unsigned(ctas), 1u, 1u};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    DP_CUDA_OK(cudaLaunchKernelEx(&cfg, pair_kernel<T>, P));
    ++g_kernel_launches;
    return DP_OK;
  }
  const long long blocks = std::min(P.rows, (long long)kRowBlocks * sm_count());
  // far enough behind that a pair's rows are done when its first gradient is drawn, no further: the L2 holds what lies between
  P.lag = std::min(P.rows, 2LL * P.T + blocks);
  DP_CUDA_OK(cudaMemsetAsync(P.ticket, 0, (1 + 2 * size_t(P.B)) * sizeof(uint32_t), st));
  preference_kernel<T><<<unsigned(blocks), kRowThreads, 0, st>>>(P);
  DP_LAUNCH_OK();
  return DP_OK;
}

}  // namespace

}  // namespace dpg

using namespace dpg;

extern "C" {

size_t dp_preference_loss_ws_bytes(int32_t B, int32_t T) {
  if (B <= 0 || T <= 0) return 0;
  return align_up((3 * 2 * size_t(B) * size_t(T) + 2 * size_t(B) + 1 + 2 * size_t(B)) * sizeof(float), 256);
}

dp_status dp_preference_loss(const void* logits, int64_t ldl, dp_dtype dt, int32_t B, int32_t T, int32_t V, const int32_t* targets,
                             const float* ref_logp, float beta, float smoothing, float scale, float* loss, float* logp, void* G,
                             int64_t ldg, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) {
  if (!logits || !targets || B <= 0 || T <= 0 || V <= 0 || ldl < V || (G && ldg < V)) return DP_ERR_INVALID_ARG;
  if (!loss && !logp && !G) return DP_ERR_INVALID_ARG;
  if (dt != DP_F32 && dt != DP_BF16) return DP_ERR_INVALID_ARG;
  if (!std::isfinite(beta) || beta < 0.f || !(smoothing >= 0.f && smoothing <= 1.f) || !std::isfinite(scale)) return DP_ERR_INVALID_ARG;
  if (G == logits && ldg != ldl) return DP_ERR_INVALID_ARG;
  if (2LL * B * T > (1LL << 30)) return DP_ERR_UNSUPPORTED;         // draws are counted in 32 bits
  const size_t es = dt == DP_F32 ? 4 : 2;
  if (!on_boundary(es, logits, G) || !on_boundary(4, targets, ref_logp, loss, logp)) return DP_ERR_ALIGNMENT;
  if (!ws || ws_bytes < dp_preference_loss_ws_bytes(B, T)) return DP_ERR_WORKSPACE;
  if (!on_boundary(4, ws)) return DP_ERR_ALIGNMENT;
  const size_t rows = 2 * size_t(B) * size_t(T);
  float* f = static_cast<float*>(ws);
  uint32_t* u = reinterpret_cast<uint32_t*>(f + 3 * rows + 2 * size_t(B));
  PrefParams P{logits, ldl, G, ldg, targets, ref_logp, loss, logp, f, f + rows, f + 2 * rows, f + 3 * rows, u, u + 1, u + 1 + B, dev_status,
               B, T, V, (long long)rows, 0, beta, smoothing, scale, g_wait_limit};
  const cudaStream_t st = (cudaStream_t)stream;
  return dt == DP_F32 ? pref_launch<float>(P, st) : pref_launch<__nv_bfloat16>(P, st);
}

}  // extern "C"
