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
// Two launches: statistics of every row, then gradients, whose launch overlaps the first one's end and whose rows go from the last to the
// first, so that the rows read last are still in the L2.  A CTA of the second adds up its pair itself, in a fixed order: 2T numbers
// against a row of logits, and no counters, no third launch.  Both are bound by memory and, in the first, by the rate of ex2 (16 a
// clock and SM: 46 us of the 76 for 206 M logits).  Measured with logits and G of (16, 2 x 128, 50257) in bf16 (412 MB each): statistics
// 76 us, both 198; a copy's time for two reads and a write is 190, for one read 127.  Persistent CTAs that draw statistics of later pairs in
// turn with gradients of earlier ones, to find every second reading in the L2, took 195 to 221 (reads and writes share the
// machine worse, and the waits between rows show); clusters of eight CTAs per pair 41 us against 18 at (2, 2 x 16, 50257).
//
// Exponents are x log2 e - c and a row's sum is fp32; a token's log-probability is ((x_target log2 e - c) - log2(sum)) ln 2,
// without the cancellation of x - (c ln 2 + log(sum)), and held in 64 bits as its sequence's sum is, since h is a small difference
// of long sums.
#include <cmath>

#include "dp_common.cuh"

namespace dpg {

namespace {

constexpr double kLog2e64 = 1.4426950408889634;
constexpr float kLog2e = float(kLog2e64), kLog2eLow = float(kLog2e64 - double(kLog2e));
// What kLog2e leaves out of x log2 e.  For logits past 2^20 that of 2^20: it only has to be alike in a row, whose logits there are 2^-3 apart at least,
// and must not outgrow the exponents.
__device__ __forceinline__ float exponent_rest(float x) { return fminf(fmaxf(x, -1048576.f), 1048576.f) * kLog2eLow; }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^d of a whole number up to 127; 0 below 2^-126, and of NaN
__device__ __forceinline__ float exp2_whole(float d) { return d >= -126.f ? __int_as_float((int(d) + 127) << 23) : 0.f; }

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
  // 2^(x log2 e + minus)
  static constexpr bool kRest = false;
  static __device__ __forceinline__ float power(float x, float minus) { return exp2_fast(fmaf(x, kLog2e, minus)); }
  // largest of U pieces (NaN apart), two values at a time
  template <int U>
  static __device__ __forceinline__ float top(const uint4 (&q)[U]) {
    __nv_bfloat162 m = two(q[0].x);
#pragma unroll
    for (int u = 0; u < U; ++u) m = __hmax2(m, __hmax2(__hmax2(two(q[u].x), two(q[u].y)), __hmax2(two(q[u].z), two(q[u].w))));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ __nv_bfloat162 two(uint32_t w) {
    __nv_bfloat162 h;
    memcpy(&h, &w, 4);
    return h;
  }
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
  static constexpr bool kRest = true;                    // log2 e in two terms
  static __device__ __forceinline__ float power(float x, float minus) {
    constexpr float kMagic = 12582912.f;                 // 1.5 * 2^23: what is added to it is rounded to a whole number, in its low bits
    const float r = fmaf(x, kLog2e, minus), u = fmaxf(r, -126.f) + kMagic;
    return exp2_fast(r - (u - kMagic) + exponent_rest(x)) * __int_as_float((__float_as_int(u) << 23) + 0x3f800000);
  }
  template <int U>
  static __device__ __forceinline__ float top(const uint4 (&q)[U]) {
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[4];
      unpack(q[u], v);
      m = fmaxf(m, fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
    }
    return m;
  }
};

// Sum of 2^(x log2 e - c) over the values seen so far; c a whole number near their maximum * log2 e, -inf of none.  The reference moves
// only when a value exceeds it by 2: nearly every warp would meet a new maximum in every piece of a row otherwise.  An exponent is
// one FMA, whose rounding is a term's error: 2^-24 of the exponent, which is at most 2 for the largest terms (a bound of 16 took the
// same time and gave fp32 gradients twice the error).  Whole references change by factors that are exact: ex2 is 5e-8 low on average where its
// argument is negative, and a row's sum meets eight to ten joins of lanes and warps (2.6e-7 in all, the same way for every token).
// fp32 logits give ex2 the part of the exponent between -0.5 and 0.5, where it is 8e-9 low, and log2 e in two terms; bf16 ones, whose own
// rounding is 4e-3, take ex2 and one term, the same in the sum and at the target (the softmax of logits 1.3e-8 smaller); so do gradients, which
// are not added up.  Error of a token's log-probability, 50257 words, on average and around it: fp32 2e-9 and 4.5e-8, bf16 1.4e-8 and
// 4.9e-8; with references that are no whole numbers and fp32 logits treated like bf16 ones 2.0e-7 and 5.1e-8, which 300 tokens add up to 1e-6 of a
// gradient (6e-8 now).  That costs the fp32 call 3 to 5 %: (8, 2 x 128, 50257) 210 us -> 217, statistics alone 87 -> 91; bf16 ones nothing that shows.
struct Softmax {
  float c, s;
  __device__ __forceinline__ float minus() const { return c == -INFINITY ? 0.f : -c; }
  __device__ __forceinline__ void reach(float top) {     // the largest of the next values, in units of c
    if (top > c + 2.f) {
      top = ceilf(top);
      s *= exp2_whole(c - top);
      c = top;
    }
  }
  template <typename T>
  __device__ __forceinline__ void add(float x) {
    reach(x * kLog2e);
    s += Quad<T>::power(x, minus());
  }
  // pieces of 16 bytes
  template <typename T, int U>
  __device__ __forceinline__ void add(const uint4 (&q)[U]) {
    constexpr int N = Quad<T>::N;
    reach(Quad<T>::template top<U>(q) * kLog2e);
    const float m = minus();
    float t[N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[N];
      Quad<T>::unpack(q[u], v);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float p = Quad<T>::power(v[e], m);
        t[e] = u ? t[e] + p : p;
      }
    }
#pragma unroll
    for (int w = N / 2; w > 0; w /= 2)
#pragma unroll
      for (int e = 0; e < w; ++e) t[e] += t[e + w];
    s += t[0];
  }
  __device__ __forceinline__ void join(float oc, float os) {
    const float top = fmaxf(c, oc);
    if (top == -INFINITY) { s += os; return; }       // nothing in either (or only NaN, which the sums carry)
    s = s * exp2_whole(c - top) + os * exp2_whole(oc - top);
    c = top;
  }
};

struct PrefParams {
  const void* logits; long long ldl;
  void* G; long long ldg;
  const int32_t* targets;
  const float* ref;
  float* loss; float* logp;
  double* row_logp; float* row_c; float* row_inv;      // [2BT] workspace
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

// elements up to the next 16-byte boundary
template <typename T>
__device__ __forceinline__ int head_of(const T* x, int V) {
  return min(V, int(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
}

constexpr float kMostReference = 1073741824.f;

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
    acc.add<T>(q);
  }
  for (; k < quads; k += n) {
    const uint4 q[1] = {xq[k]};
    acc.add<T>(q);
  }
  for (int c = tid; c < head; c += n) acc.add<T>(to_f32(x[c]));
  for (int c = head + quads * N + tid; c < V; c += n) acc.add<T>(to_f32(x[c]));
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

// in 64 bits: thousands of these are added up, and the difference of two such sums is what the loss is of
template <typename T>
__device__ __forceinline__ double token_logp(float x, const Softmax& a) {
  const double c = a.c == -INFINITY ? 0.0 : double(a.c);
  return (fma(double(x), double(kLog2e), -c) + (Quad<T>::kRest ? double(exponent_rest(x)) : 0.0) - log2(double(a.s))) * 0.6931471805599453;
}

// 16 bytes from byte `off` of a and b, a multiple of two
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, uint32_t off) {
  uint32_t w[5];
  switch (off >> 2) {
    case 0: w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; break;
    case 1: w[0] = a.y; w[1] = a.z; w[2] = a.w; w[3] = b.x; w[4] = b.y; break;
    case 2: w[0] = a.z; w[1] = a.w; w[2] = b.x; w[3] = b.y; w[4] = b.z; break;
    default: w[0] = a.w; w[1] = b.x; w[2] = b.y; w[3] = b.z; w[4] = b.w; break;
  }
  const uint32_t bits = (off & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

// This thread's share of a row's gradient: f = c / (sum of exponentials).  target < 0: zeros.
template <typename T>
__device__ __forceinline__ void write_gradient(const T* x, T* g, int V, int target, float c, float row_c, float inv, int tid, int n) {
  constexpr int N = Quad<T>::N, U = 4;
  const float f = c * inv, minus = row_c == -INFINITY ? 0.f : -row_c;
  auto grad = [&](float v, int k) {
    const float e = f * exp2_fast(fmaf(v, kLog2e, minus));
    return k == target ? c - e : -e;
  };
  // quads of g, and the columns around them.  Where x lies otherwise on its 16 bytes (dense logits, a G whose rows are padded), a quad is put
  // together from two of x, both within the row, the first `off` bytes before it.  ((8, 2 x 128, 50257) bf16: 112 us against 103 with the same
  // alignment, and 230 element by element.)
  int head = head_of(g, V);
  const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(x + head) & 15);
  int quads = (V - head) / N;
  if (off && target >= 0) {
    if (head * int(sizeof(T)) < int(off)) head = min(V, head + N);
    quads = max(0, int(((long long)(V - head) * int(sizeof(T)) + int(off)) / 16) - 1);
  }
  const uint4* xq = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(x + head) - off);
  uint4* gq = reinterpret_cast<uint4*>(g + head);
  // x and g may be one tensor: a thread has read what it writes
  auto one = [&](int k, const uint4& q) {
    float v[N];
    Quad<T>::unpack(q, v);
    const int at = head + k * N, hit = target - at;
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
  } else if (off) {
    for (int k = tid; k < quads; k += n) one(k, shifted(xq[k], xq[k + 1], off));
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

// A term of weight 0 is not there: h is infinite where a target's logit is -inf, and its other term 0.
__device__ __forceinline__ double weighted(double w, double v) { return w > 0.0 ? w * v : 0.0; }

// The factor of a pair's preferred rows (the others' is its negative); its loss and log-probabilities if `write`.
__device__ float pair_loss(const PrefParams& P, int pair, double lc, double lr, bool write) {
  const double rc = P.ref ? double(P.ref[2 * pair]) : 0.0, rr = P.ref ? double(P.ref[2 * pair + 1]) : 0.0;
  const double h = double(P.beta) * ((lc - rc) - (lr - rr)), e = double(P.smoothing);
  if (write) {
    if (P.loss) P.loss[pair] = float(weighted(1.0 - e, softplus(-h)) + weighted(e, softplus(h)));
    if (P.logp) { P.logp[2 * pair] = float(lc); P.logp[2 * pair + 1] = float(lr); }
  }
  return float(double(P.scale) * double(P.beta) * (e * logistic(h) - (1.0 - e) * logistic(-h)));
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxVocabulary = 1 << 30;                 // a thread counts columns in 32 bits, up to a block of them behind the row

// A warp per row and kWarps rows per CTA where rows are short and many, else a CTA per row.  Statistics and gradients of 4096 bf16 rows, warps
// against CTAs: 14 us against 43 with 1024 logits each, 18 against 45 with 2048, 25 against 49 with 4096, 37 against 57 with 8192; of 128 rows,
// which leave most SMs without a warp of the first form: 12 against 10 with 2048, 25 against 12 with 8192.
inline bool row_by_warp(long long rows, int V) { return V <= 8192 && rows * 512 > (long long)V * sm_count(); }

// This CTA's place: a block of rows of one pair, a warp or all of it on a row (known at compile time: so are the strides of the loops).
template <bool kByWarp>
struct Place {
  static constexpr int kRows = kByWarp ? kWarps : 1, kLanes = kByWarp ? 32 : kThreads;
  int pair, first;                         // the block's first row within the pair
  int at, who;                             // this thread's row within the pair (2T or above: none) and its number on it
  __device__ __forceinline__ Place(const PrefParams& P, unsigned block) {
    const unsigned blocks = (2u * unsigned(P.T) + kRows - 1) / kRows;
    pair = int(block / blocks);
    first = int(block % blocks) * kRows;
    at = first + (kByWarp ? int(threadIdx.x >> 5) : 0);
    who = kByWarp ? int(threadIdx.x & 31) : int(threadIdx.x);
  }
};

template <typename T, bool kByWarp>
__global__ void __launch_bounds__(kThreads, 2048 / kThreads)
row_stats_kernel(const PrefParams P) {
  __shared__ float sc[kWarps], ss[kWarps];
  cudaTriggerProgrammaticLaunchCompletion();             // the next kernel waits for this one's end itself
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Place<kByWarp> p(P, blockIdx.x);
  const bool here = p.at < 2 * P.T;
  const long long row = 2LL * P.T * p.pair + p.at;
  const int target = here ? row_target(P, row, p.who == 0) : -1;
  const T* x = static_cast<const T*>(P.logits) + row * P.ldl;
  Softmax a{-INFINITY, 0.f};
  if (target >= 0) a = warp_join(scan_row(x, P.V, p.who, p.kLanes));
  if (!kByWarp) {
    if (lane == 0) { sc[warp] = a.c; ss[warp] = a.s; }
    __syncthreads();
    if (warp == 0) a = warp_join(lane < kWarps ? Softmax{sc[lane], ss[lane]} : Softmax{-INFINITY, 0.f});
  }
  if (here && p.who == 0) {
    // past 2^30 a reference's rounding outgrows the exponents that fp32 holds; no finite logit at all, or none but the lowest
    if (!(fabsf(a.c) < kMostReference)) a.s = NAN;
    P.row_logp[row] = target < 0 ? 0.0 : token_logp<T>(to_f32(x[target]), a);
    P.row_c[row] = a.c;
    // the gradient's exponents leave the rest out: here it is that of the reference
    P.row_inv[row] = target < 0 ? 0.f : (Quad<T>::kRest ? exp2f(exponent_rest(a.c / kLog2e)) : 1.f) / a.s;
  }
}

// A pair's sequences added up, in a fixed order and by every CTA that needs them: its preferred rows' factor.
__device__ __forceinline__ float factor_of(const PrefParams& P, int pair, bool write) {
  __shared__ double part[2][kWarps];
  __shared__ float factor;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const double* l = P.row_logp + 2LL * P.T * pair;
  double s[2] = {0.0, 0.0};
  for (int t = tid; t < P.T; t += kThreads) { s[0] += l[t]; s[1] += l[P.T + t]; }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    s[q] = warp_sum(s[q]);
    if (lane == 0) part[q][warp] = s[q];
  }
  __syncthreads();
  if (tid == 0) {
    s[0] = s[1] = 0.0;
    for (int w = 0; w < kWarps; ++w) { s[0] += part[0][w]; s[1] += part[1][w]; }
    factor = pair_loss(P, pair, s[0], s[1], write);
  }
  __syncthreads();
  return factor;
}

template <typename T, bool kByWarp>
__global__ void __launch_bounds__(kThreads, 2048 / kThreads)
row_gradient_kernel(const PrefParams P) {
  const Place<kByWarp> p(P, gridDim.x - 1 - blockIdx.x);
  cudaGridDependencySynchronize();
  const float c = factor_of(P, p.pair, p.first == 0);
  if (p.at >= 2 * P.T) return;
  const long long row = 2LL * P.T * p.pair + p.at;
  write_gradient(static_cast<const T*>(P.logits) + row * P.ldl, static_cast<T*>(P.G) + row * P.ldg, P.V, row_target(P, row, false),
                 p.at < P.T ? c : -c, P.row_c[row], P.row_inv[row], p.who, p.kLanes);
}

__global__ void __launch_bounds__(kThreads) pair_loss_kernel(const PrefParams P) {
  cudaGridDependencySynchronize();
  factor_of(P, blockIdx.x, true);
}

template <typename T, bool kByWarp>
dp_status pref_launch(const PrefParams& P, cudaStream_t st) {
  constexpr int per = Place<kByWarp>::kRows;
  const unsigned blocks = unsigned(P.B) * ((2u * unsigned(P.T) + per - 1) / per);
  row_stats_kernel<T, kByWarp><<<blocks, kThreads, 0, st>>>(P);
  DP_LAUNCH_OK();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(P.G ? blocks : unsigned(P.B));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  DP_CUDA_OK(cudaLaunchKernelEx(&cfg, P.G ? row_gradient_kernel<T, kByWarp> : pair_loss_kernel, P));
  ++g_kernel_launches;
  return DP_OK;
}

}  // namespace

}  // namespace dpg

using namespace dpg;

extern "C" {

size_t dp_preference_loss_ws_bytes(int32_t B, int32_t T) {
  if (B <= 0 || T <= 0) return 0;
  return align_up(2 * size_t(B) * size_t(T) * (sizeof(double) + 2 * sizeof(float)), 256);
}

dp_status dp_preference_loss(const void* logits, int64_t ldl, dp_dtype dt, int32_t B, int32_t T, int32_t V, const int32_t* targets,
                             const float* ref_logp, float beta, float smoothing, float scale, float* loss, float* logp, void* G,
                             int64_t ldg, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) {
  if (!logits || !targets || B <= 0 || T <= 0 || V <= 0 || ldl < V || (G && ldg < V)) return DP_ERR_INVALID_ARG;
  if (!loss && !logp && !G) return DP_ERR_INVALID_ARG;
  if (dt != DP_F32 && dt != DP_BF16) return DP_ERR_INVALID_ARG;
  if (!std::isfinite(beta) || beta < 0.f || !(smoothing >= 0.f && smoothing <= 1.f) || !std::isfinite(scale)) return DP_ERR_INVALID_ARG;
  if (G == logits && ldg != ldl) return DP_ERR_INVALID_ARG;
  if (2LL * B * T > 0x7fffffffLL || V > kMaxVocabulary) return DP_ERR_UNSUPPORTED;
  const size_t es = dt == DP_F32 ? 4 : 2;
  if (!on_boundary(es, logits, G) || !on_boundary(4, targets, ref_logp, loss, logp)) return DP_ERR_ALIGNMENT;
  if (!ws || ws_bytes < dp_preference_loss_ws_bytes(B, T)) return DP_ERR_WORKSPACE;
  if (!on_boundary(8, ws)) return DP_ERR_ALIGNMENT;
  const long long rows = 2LL * B * T;
  double* l = static_cast<double*>(ws);
  float* f = reinterpret_cast<float*>(l + rows);
  PrefParams P{logits, ldl, G, ldg, targets, ref_logp, loss, logp, l, f, f + rows, dev_status,
               B, T, V, beta, smoothing, scale};
  const cudaStream_t st = (cudaStream_t)stream;
  if (row_by_warp(rows, V)) return dt == DP_F32 ? pref_launch<float, true>(P, st) : pref_launch<__nv_bfloat16, true>(P, st);
  return dt == DP_F32 ? pref_launch<float, false>(P, st) : pref_launch<__nv_bfloat16, false>(P, st);
}

}  // extern "C"
