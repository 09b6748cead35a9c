// Layer norm, forward and backward.
//
//   forward    h = (x - mean(x)) * rstd,  rstd = 1 / sqrt(var(x) + eps),  y = h * gain + shift
//   backward   u = g * gain,  dx = rstd * (u - mean(u) - h * mean(u * h))
//              per example i:  gain_sums_i = sum_t g_t * h_t,  shift_sums_i = sum_t g_t   (the two v_i of
//              vector_kernels.cu, one pass over g and x together with dx),  sq[i] += |gain_sums_i|^2 + |shift_sums_i|^2
//
// Both read every row once and keep it in registers (as stored: a bf16 row is widened where it is used), so the
// variance is a second pass over registers, not over memory, and is taken about the mean.  A row belongs to a group
// of W warps with up to four chunks of eight columns per thread; a warp alone (W = 1) does up to 1024 columns.
// Statistics, sums and everything in between are fp32; y, h and dx are rounded once.
//
// Backward: the rows of an example are shared out over a cluster of CTAs.  Every CTA adds up its rows' terms in
// registers and then in shared memory; at the end each CTA adds a slice of the columns over the cluster through
// distributed shared memory, and rank 0 adds up the squares: one launch, no workspace, a fixed order.  Where a cluster's
// CTAs are too few for a long sequence, the partial sums go through the workspace instead (ln_sums_kernel).
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "dp_common.cuh"

namespace dpg {

namespace {

namespace cg = cooperative_groups;

constexpr int kLnMaxCols = 16384;          // 16 warps x 32 lanes x 4 chunks x 8 columns
constexpr int kLnThreads = 256;

// Eight columns of a thread's chunk j.  kVec: consecutive ones (16-byte accesses); else a warp's accesses are
// consecutive and the columns of a thread a group's width apart.
template <bool kVec>
__device__ __forceinline__ int ln_col(int j, int e, int tid, int width) {
  return kVec ? (j * width + tid) * 8 + e : (j * 8 + e) * width + tid;
}

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T, bool kVec>
struct LnChunk {
  Raw8<T> raw;
  __device__ __forceinline__ void load(const T* row, int j, int tid, int width, int p) {
    if (kVec) {
      const int c = ln_col<true>(j, 0, tid, width);
      if (c < p) raw.load(row + c, 8, true);             // p is a multiple of 8 here
      else raw.zero();
    } else {
      T v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = ln_col<false>(j, e, tid, width);
        v[e] = c < p ? row[c] : from_f32<T>(0.f);
      }
      raw.load(v, 8, false);
    }
  }
};

template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float (&v)[8]) {
  uint4 q;
  __nv_bfloat162 h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
  memcpy(&q, h, 16);
  *reinterpret_cast<uint4*>(p) = q;
}

template <typename T, bool kVec>
__device__ __forceinline__ void ln_store(T* row, const float (&v)[8], int j, int tid, int width, int p) {
  if (kVec) {
    const int c = ln_col<true>(j, 0, tid, width);
    if (c < p) store8<T>(row + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = ln_col<false>(j, e, tid, width);
      if (c < p) row[c] = from_f32<T>(v[e]);
    }
  }
}

// eight values of a parameter vector, `absent` where there is none
template <bool kVec>
__device__ __forceinline__ void ln_param(const void* q, int dt, float absent, int j, int tid, int width, int p, float (&v)[8]) {
  if (!q) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = absent;
    return;
  }
  if (kVec && ln_col<true>(j, 0, tid, width) < p) {
    const int c = ln_col<true>(j, 0, tid, width);
    if (dt == DP_F32) load8<float>(static_cast<const float*>(q) + c, 8, true, v);
    else load8<__nv_bfloat16>(static_cast<const __nv_bfloat16*>(q) + c, 8, true, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = ln_col<kVec>(j, e, tid, width);
    v[e] = c >= p ? 0.f : dt == DP_F32 ? static_cast<const float*>(q)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(q)[c]);
  }
}

// Sums over the W warps of a row's group.  `red` holds 2 * 2 * W floats of the group: two slots used in turn, so one
// barrier per sum suffices (a slot is written again only after the barrier of the sum between).
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int W, int warp_in_group, int lane, int barrier, float* red, int& turn) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = warp_sum(v[k]);
  if (W == 1) return;
  float* slot = red + turn * 2 * W;
  turn ^= 1;
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) slot[k * W + warp_in_group] = v[k];
  }
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(W * 32) : "memory");
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float s = lane < W ? slot[k * W + lane] : 0.f;
    v[k] = warp_sum(s);
  }
}

struct LnForward {
  const void* X; long long ldx;
  const void* gain; const void* shift; int param_dt;
  void* Y; long long ldy;
  void* H; long long ldh;
  float* mean; float* rstd;
  long long rows;
  int p, W;
  float eps;
};

template <typename T, int NV, bool kVec>
__global__ void __launch_bounds__(512, 1)
ln_forward_kernel(const LnForward P) {
  __shared__ float red[4 * 16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int W = P.W, width = W * 32, group = warp / W, groups = (blockDim.x >> 5) / W;
  const int tid = threadIdx.x - group * width;
  float* my_red = red + group * 4 * W;
  int turn = 0;
  for (long long row = (long long)blockIdx.x * groups + group; row < P.rows; row += (long long)gridDim.x * groups) {
    const T* x = static_cast<const T*>(P.X) + row * P.ldx;
    LnChunk<T, kVec> in[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) in[j].load(x, j, tid, width, P.p);
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[8];
      in[j].raw.unpack(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += v[e];
    }
    group_sum<1>(s, W, warp - group * W, lane, 1 + group, my_red, turn);
    const float mean = s[0] / float(P.p);
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[8];
      in[j].raw.unpack(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = v[e] - mean;
        if (ln_col<kVec>(j, e, tid, width) < P.p) s[0] = fmaf(d, d, s[0]);
      }
    }
    group_sum<1>(s, W, warp - group * W, lane, 1 + group, my_red, turn);
    const float rstd = 1.f / sqrtf(s[0] / float(P.p) + P.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[8];
      in[j].raw.unpack(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (v[e] - mean) * rstd;
      if (P.H) ln_store<T, kVec>(static_cast<T*>(P.H) + row * P.ldh, v, j, tid, width, P.p);
      if (P.Y) {
        float a[8], b[8];
        ln_param<kVec>(P.gain, P.param_dt, 1.f, j, tid, width, P.p, a);
        ln_param<kVec>(P.shift, P.param_dt, 0.f, j, tid, width, P.p, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], a[e], b[e]);
        ln_store<T, kVec>(static_cast<T*>(P.Y) + row * P.ldy, v, j, tid, width, P.p);
      }
    }
    if (tid == 0) {
      if (P.mean) P.mean[row] = mean;
      if (P.rstd) P.rstd[row] = rstd;
    }
  }
}

struct LnBackward {
  const void* G; long long ldg;
  const void* X; long long ldx;
  const void* gain; int param_dt;
  const float* mean; const float* rstd;
  void* dX; long long lddx;
  float* gain_sums; float* shift_sums; float* sq;
  float* partials;               // [B][parts][2][p], or nullptr where the parts are a cluster
  int T, p, W, parts;
};

template <typename T, int NV, bool kVec>
__global__ void __launch_bounds__(512, 1)
ln_backward_kernel(const LnBackward P) {
  extern __shared__ float sums[];              // [2][p], then the groups' reduction slots and 16 squares
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int W = P.W, width = W * 32, group = warp / W, groups = (blockDim.x >> 5) / W;
  const int tid = threadIdx.x - group * width, p = P.p;
  float* red = sums + 2 * p;
  float* squares = red + 4 * (blockDim.x >> 5);
  float* my_red = red + group * 4 * W;
  int turn = 0;
  const int example = blockIdx.x / P.parts, part = blockIdx.x - example * P.parts;
  const int r0 = int((long long)P.T * part / P.parts), r1 = int((long long)P.T * (part + 1) / P.parts);
  const long long base = (long long)example * P.T;
  const float inv_p = 1.f / float(p);
  float gs[NV][8], ss[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) gs[j][e] = ss[j][e] = 0.f;
  for (int r = r0 + group; r < r1; r += groups) {
    const long long row = base + r;
    LnChunk<T, kVec> gin[NV], xin[NV];
    const T* g = static_cast<const T*>(P.G) + row * P.ldg;
    const T* x = static_cast<const T*>(P.X) + row * P.ldx;
#pragma unroll
    for (int j = 0; j < NV; ++j) { gin[j].load(g, j, tid, width, p); xin[j].load(x, j, tid, width, p); }
    const float mean = P.mean[row], rstd = P.rstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float gv[8], h[8], a[8];
      gin[j].raw.unpack(gv);
      xin[j].raw.unpack(h);
      ln_param<kVec>(P.gain, P.param_dt, 1.f, j, tid, width, p, a);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = kVec ? true : ln_col<kVec>(j, e, tid, width) < p;
        h[e] = (h[e] - mean) * rstd;
        const float u = gv[e] * a[e];                     // 0 past the row's end: its g is
        s[0] += u;
        if (in) {
          s[1] = fmaf(u, h[e], s[1]);
          gs[j][e] = fmaf(gv[e], h[e], gs[j][e]);
          ss[j][e] += gv[e];
        }
      }
    }
    if (P.dX) {
      group_sum<2>(s, W, warp - group * W, lane, 1 + group, my_red, turn);
      const float m1 = s[0] * inv_p, m2 = s[1] * inv_p;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float gv[8], h[8], a[8], d[8];
        gin[j].raw.unpack(gv);
        xin[j].raw.unpack(h);
        ln_param<kVec>(P.gain, P.param_dt, 1.f, j, tid, width, p, a);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = (fmaf(gv[e], a[e], -m1) - (h[e] - mean) * rstd * m2) * rstd;
        ln_store<T, kVec>(static_cast<T*>(P.dX) + row * P.lddx, d, j, tid, width, p);
      }
    }
  }
  if (!P.gain_sums && !P.shift_sums && !P.sq) return;          // the same for every CTA
  // this CTA's sums, its groups one after the other
  for (int k = 0; k < groups; ++k) {
    if (group == k) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = ln_col<kVec>(j, e, tid, width);
          if (c < p) {
            sums[c] = (k ? sums[c] : 0.f) + gs[j][e];
            sums[p + c] = (k ? sums[p + c] : 0.f) + ss[j][e];
          }
        }
    }
    __syncthreads();
  }
  if (P.partials) {
    float* out = P.partials + (long long)blockIdx.x * 2 * p;
    for (int c = threadIdx.x; c < 2 * p; c += blockDim.x) out[c] = sums[c];
    return;
  }
  cg::cluster_group cluster = cg::this_cluster();
  if (P.parts > 1) cluster.sync();
  const int c0 = int((long long)p * part / P.parts), c1 = int((long long)p * (part + 1) / P.parts);
  float sq = 0.f;
  for (int c = c0 + threadIdx.x; c < c1; c += blockDim.x) {
    float a = 0.f, b = 0.f;
    if (P.parts > 1) {
      for (int k = 0; k < P.parts; ++k) {
        const float* other = cluster.map_shared_rank(sums, k);
        a += other[c];
        b += other[p + c];
      }
    } else {
      a = sums[c];
      b = sums[p + c];
    }
    if (P.gain_sums) P.gain_sums[(long long)example * p + c] = a;
    if (P.shift_sums) P.shift_sums[(long long)example * p + c] = b;
    sq = fmaf(a, a, fmaf(b, b, sq));
  }
  sq = block_sum(sq, red);
  if (threadIdx.x == 0) *(P.parts > 1 ? cluster.map_shared_rank(squares + part, 0) : squares) = sq;
  if (P.parts > 1) cluster.sync();                             // no CTA leaves while its sums are read
  if (P.sq && part == 0 && threadIdx.x == 0) {
    float all = 0.f;
    for (int k = 0; k < P.parts; ++k) all += squares[k];
    P.sq[example] += all;
  }
}

// The parts' sums through the workspace: a thread per column of an example, parts in order.
__global__ void __launch_bounds__(128)
ln_sums_kernel(const float* partials, int parts, int p, float* gain_sums, float* shift_sums, float* squares) {
  __shared__ float red[32];
  const int example = blockIdx.y, c = blockIdx.x * 128 + threadIdx.x;
  float a = 0.f, b = 0.f;
  if (c < p) {
    const float* in = partials + (long long)example * parts * 2 * p + c;
#pragma unroll 4
    for (int k = 0; k < parts; ++k) {
      a += in[(long long)k * 2 * p];
      b += in[(long long)k * 2 * p + p];
    }
    if (gain_sums) gain_sums[(long long)example * p + c] = a;
    if (shift_sums) shift_sums[(long long)example * p + c] = b;
  }
  const float sq = block_sum(fmaf(a, a, b * b), red);
  if (threadIdx.x == 0) squares[example * gridDim.x + blockIdx.x] = sq;
}

// warps per row: as few as leave a thread four chunks, two where its columns are apart (a predicate each)
int ln_warps(int p, bool vec) {
  int W = 1;
  while (W < 16 && W * 32 * (vec ? 4 : 2) * 8 < p) W *= 2;
  return W;
}

bool ln_vec(const void* q, long long ld, int es) { return !q || (aligned16(q) && (ld * es) % 16 == 0); }

constexpr int kLnMaxParts = 16;            // CTAs of a cluster

// Parts an example's rows are cut into, and whether they are a cluster (else the sums go through the workspace).
struct LnParts { int parts; bool cluster; };
LnParts ln_parts(int B, int T, int p) {
  const int groups = std::max(1, 8 / ln_warps(p, true));
  const int wanted = ceil_div(2 * sm_count(), B);              // two CTAs per SM
  const int most = ceil_div(T, groups);                        // a row per group at least
  int parts = 1;
  while (parts < wanted && parts < most && parts < kLnMaxParts) parts *= 2;
  if (parts == kLnMaxParts && wanted >= 2 * kLnMaxParts && T >= 64 * groups * kLnMaxParts)
    return {std::min(wanted, T / (32 * groups)), false};
  return {parts, true};
}

template <typename T, int NV, bool kVec>
dp_status ln_back_launch(LnBackward& P, int B, bool cluster, cudaStream_t st) {
  auto* kernel = ln_backward_kernel<T, NV, kVec>;
  const int threads = std::max(kLnThreads, P.W * 32);
  const size_t smem = (size_t(2) * P.p + 4 * (threads / 32) + kLnMaxParts) * sizeof(float);
  if (first_use_on_this_device((const void*)kernel)) {
    const size_t most = (size_t(2) * kLnMaxCols + 4 * 16 + kLnMaxParts) * sizeof(float);
    DP_CUDA_OK(allow_shared(kernel, most));
    DP_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(B) * unsigned(P.parts));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {cluster ? unsigned(P.parts) : 1u, 1u, 1u};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  DP_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, P));
  ++g_kernel_launches;
  return DP_OK;
}

template <typename T, bool kVec>
dp_status ln_back_nv(LnBackward& P, int B, bool cluster, cudaStream_t st) {
  switch (ceil_div(P.p, 8 * 32 * P.W)) {
    case 1: return ln_back_launch<T, 1, kVec>(P, B, cluster, st);
    case 2: return ln_back_launch<T, 2, kVec>(P, B, cluster, st);
    case 3: return ln_back_launch<T, 3, kVec>(P, B, cluster, st);
    default: return ln_back_launch<T, 4, kVec>(P, B, cluster, st);
  }
}

template <typename T, int NV, bool kVec>
dp_status ln_fwd_launch(const LnForward& P, cudaStream_t st) {
  const int threads = std::max(kLnThreads, P.W * 32), groups = threads / 32 / P.W;
  const long long blocks = (P.rows + groups - 1) / groups;
  ln_forward_kernel<T, NV, kVec><<<unsigned(std::min<long long>(blocks, 1 << 20)), threads, 0, st>>>(P);
  DP_LAUNCH_OK();
  return DP_OK;
}

template <typename T, bool kVec>
dp_status ln_fwd_nv(const LnForward& P, cudaStream_t st) {
  switch (ceil_div(P.p, 8 * 32 * P.W)) {
    case 1: return ln_fwd_launch<T, 1, kVec>(P, st);
    case 2: return ln_fwd_launch<T, 2, kVec>(P, st);
    case 3: return ln_fwd_launch<T, 3, kVec>(P, st);
    default: return ln_fwd_launch<T, 4, kVec>(P, st);
  }
}

bool known_dtype(int dt) { return dt == DP_F32 || dt == DP_BF16; }

size_t ln_partial_bytes(const LnParts& parts, int B, int p) {
  return align_up(size_t(B) * parts.parts * 2 * p * sizeof(float), 256);
}

}  // namespace

}  // namespace dpg

using namespace dpg;

extern "C" {

dp_status dp_layernorm(const void* X, int64_t ldx, dp_dtype dt, int64_t rows, int32_t p, const void* gain, const void* shift,
                       dp_dtype param_dt, float eps, void* Y, int64_t ldy, void* X_hat, int64_t ldh, float* mean, float* rstd,
                       void* stream) {
  if (!X || rows <= 0 || p <= 0 || ldx < p || (!Y && !X_hat && !mean && !rstd)) return DP_ERR_INVALID_ARG;
  if ((Y && ldy < p) || (X_hat && ldh < p) || !known_dtype(dt) || !known_dtype(param_dt)) return DP_ERR_INVALID_ARG;
  if (!std::isfinite(eps) || eps < 0.f || (Y && Y == X_hat)) return DP_ERR_INVALID_ARG;
  if ((Y == X && ldy != ldx) || (X_hat == X && ldh != ldx)) return DP_ERR_INVALID_ARG;
  if (p > kLnMaxCols || rows > (int64_t(1) << 40)) return DP_ERR_UNSUPPORTED;
  const int es = dt == DP_F32 ? 4 : 2, ps = param_dt == DP_F32 ? 4 : 2;
  if (!on_boundary(es, X, Y, X_hat) || !on_boundary(ps, gain, shift) || !on_boundary(4, mean, rstd)) return DP_ERR_ALIGNMENT;
  const bool vec = p % 8 == 0 && ln_vec(X, ldx, es) && ln_vec(Y, ldy, es) && ln_vec(X_hat, ldh, es) && ln_vec(gain, p, ps) &&
                   ln_vec(shift, p, ps);
  const LnForward P{X, ldx, gain, shift, param_dt, Y, ldy, X_hat, ldh, mean, rstd, rows, p, ln_warps(p, vec), eps};
  const cudaStream_t st = (cudaStream_t)stream;
  if (dt == DP_F32) return vec ? ln_fwd_nv<float, true>(P, st) : ln_fwd_nv<float, false>(P, st);
  return vec ? ln_fwd_nv<__nv_bfloat16, true>(P, st) : ln_fwd_nv<__nv_bfloat16, false>(P, st);
}

size_t dp_layernorm_backward_ws_bytes(int32_t B, int32_t T, int32_t p) {
  if (B <= 0 || T <= 0 || p <= 0 || p > kLnMaxCols) return 0;
  const LnParts parts = ln_parts(B, T, p);
  if (parts.cluster) return 0;
  return ln_partial_bytes(parts, B, p) + align_up(size_t(B) * ceil_div(p, 128) * sizeof(float), 256);
}

dp_status dp_layernorm_backward(const void* G, int64_t ldg, const void* X, int64_t ldx, dp_dtype dt, int32_t B, int32_t T, int32_t p,
                                const void* gain, dp_dtype param_dt, const float* mean, const float* rstd, void* dX, int64_t lddx,
                                float* gain_sums, float* shift_sums, float* sq, void* ws, size_t ws_bytes, void* stream) {
  if (!G || !X || !mean || !rstd || B <= 0 || T <= 0 || p <= 0 || ldg < p || ldx < p) return DP_ERR_INVALID_ARG;
  if ((dX && lddx < p) || !known_dtype(dt) || !known_dtype(param_dt)) return DP_ERR_INVALID_ARG;
  const bool sums = gain_sums || shift_sums || sq;
  if (!dX && !sums) return DP_ERR_INVALID_ARG;
  if ((dX == G && lddx != ldg) || (dX == X && lddx != ldx)) return DP_ERR_INVALID_ARG;
  const int es = dt == DP_F32 ? 4 : 2, ps = param_dt == DP_F32 ? 4 : 2;
  if (!on_boundary(es, G, X, dX) || !on_boundary(ps, gain) || !on_boundary(4, mean, rstd, gain_sums, shift_sums, sq)) return DP_ERR_ALIGNMENT;
  if (p > kLnMaxCols) return DP_ERR_UNSUPPORTED;
  const LnParts parts = ln_parts(B, T, p);
  if ((long long)B * parts.parts > 0x7fffffffLL) return DP_ERR_UNSUPPORTED;
  float* partials = nullptr;
  float* squares = nullptr;
  if (!parts.cluster && sums) {
    if (!ws || ws_bytes < dp_layernorm_backward_ws_bytes(B, T, p)) return DP_ERR_WORKSPACE;
    if (!on_boundary(4, ws)) return DP_ERR_ALIGNMENT;
    partials = static_cast<float*>(ws);
    squares = reinterpret_cast<float*>(static_cast<char*>(ws) + ln_partial_bytes(parts, B, p));
  }
  const bool vec = p % 8 == 0 && ln_vec(G, ldg, es) && ln_vec(X, ldx, es) && ln_vec(dX, lddx, es) &&
                   ln_vec(gain, p, ps);
  LnBackward P{G, ldg, X, ldx, gain, param_dt, mean, rstd, dX, lddx, gain_sums, shift_sums, sq, partials, T, p, ln_warps(p, vec), parts.parts};
  const cudaStream_t st = (cudaStream_t)stream;
  const bool cluster = parts.cluster;
  dp_status r;
  if (dt == DP_F32) r = vec ? ln_back_nv<float, true>(P, B, cluster, st) : ln_back_nv<float, false>(P, B, cluster, st);
  else r = vec ? ln_back_nv<__nv_bfloat16, true>(P, B, cluster, st) : ln_back_nv<__nv_bfloat16, false>(P, B, cluster, st);
  if (r != DP_OK || !partials) return r;
  const int slabs = ceil_div(p, 128);
  ln_sums_kernel<<<dim3(slabs, B), 128, 0, st>>>(partials, parts.parts, p, gain_sums, shift_sums, squares);
  DP_LAUNCH_OK();
  return sq ? launch_reduce_partials(squares, slabs, B, sq, 1.f, nullptr, st) : DP_OK;
}

}  // extern "C"
