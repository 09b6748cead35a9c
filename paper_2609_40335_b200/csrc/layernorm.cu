// Layer norm, forward and backward.
//
//   forward    h = (x - mean(x)) * rstd,  rstd = 1 / sqrt(var(x) + eps),  y = h * gain + shift
//   backward   u = g * gain,  dx = rstd * (u - mean(u) - h * mean(u * h))
//              per example i:  gain_sums_i = sum_t g_t * h_t,  shift_sums_i = sum_t g_t   (the two v_i of
//              vector_kernels.cu, one pass over g and x together with dx),  sq[i] += |gain_sums_i|^2 + |shift_sums_i|^2
//
// Statistics, sums and everything in between are fp32; y, h and dx are rounded once.
//
// Forward: a row belongs to a group of W warps with up to four chunks of eight columns per thread, which stay in registers (as stored:
// a bf16 row is widened where it is used), so the variance is a second pass over registers, not over memory, and is taken about
// the mean.  A warp alone (W = 1) does up to 1024 columns.
//
// Backward: a row's two means run along the row, the parameters' sums across rows.  Rows come to shared memory in tiles (bulk copies, two
// or more tiles in flight); a warp takes a row's means, then each thread takes the same 16 bytes of columns of every row, writes
// dx and keeps its columns' sums in registers.  (With a row's columns spread over a warp's registers, sums and all, GPT-2 medium's norm at
// B = 64, T = 512 took 204 us: 128 registers with spills, too few rows in flight.)
// The rows of an example are shared out over a cluster of CTAs: at the end each CTA adds a slice of the columns over the cluster through
// distributed shared memory, and rank 0 adds up the squares: one launch, no workspace, a fixed order.  Where a cluster's CTAs are too few
// for a long sequence, the partial sums go through the workspace instead (ln_sums_kernel).
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "dp_common.cuh"
#include "ptx_sm100.cuh"

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

// four blocks of 256 threads per SM (64 registers): what hides the latency is rows in flight
template <typename T, int NV, bool kVec, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
ln_forward_kernel(const LnForward P) {
  __shared__ float red[4 * (kThreads / 32)];
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
  int T, p, parts;
  int bulk;                      // rows come by bulk copies: 16-byte boundaries, p % 8 == 0
  int vec_out;                   // dX is written in 16-byte pieces
  int rows, buffers;             // of a tile; tiles in shared memory
};

// Shared memory of a block: buffers of tiles of G and X rows (16-byte pitch), which the sums take over at the end; the gain as
// floats; per row of each buffer its mean and rstd; the warps' parts of the means of a tile's rows; barriers; squares.
struct LnSmem {
  int pitch;                     // bytes of a row
  size_t tile, gain, stats, means, bars, squares, red, bytes;
  __host__ __device__ LnSmem(int p, int es, int rows, int buffers, int warps) {
    pitch = (p * es + 15) / 16 * 16;
    tile = size_t(rows) * 2 * pitch;
    size_t at = tile * buffers;
    if (at < size_t(2) * p * sizeof(float)) at = size_t(2) * p * sizeof(float);
    gain = at = (at + 15) / 16 * 16;
    at += size_t(pitch / es) * sizeof(float);
    stats = at; at += size_t(buffers) * rows * 2 * sizeof(float);
    means = at; at += size_t(rows) * warps * 2 * sizeof(float);
    bars = at = (at + 15) / 16 * 16;
    at += size_t(buffers) * sizeof(uint64_t);
    squares = at; at += 16 * sizeof(float);
    red = at; at += 32 * sizeof(float);
    bytes = at;
  }
};

constexpr int kLnMaxRows = 16, kLnMaxBuffers = 4;

template <typename T> struct Piece;                    // 16 bytes of a row
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Piece<__nv_bfloat16> {
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
    uint4 q;
    __nv_bfloat162 h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
    memcpy(&q, h, 16);
    return q;
  }
};

// NV: pieces of 16 bytes per thread and row
template <typename T, int NV, int kThreads>
__global__ void __launch_bounds__(kThreads)
ln_backward_kernel(const LnBackward P) {
  constexpr int N = Piece<T>::N;
  extern __shared__ __align__(16) uint8_t smem[];
  const int p = P.p, R = P.rows, nb = P.buffers, warps = blockDim.x >> 5;
  const LnSmem at(p, sizeof(T), R, nb, warps);
  float* sums = reinterpret_cast<float*>(smem);
  float* gain = reinterpret_cast<float*>(smem + at.gain);
  float* stats = reinterpret_cast<float*>(smem + at.stats);
  float* means = reinterpret_cast<float*>(smem + at.means);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + at.bars);
  float* squares = reinterpret_cast<float*>(smem + at.squares);
  float* red = reinterpret_cast<float*>(smem + at.red);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int example = blockIdx.x / P.parts, part = blockIdx.x - example * P.parts;
  const int r0 = int((long long)P.T * part / P.parts), r1 = int((long long)P.T * (part + 1) / P.parts);
  const long long base = (long long)example * P.T;
  const int tiles = (r1 - r0 + R - 1) / R, pieces = at.pitch / 16;
  const float inv_p = 1.f / float(p);

  // tile k to its buffer: a bulk copy per row of G and of X, or element by element with zeros behind the row
  auto fill = [&](int k) {
    uint8_t* to = smem + size_t(k % nb) * at.tile;
    const int first = r0 + k * R, n = min(R, r1 - first);
    if (P.bulk) {
      if (warp == 0) {
        uint64_t* bar = full + k % nb;
        const uint32_t bytes = uint32_t(p) * sizeof(T);
        if (lane == 0) ptx::mbar_arrive_expect_tx(bar, 2 * uint32_t(n) * bytes);
        __syncwarp();
        if (lane < n) {
          const long long row = base + first + lane;
          ptx::bulk_load(to + size_t(2 * lane) * at.pitch, static_cast<const T*>(P.G) + row * P.ldg, bytes, bar);
          ptx::bulk_load(to + size_t(2 * lane + 1) * at.pitch, static_cast<const T*>(P.X) + row * P.ldx, bytes, bar);
        }
      }
    } else {
      const int cols = at.pitch / int(sizeof(T));
      for (int r = 0; r < n; ++r) {
        const long long row = base + first + r;
        const T* g = static_cast<const T*>(P.G) + row * P.ldg;
        const T* x = static_cast<const T*>(P.X) + row * P.ldx;
        T* tg = reinterpret_cast<T*>(to + size_t(2 * r) * at.pitch);
        T* tx = reinterpret_cast<T*>(to + size_t(2 * r + 1) * at.pitch);
        for (int c = tid; c < cols; c += blockDim.x) {
          tg[c] = c < p ? g[c] : from_f32<T>(0.f);
          tx[c] = c < p ? x[c] : from_f32<T>(0.f);
        }
      }
    }
    if (tid < 2 * n)
      stats[(k % nb) * 2 * R + tid] = (tid & 1 ? P.rstd : P.mean)[base + first + (tid >> 1)];
  };

  if (tid == 0 && P.bulk) {
    for (int k = 0; k < nb; ++k) ptx::mbar_init(full + k, 1);
    ptx::fence_mbar_init();
  }
  for (int c = tid; c < pieces * N; c += blockDim.x)
    gain[c] = !P.gain ? 1.f : c >= p ? 0.f : P.param_dt == DP_F32 ? static_cast<const float*>(P.gain)[c]
                                                                 : __bfloat162float(static_cast<const __nv_bfloat16*>(P.gain)[c]);
  __syncthreads();
  for (int k = 0; k < min(nb, tiles); ++k) fill(k);

  // this thread's rows of a tile and its pieces of a row
  const int groups = NV == 1 ? max(1, int(blockDim.x) / pieces) : 1;
  const int group = NV == 1 ? tid / pieces : 0;
  const int piece0 = NV == 1 ? tid - group * pieces : tid;
  float gs[NV][N], ss[NV][N], a[NV][N];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int piece = piece0 + j * blockDim.x;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      gs[j][e] = ss[j][e] = 0.f;
      a[j][e] = piece < pieces ? gain[piece * N + e] : 0.f;
    }
  }
  // warps per row for the means, and how many rows they take at once
  const int per_row = max(1, warps / R), at_once = warps / per_row;

  for (int k = 0; k < tiles; ++k) {
    const uint8_t* tile = smem + size_t(k % nb) * at.tile;
    const float* st = stats + (k % nb) * 2 * R;
    const int first = r0 + k * R, n = min(R, r1 - first);
    if (!P.bulk) __syncthreads();                      // filled by every thread (and the statistics with it)
    else {
      if (k < nb || nb == 1) __syncthreads();          // the statistics; with more buffers later tiles' are a sync older
      const long long t0 = clock64();
      while (!ptx::mbar_try_wait(full + k % nb, (k / nb) & 1))
        if (clock64() - t0 > ptx::kDefaultWaitLimit) break;      // copies of this block's own: they end
    }
    if (P.dX) {
      for (int r = warp / per_row; r < n && warp < per_row * at_once; r += at_once) {
        const uint4* g = reinterpret_cast<const uint4*>(tile + size_t(2 * r) * at.pitch);
        const uint4* x = reinterpret_cast<const uint4*>(tile + size_t(2 * r + 1) * at.pitch);
        const float mean = st[2 * r], rstd = st[2 * r + 1];
        float s1 = 0.f, s2 = 0.f;
        for (int c = (warp % per_row) * 32 + lane; c < pieces; c += per_row * 32) {
          float gv[N], h[N];
          Piece<T>::unpack(g[c], gv);
          Piece<T>::unpack(x[c], h);
          const float4* w = reinterpret_cast<const float4*>(gain + c * N);
#pragma unroll
          for (int q = 0; q < N / 4; ++q) {
            const float4 b = w[q];
            const float bb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float u = gv[4 * q + e] * bb[e];   // 0 behind the row
              s1 += u;
              s2 = fmaf(u, (h[4 * q + e] - mean) * rstd, s2);
            }
          }
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (lane == 0) {
          means[(r * warps + warp % per_row) * 2] = s1;
          means[(r * warps + warp % per_row) * 2 + 1] = s2;
        }
      }
      __syncthreads();
    }
    if (group < groups) {
      for (int r = group; r < n; r += groups) {
        const uint4* g = reinterpret_cast<const uint4*>(tile + size_t(2 * r) * at.pitch);
        const uint4* x = reinterpret_cast<const uint4*>(tile + size_t(2 * r + 1) * at.pitch);
        const float mean = st[2 * r], rstd = st[2 * r + 1];
        float m1 = 0.f, m2 = 0.f;
        if (P.dX) {
          for (int w = 0; w < per_row; ++w) { m1 += means[(r * warps + w) * 2]; m2 += means[(r * warps + w) * 2 + 1]; }
          m1 *= inv_p;
          m2 *= inv_p;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int piece = piece0 + j * blockDim.x;
          if (NV > 1 && piece >= pieces) break;
          float gv[N], h[N], d[N];
          Piece<T>::unpack(g[piece], gv);
          Piece<T>::unpack(x[piece], h);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            h[e] = (h[e] - mean) * rstd;
            gs[j][e] = fmaf(gv[e], h[e], gs[j][e]);
            ss[j][e] += gv[e];
            d[e] = (fmaf(gv[e], a[j][e], -m1) - h[e] * m2) * rstd;
          }
          if (P.dX) {
            T* out = static_cast<T*>(P.dX) + (base + first + r) * P.lddx + piece * N;
            if (P.vec_out) *reinterpret_cast<uint4*>(out) = Piece<T>::pack(d);
            else {
#pragma unroll
              for (int e = 0; e < N; ++e) if (piece * N + e < p) out[e] = from_f32<T>(d[e]);
            }
          }
        }
      }
    }
    __syncthreads();                                   // the buffer has been read
    if (k + nb < tiles) fill(k + nb);
  }
  if (!P.gain_sums && !P.shift_sums && !P.sq) return;          // the same for every CTA
  // this CTA's sums, its groups one after the other
  if (tiles == 0) {
    for (int c = tid; c < 2 * p; c += blockDim.x) sums[c] = 0.f;
  }
  for (int q = 0; q < groups && tiles; ++q) {
    if (group == q) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int c = (piece0 + j * int(blockDim.x)) * N + e;
          if (c < p) {
            sums[c] = (q ? sums[c] : 0.f) + gs[j][e];
            sums[p + c] = (q ? sums[p + c] : 0.f) + ss[j][e];
          }
        }
    }
    __syncthreads();
  }
  __syncthreads();
  if (P.partials) {
    float* out = P.partials + (long long)blockIdx.x * 2 * p;
    for (int c = tid; c < 2 * p; c += blockDim.x) out[c] = sums[c];
    return;
  }
  cg::cluster_group cluster = cg::this_cluster();
  if (P.parts > 1) cluster.sync();
  const int c0 = int((long long)p * part / P.parts), c1 = int((long long)p * (part + 1) / P.parts);
  float sq = 0.f;
  for (int c = c0 + tid; c < c1; c += blockDim.x) {
    float u = 0.f, v = 0.f;
    if (P.parts > 1) {
      for (int q = 0; q < P.parts; ++q) {
        const float* other = cluster.map_shared_rank(sums, q);
        u += other[c];
        v += other[p + c];
      }
    } else {
      u = sums[c];
      v = sums[p + c];
    }
    if (P.gain_sums) P.gain_sums[(long long)example * p + c] = u;
    if (P.shift_sums) P.shift_sums[(long long)example * p + c] = v;
    sq = fmaf(u, u, fmaf(v, v, sq));
  }
  sq = block_sum(sq, red);
  if (tid == 0) *(P.parts > 1 ? cluster.map_shared_rank(squares + part, 0) : squares) = sq;
  if (P.parts > 1) cluster.sync();                             // no CTA leaves while its sums are read
  if (P.sq && part == 0 && tid == 0) {
    float all = 0.f;
    for (int q = 0; q < P.parts; ++q) all += squares[q];
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

// warps per row of the forward pass: as few as leave a thread three chunks (four spill), two where its columns are apart (a
// predicate each)
int ln_warps(int p, bool vec) {
  int W = 1;
  while (W < 16 && W * 32 * (vec ? 3 : 2) * 8 < p) W *= 2;
  return W;
}

bool ln_vec(const void* q, long long ld, int es) { return !q || (aligned16(q) && (ld * es) % 16 == 0); }

constexpr int kLnMaxParts = 16;            // CTAs of a cluster

// Parts an example's rows are cut into, and whether they are a cluster (else the sums go through the workspace): about three
// CTAs per SM, eight rows each at least.
struct LnParts { int parts; bool cluster; };
LnParts ln_parts(int B, int T) {
  const int wanted = std::max(1, 3 * sm_count() / B);
  const int most = ceil_div(T, 8);
  if (wanted > 2 * kLnMaxParts && T >= 1024 * kLnMaxParts) return {std::min(wanted, T / 512), false};
  return {std::max(1, std::min(std::min(wanted, most), kLnMaxParts)), true};
}

template <typename T, int NV, int kThreads>
dp_status ln_back_launch(LnBackward& P, int B, int threads, bool cluster, cudaStream_t st) {
  auto* kernel = ln_backward_kernel<T, NV, kThreads>;
  // rows per tile and tiles: a third of an SM's shared memory where three CTAs share it, all of it for a CTA alone
  const size_t most = (long long)B * P.parts > sm_count() ? 72 * 1024 : 200 * 1024;
  const int pitch = (P.p * int(sizeof(T)) + 15) / 16 * 16;
  P.rows = std::max(1, std::min(kLnMaxRows, int(24 * 1024 / (2 * pitch))));
  P.rows = std::min(P.rows, std::max(1, ceil_div(P.T, P.parts)));
  P.buffers = P.bulk ? kLnMaxBuffers : 1;
  while (P.buffers > 1 && LnSmem(P.p, sizeof(T), P.rows, P.buffers, threads / 32).bytes > most) --P.buffers;
  if (P.buffers == 1 && P.bulk && LnSmem(P.p, sizeof(T), P.rows, 2, threads / 32).bytes <= 225 * 1024) P.buffers = 2;
  const LnSmem smem(P.p, sizeof(T), P.rows, P.buffers, threads / 32);
  if (first_use_on_this_device((const void*)kernel)) {
    DP_CUDA_OK(allow_shared(kernel, 227 * 1024));
    DP_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(B) * unsigned(P.parts));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem.bytes;
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

// Threads: as many whole rows of pieces as fill most of a block, 256 or so; wide rows take 512 threads and several pieces each.
template <typename T>
dp_status ln_back(LnBackward& P, int B, bool cluster, cudaStream_t st) {
  const int pieces = ceil_div(P.p * int(sizeof(T)), 16);
  if (pieces <= 512) {
    int best = 0, used = 0;
    for (int threads = 128; threads <= 512; threads += 32) {
      if (threads < pieces) continue;
      const int score = threads / pieces * pieces * 1024 / threads - std::abs(threads - 256) / 4;
      if (!best || score > used) { best = threads; used = score; }
    }
    return best <= 256 ? ln_back_launch<T, 1, 256>(P, B, best, cluster, st) : ln_back_launch<T, 1, 512>(P, B, best, cluster, st);
  }
  switch (ceil_div(pieces, 512)) {
    case 2: return ln_back_launch<T, 2, 512>(P, B, 512, cluster, st);
    case 3: return ln_back_launch<T, 3, 512>(P, B, 512, cluster, st);
    case 4: return ln_back_launch<T, 4, 512>(P, B, 512, cluster, st);
    default: return ln_back_launch<T, 8, 512>(P, B, 512, cluster, st);
  }
}

template <typename T, int NV, bool kVec>
dp_status ln_fwd_launch(const LnForward& P, cudaStream_t st) {
  const int threads = std::max(kLnThreads, P.W * 32), groups = threads / 32 / P.W;
  const unsigned blocks = unsigned(std::min<long long>((P.rows + groups - 1) / groups, 1 << 20));
  if (threads == 512) ln_forward_kernel<T, NV, kVec, 512><<<blocks, threads, 0, st>>>(P);
  else ln_forward_kernel<T, NV, kVec, 256><<<blocks, threads, 0, st>>>(P);
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
  const LnParts parts = ln_parts(B, T);
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
  const LnParts parts = ln_parts(B, T);
  if ((long long)B * parts.parts > 0x7fffffffLL) return DP_ERR_UNSUPPORTED;
  float* partials = nullptr;
  float* squares = nullptr;
  if (!parts.cluster && sums) {
    if (!ws || ws_bytes < dp_layernorm_backward_ws_bytes(B, T, p)) return DP_ERR_WORKSPACE;
    if (!on_boundary(4, ws)) return DP_ERR_ALIGNMENT;
    partials = static_cast<float*>(ws);
    squares = reinterpret_cast<float*>(static_cast<char*>(ws) + ln_partial_bytes(parts, B, p));
  }
  LnBackward P{};
  P.G = G; P.ldg = ldg; P.X = X; P.ldx = ldx; P.gain = gain; P.param_dt = param_dt; P.mean = mean; P.rstd = rstd; P.dX = dX; P.lddx = lddx;
  P.gain_sums = gain_sums; P.shift_sums = shift_sums; P.sq = sq; P.partials = partials;
  P.T = T; P.p = p; P.parts = parts.parts;
  P.bulk = p % 8 == 0 && ln_vec(G, ldg, es) && ln_vec(X, ldx, es);
  P.vec_out = p % 8 == 0 && ln_vec(dX, lddx, es);
  const cudaStream_t st = (cudaStream_t)stream;
  const dp_status r = dt == DP_F32 ? ln_back<float>(P, B, parts.cluster, st) : ln_back<__nv_bfloat16>(P, B, parts.cluster, st);
  if (r != DP_OK || !partials) return r;
  const int slabs = ceil_div(p, 128);
  ln_sums_kernel<<<dim3(slabs, B), 128, 0, st>>>(partials, parts.parts, p, gain_sums, shift_sums, squares);
  DP_LAUNCH_OK();
  return sq ? launch_reduce_partials(squares, slabs, B, sq, 1.f, nullptr, st) : DP_OK;
}

}  // extern "C"
