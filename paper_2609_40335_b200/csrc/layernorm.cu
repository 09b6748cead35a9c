// Layer norm, forward and backward.
//
//   forward    h = (x - mean(x)) * rstd,  rstd = 1 / sqrt(var(x) + eps),  y = h * gain + shift
//   backward   u = g * gain,  dx = rstd * (u - mean(u) - h * mean(u * h))
//              per example i:  gain_sums_i = sum_t g_t * h_t,  shift_sums_i = sum_t g_t   (the two v_i of
//              vector_kernels.cu, one pass over g and x together with dx),  sq[i] += |gain_sums_i|^2 + |shift_sums_i|^2
//
// Statistics, sums and everything in between are fp32; y, h and dx are rounded once.  The variance is a second pass over registers,
// not over memory, and is taken about the mean.
//
// A row belongs to a group of lanes (part of a warp for narrow rows, up to 16 warps for wide ones), each with 16-byte pieces of it, at most
// 32 columns, as fp32 in registers: one conversion per element and pass.  Rows on 16-byte boundaries come to shared memory by bulk copies
// that a warp of its own issues several tiles ahead, a tile being a row per group; so few warps with many registers are enough.  Other
// rows are loaded element by element, a warp's accesses side by side.  The backward pass keeps the sums for its columns of gain and shift in
// registers too.  (GPT-2 medium's norm at B = 64, T = 512, backward: loads straight into registers, spilling at 128 of them, 204 us; means
// by rows and sums by columns from shared memory, each element converted twice, 66 to 74; in this form 49.)
//
// Backward: the rows of an example are shared out over a cluster of CTAs: at the end each CTA adds a slice of the columns over the cluster
// through distributed shared memory, and rank 0 adds up the squares: one launch, no workspace, a fixed order.  Where too few clusters fit
// the chip at once, the partial sums go through the workspace instead (ln_sums_kernel).
#include <cooperative_groups.h>

#include <algorithm>
#include <array>
#include <cmath>
#include <map>
#include <mutex>
#include <utility>

#include "dp_common.cuh"
#include "ptx_sm100.cuh"

namespace dpg {

namespace {

namespace cg = cooperative_groups;

constexpr int kLnMaxCols = 16384;          // 16 warps x 32 lanes x 32 columns
constexpr int kLnMaxBuffers = 8;           // tiles in flight
constexpr int kLnMaxParts = 16;            // CTAs of a cluster
constexpr int kLnMaxTokens = 1 << 30;      // rows of an example: the backward pass counts them, a tile or two ahead, in 32 bits

// Two columns.  (As fma.rn.f32x2 and the like these took longer: 66 us instead of 59 for the backward pass above.)
struct F2 { float x, y; };
__device__ __forceinline__ F2 f2(float x, float y) { return F2{x, y}; }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { return F2{a.x + b.x, a.y + b.y}; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { return F2{a.x * b.x, a.y * b.y}; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { return F2{fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)}; }
__device__ __forceinline__ float2 floats(F2 v) { return make_float2(v.x, v.y); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// 16 bytes of a row
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void open(const uint4& q, F2 (&v)[2]) {
    v[0] = f2(__uint_as_float(q.x), __uint_as_float(q.y));
    v[1] = f2(__uint_as_float(q.z), __uint_as_float(q.w));
  }
  static __device__ __forceinline__ uint4 close(const F2 (&v)[2]) {
    const float2 a = floats(v[0]), b = floats(v[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
};
template <> struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void open(const uint4& q, F2 (&v)[4]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = f2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 close(const F2 (&v)[4]) {
    uint4 q;
    __nv_bfloat162 h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = floats(v[e]);
      h[e] = __floats2bfloat162_rn(f.x, f.y);
    }
    memcpy(&q, h, 16);
    return q;
  }
};

// How a kernel's threads share out rows.
struct LnShape {
  int lanes, W;              // lanes of a warp that a row has, warps of a row (with all their lanes)
  int columns;               // of a lane, as its kernel is compiled
  int groups;                // rows at a time, which are a tile
  int buffers;               // tiles in shared memory
  int pitch;                 // bytes of a row there
};

// Shared memory of a block: the tiles of `rows` tensors, whose place the groups' sums take at the end; gain and shift as floats; the
// warps' parts of a row's sums; barriers; squares; a reduction's slots.
struct LnSmem {
  size_t tile, gain, shift, parts, bars, squares, red, bytes;
  __host__ __device__ LnSmem(const LnShape& S, int p, int rows, bool sums, int warps) {
    tile = size_t(S.groups) * rows * S.pitch;
    size_t at = tile * size_t(S.buffers);              // no buffers: rows are loaded, not copied
    const size_t most = sums ? size_t(S.groups) * 2 * p * sizeof(float) : 0;
    if (at < most) at = most;
    // all pieces of every lane (see LnRow::place), and unaligned rows' columns
    const int width = S.lanes * S.W, padded = S.columns * width > p ? S.columns * width : (p + 3) / 4 * 4;
    gain = at = (at + 15) / 16 * 16;
    at += size_t(padded) * sizeof(float);
    shift = at; at += sums ? 0 : size_t(padded) * sizeof(float);
    parts = at; at += size_t(warps) * 4 * sizeof(float);
    bars = at = (at + 15) / 16 * 16;
    at += size_t(2) * S.buffers * sizeof(uint64_t);
    squares = at; at += 16 * sizeof(float);
    red = at; at += 32 * sizeof(float);
    bytes = at;
  }
};

// A parameter vector as floats, `absent` where there is none.
__device__ __forceinline__ float ln_param(const void* q, int dt, float absent, int c) {
  return !q ? absent : dt == DP_F32 ? static_cast<const float*>(q)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(q)[c]);
}

// The copying warp's part of a tile: n rows of one tensor, `pitch` bytes apart in shared memory.  Returns the bytes that this lane has to
// announce; go: makes the copies.
template <typename T>
__device__ __forceinline__ uint32_t ln_copy(const T* first, long long ld, int p, int n, uint8_t* to, int pitch, bool whole, uint64_t* bar,
                                            int lane, bool go) {
  uint32_t bytes = 0;
  if (whole) {                                         // rows follow one another: one copy
    if (lane == 0) {
      bytes = uint32_t(n) * uint32_t(pitch);
      if (go) ptx::bulk_load(to, first, bytes, bar);
    }
    return bytes;
  }
  for (int r = lane; r < n; r += 32) {
    if (go) ptx::bulk_load(to + size_t(r) * pitch, first + r * ld, uint32_t(pitch), bar);
    bytes += uint32_t(pitch);
  }
  return bytes;
}

// A lane's pieces of a row.  kAligned: 16 bytes each; else columns 32 apart, so that a warp's accesses are consecutive, their distances
// constants, and whether a column is in the row one comparison with a constant (with columns as far apart as the row has pieces the forward pass
// issued 67 instructions per column).
template <typename T, int NP, bool kAligned>
struct LnRow {
  static constexpr int N = Piece<T>::N, H = N / 2;
  int tid, width, limit;     // limit: pieces of the row; else this lane's columns
  int first;                 // not aligned: this lane's first column; its others are 32 apart, a warp's all within 32 NP N
  __device__ __forceinline__ LnRow(int tid, int width, int p) : tid(tid), width(width), first(tid / 32 * (32 * NP * N) + tid % 32) {
    limit = kAligned ? (p + N - 1) / N : p > first ? (p - first + 31) / 32 : 0;
  }
  __device__ __forceinline__ int piece(int j) const { return tid + j * width; }
  __device__ __forceinline__ int column(int j, int e) const { return kAligned ? piece(j) * N + e : first + (j * N + e) * 32; }
  __device__ __forceinline__ bool has(int j) const { return kAligned ? piece(j) < limit : j * N < limit; }
  __device__ __forceinline__ bool has(int j, int e) const { return kAligned ? piece(j) < limit : j * N + e < limit; }
  // Zeros behind the row, and all zeros where `there` is false.  kAny: any values of the row behind it, for lanes of several pieces,
  // whose row is there or not for the whole warp, where zeros in the vectors take them out (selecting took a sixth of the backward
  // pass's instructions).
  template <bool kAny>
  __device__ __forceinline__ void open(const void* row, bool there, F2 (&v)[NP][H]) const {
    const int most = there ? limit : 0;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      if (kAligned) {
        uint4 q = make_uint4(0u, 0u, 0u, 0u);
        if (kAny && NP > 1) q = static_cast<const uint4*>(row)[has(j) ? piece(j) : tid];
        else if (there && has(j)) q = static_cast<const uint4*>(row)[piece(j)];
        Piece<T>::open(q, v[j]);
      } else {
        const T* x = static_cast<const T*>(row) + first;
#pragma unroll
        for (int e = 0; e < H; ++e) {
          v[j][e] = f2(j * N + 2 * e < most ? to_f32(x[(j * N + 2 * e) * 32]) : 0.f, j * N + 2 * e + 1 < most ? to_f32(x[(j * N + 2 * e + 1) * 32]) : 0.f);
        }
      }
    }
  }
  // Where a vector of floats has column c in shared memory.  kAligned: quads of columns in the order in which a warp's lanes read them,
  // 16 bytes beside 16 bytes (in the columns' own order a lane's eight lie 32 bytes from its neighbour's: four lanes to a bank, which
  // cost the backward pass a third of its time).
  __device__ __forceinline__ int place(int c) const {
    if (!kAligned) return c;
    const int q = c / N, j = q / width, t = q - j * width, e = c - q * N;
    return ((j * (N / 4) + e / 4) * width + t) * 4 + (e & 3);
  }
  __device__ __forceinline__ void vector(const float* v, int j, F2 (&f)[H]) const {
    if (kAligned) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) {
        const float4 w = reinterpret_cast<const float4*>(v)[(j * (N / 4) + q) * width + tid];
        f[2 * q] = f2(w.x, w.y);
        f[2 * q + 1] = f2(w.z, w.w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < H; ++e) {
        f[e] = f2(v[column(j, 2 * e)], v[column(j, 2 * e + 1)]);        // (the vectors go on behind the row)
      }
    }
  }
  __device__ __forceinline__ void store(T* out, bool vec, int j, const F2 (&v)[H]) const {
    if (!has(j)) return;
    if (kAligned && vec) {
      reinterpret_cast<uint4*>(out)[piece(j)] = Piece<T>::close(v);
      return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float2 f = floats(v[e / 2]);
      if (has(j, e)) out[column(j, e)] = from_f32<T>(e & 1 ? f.y : f.x);
    }
  }
};

// Sums over a row's lanes.  Across warps they meet in `slots` (4 W floats of the group): two halves used in turn, so that one barrier per
// sum suffices (a half is written again only behind the barrier of the sum between).
template <int K>
__device__ __forceinline__ void row_sum(float (&v)[K], const LnShape& S, int warp_in_group, int lane, int barrier, float* slots, int& turn) {
  if (S.lanes == 32) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
  } else {
    for (int o = S.lanes >> 1; o > 0; o >>= 1) {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
  }
  if (S.W == 1) return;
  float* half = slots + turn * 2 * S.W;
  turn ^= 1;
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) half[k * S.W + warp_in_group] = v[k];
  }
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(S.W * 32) : "memory");
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = 0.f;
    for (int w = 0; w < S.W; ++w) v[k] += half[k * S.W + w];
  }
}

struct LnForward {
  const void* X; long long ldx;
  const void* gain; const void* shift; int param_dt;
  void* Y; long long ldy;
  void* H; long long ldh;
  float* mean; float* rstd;
  long long rows;
  int p;
  int whole, vec_y, vec_h;       // X's rows follow one another; outputs are written in 16-byte pieces (rows read in such)
  float eps;
  LnShape S;
  int* dev_status;
  long long wait_limit;
};

template <typename T, int NP, bool kAligned, int kThreads, int kBlocks>
__global__ void __launch_bounds__(kThreads, kBlocks)
ln_forward_kernel(const LnForward P) {
  constexpr int N = Piece<T>::N, H = N / 2;
  extern __shared__ __align__(128) uint8_t smem[];
  const LnShape& S = P.S;
  const int p = P.p, warps = (blockDim.x >> 5) - (kAligned ? 1 : 0);       // the last warp copies
  const LnSmem at(S, p, 1, false, warps);
  float* gain = reinterpret_cast<float*>(smem + at.gain);
  float* shift = reinterpret_cast<float*>(smem + at.shift);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + at.bars);
  uint64_t* empty = full + S.buffers;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long r0 = P.rows * blockIdx.x / gridDim.x, r1 = P.rows * (blockIdx.x + 1) / gridDim.x;
  const int tiles = int((r1 - r0 + S.groups - 1) / S.groups);
  const T* X = static_cast<const T*>(P.X);
  if (tid == 0) {
    for (int k = 0; k < S.buffers; ++k) { ptx::mbar_init(full + k, 32); ptx::mbar_init(empty + k, warps); }
    ptx::fence_mbar_init();
  }
  __syncthreads();
  if (kAligned && warp == warps) {
    int b = 0;
    uint32_t phase = 1;                                  // of the use before
    int issued = 0;
    for (; issued < tiles; ++issued) {
      const int k = issued;
      if (k >= S.buffers && !ptx::warp_ok(ptx::mbar_wait_own(empty + b, phase, P.wait_limit))) break;
      const long long first = r0 + (long long)k * S.groups;
      const int n = int(min((long long)S.groups, r1 - first));
      uint8_t* to = smem + size_t(b) * at.tile;
      ptx::mbar_arrive_expect_tx(full + b, ln_copy<T>(X + first * P.ldx, P.ldx, p, n, to, S.pitch, P.whole, full + b, lane, false));
      ln_copy<T>(X + first * P.ldx, P.ldx, p, n, to, S.pitch, P.whole, full + b, lane, true);
      if (++b == S.buffers) { b = 0; phase ^= 1; }
    }
    if (lane == 0) ptx::drain_issued_copies(full, S.buffers, uint32_t(issued));       // before the block ends, also where a wait has run out
    return;
  }
  const int per_row = S.lanes * S.W, group = tid / per_row;
  const LnRow<T, NP, kAligned> R(tid - group * per_row, per_row, p);
  for (int c = tid; c < max(p, per_row * NP * N); c += warps * 32) {
    gain[R.place(c)] = c < p ? ln_param(P.gain, P.param_dt, 1.f, c) : 0.f;
    shift[R.place(c)] = c < p ? ln_param(P.shift, P.param_dt, 0.f, c) : 0.f;
  }
  asm volatile("bar.sync 15, %0;" ::"r"(warps * 32) : "memory");
  float* slots = reinterpret_cast<float*>(smem + at.parts) + (S.W > 1 ? group * 4 * S.W : 0);
  const float inv_p = 1.f / float(p);
  int b = 0, turn = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (int k = 0; k < tiles; ++k) {
    // a warp whose wait has run out goes on without waiting: others meet it at barriers
    if (kAligned && ok && !ptx::mbar_wait_own(full + b, phase, P.wait_limit)) {
      ok = false;
      if (P.dev_status && lane == 0) atomicOr(P.dev_status, DP_DEV_TIMEOUT);
    }
    const long long row = r0 + (long long)k * S.groups + group;
    const bool mine = group < S.groups && row < r1;
    F2 v[NP][H];
    if (kAligned) {
      R.template open<false>(smem + size_t(b) * at.tile + size_t(mine ? group : 0) * S.pitch, mine, v);
      ptx::release_to_copies(empty + b, lane);           // the row is in registers
      if (++b == S.buffers) { b = 0; phase ^= 1; }
    } else {
      R.template open<false>(X + (mine ? row : r0) * P.ldx, mine, v);
    }
    F2 sum = f2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int e = 0; e < H; ++e) sum = add2(sum, v[j][e]);
    float s[1] = {floats(sum).x + floats(sum).y};
    row_sum<1>(s, S, warp % S.W, lane, 1 + group, slots, turn);
    // a true quotient where it is cheap: 1 / p rounded would move the mean by half a rounding more
    const float mean = s[0] / float(p);
    const F2 minus = f2(-mean, -mean);
    sum = f2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int e = 0; e < H; ++e) {
        v[j][e] = add2(v[j][e], minus);
        if (!R.has(j)) v[j][e] = f2(0.f, 0.f);
        else if (!kAligned) {
          const float2 f = floats(v[j][e]);
          v[j][e] = f2(R.has(j, 2 * e) ? f.x : 0.f, R.has(j, 2 * e + 1) ? f.y : 0.f);
        }
        sum = fma2(v[j][e], v[j][e], sum);
      }
    s[0] = floats(sum).x + floats(sum).y;
    row_sum<1>(s, S, warp % S.W, lane, 1 + group, slots, turn);
    const float rstd = 1.f / sqrtf(s[0] * inv_p + P.eps);
    if (!mine) continue;
    const F2 scale = f2(rstd, rstd);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
#pragma unroll
      for (int e = 0; e < H; ++e) v[j][e] = mul2(v[j][e], scale);
      if (P.H) R.store(static_cast<T*>(P.H) + row * P.ldh, P.vec_h, j, v[j]);
      if (P.Y && R.has(j)) {
        F2 a[H], c[H];
        R.vector(gain, j, a);
        R.vector(shift, j, c);
#pragma unroll
        for (int e = 0; e < H; ++e) v[j][e] = fma2(v[j][e], a[e], c[e]);
        R.store(static_cast<T*>(P.Y) + row * P.ldy, P.vec_y, j, v[j]);
      }
    }
    if (R.tid == 0) {
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
  int whole_g, whole_x, vec_out;
  LnShape S;
  int* dev_status;
  long long wait_limit;
};

template <typename T, int NP, bool kAligned, int kThreads, int kBlocks>
__global__ void __launch_bounds__(kThreads, kBlocks)
ln_backward_kernel(const LnBackward P) {
  constexpr int N = Piece<T>::N, H = N / 2;
  extern __shared__ __align__(128) uint8_t smem[];
  const LnShape& S = P.S;
  const int p = P.p, warps = (blockDim.x >> 5) - (kAligned ? 1 : 0);       // the last warp copies
  const LnSmem at(S, p, 2, true, warps);
  float* sums = reinterpret_cast<float*>(smem);
  float* gain = reinterpret_cast<float*>(smem + at.gain);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + at.bars);
  uint64_t* empty = full + S.buffers;
  float* squares = reinterpret_cast<float*>(smem + at.squares);
  float* red = reinterpret_cast<float*>(smem + at.red);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int example = blockIdx.x / P.parts, part = blockIdx.x - example * P.parts;
  const int r0 = int((long long)P.T * part / P.parts), r1 = int((long long)P.T * (part + 1) / P.parts);
  const long long base = (long long)example * P.T;
  const int tiles = (r1 - r0 + S.groups - 1) / S.groups;
  const T* G = static_cast<const T*>(P.G);
  const T* X = static_cast<const T*>(P.X);
  if (tid == 0) {
    for (int k = 0; k < S.buffers; ++k) { ptx::mbar_init(full + k, 32); ptx::mbar_init(empty + k, warps); }
    ptx::fence_mbar_init();
  }
  __syncthreads();
  const int per_row = S.lanes * S.W, group = tid / per_row;
  const LnRow<T, NP, kAligned> R(tid - group * per_row, per_row, p);
  F2 gs[NP][H], ss[NP][H];
#pragma unroll
  for (int j = 0; j < NP; ++j)
#pragma unroll
    for (int e = 0; e < H; ++e) gs[j][e] = ss[j][e] = f2(0.f, 0.f);

  if (kAligned && warp == warps) {
    // ------------------------------------------------------------------ copies
    int b = 0;
    uint32_t phase = 1;                                  // of the use before
    int issued = 0;
    for (; issued < tiles; ++issued) {
      const int k = issued;
      if (k >= S.buffers && !ptx::warp_ok(ptx::mbar_wait_own(empty + b, phase, P.wait_limit))) break;
      const int first = r0 + k * S.groups, n = min(S.groups, r1 - first);
      const T* g = G + (base + first) * P.ldg;
      const T* x = X + (base + first) * P.ldx;
      uint8_t* to = smem + size_t(b) * at.tile;
      uint8_t* to_x = to + size_t(S.groups) * S.pitch;
      ptx::mbar_arrive_expect_tx(full + b, ln_copy<T>(g, P.ldg, p, n, to, S.pitch, P.whole_g, full + b, lane, false) +
                                               ln_copy<T>(x, P.ldx, p, n, to_x, S.pitch, P.whole_x, full + b, lane, false));
      ln_copy<T>(g, P.ldg, p, n, to, S.pitch, P.whole_g, full + b, lane, true);
      ln_copy<T>(x, P.ldx, p, n, to_x, S.pitch, P.whole_x, full + b, lane, true);
      if (++b == S.buffers) { b = 0; phase ^= 1; }
    }
    // copies in flight land before the block ends, also where a wait has run out
    if (lane == 0) ptx::drain_issued_copies(full, S.buffers, uint32_t(issued));
  } else {
    // -------------------------------------------------------------------- work
    for (int c = tid; c < max(p, per_row * NP * N); c += warps * 32)
      gain[R.place(c)] = c < p ? ln_param(P.gain, P.param_dt, 1.f, c) : 0.f;
    asm volatile("bar.sync 15, %0;" ::"r"(warps * 32) : "memory");
    float* slots = reinterpret_cast<float*>(smem + at.parts) + (S.W > 1 ? group * 4 * S.W : 0);
    const float inv_p = 1.f / float(p);
    int b = 0, turn = 0;
    uint32_t phase = 0;
    bool ok = true;
    T* out = static_cast<T*>(P.dX) + (base + r0 + group) * P.lddx;
    const long long out_step = S.groups * P.lddx;      // (a row that is not there is a group's last)
    // a row's statistics are fetched a tile ahead
    float next_mean = 0.f, next_rstd = 0.f;
    auto look = [&](int k) {
      const int r = r0 + k * S.groups + group;
      const bool there = group < S.groups && r < r1;
      next_mean = there ? P.mean[base + r] : 0.f;
      next_rstd = there ? P.rstd[base + r] : 0.f;
    };
    look(0);
    for (int k = 0; k < tiles; ++k) {
      // a warp whose wait has run out goes on without waiting: others meet it at barriers
      if (kAligned && ok && !ptx::mbar_wait_own(full + b, phase, P.wait_limit)) {
        ok = false;
        if (P.dev_status && lane == 0) atomicOr(P.dev_status, DP_DEV_TIMEOUT);
      }
      const int r = r0 + k * S.groups + group;
      const bool mine = group < S.groups && r < r1;
      const long long row = base + (mine ? r : r0 + k * S.groups);
      // nothing of a row that is not there enters the sums: zeros, mean and rstd among them
      const float mean = next_mean, rstd = next_rstd;
      look(k + 1);
      F2 g[NP][H], c[NP][H];
      if (kAligned) {
        const uint8_t* from = smem + size_t(b) * at.tile + size_t(mine ? group : 0) * S.pitch;
        R.template open<true>(from, mine, g);
        R.template open<true>(from + size_t(S.groups) * S.pitch, mine, c);
        ptx::release_to_copies(empty + b, lane);         // the row is in registers
        if (++b == S.buffers) { b = 0; phase ^= 1; }
      } else {
        R.template open<true>(G + row * P.ldg, mine, g);
        R.template open<true>(X + row * P.ldx, mine, c);
      }
      if (NP > 1 && !mine) continue;                     // whole warps, and all of a group's
      const F2 minus = f2(-mean, -mean), scale = f2(rstd, rstd);
      F2 a1 = f2(0.f, 0.f), a2 = a1;
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        F2 w[H];
        R.vector(gain, j, w);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          c[j][e] = add2(c[j][e], minus);
          ss[j][e] = add2(ss[j][e], g[j][e]);
          g[j][e] = mul2(g[j][e], scale);
          gs[j][e] = fma2(g[j][e], c[j][e], gs[j][e]);
          g[j][e] = mul2(g[j][e], w[e]);                 // rstd u
          a1 = add2(a1, g[j][e]);
          a2 = fma2(g[j][e], c[j][e], a2);
        }
      }
      if (P.dX) {
        // dx = rstd u - mean(rstd u) - (x - mean) rstd^2 mean(rstd u (x - mean))
        float s[2] = {a1.x + a1.y, a2.x + a2.y};
        row_sum<2>(s, S, warp % S.W, lane, 1 + group, slots, turn);
        const float k1 = -s[0] * inv_p, k2 = -rstd * rstd * (s[1] * inv_p);
        const F2 kk1 = f2(k1, k1), kk2 = f2(k2, k2);
        if (mine) {
#pragma unroll
          for (int j = 0; j < NP; ++j) {
#pragma unroll
            for (int e = 0; e < H; ++e) g[j][e] = add2(g[j][e], fma2(c[j][e], kk2, kk1));
            R.store(out, P.vec_out, j, g[j]);
          }
        }
        out += out_step;
      }
    }
  }
  if (!P.gain_sums && !P.shift_sums && !P.sq) return;          // the same for every CTA
  // this CTA's sums: every group's in the place of the tiles, then added in order
  __syncthreads();
  if (warp < warps && group < S.groups) {
    float* mine = sums + size_t(group) * 2 * p;
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 u = floats(gs[j][e / 2]), v = floats(ss[j][e / 2]);
        const int c = R.column(j, e);
        if (R.has(j, e)) { mine[c] = e & 1 ? u.y : u.x; mine[p + c] = e & 1 ? v.y : v.x; }
      }
  }
  __syncthreads();
  if (S.groups > 1) {
    for (int c = tid; c < 2 * p; c += blockDim.x) {
      float u = sums[c];
#pragma unroll 4
      for (int q = 1; q < S.groups; ++q) u += sums[size_t(q) * 2 * p + c];
      sums[c] = u;
    }
    __syncthreads();
  }
  if (P.partials) {
    cudaTriggerProgrammaticLaunchCompletion();
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
      for (int q = 0; q < P.parts; q += 4) {             // four CTAs' loads in flight
        float t[4], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* other = cluster.map_shared_rank(sums, min(q + i, P.parts - 1));
          t[i] = other[c];
          w[i] = other[p + c];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (q + i < P.parts) { u += t[i]; v += w[i]; }
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

// The parts' sums through the workspace: a thread per column, parts in order, an example's columns over a cluster whose rank 0 adds up the
// squares.  Its launch overlaps the end of the other one.
constexpr int kLnSumThreads = 128;
__global__ void __launch_bounds__(kLnSumThreads)
ln_sums_kernel(const float* partials, int parts, int p, float* gain_sums, float* shift_sums, float* sq) {
  __shared__ float red[32], squares[8];
  cg::cluster_group cluster = cg::this_cluster();
  auto begun = cluster.barrier_arrive();               // rank 0's memory is written only once its CTA runs
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank(), example = blockIdx.x / ctas;
  cudaGridDependencySynchronize();
  float square = 0.f;
  for (int c = rank * kLnSumThreads + threadIdx.x; c < p; c += ctas * kLnSumThreads) {
    const float* in = partials + (long long)example * parts * 2 * p + c;
    float a = 0.f, b = 0.f;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) {
      a += in[(long long)k * 2 * p];
      b += in[(long long)k * 2 * p + p];
    }
    if (gain_sums) gain_sums[(long long)example * p + c] = a;
    if (shift_sums) shift_sums[(long long)example * p + c] = b;
    square = fmaf(a, a, fmaf(b, b, square));
  }
  square = block_sum(square, red);
  cluster.barrier_wait(std::move(begun));
  if (threadIdx.x == 0) *cluster.map_shared_rank(squares + rank, 0) = square;
  cluster.sync();
  if (sq && rank == 0 && threadIdx.x == 0) {
    float all = 0.f;
    for (int q = 0; q < ctas; ++q) all += squares[q];
    sq[example] += all;
  }
}

bool ln_vec(const void* q, long long ld, int es) { return !q || (aligned16(q) && (ld * es) % 16 == 0); }

// Lanes and warps of a row: 16-byte pieces, at most 32 columns a lane; whole warps for rows that are not aligned.
LnShape ln_shape(int p, int es, bool aligned) {
  LnShape S{};
  const int pieces = ceil_div(p * es, 16), most = 2 * es;              // pieces per lane
  S.lanes = aligned ? 1 : 32;
  while (S.lanes < 32 && S.lanes < pieces) S.lanes *= 2;
  S.W = 1;
  while (S.W * 32 * most < pieces) S.W *= 2;
  S.pitch = pieces * 16;
  return S;
}

// Pieces per lane that a kernel is compiled for.
int ln_pieces(const LnShape& S, int p, int es) {
  const int n = ceil_div(ceil_div(p * es, 16), S.lanes * S.W);
  return es == 4 && n > 2 ? (n + 1) / 2 * 2 : n;
}

template <typename K>
dp_status ln_smem_setup(K* kernel) {
  DP_SET_UP_ONCE((const void*)kernel, {
    DP_CUDA_OK(allow_shared(kernel, 227 * 1024));
    DP_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  });
  return DP_OK;
}

// Rows at a time and tiles in flight: an SM's shared memory divided by the blocks that share it, 48 KiB a tile at most.
bool ln_fit(LnShape& S, int p, int rows, bool sums, int warps, int blocks, bool copied) {
  S.groups = S.W > 1 ? warps / S.W : warps * 32 / S.lanes;
  const size_t most = (blocks == 1 ? 224 : blocks == 2 ? 112 : 74) * 1024;
  if (!copied) {
    S.buffers = 0;
    return LnSmem(S, p, rows, sums, warps).bytes <= 226 * 1024;
  }
  S.groups = std::max(1, std::min(S.groups, int(48 * 1024 / (rows * S.pitch))));
  for (S.buffers = kLnMaxBuffers; S.buffers > 1; --S.buffers)
    if (LnSmem(S, p, rows, sums, warps).bytes <= most) return true;
  return LnSmem(S, p, rows, sums, warps).bytes <= 226 * 1024;
}

// Working warps of a block and blocks per SM, by the registers that a lane's columns take: four of each in the backward pass, two in the
// forward pass.
constexpr int ln_columns(int NP, int es) { return NP * 16 / es; }
struct LnBlock { int warps, blocks; };
constexpr LnBlock ln_back_block(int columns, bool widest) {
  return widest ? LnBlock{16, 1} : columns > 24 ? LnBlock{10, 1} : columns > 16 ? LnBlock{14, 1} : columns > 8 ? LnBlock{8, 2} : LnBlock{8, 3};
}
constexpr LnBlock ln_forward_block(bool widest) { return widest ? LnBlock{16, 1} : LnBlock{8, 2}; }

// [c]: clusters of c CTAs, one CTA per SM, that run at once on the current device: fewer than SMs / c, since a cluster stays within a group of
// SMs (7 of 16, 15 of 8, 37 of 4 on a B200 with 148).
using LnClusters = std::array<int, kLnMaxParts + 1>;
const LnClusters& clusters_at_once() {
  static std::mutex mutex;
  static std::map<int, LnClusters> known;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) dev = -1;
  std::lock_guard<std::mutex> lock(mutex);
  const auto seen = known.find(dev);
  if (seen != known.end()) return seen->second;
  LnClusters& most = known[dev];                       // stays where it is
  auto* kernel = ln_backward_kernel<__nv_bfloat16, 4, true, (ln_back_block(32, true).warps + 1) * 32, ln_back_block(32, true).blocks>;
  for (int c = 1; c <= kLnMaxParts; ++c) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(c));
    cfg.blockDim = dim3((ln_back_block(32, true).warps + 1) * 32);
    cfg.dynamicSmemBytes = 200 * 1024;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {unsigned(c), 1u, 1u};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (dev < 0 || ln_smem_setup(kernel) != DP_OK || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      n = std::max(1, device_sm_count() / (c + c / 4));
    }
    most[c] = n;
  }
  return most;
}

// Parts an example's rows are cut into, and whether they are a cluster (else the sums go through the workspace): whichever takes least, in
// rows of a CTA.  A wave of CTAs costs 128 rows beside its own, the other launch 64 and one per part.  16 rows per part at least.
// Measured with T = 1024, p = 768 in bf16, clusters of 16, of 8 and the workspace (37 to 148 CTAs in all): 16, 21 and 19 us of 6 examples, 30, 21 and 20 of
// 8, 40, 41 and 23 of 16; p = 256: 11, 15 and 24; 12, 16 and 23; 16, 18 and 19.
struct LnParts { int parts; bool cluster; };
LnParts ln_parts(int B, int T, int blocks) {
  const int sms = device_sm_count();
  const LnClusters& at_once = clusters_at_once();
  LnParts best{1, true};
  long long least = 0;
  for (int c = 1; c <= std::min(kLnMaxParts, ceil_div(T, 16)); c *= 2) {
    const long long n = blocks * at_once[c], waves = (B + n - 1) / n, cost = waves * (ceil_div(T, c) + 128);
    if (c == 1 || cost < least) { least = cost; best = {c, true}; }
  }
  const int through = std::min(std::min(blocks * sms / B, ceil_div(T, 16)), int(std::sqrt(double(T))));
  if (through > 1 && ceil_div(T, through) + 192 + through < least) best = {through, false};
  return best;
}

template <typename T, int NP, bool kAligned, bool kWidest>
dp_status ln_back_launch(LnBackward& P, int B, LnParts parts, cudaStream_t st) {
  constexpr LnBlock kBlock = ln_back_block(ln_columns(NP, sizeof(T)), kWidest);
  auto* kernel = ln_backward_kernel<T, NP, kAligned, (kBlock.warps + 1) * 32, kBlock.blocks>;
  const int warps = P.S.W > 1 ? kBlock.warps / P.S.W * P.S.W : kBlock.warps;
  P.S.columns = ln_columns(NP, sizeof(T));
  if (!ln_fit(P.S, P.p, 2, true, warps, kBlock.blocks, kAligned)) return DP_ERR_UNSUPPORTED;
  const dp_status r = ln_smem_setup(kernel);
  if (r != DP_OK) return r;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(B) * unsigned(P.parts));
  cfg.blockDim = dim3((warps + (kAligned ? 1 : 0)) * 32);
  cfg.dynamicSmemBytes = LnSmem(P.S, P.p, 2, true, warps).bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {parts.cluster ? unsigned(P.parts) : 1u, 1u, 1u};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  DP_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, P));
  ++g_kernel_launches;
  return DP_OK;
}

template <typename T, int NP, bool kAligned, bool kWidest>
dp_status ln_fwd_launch(LnForward& P, cudaStream_t st) {
  constexpr LnBlock kBlock = ln_forward_block(kWidest);
  auto* kernel = ln_forward_kernel<T, NP, kAligned, (kBlock.warps + 1) * 32, kBlock.blocks>;
  const int warps = P.S.W > 1 ? kBlock.warps / P.S.W * P.S.W : kBlock.warps;
  P.S.columns = ln_columns(NP, sizeof(T));
  if (!ln_fit(P.S, P.p, 1, false, warps, kBlock.blocks, kAligned)) return DP_ERR_UNSUPPORTED;
  const long long blocks = std::min((P.rows + P.S.groups - 1) / P.S.groups, (long long)kBlock.blocks * sm_count());
  if (P.rows / blocks / P.S.groups >= 0x7fffffffLL - 1) return DP_ERR_UNSUPPORTED;       // a block counts its tiles in 32 bits
  const dp_status r = ln_smem_setup(kernel);
  if (r != DP_OK) return r;
  kernel<<<unsigned(blocks), (warps + (kAligned ? 1 : 0)) * 32, LnSmem(P.S, P.p, 1, false, warps).bytes, st>>>(P);
  DP_LAUNCH_OK();
  return DP_OK;
}

// f.template run<T, NP, kAligned, kWidest>() for the pieces per lane at hand
template <typename T, bool kAligned, typename F>
dp_status ln_dispatch(int pieces, bool widest, F f) {
  if (widest) return f.template run<T, sizeof(T) == 4 ? 8 : 4, kAligned, true>();
  switch (pieces) {
    case 1: return f.template run<T, 1, kAligned, false>();
    case 2: return f.template run<T, 2, kAligned, false>();
    case 3: return f.template run<T, sizeof(T) == 4 ? 4 : 3, kAligned, false>();
    case 4: return f.template run<T, 4, kAligned, false>();
    case 6: return f.template run<T, sizeof(T) == 4 ? 6 : 4, kAligned, false>();
    default: return f.template run<T, sizeof(T) == 4 ? 8 : 4, kAligned, false>();
  }
}

struct RunForward {
  LnForward& P;
  cudaStream_t st;
  template <typename T, int NP, bool kAligned, bool kWidest>
  dp_status run() { return ln_fwd_launch<T, NP, kAligned, kWidest>(P, st); }
};
struct RunBackward {
  LnBackward& P;
  int B;
  LnParts parts;
  cudaStream_t st;
  template <typename T, int NP, bool kAligned, bool kWidest>
  dp_status run() { return ln_back_launch<T, NP, kAligned, kWidest>(P, B, parts, st); }
};
template <typename F>
dp_status ln_run(dp_dtype dt, bool aligned, int pieces, bool widest, F f) {
  if (dt == DP_F32) return aligned ? ln_dispatch<float, true>(pieces, widest, f) : ln_dispatch<float, false>(pieces, widest, f);
  return aligned ? ln_dispatch<__nv_bfloat16, true>(pieces, widest, f) : ln_dispatch<__nv_bfloat16, false>(pieces, widest, f);
}

LnParts ln_parts_of(int B, int T, int p, int es) {
  const LnShape S = ln_shape(p, es, true);             // (the number of pieces per lane is the same for other rows)
  return ln_parts(B, T, ln_back_block(ln_columns(ln_pieces(S, p, es), es), S.W == 16).blocks);
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
                       int32_t* dev_status, void* stream) try {
  if (!X || rows <= 0 || p <= 0 || ldx < p || (!Y && !X_hat && !mean && !rstd)) return DP_ERR_INVALID_ARG;
  if ((Y && ldy < p) || (X_hat && ldh < p) || !known_dtype(dt) || !known_dtype(param_dt)) return DP_ERR_INVALID_ARG;
  if (!std::isfinite(eps) || eps < 0.f || (Y && Y == X_hat)) return DP_ERR_INVALID_ARG;
  if ((Y == X && ldy != ldx) || (X_hat == X && ldh != ldx)) return DP_ERR_INVALID_ARG;
  if (p > kLnMaxCols || rows > (int64_t(1) << 36)) return DP_ERR_UNSUPPORTED;
  const int es = dt == DP_F32 ? 4 : 2, ps = param_dt == DP_F32 ? 4 : 2;
  if (!on_boundary(es, X, Y, X_hat) || !on_boundary(ps, gain, shift) || !on_boundary(4, mean, rstd)) return DP_ERR_ALIGNMENT;
  LnForward P{};
  P.X = X; P.ldx = ldx; P.gain = gain; P.shift = shift; P.param_dt = param_dt; P.Y = Y; P.ldy = ldy; P.H = X_hat; P.ldh = ldh;
  P.mean = mean; P.rstd = rstd; P.rows = rows; P.p = p; P.eps = eps; P.dev_status = dev_status;
  P.wait_limit = g_wait_limit;
  const bool aligned = p * es % 16 == 0 && ln_vec(X, ldx, es);
  P.S = ln_shape(p, es, aligned);
  P.whole = aligned && ldx == p;
  P.vec_y = ln_vec(Y, ldy, es);
  P.vec_h = ln_vec(X_hat, ldh, es);
  return ln_run(dt, aligned, ln_pieces(P.S, p, es), P.S.W == 16, RunForward{P, (cudaStream_t)stream});
} catch (...) {                                        // host memory for the set-up of a device
  return DP_ERR_UNSUPPORTED;
}

size_t dp_layernorm_backward_ws_bytes(int32_t B, int32_t T, int32_t p) try {
  if (B <= 0 || T <= 0 || p <= 0 || p > kLnMaxCols || T > kLnMaxTokens) return 0;
  size_t most = 0;                                    // of either type of G and X
  for (const int es : {2, 4}) {
    const LnParts parts = ln_parts_of(B, T, p, es);
    if (!parts.cluster) most = std::max(most, ln_partial_bytes(parts, B, p));
  }
  return most;
} catch (...) {
  return 0;
}

dp_status dp_layernorm_backward(const void* G, int64_t ldg, const void* X, int64_t ldx, dp_dtype dt, int32_t B, int32_t T, int32_t p,
                                const void* gain, dp_dtype param_dt, const float* mean, const float* rstd, void* dX, int64_t lddx,
                                float* gain_sums, float* shift_sums, float* sq, void* ws, size_t ws_bytes, int32_t* dev_status,
                                void* stream) try {
  if (!G || !X || !mean || !rstd || B <= 0 || T <= 0 || p <= 0 || ldg < p || ldx < p) return DP_ERR_INVALID_ARG;
  if ((dX && lddx < p) || !known_dtype(dt) || !known_dtype(param_dt)) return DP_ERR_INVALID_ARG;
  const bool sums = gain_sums || shift_sums || sq;
  if (!dX && !sums) return DP_ERR_INVALID_ARG;
  if ((dX == G && lddx != ldg) || (dX == X && lddx != ldx)) return DP_ERR_INVALID_ARG;
  const int es = dt == DP_F32 ? 4 : 2, ps = param_dt == DP_F32 ? 4 : 2;
  if (!on_boundary(es, G, X, dX) || !on_boundary(ps, gain) || !on_boundary(4, mean, rstd, gain_sums, shift_sums, sq)) return DP_ERR_ALIGNMENT;
  if (p > kLnMaxCols || T > kLnMaxTokens) return DP_ERR_UNSUPPORTED;
  const LnParts parts = ln_parts_of(B, T, p, es);
  if ((long long)B * parts.parts > 0x7fffffffLL) return DP_ERR_UNSUPPORTED;
  float* partials = nullptr;
  if (!parts.cluster && sums) {
    if (!ws || ws_bytes < dp_layernorm_backward_ws_bytes(B, T, p)) return DP_ERR_WORKSPACE;
    if (!on_boundary(4, ws)) return DP_ERR_ALIGNMENT;
    partials = static_cast<float*>(ws);
  }
  LnBackward P{};
  P.G = G; P.ldg = ldg; P.X = X; P.ldx = ldx; P.gain = gain; P.param_dt = param_dt; P.mean = mean; P.rstd = rstd; P.dX = dX; P.lddx = lddx;
  P.gain_sums = gain_sums; P.shift_sums = shift_sums; P.sq = sq; P.partials = partials;
  P.T = T; P.p = p; P.parts = parts.parts; P.dev_status = dev_status; P.wait_limit = g_wait_limit;
  const bool aligned = p * es % 16 == 0 && ln_vec(G, ldg, es) && ln_vec(X, ldx, es);
  P.S = ln_shape(p, es, aligned);
  P.whole_g = aligned && ldg == p;
  P.whole_x = aligned && ldx == p;
  P.vec_out = ln_vec(dX, lddx, es);
  const cudaStream_t st = (cudaStream_t)stream;
  const dp_status r = ln_run(dt, aligned, ln_pieces(P.S, p, es), P.S.W == 16, RunBackward{P, B, parts, st});
  if (r != DP_OK || !partials) return r;
  const unsigned ctas = unsigned(std::min(8, ceil_div(p, kLnSumThreads)));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(B) * ctas);
  cfg.blockDim = dim3(kLnSumThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {ctas, 1u, 1u};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  DP_CUDA_OK(cudaLaunchKernelEx(&cfg, ln_sums_kernel, (const float*)partials, parts.parts, p, gain_sums, shift_sums, sq));
  ++g_kernel_launches;
  return DP_OK;
} catch (...) {
  return DP_ERR_UNSUPPORTED;
}

}  // extern "C"
