// Orthogonalised updates: Newton-Schulz products on the noised sums of weight matrices.
//
//   X_0 = M / (|M|_F + eps),   A = X X^T,   B = b A + c A A,   X <- a X + B X   (once per step, coefficients per step)
//
// turns a matrix into the nearest one with orthonormal rows (columns), as far as the polynomial's steps go; applied to a
// noised sum it is post-processing, so it costs no privacy.  A matrix with more rows than columns is transposed on the way in
// and out, so that X is m x n with m <= n and A, B are m x m.
//
// Every product runs on the tensor cores in three bf16-rate products of fp16 operands: X, A and B are kept as two planes
// of fp16, high and low terms (22 bits), scaled by powers of two that the host derives from bounds of the polynomials (|X| <= s
// in the spectral norm gives |A| <= s^2 and so on), so that nothing overflows and small entries keep their low terms: one
// bf16 product per product is off by 1e-2 after five steps, two bf16 terms by 2e-5, these by what the sums round.
// An MMA rounds its sum towards zero, by as much as the sum is large.  So sums are taken in K steps of 64, each in an
// accumulator of its own, that the epilogue adds up in registers to nearest: error of DistilGPT2's updates against 64 bits 2.2e-5
// with one accumulator per tile (the diagonal of A, a sum of squares, came out 6e-6 too small in the longest sums).
//
// Nothing is added to a product but on the diagonal, so no epilogue reads matrices: B = a I + b A + c A A = c A A' + a I with
// A' = A + (b / c) I, which differs from A on the diagonal: A' is a copy of the diagonal's tiles.  X' = B X.  (Completing the square,
// c A'' A'' with A'' = A + (b / 2c) I, would do too, but in a sum that one large term dominates the others are truncated at that
// one's exponent: error of DistilGPT2's updates 2.7e-6 against 1.3e-6.  A polynomial whose c is so small that b / c would drown A adds b A
// instead.)
//
// Several steps go by A alone where X is longer than high: A_1 = B_0 A_0 B_0 and so on, all of them symmetric products of m x m, and X
// meets the product of the Bs once at the end.  For a GPT-2 block 3 + 2 steps at once take 36 % less work, 2 + 2 + 1 24 %.  A's error
// grows by max |B|^2 a step (11.8 for the usual quintic) relative to its small eigenvalues, B = a I + ... sees it next to a.  Errors of the updates of
// layers of d = 256, 768, 1000 (and the square one among them), in 1e-6: one by one 2.4 (1.4), 1.3 (1.4), 1.4 (1.4); two at once 1.9
// (3.2), 2.8 (3.3), 3.4 (3.2); three 8.9 (5.4), 3.2 (4.3), 2.0 (3.6); five 22 (170), 13 (60), 14 (48); plain fp32 products
// 2.5 (1.7), 2.8 (2.6), 3.3 (2.8).  What grows is largest beside one dominant direction, where the others, 1e-3 of it, are amplified 485 times:
// five steps at once then are 2.3e-2 off (of (512, 1500); plain fp32 products 1.5e-4), 3 + 2 less than shows beside bf16's rounding, 1.7e-3.  So bf16
// updates take three steps at once.  fp32 ones take two from m = 640 on, where no such matrix was more than 1.3 times as far off as plain fp32
// products make it (at (512, 2048) 1.6 times, 4.3e-6 against 2.7e-6).
//
// A and A A are symmetric: tiles on and below the diagonal are computed and stored, and a product that needs one above it reads the
// stored one with rows and columns exchanged (the tensor core takes either order).
//
// One kernel for all three products and all matrices of a call: persistent, work items are output tiles.  kPair: CTA pairs
// (cta_group::2) with 256 x 256 tiles; else single CTAs with 128 x 128 tiles, for calls with few tiles.  Roles: two producer
// warps (TMA, 64-wide K steps of the left and the right operand), the MMA issuer, a relay (pairs: tells rank 0's issuer
// that rank 1's half of a stage has landed), 16 epilogue warps; two accumulators, so adding up a chunk and the epilogue of a
// tile overlap the next ones.  Calls whose matrices all have at most 64 by 256 numbers take ns_small_kernel.
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <utility>
#include <vector>

#include "dp_common.cuh"
#include "ptx_sm100.cuh"
#include "tma_host.cuh"

namespace dpg {

namespace {

constexpr int kBK = 64;
constexpr int kBoxBytes = 64 * 128;                   // 64 rows x 64 fp16
constexpr int kPartBytes = 2 * kBoxBytes;             // 128 rows (or columns) of an operand
constexpr int kStageBytes = 4 * kPartBytes;           // high and low terms of the left and of the right operand
constexpr int kStages = 3;
constexpr int kStagingBytes = 32 * 64;                // a warp's 32 rows x 32 fp16 on their way out
constexpr int kRelayWarp = 2, kProducerQWarp = 3, kEpiWarp0 = 4, kEpiWarps = 16;
constexpr int kThreads = (kEpiWarp0 + kEpiWarps) * 32;
constexpr size_t kSmemBytes = size_t(kStages) * kStageBytes + kEpiWarps * kStagingBytes + 1024 + 512;
constexpr int kNsMaxMats = 48;                        // matrices per launch (parameter-block limit)
constexpr int kNormParts = 32;                        // partial sums of a matrix's squares

enum Product { kGram, kSym, kApply };                 // X X^T; symmetric times symmetric, commuting; symmetric times X

struct NsMat {
  const __half* add;         // kSym: planes that are added, or nullptr
  void* out;                 // the call's output, or nullptr: planes, through tmD
  long long plane_add, ldo;
  int ld_add;
  int M, N, ksteps;
  int item_begin;
  int transposed;            // out is X'^T
  float out_scale;
};

struct __align__(64) NsParams {
  CUtensorMap tmP[kNsMaxMats];
  CUtensorMap tmQ[kNsMaxMats];
  CUtensorMap tmD[kNsMaxMats];
  CUtensorMap tmE[kNsMaxMats];       // the copy of the diagonal's tiles: written beside tmD, or read
  NsMat mat[kNsMaxMats];
  int n_mats, total_items;
  int out_dt;
  int shifted;               // kSym: the right operand's tiles on the diagonal come from tmE
  int copy;                  // the diagonal's tiles go to tmE too, with `diagonal` there and not in tmD
  float f_acc;               // written value = f_acc * product
  float f_add, diagonal;     //   + f_add * (high + low term of `add`), + diagonal where row = column
  int* dev_status;
  long long wait_limit;
};
static_assert(sizeof(NsParams) <= 32764, "kernel parameter block too large");

struct Item { int mat, tm, tn; };

template <Product kProduct, int kTile>
__device__ __forceinline__ Item decode_item(const NsParams& P, int item, int& l) {
  while (l + 1 < P.n_mats && item >= P.mat[l + 1].item_begin) ++l;
  const NsMat& L = P.mat[l];
  int local = item - L.item_begin;
  Item it;
  it.mat = l;
  if (kProduct == kApply) {                           // tiles of the same columns of X, which B's rows all meet, together
    const int tiles_m = (L.M + kTile - 1) / kTile;
    it.tn = local / tiles_m;
    it.tm = local - it.tn * tiles_m;
  } else {                                            // rows of the lower triangle, the diagonal in them
    it.tm = 0;
    while (local > it.tm) { local -= it.tm + 1; ++it.tm; }
    it.tn = local;
  }
  return it;
}

// Whether a K step of a symmetric operand's row tile `t` lies above the diagonal's tiles: there the stored tile is the transpose,
// contiguous along the rows that are wanted.
template <Product kProduct, int kTile>
__device__ __forceinline__ bool exchanged(bool right, int t, int k) {
  if (kProduct == kApply && right) return true;       // X: K rows, contiguous along N
  return kProduct != kGram && k * kBK / kTile > t;
}

__device__ __forceinline__ void split_fp16(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}

__device__ __forceinline__ uint32_t high_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  uint32_t w;
  memcpy(&w, &h, 4);
  return w;
}
__device__ __forceinline__ uint32_t low_pair(float a, float b) {
  const float2 h = __half22float2(__floats2half2_rn(a, b));
  return high_pair(a - h.x, b - h.y);
}

// v += f * (16 consecutive values of two planes)
__device__ __forceinline__ void add_planes(const __half* p, long long plane, float f, float* v) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint4 a = reinterpret_cast<const uint4*>(p)[h], b = reinterpret_cast<const uint4*>(p + plane)[h];
    const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&aw[e]));
      const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&bw[e]));
      v[8 * h + 2 * e] = fmaf(f, x.x + y.x, v[8 * h + 2 * e]);
      v[8 * h + 2 * e + 1] = fmaf(f, x.y + y.y, v[8 * h + 2 * e + 1]);
    }
  }
}

// 16 columns of the result, `left` of which exist
__device__ __forceinline__ void store_out(const NsMat& L, int dt, int row, int col, int left, const float* v) {
  if (L.transposed) {                                  // a warp's lanes lie side by side
    const size_t at = size_t(col) * L.ldo + row;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (e >= left) continue;
      if (dt == DP_F32) static_cast<float*>(L.out)[at + e * L.ldo] = v[e];
      else static_cast<__nv_bfloat16*>(L.out)[at + e * L.ldo] = __float2bfloat16_rn(v[e]);
    }
    return;
  }
  const size_t at = size_t(row) * L.ldo + col;
  if (dt == DP_F32) {
    float* o = static_cast<float*>(L.out) + at;
    if (left >= 16 && (reinterpret_cast<uintptr_t>(o) & 31) == 0) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = v[8 * h + e];
        ptx::st_global_v8(o + 8 * h, w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) if (e < left) o[e] = v[e];
    }
  } else {
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(L.out) + at;
    if (left >= 16 && (reinterpret_cast<uintptr_t>(o) & 31) == 0) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        memcpy(&w[e], &h, 4);
      }
      ptx::st_global_v8(reinterpret_cast<float*>(o), w);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) if (e < left) o[e] = __float2bfloat16_rn(v[e]);
    }
  }
}

// A call's launches overlap: the next one's CTAs start where this one's leave room, set themselves up and wait here for its end (and so,
// since every CTA waits, for the ends of all before it).  132 us -> 99 for a
// 128 x 128 in 17 launches, 206 -> 176 for the layers of a block of width 256.
__device__ __forceinline__ void follow_the_launch_before() {
  cudaTriggerProgrammaticLaunchCompletion();
  cudaGridDependencySynchronize();
}

template <Product kProduct, bool kPair>
__global__ void __launch_bounds__(kThreads, 1)
ns_product_kernel(const __grid_constant__ NsParams P) {
  constexpr int kTile = kPair ? 256 : 128;             // output tile; also columns of an accumulator
  const uint32_t rank = kPair ? ptx::cluster_ctarank() : 0u;
  const int first_item = kPair ? int(blockIdx.x >> 1) : int(blockIdx.x);
  const int item_stride = kPair ? int(gridDim.x >> 1) : int(gridDim.x);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = tiles + size_t(kStages) * kStageBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(staging + kEpiWarps * kStagingBytes);
  uint64_t* full = bars;                      // both producers' TMA loads landed
  uint64_t* ready = bars + kStages;           // pair: in both CTAs (rank 0's copy)
  uint64_t* empty = bars + 2 * kStages;       // MMAs retired
  uint64_t* acc_full = bars + 3 * kStages;    // [2]
  uint64_t* acc_empty = acc_full + 2;         // [2]
  uint64_t* mma_done = acc_empty + 2;         // only used where a wait ran out
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* sink = tmem_slot + 2;             // [kStages] written by st.async, never read

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t tiles_a = ptx::smem_u32(tiles);
  const uint32_t full_a = ptx::smem_u32(full), ready_a = ptx::smem_u32(ready), empty_a = ptx::smem_u32(empty);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(&full[s], 2);
      ptx::mbar_init(&ready[s], 1);           // rank 0's relay arrives and announces 4 bytes, rank 1's sends them
      ptx::mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(&acc_full[b], 1);
      ptx::mbar_init(&acc_empty[b], kEpiWarps);    // pair: + 4 bytes from each of rank 1's
    }
    ptx::mbar_init(mma_done, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 1) {
    if (kPair) { ptx::tmem_alloc_pair(tmem_slot, 2 * kTile); ptx::tmem_relinquish_pair(); }
    else { ptx::tmem_alloc(tmem_slot, 2 * kTile); ptx::tmem_relinquish(); }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (kPair) ptx::cluster_sync_all();         // the partner's barriers exist before anyone arrives on them
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  uint32_t issued = 0;                        // a producer's stages so far
  follow_the_launch_before();

  if (warp == 0 || warp == kProducerQWarp) {
    // ------------------------------------------------------------- TMA producers
    // producers, issuer and relay: the whole warp runs the loop, an elected lane issues (see ptx::warp_ok)
    const bool right = warp != 0;
    uint32_t stage = 0, phase = 0;
    int lay = 0;
    bool ok = true;
    for (int item = first_item; item < P.total_items && ok; item += item_stride) {
      const Item it = decode_item<kProduct, kTile>(P, item, lay);
      const uint64_t tm = reinterpret_cast<uint64_t>(right ? &P.tmQ[it.mat] : &P.tmP[it.mat]);
      const int ksteps = P.mat[it.mat].ksteps;
      // first of this CTA's 128 rows (columns) of the operand
      const int r0 = (right ? it.tn : it.tm) * kTile + int(rank) * 128;
      for (int k = 0; k < ksteps; ++k) {
        ok = ptx::warp_ok(ptx::mbar_wait_a(empty_a + 8 * stage, phase ^ 1, abort_flag, P.wait_limit));
        if (!ok) break;
        const uint32_t bar = full_a + 8 * stage;
        const uint32_t dst = tiles_a + stage * kStageBytes + (right ? 2 * kPartBytes : 0);
        const bool x = exchanged<kProduct, kTile>(right, right ? it.tn : it.tm, k);
        const bool diagonal = kProduct == kSym && right && P.shifted && k * kBK / kTile == it.tn;
        const uint64_t from = diagonal ? reinterpret_cast<uint64_t>(&P.tmE[it.mat]) : tm;
        if (ptx::elect_one()) {
          ptx::mbar_arrive_expect_tx_a(bar, uint32_t(2 * kPartBytes));
#pragma unroll
          for (int b = 0; b < 4; ++b) {                // two boxes of high terms, two of low ones
            const int r = r0 + (b & 1) * 64;
            ptx::tma_load_3d_a(dst + b * kBoxBytes, from, bar, x ? r : k * kBK, x ? k * kBK : r, b >> 1);
          }
        }
        __syncwarp();
        ++issued;
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
    }
    if (!ok && ptx::elect_one()) {
      *abort_flag = 1;
      if (P.dev_status) atomicOr(P.dev_status, DP_DEV_TIMEOUT);
    }
  } else if (warp == 1) {
    // --------------------------------------------------------------- MMA issuer
    if (rank == 0) {
      // fp16 operands: format 0 in place of bf16's 1 in bits 7 and 10; bits 15, 16: left, right operand contiguous along M, N
      constexpr uint32_t idesc0 = ptx::idesc_bf16_f32(kTile, kTile, 0, 0) & ~((1u << 7) | (1u << 10));
      // K-major: groups of 8 rows 1 KiB apart, 16 columns further 32 bytes; MN-major: 64-column boxes apart, 16 rows 2 KiB
      constexpr uint64_t dk = ptx::smem_desc_base(16, 1024, ptx::SWIZZLE_128B);
      constexpr uint64_t dmn = ptx::smem_desc_base(kBoxBytes, 1024, ptx::SWIZZLE_128B);
      constexpr uint32_t desc_hi = uint32_t(dk >> 32);
      static_assert(desc_hi == uint32_t(dmn >> 32), "descriptors differ in the low word only");
      const uint32_t base = (tiles_a >> 4) & 0x3FFF;
      const uint32_t go_a = kPair ? ready_a : full_a;
      uint32_t stage = 0, phase = 0, n_acc = 0;
      int lay = 0;
      bool ok = true;
      for (int item = first_item; item < P.total_items && ok; item += item_stride) {
        const Item it = decode_item<kProduct, kTile>(P, item, lay);
        const int ksteps = P.mat[it.mat].ksteps;
        for (int k = 0; k < ksteps; ++k, ++n_acc) {
          const uint32_t buf = n_acc & 1, d_tmem = tmem_base + buf * kTile;
          ok = ptx::warp_ok(kPair ? ptx::mbar_wait_cluster(&acc_empty[buf], ((n_acc >> 1) & 1) ^ 1, abort_flag, P.wait_limit)
                                  : ptx::mbar_wait(&acc_empty[buf], ((n_acc >> 1) & 1) ^ 1, abort_flag, P.wait_limit));
          if (!ok) break;
          ok = ptx::warp_ok(kPair ? ptx::mbar_wait_cluster_a(go_a + 8 * stage, phase, abort_flag, P.wait_limit)
                                  : ptx::mbar_wait_a(go_a + 8 * stage, phase, abort_flag, P.wait_limit));
          if (!ok) break;
          ptx::tc_fence_after();
          const bool xp = exchanged<kProduct, kTile>(false, it.tm, k), xq = exchanged<kProduct, kTile>(true, it.tn, k);
          const uint32_t idesc = idesc0 | (xp ? 1u << 15 : 0u) | (xq ? 1u << 16 : 0u);
          const uint32_t lo_p = (xp ? uint32_t(dmn) : uint32_t(dk)) | (base + stage * (kStageBytes >> 4));
          const uint32_t lo_q = (xq ? uint32_t(dmn) : uint32_t(dk)) | (base + stage * (kStageBytes >> 4) + (2 * kPartBytes >> 4));
          const uint32_t dp = xp ? 128 : 2, dq = xq ? 128 : 2;
          if (ptx::elect_one()) {
#pragma unroll
            for (int t = 0; t < 3; ++t) {              // lo hi', hi lo', hi hi': the small products while the sum is small
              constexpr uint32_t low = kPartBytes >> 4;
#pragma unroll
              for (int kk = 0; kk < kBK / 16; ++kk) {
                const uint32_t p = lo_p + (t == 0 ? low : 0u) + kk * dp, q = lo_q + (t == 1 ? low : 0u) + kk * dq;
                const uint32_t more = t || kk ? 1u : 0u;
                if (kPair) ptx::mma_bf16_ss_pair_lh(d_tmem, p, q, desc_hi, idesc, more);
                else ptx::mma_bf16_ss_lh(d_tmem, p, q, desc_hi, idesc, more);
              }
            }
            if (kPair) ptx::mma_commit_pair_a(empty_a + 8 * stage, 3);     // stage reusable once these MMAs retire
            else ptx::mma_commit_a(empty_a + 8 * stage);
            if (kPair) ptx::mma_commit_pair(&acc_full[buf], 3);
            else ptx::mma_commit(&acc_full[buf]);
          }
          __syncwarp();
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
      }
      // what rank 1's epilogue tells this CTA's barriers last has to arrive before the CTA ends
      if (kPair)
        for (uint32_t n = n_acc > 2 ? n_acc - 2 : 0; n < n_acc && ok; ++n)
          ok = ptx::warp_ok(ptx::mbar_wait_cluster(&acc_empty[n & 1], (n >> 1) & 1, abort_flag, P.wait_limit));
      if (!ok && ptx::elect_one()) {
        *abort_flag = 1;
        if (P.dev_status) atomicOr(P.dev_status, DP_DEV_TIMEOUT);
      }
    }
  } else if (warp == kRelayWarp) {
    // -------------------------------------------------------------------- relay
    // Rank 0's relay arrives on its own `ready` barrier and announces 4 more bytes; rank 1's, which has acquired its `full`
    // barrier, delivers them with an asynchronous store whose completion is a release at cluster scope.
    if (kPair) {
      const uint32_t ready_remote = ptx::mapa_u32(ready_a, 0), sink_remote = ptx::mapa_u32(ptx::smem_u32(sink), 0);
      uint32_t stage = 0, phase = 0;
      int lay = 0;
      bool ok = true;
      for (int item = first_item; item < P.total_items && ok; item += item_stride) {
        const Item it = decode_item<kProduct, kTile>(P, item, lay);
        for (int k = P.mat[it.mat].ksteps; k > 0; --k) {
          ok = ptx::warp_ok(ptx::mbar_wait_a(full_a + 8 * stage, phase, abort_flag, P.wait_limit));
          if (!ok) break;
          if (ptx::elect_one()) {
            if (rank == 0) ptx::mbar_arrive_expect_tx_a(ready_a + 8 * stage, 4);
            else ptx::st_async_signal_a(ready_remote + 8 * stage, sink_remote + 4 * stage);
          }
          __syncwarp();
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
      }
      if (!ok && ptx::elect_one()) {
        *abort_flag = 1;
        if (P.dev_status) atomicOr(P.dev_status, DP_DEV_TIMEOUT);
      }
    }
  } else {
    // ----------------------------------------------------------------- epilogue
    const int q = warp & 3;                          // TMEM lane quarter this warp may read
    const int ew = warp - kEpiWarp0;
    constexpr int kCols = kTile / (kEpiWarps / 4);   // columns of a warp
    const uint32_t acc_empty_a = ptx::smem_u32(acc_empty);
    const uint32_t acc_empty_remote = kPair ? ptx::mapa_u32(acc_empty_a, 0) : 0u;
    const uint32_t sink_remote = kPair ? ptx::mapa_u32(ptx::smem_u32(sink), 0) : 0u;
    auto free_acc = [&](uint32_t buf) {              // see gemm_gta_tc.cu
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (!kPair) ptx::mbar_arrive(&acc_empty[buf]);
        else if (rank == 0) ptx::mbar_arrive_expect_tx_a(acc_empty_a + 8 * buf, 4);
        else ptx::st_async_signal_a(acc_empty_remote + 8 * buf, sink_remote);
      }
    };
    uint32_t n_acc = 0;
    uint8_t* my_staging = staging + ew * kStagingBytes;
    const uint32_t my_staging_a = ptx::smem_u32(my_staging);
    int lay = 0;
    bool ok = true;
    for (int item = first_item; item < P.total_items && ok; item += item_stride) {
      const Item it = decode_item<kProduct, kTile>(P, item, lay);
      const NsMat& L = P.mat[it.mat];
      float sum[kCols];
#pragma unroll
      for (int e = 0; e < kCols; ++e) sum[e] = 0.f;
      for (int left = L.ksteps; left > 0; --left, ++n_acc) {
        const uint32_t buf = n_acc & 1;
        // no sleep between polls: the accumulator is wanted again in a K step's time
        ok = ptx::warp_ok(ptx::mbar_wait(&acc_full[buf], (n_acc >> 1) & 1, abort_flag, P.wait_limit));
        if (!ok) break;
        ptx::tc_fence_after();
        const uint32_t t0 = tmem_base + (uint32_t(q * 32) << 16) + buf * kTile + (ew >> 2) * kCols;
#pragma unroll
        for (int c = 0; c < kCols; c += 16) {
          uint32_t r[16];
          ptx::tmem_ld_32x32b_x16(t0 + c, r);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) sum[c + e] += __uint_as_float(r[e]);
        }
        free_acc(buf);
      }
      if (!ok) break;
      const int row0 = it.tm * kTile + int(rank) * 128 + q * 32, row = row0 + lane;
      const int col0 = it.tn * kTile + (ew >> 2) * kCols;
      const float f_acc = P.f_acc * L.out_scale;
      if (row0 >= L.M) continue;
#pragma unroll
      for (int g = 0; g < kCols / 32; ++g) {
        const int col = col0 + 32 * g;
        if (col >= L.N) continue;
        float* v = sum + 32 * g;
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] *= f_acc;
        if (kProduct == kSym && L.add && row < L.M) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (col + 16 * h < L.N) add_planes(L.add + size_t(row) * L.ld_add + col + 16 * h, L.plane_add, P.f_add, v + 16 * h);
        }
        if (kProduct == kApply && L.out) {
          if (row < L.M) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (col + 16 * h < L.N) store_out(L, P.out_dt, row, col + 16 * h, L.N - col - 16 * h, v + 16 * h);
          }
          continue;
        }
        // 32 x 32 of each plane through shared memory to a TMA store, which leaves out what lies outside the matrix
        const bool on_diagonal = kProduct != kApply && it.tm == it.tn;
        const int copies = on_diagonal && P.copy ? 2 : 1;
#pragma unroll 1
        for (int t = 0; t < copies; ++t) {
          const uint64_t tm = reinterpret_cast<uint64_t>(t ? &P.tmE[it.mat] : &P.tmD[it.mat]);
          if (on_diagonal && t == P.copy) {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] += col + e == row ? P.diagonal : 0.f;
          }
#pragma unroll
          for (int plane = 0; plane < 2; ++plane) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = plane ? low_pair(v[2 * e], v[2 * e + 1]) : high_pair(v[2 * e], v[2 * e + 1]);
            if (lane == 0) ptx::tma_store_wait_read();
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 4; ++c)                // 64-byte swizzle: no two of a quarter-warp's stores share a bank
              *reinterpret_cast<uint4*>(my_staging + lane * 64 + ((c ^ (lane >> 1 & 3)) << 4)) =
                  make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::tma_store_3d_a(tm, my_staging_a, col, row0, plane);
          }
        }
      }
      __syncwarp();
    }
    if (lane == 0) ptx::tma_store_wait();
    if (!ok && lane == 0) {
      *abort_flag = 1;
      if (P.dev_status) atomicOr(P.dev_status, DP_DEV_TIMEOUT);
    }
  }

  ptx::tc_fence_before();
  __syncthreads();
  ptx::settle_after_abort(abort_flag, (warp == 0 || warp == kProducerQWarp) && lane == 0, full, kStages, issued,
                          warp == 1 && rank == 0 && ptx::elect_one(), mma_done, kPair);
  if (kPair) ptx::cluster_sync_all();         // neither CTA leaves while the partner may still use its memory
  if (warp == 1) {
    ptx::tc_fence_after();
    if (kPair) ptx::tmem_dealloc_pair(tmem_base, 2 * kTile);
    else ptx::tmem_dealloc(tmem_base, 2 * kTile);
  }
}

// ---- the way in: norms, scaled and split matrices ------------------------------------------------

struct NsIn {
  const void* M;
  long long ldm, plane;
  __half* X;                 // planes of the m x n matrix
  int p, d, ldx;
  int transposed, vec;       // vec: rows on 16-byte boundaries
  int block_begin;
};
struct NsInParams {
  NsIn mat[kNsMaxMats];
  int n_mats, dt;
  double* partials;          // [matrix][kNormParts]
  double eps;
  float scale;
};

// eight columns of a row, zeros past its end
__device__ __forceinline__ void ns_load8(const NsIn& L, int dt, int r, int c, float (&v)[8]) {
  const size_t at = size_t(r) * size_t(L.ldm) + c;
  if (dt == DP_F32) load8<float>(static_cast<const float*>(L.M) + at, L.d - c, L.vec, v);
  else load8<__nv_bfloat16>(static_cast<const __nv_bfloat16*>(L.M) + at, L.d - c, L.vec, v);
}

// squares of a matrix, kNormParts blocks each; in 64 bits, whose range holds the square of every fp32 number
__global__ void __launch_bounds__(256)
ns_norm_kernel(const __grid_constant__ NsInParams P) {
  __shared__ double red[8];
  cudaTriggerProgrammaticLaunchCompletion();
  const int l = blockIdx.x / kNormParts, part = blockIdx.x % kNormParts;
  const NsIn& L = P.mat[l];
  const int chunks = (L.d + 7) / 8;                   // of eight columns; a thread's lie 256 * kNormParts apart
  const long long total = (long long)chunks * L.p, stride = 256LL * kNormParts;
  const int step_r = int(stride / chunks), step_c = int(stride % chunks);
  long long k = part * 256LL + threadIdx.x;
  int r = int(k / chunks), c = int(k % chunks);
  double s = 0.0;
  while (k < total) {
    float v[4][8];
    int n = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (k < total) { ns_load8(L, P.dt, r, 8 * c, v[u]); ++n; }
      k += stride;
      r += step_r;
      c += step_c;
      if (c >= chunks) { c -= chunks; ++r; }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (u < n)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fma(double(v[u][e]), double(v[u][e]), s);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = 0.0;
    for (int w = 0; w < 8; ++w) all += red[w];
    P.partials[l * kNormParts + part] = all;
  }
}

// f as a number in [1, 2) and two powers of two, since fp32 may hold neither it nor its inverse
__device__ __forceinline__ void ns_factor(double f, float (&factor)[3]) {
  int e = 0;
  if (f > 0 && f <= 1.7e308) e = ilogb(f);
  factor[0] = float(scalbn(f, -e));
  factor[1] = float(scalbn(1.0, e / 2));
  factor[2] = float(scalbn(1.0, e - e / 2));
}

// 64 x 64 blocks of M / (|M| + eps), scaled and split, transposed where M has more rows than columns
__global__ void __launch_bounds__(256)
ns_split_kernel(const __grid_constant__ NsInParams P) {
  __shared__ float tile[64][65];
  __shared__ float factor[3];
  follow_the_launch_before();
  int lo = 0, hi = P.n_mats - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (int(blockIdx.x) >= P.mat[mid].block_begin) lo = mid; else hi = mid - 1;
  }
  const NsIn& L = P.mat[lo];
  if (threadIdx.x < 32) {
    double s = P.partials[lo * kNormParts + threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x == 0) ns_factor(double(P.scale) / (sqrt(s) + P.eps), factor);
  }
  const int local = blockIdx.x - L.block_begin, tiles_c = (L.d + 63) / 64;
  const int r0 = local / tiles_c * 64, c0 = local % tiles_c * 64;
  const int x = (threadIdx.x & 7) * 8, y0 = threadIdx.x >> 3;        // eight columns of rows y0 and y0 + 32
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + y0 + 32 * h;
    if (r < L.p && c0 + x < L.d) ns_load8(L, P.dt, r, c0 + x, v[h]);
    else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[h][e] = 0.f;
    }
  }
  if (L.transposed) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[y0 + 32 * h][x + e] = v[h][e];
  }
  __syncthreads();
  const float f0 = factor[0], f1 = factor[1], f2 = factor[2];
  const int rows = L.transposed ? L.d : L.p, cols = L.transposed ? L.p : L.d;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = (L.transposed ? c0 : r0) + y0 + 32 * h, c = (L.transposed ? r0 : c0) + x;
    if (r < rows && c < cols) {                        // whole chunks of eight: rows of X are padded to 16
      __half a[8], b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = L.transposed ? tile[x + e][y0 + 32 * h] : v[h][e];
        split_fp16(w * f1 * f2 * f0, a[e], b[e]);
      }
      __half* to = L.X + size_t(r) * L.ldx + c;
      uint4 q;
      memcpy(&q, a, 16);
      *reinterpret_cast<uint4*>(to) = q;
      memcpy(&q, b, 16);
      *reinterpret_cast<uint4*>(to + L.plane) = q;
    }
  }
}

// ---- small matrices: all steps of a matrix in one CTA ----------------------------------------------
// X transposed, A and B in shared memory; products in fp32 FMAs, 4 x 4 sums per thread: 32 bytes of shared memory per 16 FMAs, which
// bounds it (63 % of its rate; tiles on one side of the diagonal only, or twice the width, took the same time).  One launch instead of 17
// that wait for one another: 40 us against 97 for one 64 x 64, 17 against 75 for 24 x 24; for the four layers of a block of width 64, the longest of
// 256, 102 against 95, for those of 24 blocks 103 against 322.

constexpr int kSmallM = 64, kSmallN = 256, kSmallPitch = kSmallM + 4, kSmallThreads = 512;
constexpr int kSmallSteps = 16, kSmallMats = 96;      // per launch (parameter block)

struct NsSmallMat {
  const void* M; void* out;
  long long ldm, ldo;
  int p, d;
  float scale;
};
struct NsSmallParams {
  NsSmallMat mat[kSmallMats];
  float coef[kSmallSteps][3];
  double eps;
  int steps, dt, out_dt;
};
__device__ __forceinline__ void ns_small_add(float4& to, float f, const float4& v) {
  to.x = fmaf(f, v.x, to.x);
  to.y = fmaf(f, v.y, to.y);
  to.z = fmaf(f, v.z, to.z);
  to.w = fmaf(f, v.w, to.w);
}

struct NsSmallSmem {
  float X[kSmallN][kSmallPitch];                       // X[k][i]: column k of X, zeros from row m on
  float A[kSmallM][kSmallPitch], B[kSmallM][kSmallPitch];
  double red[kSmallThreads / 32];
  float factor[3];
};

// sum over k0 <= k < k1 of U[k][i..i+3] U[k][j..j+3]; acc[c] are row j + c's four
__device__ __forceinline__ void ns_small_square(const float (*U)[kSmallPitch], int k0, int k1, int i, int j, float4 (&acc)[4]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int k = k0; k < k1; ++k) {
    const float4 x = *reinterpret_cast<const float4*>(&U[k][i]), y = *reinterpret_cast<const float4*>(&U[k][j]);
    ns_small_add(acc[0], y.x, x);
    ns_small_add(acc[1], y.y, x);
    ns_small_add(acc[2], y.z, x);
    ns_small_add(acc[3], y.w, x);
  }
}

__device__ __forceinline__ void ns_small_store(float (*to)[kSmallPitch], int i, int j, const float4 (&v)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) *reinterpret_cast<float4*>(&to[j + r][i]) = v[r];
}

// X <- a X + B X for four columns of X from c0 on, which a half-warp (`lanes`) alone reads and writes; rows i .. i + 3
__device__ __forceinline__ void ns_small_apply(NsSmallSmem& S, float a, int m4, int i, int c0, uint32_t lanes) {
  float4 sum[4];
  if (i < m4) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float4 x = *reinterpret_cast<const float4*>(&S.X[c0 + r][i]);
      sum[r] = make_float4(a * x.x, a * x.y, a * x.z, a * x.w);
    }
#pragma unroll 2
    for (int k = 0; k < m4; k += 4) {
      float4 b[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) b[q] = *reinterpret_cast<const float4*>(&S.B[k + q][i]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float4 x = *reinterpret_cast<const float4*>(&S.X[c0 + r][k]);
        ns_small_add(sum[r], x.x, b[0]);
        ns_small_add(sum[r], x.y, b[1]);
        ns_small_add(sum[r], x.z, b[2]);
        ns_small_add(sum[r], x.w, b[3]);
      }
    }
  }
  __syncwarp(lanes);
  if (i < m4) {
#pragma unroll
    for (int r = 0; r < 4; ++r) *reinterpret_cast<float4*>(&S.X[c0 + r][i]) = sum[r];
  }
}

__global__ void __launch_bounds__(kSmallThreads)
ns_small_kernel(const __grid_constant__ NsSmallParams P) {
  extern __shared__ uint8_t smem_raw[];
  NsSmallSmem& S = *reinterpret_cast<NsSmallSmem*>(smem_raw);
  const NsSmallMat& L = P.mat[blockIdx.x];
  const int tid = threadIdx.x, total = L.p * L.d;
  const bool transposed = L.p > L.d;
  const int m = transposed ? L.d : L.p, n = transposed ? L.p : L.d;
  const int m4 = (m + 3) & ~3;
  double s = 0.0;
  for (int k0 = tid; k0 < total; k0 += 8 * kSmallThreads) {        // eight loads on their way at once
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = k0 + u * kSmallThreads, r = k / L.d, c = k - r * L.d;
      const size_t at = size_t(r) * size_t(L.ldm) + c;
      if (k < total) v[u] = P.dt == DP_F32 ? static_cast<const float*>(L.M)[at] : to_f32(static_cast<const __nv_bfloat16*>(L.M)[at]);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = k0 + u * kSmallThreads, r = k / L.d, c = k - r * L.d;
      if (k >= total) continue;
      if (transposed) S.X[r][c] = v[u]; else S.X[c][r] = v[u];
      s = fma(double(v[u]), double(v[u]), s);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((tid & 31) == 0) S.red[tid >> 5] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.0;
    for (int w = 0; w < kSmallThreads / 32; ++w) s += S.red[w];
    ns_factor(1.0 / (sqrt(s) + P.eps), S.factor);
  }
  __syncthreads();
  const float f0 = S.factor[0], f1 = S.factor[1], f2 = S.factor[2];
  for (int k = tid; k < ((n + 3) & ~3) * kSmallM; k += kSmallThreads) {
    float& x = S.X[k / kSmallM][k % kSmallM];
    x = k % kSmallM < m && k / kSmallM < n ? x * f1 * f2 * f0 : 0.f;
  }
  __syncthreads();
  // products of 64 x 64: 256 threads on each half of the sum, the second's added by the first
  const int half = tid >> 8, i = 4 * (tid & 15), j = 4 * (tid >> 4 & 15);
  const bool here = i < m && j < m;
  const int n_half = (n + 1) / 2, m_half = m4 / 2;
  for (int step = 0; step < P.steps; ++step) {
    const float a = P.coef[step][0], b = P.coef[step][1], c = P.coef[step][2];
    float4 acc[4];
    if (here) ns_small_square(S.X, half ? n_half : 0, half ? n : n_half, i, j, acc);
    if (here && half) ns_small_store(S.A, i, j, acc);
    __syncthreads();
    if (here && !half) {
#pragma unroll
      for (int r = 0; r < 4; ++r) ns_small_add(acc[r], 1.f, *reinterpret_cast<const float4*>(&S.A[j + r][i]));
      ns_small_store(S.A, i, j, acc);
    }
    __syncthreads();
    if (here) ns_small_square(S.A, half ? m_half : 0, half ? m4 : m_half, i, j, acc);   // rows from m on are zeros
    if (here && half) ns_small_store(S.B, i, j, acc);
    __syncthreads();
    if (here && !half) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float4 x = *reinterpret_cast<const float4*>(&S.A[j + r][i]);
        ns_small_add(acc[r], 1.f, *reinterpret_cast<const float4*>(&S.B[j + r][i]));
        acc[r] = make_float4(fmaf(c, acc[r].x, b * x.x), fmaf(c, acc[r].y, b * x.y), fmaf(c, acc[r].z, b * x.z), fmaf(c, acc[r].w, b * x.w));
      }
      ns_small_store(S.B, i, j, acc);
    }
    __syncthreads();
    const uint32_t lanes = 0xffffu << (tid & 16);
    for (int c0 = 4 * (tid >> 4); c0 < n; c0 += 4 * (kSmallThreads / 16)) ns_small_apply(S, a, m4, i, c0, lanes);
    __syncthreads();
  }
  for (int k = tid; k < total; k += kSmallThreads) {
    const int r = k / L.d, c = k - r * L.d;
    const size_t at = size_t(r) * size_t(L.ldo) + c;
    const float v = L.scale * (transposed ? S.X[r][c] : S.X[c][r]);
    if (P.out_dt == DP_F32) static_cast<float*>(L.out)[at] = v; else static_cast<__nv_bfloat16*>(L.out)[at] = __float2bfloat16_rn(v);
  }
}

// ---- host ----------------------------------------------------------------------------------------

bool ns_small(const dp_matrix_desc* mats, int n, int steps) {
  for (int k = 0; k < n; ++k)
    if (std::min(mats[k].p, mats[k].d) > kSmallM || std::max(mats[k].p, mats[k].d) > kSmallN) return false;
  return steps <= kSmallSteps;
}

dp_status ns_small_launch(const dp_matrix_desc* mats, int n, dp_dtype dt, dp_dtype out_dt, const float* coefs, int steps, float eps,
                          cudaStream_t st) {
  NsSmallParams P;
  P.steps = steps; P.dt = dt; P.out_dt = out_dt; P.eps = eps;
  std::memcpy(P.coef, coefs, sizeof(float) * 3 * size_t(steps));
  DP_SET_UP_ONCE((const void*)ns_small_kernel, DP_CUDA_OK(allow_shared(ns_small_kernel, sizeof(NsSmallSmem))));
  for (int k0 = 0; k0 < n; k0 += kSmallMats) {
    const int here = std::min(kSmallMats, n - k0);
    for (int k = 0; k < here; ++k) {
      const dp_matrix_desc& D = mats[k0 + k];
      P.mat[k] = {D.M, D.out, D.ldm, D.ldo, D.p, D.d, D.scale};
    }
    ns_small_kernel<<<here, kSmallThreads, sizeof(NsSmallSmem), st>>>(P);
    DP_LAUNCH_OK();
  }
  return DP_OK;
}

struct NsShape {
  int m, n, ldx, lda;
  bool transposed;
  size_t x_bytes, a_bytes;             // of both planes
  NsShape() = default;
  explicit NsShape(const dp_matrix_desc& D) {
    transposed = D.p > D.d;
    m = std::min(D.p, D.d);
    n = std::max(D.p, D.d);
    ldx = (n + 15) / 16 * 16;
    lda = (m + 15) / 16 * 16;
    x_bytes = align_up(2 * size_t(m) * ldx * sizeof(__half), 256);
    a_bytes = align_up(2 * size_t(m) * lda * sizeof(__half), 256);
  }
  size_t bytes() const { return 2 * x_bytes + 7 * a_bytes; }
};

// The power of two that brings values of at most `bound` below half of fp16's largest.  (Bounds below 1e-30 are those of results that fp32
// does not hold.)
float scale_for(double bound) {
  int e = 0;
  frexp(std::max(bound, 1e-30), &e);                 // bound < 2^e
  return float(ldexp(1.0, 15 - e));
}

// Bounds of a step on a matrix whose singular values are at most s: of |a + b l + c l^2| for l <= s^2, of |a x + b x^3 + c x^5|.
void step_bounds(double a, double b, double c, double s, double* poly, double* next) {
  auto f = [&](double l) { return std::fabs(a + b * l + c * l * l); };
  auto g = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
  *poly = std::max(std::fabs(a), f(s * s));
  *next = g(s);
  if (c != 0.0) {
    const double l = -b / (2 * c);
    if (l > 0 && l < s * s) *poly = std::max(*poly, f(l));
    const double disc = 9 * b * b - 20 * a * c;      // a + 3 b y + 5 c y^2 = 0, y = x^2
    if (disc >= 0)
      for (int sign = -1; sign <= 1; sign += 2) {
        const double y = (-3 * b + sign * std::sqrt(disc)) / (10 * c);
        if (y > 0 && y < s * s) *next = std::max(*next, g(std::sqrt(y)));
      }
  } else if (b != 0.0) {
    const double y = -a / (3 * b);
    if (y > 0 && y < s * s) *next = std::max(*next, g(std::sqrt(y)));
  }
}

// A step: B = c A A' + a I of A' = A + q I, or (added) c A A + b A + a I; bounds of singular values before and after, and of |B|.
struct NsStep { double a, b, c, q, before, after, poly; bool added; };

constexpr double kMargin = 1.01;                     // on a bound, for what the products round
constexpr double kMaxBound = 1e6;

bool plan_steps(const float* coefs, int steps, std::vector<NsStep>& plan) {
  double s = 1.0;
  for (int k = 0; k < steps; ++k) {
    const double a = coefs[3 * k], b = coefs[3 * k + 1], c = coefs[3 * k + 2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    NsStep S{};
    S.before = s * kMargin;
    step_bounds(a, b, c, s, &S.poly, &S.after);
    if (!(S.poly <= kMaxBound) || !(S.after <= kMaxBound)) return false;
    S.a = a;
    S.c = c;
    // A' within a few times A: two or three bits of its terms
    S.added = std::fabs(b) > 16.0 * s * s * std::fabs(c);
    if (S.added) S.b = b;
    else if (c != 0.0) S.q = b / c;
    S.poly *= kMargin;
    S.after *= kMargin;
    s = S.after;
    plan.push_back(S);
  }
  return true;
}

// Steps from k on that go by A alone, given how far A's error may grow on the way (see the top of the file).
int fused_steps(const std::vector<NsStep>& plan, size_t k, double most) {
  double growth = 1.0;
  int n = 1;
  for (; k + n < plan.size(); ++n) {
    growth *= plan[k + n - 1].poly * plan[k + n - 1].poly;
    if (growth > most) break;
  }
  return n;
}

template <Product kProduct, bool kPair>
dp_status ns_launch(const NsParams& P, cudaStream_t st) {
  auto* kernel = ns_product_kernel<kProduct, kPair>;
  DP_SET_UP_ONCE((const void*)kernel, DP_CUDA_OK(allow_shared(kernel, kSmemBytes)));
  const int units = kPair ? sm_count() / 2 : sm_count();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((kPair ? 2 : 1) * std::min(P.total_items, units));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {2u, 1u, 1u};
  cfg.attrs = attr;
  cfg.numAttrs = kPair ? 2 : 1;
  DP_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, P));
  ++g_kernel_launches;
  return DP_OK;
}

int tiles_of(Product product, int m, int n, int tile) {
  const int tm = ceil_div(m, tile);
  return product == kApply ? tm * ceil_div(n, tile) : tm * (tm + 1) / 2;
}

// How a group of matrices runs: on CTA pairs or single CTAs, the same for all products, since symmetric matrices are stored by the tile; and
// how far A's error may grow in fused steps, 1 where each is by itself.  Whichever takes less time in whole waves of K steps, a launch counting
// three more.  A pair's K step is 1.7 times as long for twice the work per CTA: a single CTA's reads 64 KB of shared memory's tiles anew for half
// of the MMAs (tensor pipe at 45 %).  Pairs against single CTAs: layers of 6 blocks of width 768 in fp32 1.61 ms against 1.88, of 24 of 1024 to bf16
// 11.9 against 12.9; of one of 768 in fp32, which leave pairs without work, 0.66 against 0.58.
struct NsForm { bool pair; double growth; };
NsForm choose_form(const std::vector<NsShape>& shapes, const std::vector<NsStep>& plan, bool bf16_out) {
  int least_m = shapes[0].m;
  for (const NsShape& s : shapes) least_m = std::min(least_m, s.m);
  const double most = bf16_out ? 150.0 : least_m >= 640 ? 13.0 : 1.0;   // three, two and one of the usual quintic's steps
  NsForm best{};
  double least = INFINITY;
  for (int form = 0; form < 4; ++form) {
    const NsForm f{(form & 1) != 0, form & 2 ? most : 1.0};
    const int tile = f.pair ? 256 : 128, units = f.pair ? sm_count() / 2 : sm_count();
    double cost[3];
    for (const Product q : {kGram, kSym, kApply}) {
      long long tiles = 0, work = 0, longest = 0;
      for (const NsShape& s : shapes) {
        const long long t = tiles_of(q, s.m, s.n, tile), k = ceil_div(q == kGram ? s.n : s.m, kBK);
        tiles += t;
        work += t * k;
        longest = std::max(longest, k);
      }
      const double waves = double((tiles + units - 1) / units);
      cost[q] = 3.0 + (f.pair ? 1.7 : 1.0) * std::max(double(longest), waves * double(work) / double(tiles));
    }
    double all = 0;
    for (size_t k = 0; k < plan.size();) {
      const int n = fused_steps(plan, k, f.growth);
      all += cost[kGram] + (1 + 4 * (n - 1)) * cost[kSym] + cost[kApply];
      k += n;
    }
    if (all < least) { least = all; best = f; }
  }
  return best;
}

// One product of all matrices of a group.
dp_status ns_product(Product product, NsParams& P, bool pair, cudaStream_t st) {
  if (pair) {
    return product == kGram ? ns_launch<kGram, true>(P, st) : product == kSym ? ns_launch<kSym, true>(P, st)
                                                                              : ns_launch<kApply, true>(P, st);
  }
  return product == kGram ? ns_launch<kGram, false>(P, st) : product == kSym ? ns_launch<kSym, false>(P, st)
                                                                             : ns_launch<kApply, false>(P, st);
}

enum { kX0, kX1, kA, kDiagonal, kT, kB0, kB, kB1, kB2, kPlaces };
struct NsPlace {
  NsShape s;
  __half* at[kPlaces];
  CUtensorMap load[kPlaces], store[kPlaces];
};

dp_status ns_group(const dp_matrix_desc* mats, int n, dp_dtype dt, dp_dtype out_dt, const std::vector<NsStep>& plan, float eps,
                   double* partials, char* base, int* dev_status, cudaStream_t st) {
  // The matrices kept of each: X and the next one; A and the copy of its diagonal's tiles; B; a product on the way from one A to the
  // next; the product of the Bs of fused steps and the next one.  The last four are as large as A.
  std::vector<NsPlace> places(n);
  std::vector<NsShape> shapes;
  NsInParams In;
  int blocks = 0;
  for (int k = 0; k < n; ++k) {
    NsPlace& p = places[k];
    p.s = NsShape(mats[k]);
    shapes.push_back(p.s);
    for (int j = 0; j < kPlaces; ++j) {
      const bool x = j == kX0 || j == kX1;
      p.at[j] = reinterpret_cast<__half*>(base);
      base += x ? p.s.x_bytes : p.s.a_bytes;
      const int ld = x ? p.s.ldx : p.s.lda, cols = x ? p.s.n : p.s.m;
      dp_status r = make_tmap_bf16_3d(&p.load[j], p.at[j], ld, cols, p.s.m, 2, 64, 64);
      if (r == DP_OK) r = make_tmap_store16_3d(&p.store[j], p.at[j], ld, cols, p.s.m, 2);
      if (r != DP_OK) return r;
    }
    In.mat[k] = {mats[k].M, mats[k].ldm, (long long)p.s.m * p.s.ldx, p.at[kX0], mats[k].p, mats[k].d, p.s.ldx, p.s.transposed,
                 aligned16(mats[k].M) && mats[k].ldm * (dt == DP_F32 ? 4 : 2) % 16 == 0, blocks};
    blocks += ceil_div(mats[k].p, 64) * ceil_div(mats[k].d, 64);
  }
  double sx = scale_for(plan[0].before);
  In.n_mats = n; In.dt = dt; In.partials = partials; In.eps = eps; In.scale = float(sx);
  ns_norm_kernel<<<n * kNormParts, 256, 0, st>>>(In);
  DP_LAUNCH_OK();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  DP_CUDA_OK(cudaLaunchKernelEx(&cfg, ns_split_kernel, In));
  ++g_kernel_launches;

  const NsForm form = choose_form(shapes, plan, out_dt == DP_BF16);
  NsParams P;
  P.n_mats = n; P.out_dt = out_dt; P.dev_status = dev_status; P.wait_limit = g_wait_limit;
  // D = f_acc * P Q + f_add * add [+ diagonal I: in D, or in the copy of the diagonal's tiles]
  auto product = [&](Product kind, int left, int right, int to, double f_acc, double f_add, double diagonal, bool copy, bool last) {
    P.total_items = 0;
    P.f_acc = float(f_acc); P.f_add = float(f_add); P.diagonal = float(diagonal);
    P.copy = copy;
    P.shifted = kind == kSym && left == kA && right == kA && f_add == 0.0;
    for (int i = 0; i < n; ++i) {
      const NsPlace& p = places[i];
      NsMat& L = P.mat[i];
      L = {};
      L.M = p.s.m;
      L.N = kind == kApply ? p.s.n : p.s.m;
      L.ksteps = ceil_div(kind == kGram ? p.s.n : p.s.m, kBK);
      L.out_scale = 1.f;
      L.item_begin = P.total_items;
      P.total_items += tiles_of(kind, p.s.m, p.s.n, form.pair ? 256 : 128);
      P.tmP[i] = p.load[left];
      P.tmQ[i] = p.load[right];
      P.tmD[i] = p.store[to];
      P.tmE[i] = copy ? p.store[kDiagonal] : p.load[kDiagonal];
      if (f_add != 0.0) { L.add = p.at[kA]; L.plane_add = (long long)p.s.m * p.s.lda; L.ld_add = p.s.lda; }
      if (last) { L.out = mats[i].out; L.ldo = mats[i].ldo; L.transposed = p.s.transposed; L.out_scale = mats[i].scale; }
    }
    return ns_product(kind, P, form.pair, st);
  };
  int x = kX0;
  for (size_t k = 0; k < plan.size();) {
    const int fused = fused_steps(plan, k, form.growth);
    int acc = kB0;                                     // the product of the group's Bs so far
    double s_acc = 0, sA = 0, acc_bound = 1;
    for (int f = 0; f < fused; ++f) {
      const NsStep& S = plan[k + f];
      const double old_sA = sA, a_bound = S.before * S.before;
      sA = scale_for(a_bound + std::fabs(S.q));
      const bool copy = !S.added;
      dp_status r;
      if (f == 0) {
        r = product(kGram, x, x, kA, sA / (sx * sx), 0.0, S.q * sA, copy, false);
      } else {
        // A <- B A B; B of the step before is in kB0 (the group's first) or kB
        const NsStep& before = plan[k + f - 1];
        const int B = f == 1 ? kB0 : kB;
        const double sB = scale_for(before.poly), sT = scale_for(before.before * before.after);
        r = product(kSym, B, kA, kT, sT / (sB * old_sA), 0.0, 0.0, false, false);
        if (r == DP_OK) r = product(kSym, kT, B, kA, sA / (sT * sB), 0.0, S.q * sA, copy, false);
      }
      if (r != DP_OK) return r;
      const double sB = scale_for(S.poly);
      const int to = f == 0 ? kB0 : kB;
      r = product(kSym, kA, kA, to, S.c * sB / (sA * sA), S.b * sB / sA, S.a * sB, false, false);
      if (r != DP_OK) return r;
      acc_bound *= S.poly;
      if (f == 0) {
        s_acc = sB;
      } else {
        const int next = acc == kB1 ? kB2 : kB1;
        const double s_next = scale_for(acc_bound);
        r = product(kSym, kB, acc, next, s_next / (sB * s_acc), 0.0, 0.0, false, false);
        if (r != DP_OK) return r;
        acc = next;
        s_acc = s_next;
      }
    }
    k += fused;
    const bool last = k == plan.size();
    const int next = x == kX0 ? kX1 : kX0;
    const double to = last ? 1.0 : scale_for(plan[k].before);
    const dp_status r = product(kApply, acc, x, next, to / (s_acc * sx), 0.0, 0.0, false, last);
    if (r != DP_OK) return r;
    x = next;
    sx = to;
  }
  return DP_OK;
}

size_t ns_partial_bytes(int n) { return size_t(std::min(n, kNsMaxMats)) * kNormParts * sizeof(double); }

dp_status check_matrix(const dp_matrix_desc& D, bool pointers) {
  if (D.p <= 0 || D.d <= 0) return DP_ERR_INVALID_ARG;
  if (D.p > (1 << 20) || D.d > (1 << 20)) return DP_ERR_UNSUPPORTED;
  if (pointers && (!D.M || !D.out || D.ldm < D.d || D.ldo < D.d || !std::isfinite(D.scale))) return DP_ERR_INVALID_ARG;
  return DP_OK;
}

// No two matrices share an output, and no output is another matrix's input: matrices of a call run together.
bool distinct_outputs(const dp_matrix_desc* mats, int n) {
  std::vector<std::pair<const void*, int>> outs(n);
  for (int k = 0; k < n; ++k) outs[k] = {mats[k].out, k};
  std::sort(outs.begin(), outs.end());
  for (int k = 1; k < n; ++k)
    if (outs[k].first == outs[k - 1].first) return false;
  for (int k = 0; k < n; ++k) {
    const auto at = std::lower_bound(outs.begin(), outs.end(), std::make_pair(mats[k].M, 0));
    if (at != outs.end() && at->first == mats[k].M && at->second != k) return false;
  }
  return true;
}

// The order in which matrices are taken: long sums first, so that the tiles of a last wave are the short ones.
std::vector<int> ns_order(const dp_matrix_desc* mats, int n) {
  std::vector<int> order(n);
  for (int k = 0; k < n; ++k) order[k] = k;
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) {
    return std::max(mats[a].p, mats[a].d) > std::max(mats[b].p, mats[b].d);
  });
  return order;
}

// Launches' groups: of equal size, every so-manieth matrix of the order, so that they are alike.  They run one after the other in the
// same memory.
int ns_groups(int n) { return ceil_div(n, kNsMaxMats); }

}  // namespace

}  // namespace dpg

using namespace dpg;

extern "C" {

size_t dp_orthogonalize_ws_bytes(const dp_matrix_desc* mats, int32_t n) try {
  if (!mats || n <= 0) return 0;
  for (int k = 0; k < n; ++k)
    if (check_matrix(mats[k], false) != DP_OK) return 0;
  const std::vector<int> order = ns_order(mats, n);
  const int groups = ns_groups(n);
  size_t most = 0;
  for (int g = 0; g < groups; ++g) {
    size_t need = 0;
    for (int k = g; k < n; k += groups) need += NsShape(mats[order[k]]).bytes();
    most = std::max(most, need);
  }
  return ns_partial_bytes(n) + most;
} catch (...) {
  return 0;
}

int32_t dp_debug_orthogonalize_form(const dp_matrix_desc* mats, int32_t n, dp_dtype out_dt, const float* coefs, int32_t steps) try {
  if (!mats || n <= 0 || !coefs || steps <= 0) return -1;
  for (int k = 0; k < n; ++k)
    if (check_matrix(mats[k], false) != DP_OK) return -1;
  std::vector<NsStep> plan;
  if (!plan_steps(coefs, steps, plan)) return -1;
  if (ns_small(mats, n, steps)) return 0;
  const std::vector<int> order = ns_order(mats, n);
  const int groups = ns_groups(n);
  std::vector<NsShape> shapes;
  for (int k = 0; k < n; k += groups) shapes.push_back(NsShape(mats[order[k]]));
  const NsForm form = choose_form(shapes, plan, out_dt == DP_BF16);
  return 2 * fused_steps(plan, 0, form.growth) + (form.pair ? 1 : 0);
} catch (...) {
  return -1;
}

dp_status dp_orthogonalize(const dp_matrix_desc* mats, int32_t n, dp_dtype dt, dp_dtype out_dt, const float* coefs, int32_t steps,
                           float eps, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) try {
  if (!mats || n <= 0 || !coefs || steps <= 0 || !std::isfinite(eps) || eps < 0.f) return DP_ERR_INVALID_ARG;
  if ((dt != DP_F32 && dt != DP_BF16) || (out_dt != DP_F32 && out_dt != DP_BF16)) return DP_ERR_INVALID_ARG;
  for (int k = 0; k < n; ++k) {
    const dp_status r = check_matrix(mats[k], true);
    if (r != DP_OK) return r;
    if (!on_boundary(dt == DP_F32 ? 4 : 2, mats[k].M) || !on_boundary(out_dt == DP_F32 ? 4 : 2, mats[k].out)) return DP_ERR_ALIGNMENT;
  }
  if (!distinct_outputs(mats, n)) return DP_ERR_INVALID_ARG;
  std::vector<NsStep> plan;
  if (!plan_steps(coefs, steps, plan)) return DP_ERR_INVALID_ARG;
  if (!ws || ws_bytes < dp_orthogonalize_ws_bytes(mats, n)) return DP_ERR_WORKSPACE;
  if (!aligned16(ws)) return DP_ERR_ALIGNMENT;
  if (ns_small(mats, n, steps)) return ns_small_launch(mats, n, dt, out_dt, coefs, steps, eps, (cudaStream_t)stream);
  const std::vector<int> order = ns_order(mats, n);
  const int groups = ns_groups(n);
  for (int g = 0; g < groups; ++g) {
    std::vector<dp_matrix_desc> group;
    for (int k = g; k < n; k += groups) group.push_back(mats[order[k]]);
    const dp_status r = ns_group(group.data(), int(group.size()), dt, out_dt, plan, eps, static_cast<double*>(ws),
                                 static_cast<char*>(ws) + ns_partial_bytes(n), dev_status, (cudaStream_t)stream);
    if (r != DP_OK) return r;
  }
  return DP_OK;
} catch (...) {                                        // host memory for a call of this size
  return DP_ERR_UNSUPPORTED;
}

}  // extern "C"
