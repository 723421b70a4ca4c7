// psa_ffn / psa_ffn_bwd: the gated feed-forward block of a decoder layer,
//     G = X Wg,  U = X Wu,  H = silu(G) * U,  Y = H Wd,         silu(g) = g * sigmoid(g),
// and its gradient for dY:
//     dH = dY Wd^T,  dU = dH * silu(G),  dG = dH * U * sigmoid(G) * (1 + G * (1 - sigmoid(G))),
//     dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU,  dWd = H^T dY.
// Six kinds of product, one kernel: C[M, N] = sum over K of A B with bf16 operands and fp32 sums in TMEM.  An operand lies
// in memory with K innermost (K-major) or with M or N innermost (MN-major); tcgen05.mma reads either from a 128-byte-
// swizzled tile, so no matrix is ever transposed in memory.  What differs is the end of a tile:
//     the forward's first product computes a tile of G and the same tile of U, so that one thread holds both values of
//     an element and writes H (and, for a backward pass, G and U) from registers;
//     dH is never written: its tile meets G and U in registers and leaves as dG, dU and H;
//     dX sums over two pairs of operands, one after the other; dWg and dWu are two outputs of one launch.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "psa.h"
#include "psa_device.cuh"
#include "psa_internal.h"
#include "psa_launch.cuh"
#include "psa_tensormap.h"

namespace psa {
namespace {

using namespace dev;

constexpr int kBK = 64;                // K per stage: one 128-byte swizzle row of bf16
constexpr int kChunk = 64;             // columns of an MN-major sub-tile
constexpr int kSmCount = 148;

enum Epilogue {
  kEpiOut,        // C rounded to bf16, or an fp32 partial sum where K is split
  kEpiGate,       // columns [0, BN/2) are G, [BN/2, BN) are U of the same features
  kEpiGateBwd,    // C is dH
};

struct GemmParams {
  int32_t M, N;                // rows and columns of one output
  int32_t k_tiles;             // stages of one operand pair
  int32_t k_pairs;             // operand pairs that are summed
  int32_t n_tiles;             // tiles along N of one output
  int32_t n_outputs;           // outputs side by side (each with a B of its own)
  int32_t splits;              // parts of K
  __nv_bfloat16 *out[2];       // kEpiOut: C;  kEpiGate: G, U (may be null);  kEpiGateBwd: dG, dU
  __nv_bfloat16 *h;            // kEpiGate, kEpiGateBwd
  const __nv_bfloat16 *gate, *up;   // kEpiGateBwd
  float* partial;              // [splits][n_outputs][M][N]
  int32_t* status;
};

__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }

// dH, G, U of an element -> dG and dU (over G and U) and H.
__device__ __forceinline__ void gate_bwd(float dh, float& g, float& u, float& h) {
  const float s = sigmoid(g), act = g * s;
  h = act * u;
  const float dg = dh * u * (s * (1.0f + g * (1.0f - s)));
  u = dh * act;
  g = dg;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight fp32 values as 16 bytes of bf16.
__device__ __forceinline__ uint4 pack8(const float* v) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void unpack8(const uint4& w, float* v) {
  v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
  v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
}

// ---------------------------------------------------------------- one CTA per tile of 128 x 128
// Warps 0-3: end of the tile (TMEM lane = row of the tile), warp 4: TMA, warp 5: UMMA.
constexpr int kSmallBM = 128, kSmallBN = 128, kSmallStages = 3, kSmallThreads = 192;
constexpr uint32_t kSmallStageBytes = uint32_t(kSmallBM + kSmallBN) * kBK * 2;
constexpr uint32_t kSmallSmem = kSmallStages * kSmallStageBytes + 1024 + 256;

template <bool A_MN, bool B_MN, int EPI>
__global__ void __launch_bounds__(kSmallThreads)
ffn_small_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap a1,
                 const __grid_constant__ CUtensorMap b0, const __grid_constant__ CUtensorMap b1, const GemmParams prm) {
  constexpr int kBN = kSmallBN, kStages = kSmallStages;
  constexpr int kTileN = EPI == kEpiGate ? kBN / 2 : kBN;      // features per tile
  constexpr uint32_t kABytes = kSmallBM * kBK * 2, kSub = kChunk * kBK * 2;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + kStages * kSmallStageBytes;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (kStages + s); };
  const uint32_t done = bars + 16u * kStages;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + kStages * kSmallStageBytes + 128);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_base + kStages * kSmallStageBytes + 136);
  const WaitCtx wctx{abort_flag, prm.status, kWaitLimitClocks};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  const int m0 = int(blockIdx.x) * kSmallBM;
  const int sel = int(blockIdx.y) / prm.n_tiles, n0 = (int(blockIdx.y) % prm.n_tiles) * kTileN;
  const int total = prm.k_tiles * prm.k_pairs;
  const int it0 = int(int64_t(total) * blockIdx.z / prm.splits), it1 = int(int64_t(total) * (blockIdx.z + 1) / prm.splits);

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(done, 1);
    fence_mbar_init();
  }
  if (warp == 5) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kBN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 4) {
    if (lane == 0) {
      int n = 0;   // stages filled
      for (int it = it0; it < it1; ++it, ++n) {
        const int s = n % kStages;
        if (n >= kStages) mbar_wait(empty(s), (n / kStages - 1) & 1, wctx);
        if (*abort_flag) break;
        const bool second = it >= prm.k_tiles;
        const int k0 = (second ? it - prm.k_tiles : it) * kBK;
        const CUtensorMap* am = second ? &a1 : &a0;
        const uint32_t sa = base + s * kSmallStageBytes, sb = sa + kABytes;
        mbar_expect_tx(full(s), kSmallStageBytes);
        if (A_MN) {
          for (int c = 0; c < kSmallBM / kChunk; ++c) tma_load_3d(sa + c * kSub, am, m0 + c * kChunk, 0, k0, full(s));
        } else {
          tma_load_3d(sa, am, k0, 0, m0, full(s));
        }
        if (EPI == kEpiGate) {   // the same features of two weights
          tma_load_3d(sb, &b0, n0, 0, k0, full(s));
          tma_load_3d(sb + kSub, &b1, n0, 0, k0, full(s));
        } else {
          const CUtensorMap* bm = second || sel ? &b1 : &b0;
          if (B_MN) {
            for (int c = 0; c < kBN / kChunk; ++c) tma_load_3d(sb + c * kSub, bm, n0 + c * kChunk, 0, k0, full(s));
          } else {
            tma_load_3d(sb, bm, k0, 0, n0, full(s));
          }
        }
      }
      if (*abort_flag) {   // shared memory must outlive the copies in flight
        const long long t0 = clock64();
        for (int i = n > kStages ? n - kStages : 0; i < n; ++i)
          while (!mbar_try_wait(full(i % kStages), (i / kStages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
      }
    }
    __syncwarp();
  } else if (warp == 5) {
    const uint32_t issuer = elect_one();
    constexpr uint32_t idesc = umma_idesc_bf16(kSmallBM, kBN, A_MN, B_MN);
    for (int it = it0, n = 0; it < it1; ++it, ++n) {
      const int s = n % kStages;
      mbar_wait(full(s), (n / kStages) & 1, wctx);
      tc_fence_after();
      const uint32_t sa = base + s * kSmallStageBytes;
      const uint32_t a = smem_desc_lo(sa, A_MN ? kSub : 16), b = smem_desc_lo(sa + kABytes, B_MN ? kSub : 16);
#pragma unroll
      for (int kk = 0; kk < kBK / 16; ++kk)
        umma_ss_w(tmem, a + kk * ((A_MN ? 2048 : 32) >> 4), b + kk * ((B_MN ? 2048 : 32) >> 4), idesc, n > 0 || kk > 0, issuer);
      umma_commit_w(empty(s), issuer);
    }
    umma_commit_w(done, issuer);
    __syncwarp();
  } else {
    mbar_wait(done, 0, wctx);
    tc_fence_after();
    const int row = m0 + warp * 32 + lane;
    const uint32_t lanes = tmem + (uint32_t(warp * 32) << 16);
    const bool live = row < prm.M && !*abort_flag;
    uint32_t v[32];
    if (EPI == kEpiGate) {
      for (int c = 0; c < kTileN; c += 32) {
        uint32_t u[32];
        tmem_ld32_wait(lanes + c, v);
        tmem_ld32_wait(lanes + kTileN + c, u);
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
          const int col = n0 + c + j;
          const int64_t at = int64_t(row) * prm.N + col;
          if (!live || col >= prm.N || !PSA_IN_BOUNDS(at + 7, int64_t(prm.M) * prm.N, prm.status)) continue;
          float g[8], w[8], h[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            g[i] = __uint_as_float(v[j + i]);
            w[i] = __uint_as_float(u[j + i]);
            h[i] = g[i] * sigmoid(g[i]) * w[i];
          }
          if (prm.out[0]) {
            *reinterpret_cast<uint4*>(prm.out[0] + at) = pack8(g);
            *reinterpret_cast<uint4*>(prm.out[1] + at) = pack8(w);
          }
          *reinterpret_cast<uint4*>(prm.h + at) = pack8(h);
        }
      }
    } else {
      for (int c = 0; c < kTileN; c += 32) {
        tmem_ld32_wait(lanes + c, v);
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
          const int col = n0 + c + j;
          const int64_t at = int64_t(row) * prm.N + col;
          if (!live || col >= prm.N || !PSA_IN_BOUNDS(at + 7, int64_t(prm.M) * prm.N, prm.status)) continue;
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[j + i]);
          if (EPI == kEpiGateBwd) {
            float g[8], u[8], h[8];
            unpack8(*reinterpret_cast<const uint4*>(prm.gate + at), g);
            unpack8(*reinterpret_cast<const uint4*>(prm.up + at), u);
#pragma unroll
            for (int i = 0; i < 8; ++i) gate_bwd(x[i], g[i], u[i], h[i]);
            *reinterpret_cast<uint4*>(prm.out[0] + at) = pack8(g);
            *reinterpret_cast<uint4*>(prm.out[1] + at) = pack8(u);
            *reinterpret_cast<uint4*>(prm.h + at) = pack8(h);
          } else if (prm.splits > 1) {
            float4* dst = reinterpret_cast<float4*>(prm.partial + (int64_t(blockIdx.z) * prm.n_outputs + sel) * prm.M * prm.N + at);
            dst[0] = make_float4(x[0], x[1], x[2], x[3]);
            dst[1] = make_float4(x[4], x[5], x[6], x[7]);
          } else {
            *reinterpret_cast<uint4*>((sel ? prm.out[1] : prm.out[0]) + at) = pack8(x);
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 5) {
    tc_fence_after();
    tmem_dealloc(tmem, kBN);
  }
}

// ---------------------------------------------------------------- two CTAs per tile of 256 x 256
// A persistent kernel: 74 clusters of two CTAs take every 74th tile.  A tile's product is one UMMA stream of the pair
// (M = 256, N = 256): each CTA loads its 128 rows of A and 128 of the tile's 256 columns of B, so a stage brings 32 KB to each
// SM for the work of which a CTA alone would need 48.  The accumulator takes half of TMEM: while the end of one tile
// drains it, the next tile's UMMAs fill the other half.
// Warps: 0 TMA, 1 UMMA (in the CTA of rank 0), 2 TMEM, 4-7 the end of a tile, each for 32 rows of its CTA.
// A result leaves by TMA stores of 32 rows x 64 columns, from four buffers that each warp owns: no barrier but the warp's own,
// and the tensor map clips what lies behind the last row or column.
constexpr int kBigBM = 256, kBigBN = 256, kBigStages = 5, kBigThreads = 256, kBigBufs = 4;
constexpr uint32_t kBigHalf = 128 * kBK * 2;                       // one operand's half of a stage
constexpr uint32_t kBigStageBytes = 2 * kBigHalf;
constexpr uint32_t kBufBytes = 32 * 64 * 2;
constexpr uint32_t kBigBufsAt = kBigStages * kBigStageBytes;
constexpr uint32_t kBigBarsAt = kBigBufsAt + 4 * kBigBufs * kBufBytes;
constexpr uint32_t kBigSmem = kBigBarsAt + 256 + 1024;
static_assert(kBigSmem <= 227 * 1024, "shared memory of one CTA");

struct BigMaps {
  CUtensorMap a[2], b[2], out[3], in[2];    // out: C of both outputs, or G / dG, U / dU, H;  in: G, U
};

template <bool A_MN, bool B_MN, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kBigThreads, 1)
ffn_big_kernel(const __grid_constant__ BigMaps maps, const GemmParams prm) {
  constexpr int kTileN = EPI == kEpiGate ? kBigBN / 2 : kBigBN;
  constexpr uint32_t kSub = kChunk * kBK * 2;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + kBigBarsAt;
  auto full = [&](int s) { return bars + 8u * s; };                    // of rank 0: both CTAs' loads
  auto empty = [&](int s) { return bars + 8u * (kBigStages + s); };
  auto acc_full = [&](int i) { return bars + 8u * (2 * kBigStages + i); };
  auto acc_empty = [&](int i) { return bars + 8u * (2 * kBigStages + 2 + i); };   // of rank 0: both CTAs' warps
  auto in_full = [&](int w) { return bars + 8u * (2 * kBigStages + 4 + w); };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + kBigBarsAt + 192);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_base + kBigBarsAt + 200);
  const WaitCtx wctx{abort_flag, prm.status, kWaitLimitClocks};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int cluster = int(blockIdx.x) >> 1, n_clusters = int(gridDim.x) >> 1;

  const int m_tiles = (prm.M + kBigBM - 1) / kBigBM, n_all = prm.n_tiles * prm.n_outputs, n_work = m_tiles * n_all;
  const int total = prm.k_tiles * prm.k_pairs;
  // Tiles run down kGroup rows of tiles before they move one column on: the 74 tiles in flight share kGroup strips of A
  // and about 74 / kGroup of B, which stay in L2.
  constexpr int kGroup = 8;
  struct Place { int m0, n0, sel; };
  auto place = [&](int tile) {
    const int per_group = kGroup * n_all, group = tile / per_group, first = group * kGroup;
    const int rows = min(kGroup, m_tiles - first), in = tile - group * per_group;
    const int n = in / rows;
    return Place{(first + in % rows) * kBigBM, (n % prm.n_tiles) * kTileN, n / prm.n_tiles};
  };

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kBigStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(acc_full(i), 1); mbar_init(acc_empty(i), 8); }
    for (int w = 0; w < 4; ++w) mbar_init(in_full(w), 1);
    fence_mbar_init();
    for (int i = 0; i < 2; ++i) { tma_prefetch_desc(&maps.a[i]); tma_prefetch_desc(&maps.b[i]); }
  }
  if (warp == 2) tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();     // the other CTA's barriers are there
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      int n = 0;
      for (int tile = cluster; tile < n_work && !*abort_flag; tile += n_clusters) {
        const Place at = place(tile);
        const int m0 = at.m0 + 128 * int(rank);
        for (int it = 0; it < total; ++it, ++n) {
          const int s = n % kBigStages;
          if (n >= kBigStages) mbar_wait(empty(s), (n / kBigStages - 1) & 1, wctx);
          if (*abort_flag) break;
          const bool second = it >= prm.k_tiles;
          const int k0 = (second ? it - prm.k_tiles : it) * kBK;
          const uint32_t sa = base + s * kBigStageBytes, sb = sa + kBigHalf, bar = cluster_map(full(s), 0);
          const CUtensorMap* am = &maps.a[second];
          if (rank == 0) mbar_expect_tx(full(s), 2 * kBigStageBytes);
          if (A_MN) {
            tma_load_3d_pair(sa, am, m0, 0, k0, bar);
            tma_load_3d_pair(sa + kSub, am, m0 + kChunk, 0, k0, bar);
          } else {
            tma_load_3d_pair(sa, am, k0, 0, m0, bar);
          }
          // Gate: rank 0 loads the tile's features of Wg, rank 1 the same features of Wu.
          const CUtensorMap* bm = &maps.b[EPI == kEpiGate ? int(rank) : (second || at.sel)];
          const int n0 = EPI == kEpiGate ? at.n0 : at.n0 + 128 * int(rank);
          if (B_MN) {
            tma_load_3d_pair(sb, bm, n0, 0, k0, bar);
            tma_load_3d_pair(sb + kSub, bm, n0 + kChunk, 0, k0, bar);
          } else {
            tma_load_3d_pair(sb, bm, k0, 0, n0, bar);
          }
        }
      }
      if (*abort_flag) {   // shared memory must outlive the copies in flight (the cluster's last barrier holds the other CTA)
        const long long t0 = clock64();
        if (rank == 0)
          for (int i = n > kBigStages ? n - kBigStages : 0; i < n; ++i)
            while (!mbar_try_wait(full(i % kBigStages), (i / kBigStages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
        while (clock64() - t0 < 1000000) {}
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t issuer = elect_one();
      constexpr uint32_t idesc = umma_idesc_bf16(kBigBM, kBigBN, A_MN, B_MN);
      int n = 0, i = 0;
      for (int tile = cluster; tile < n_work && !*abort_flag; tile += n_clusters, ++i) {
        const uint32_t acc = tmem + uint32_t(i & 1) * 256;
        mbar_wait_cluster(acc_empty(i & 1), ((i >> 1) & 1) ^ 1, wctx);
        tc_fence_after();
        for (int it = 0; it < total; ++it, ++n) {
          const int s = n % kBigStages;
          mbar_wait_cluster(full(s), (n / kBigStages) & 1, wctx);
          if (*abort_flag) break;
          tc_fence_after();
          const uint32_t sa = base + s * kBigStageBytes;
          const uint32_t a = smem_desc_lo(sa, A_MN ? kSub : 16), b = smem_desc_lo(sa + kBigHalf, B_MN ? kSub : 16);
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk)
            umma_ss_pair_w(acc, a + kk * ((A_MN ? 2048 : 32) >> 4), b + kk * ((B_MN ? 2048 : 32) >> 4), idesc, it > 0 || kk > 0, issuer);
          umma_commit_pair_w(empty(s), issuer);
        }
        umma_commit_pair_w(acc_full(i & 1), issuer);
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    const int w = warp - 4;
    const uint32_t bufs = base + kBigBufsAt + uint32_t(w) * kBigBufs * kBufBytes;
    auto buf = [&](uint32_t use) { return bufs + (use % kBigBufs) * kBufBytes; };
    // 16 bytes (8 columns) of this thread's row in a buffer, in the 128-byte-swizzled layout of the tensor maps
    auto cell = [&](uint32_t b, int eight) { return b + uint32_t(lane) * 128 + ((uint32_t(eight) ^ uint32_t(lane & 7)) << 4); };
    uint32_t use = 0;      // buffers used so far; each is one group of stores
    int i = 0, n_in = 0;   // n_in: loads of G and U requested so far
    for (int tile = cluster; tile < n_work && !*abort_flag; tile += n_clusters, ++i) {
      const Place at = place(tile);
      const int row0 = at.m0 + 128 * int(rank) + 32 * w;
      const uint32_t lanes = tmem + uint32_t(i & 1) * 256 + (uint32_t(w * 32) << 16);
      auto store = [&](const CUtensorMap* m, uint32_t b, int col) {    // by one lane, after the warp's writes
        if (row0 < prm.M && col < prm.N) tma_store_3d(m, b, col, 0, row0);
        tma_commit_group();
      };
      if (EPI != kEpiGateBwd) {
        mbar_wait(acc_full(i & 1), (i >> 1) & 1, wctx);
        tc_fence_after();
        if (*abort_flag) break;
      }
      if (EPI == kEpiOut) {
#pragma unroll 1
        for (int c = 0; c < kBigBN / 64; ++c, ++use) {
          uint32_t v[64];
          tmem_ld64_wait(lanes + c * 64, v);
          if (c == kBigBN / 64 - 1) {      // the accumulator is read
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(cluster_map(acc_empty(i & 1), 0));
          }
          if (lane == 0) tma_wait_group_read<kBigBufs - 1>();
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float* x = reinterpret_cast<const float*>(v) + 8 * j;
            const uint4 p = pack8(x);
            st_shared_v4(cell(buf(use), j), p.x, p.y, p.z, p.w);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) store(&maps.out[at.sel], buf(use), at.n0 + c * 64);
        }
      } else if (EPI == kEpiGate) {
        const bool keep = prm.out[0] != nullptr;
        const int n_bufs = keep ? 3 : 1;
#pragma unroll 1
        for (int c = 0; c < kTileN / 64; ++c, use += n_bufs) {
          if (lane == 0) {
            if (keep) tma_wait_group_read<kBigBufs - 3>(); else tma_wait_group_read<kBigBufs - 1>();
          }
          __syncwarp();
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            uint32_t g[32], u[32];
            tmem_ld32_wait(lanes + c * 64 + half * 32, g);
            tmem_ld32_wait(lanes + kTileN + c * 64 + half * 32, u);
            if (c == kTileN / 64 - 1 && half) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive_cluster(cluster_map(acc_empty(i & 1), 0));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float *gf = reinterpret_cast<const float*>(g) + 8 * j, *uf = reinterpret_cast<const float*>(u) + 8 * j;
              float h[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) h[k] = gf[k] * sigmoid(gf[k]) * uf[k];
              const int at8 = half * 4 + j;
              uint4 p = pack8(h);
              st_shared_v4(cell(buf(use), at8), p.x, p.y, p.z, p.w);
              if (keep) {
                p = pack8(gf);
                st_shared_v4(cell(buf(use + 1), at8), p.x, p.y, p.z, p.w);
                p = pack8(uf);
                st_shared_v4(cell(buf(use + 2), at8), p.x, p.y, p.z, p.w);
              }
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            store(&maps.out[2], buf(use), at.n0 + c * 64);
            if (keep) {
              store(&maps.out[0], buf(use + 1), at.n0 + c * 64);
              store(&maps.out[1], buf(use + 2), at.n0 + c * 64);
            }
          }
        }
      } else {
        // G and U of the tile arrive in two buffers, and leave from them as dG and dU.
#pragma unroll 1
        for (int c = 0; c < kBigBN / 64; ++c, use += 3) {
          if (lane == 0) {
            tma_wait_group_read<kBigBufs - 3>();
            mbar_expect_tx(in_full(w), 2 * kBufBytes);
            tma_load_3d(buf(use), &maps.in[0], at.n0 + c * 64, 0, row0, in_full(w));
            tma_load_3d(buf(use + 1), &maps.in[1], at.n0 + c * 64, 0, row0, in_full(w));
          }
          if (c == 0) {
            mbar_wait(acc_full(i & 1), (i >> 1) & 1, wctx);
            tc_fence_after();
          }
          mbar_wait(in_full(w), n_in & 1, wctx);
          ++n_in;
          __syncwarp();
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            uint32_t v[32];
            tmem_ld32_wait(lanes + c * 64 + half * 32, v);
            if (c == kBigBN / 64 - 1 && half) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive_cluster(cluster_map(acc_empty(i & 1), 0));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float* x = reinterpret_cast<const float*>(v) + 8 * j;
              const int at8 = half * 4 + j;
              float g[8], u[8], h[8];
              unpack8(ld_shared_v4(cell(buf(use), at8)), g);
              unpack8(ld_shared_v4(cell(buf(use + 1), at8)), u);
#pragma unroll
              for (int k = 0; k < 8; ++k) gate_bwd(x[k], g[k], u[k], h[k]);
              uint4 p = pack8(g);
              st_shared_v4(cell(buf(use), at8), p.x, p.y, p.z, p.w);
              p = pack8(u);
              st_shared_v4(cell(buf(use + 1), at8), p.x, p.y, p.z, p.w);
              p = pack8(h);
              st_shared_v4(cell(buf(use + 2), at8), p.x, p.y, p.z, p.w);
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (*abort_flag) break;
          if (lane == 0) {
            store(&maps.out[0], buf(use), at.n0 + c * 64);
            store(&maps.out[1], buf(use + 1), at.n0 + c * 64);
            store(&maps.out[2], buf(use + 2), at.n0 + c * 64);
          }
        }
      }
    }
    if (lane == 0) {
      if (EPI == kEpiGateBwd && *abort_flag && n_in > 0) {   // loads of G and U in flight
        const long long t0 = clock64();
        while (!mbar_try_wait(in_full(w), (n_in - 1) & 1) && clock64() - t0 < kWaitLimitClocks) {}
      }
      tma_wait_group_read<0>();   // shared memory must outlive the stores' reads
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();     // no CTA leaves while the pair's UMMAs or arrivals may still reach it
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// The parts of K summed in their order and rounded once.  blockIdx.y: output.
__global__ void __launch_bounds__(256)
ffn_sum_kernel(const float* partial, __nv_bfloat16* out0, __nv_bfloat16* out1, int64_t n, int32_t splits) {
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  const float* p = partial + int64_t(blockIdx.y) * n + i;
  const int64_t step = int64_t(gridDim.y) * n;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const float4 a = *reinterpret_cast<const float4*>(p + s * step), b = *reinterpret_cast<const float4*>(p + s * step + 4);
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
    v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
  }
  *reinterpret_cast<uint4*>((blockIdx.y ? out1 : out0) + i) = pack8(v);
}

// ---------------------------------------------------------------- host
// A row-major matrix, `rows` x `cols`, read in boxes of `box_rows` x 64.
bool matrix_map(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int box_rows) {
  return make_tile_map(m, p, rows, 1, int(cols), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, kBK, box_rows);
}

// One product: operands as they lie in memory.
struct Product {
  int64_t M, N, K;
  const void *a[2] = {nullptr, nullptr}, *b[2] = {nullptr, nullptr};
  int k_pairs = 1, n_outputs = 1;
};

bool takes_big(int64_t M, int64_t N, int n_outputs);

int split_count(int64_t M, int64_t N, int64_t K, int k_pairs, int n_outputs) {
  const int64_t tiles = ((M + kSmallBM - 1) / kSmallBM) * ((N + kSmallBN - 1) / kSmallBN) * n_outputs;
  if (tiles == 0) return 1;
  const int64_t its = (K + kBK - 1) / kBK * k_pairs;
  return int(std::max<int64_t>(1, std::min<int64_t>(2 * kSmCount / tiles, its / 8)));
}

int64_t partial_bytes(int64_t M, int64_t N, int64_t K, int k_pairs, int n_outputs) {
  if (takes_big(M, N, n_outputs)) return 0;
  const int s = split_count(M, N, K, k_pairs, n_outputs);
  return s > 1 ? 4 * M * N * n_outputs * s : 0;
}

bool takes_big(int64_t M, int64_t N, int n_outputs) {
  return ((M + kBigBM - 1) / kBigBM) * ((N + kBigBN - 1) / kBigBN) * n_outputs >= kSmCount / 2;
}

template <bool A_MN, bool B_MN, int EPI>
psa_status_t launch_big(const Product& p, GemmParams prm, cudaStream_t stream) {
  constexpr int kTileN = EPI == kEpiGate ? kBigBN / 2 : kBigBN;
  BigMaps maps;
  bool ok = true;
  for (int i = 0; i < 2; ++i) {
    const void *pa = p.a[i] ? p.a[i] : p.a[0], *pb = p.b[i] ? p.b[i] : p.b[0];
    ok = ok && (A_MN ? matrix_map(&maps.a[i], pa, p.K, p.M, kBK) : matrix_map(&maps.a[i], pa, p.M, p.K, 128));
    ok = ok && (B_MN ? matrix_map(&maps.b[i], pb, p.K, p.N, kBK) : matrix_map(&maps.b[i], pb, p.N, p.K, 128));
    const void *out = prm.out[i] ? prm.out[i] : prm.out[0], *in = i ? prm.up : prm.gate;
    ok = ok && matrix_map(&maps.out[i], out ? out : prm.h, p.M, p.N, 32);
    maps.in[i] = maps.a[i];
    if (EPI == kEpiGateBwd) ok = ok && matrix_map(&maps.in[i], in, p.M, p.N, 32);
  }
  ok = ok && matrix_map(&maps.out[2], prm.h ? prm.h : prm.out[0], p.M, p.N, 32);
  if (!ok) return PSA_ERR_CUDA;
  prm.M = int32_t(p.M);
  prm.N = int32_t(p.N);
  prm.k_tiles = int32_t((p.K + kBK - 1) / kBK);
  prm.k_pairs = p.k_pairs;
  prm.n_tiles = int32_t((p.N + kTileN - 1) / kTileN);
  prm.n_outputs = p.n_outputs;
  prm.splits = 1;
  auto kernel = ffn_big_kernel<A_MN, B_MN, EPI>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBigSmem) != cudaSuccess) return PSA_ERR_CUDA;
  const int64_t tiles = (p.M + kBigBM - 1) / kBigBM * prm.n_tiles * p.n_outputs;
  const unsigned grid = unsigned(2 * std::min<int64_t>(tiles, kSmCount / 2));
  kernel<<<grid, kBigThreads, kBigSmem, stream>>>(maps, prm);
  return check_last_cuda_error("psa_ffn launch");
}

template <bool A_MN, bool B_MN, int EPI>
psa_status_t launch_product(const Product& p, GemmParams prm, cudaStream_t stream) {
  if (takes_big(p.M, EPI == kEpiGate ? 2 * p.N : p.N, p.n_outputs)) return launch_big<A_MN, B_MN, EPI>(p, prm, stream);
  constexpr int kTileN = EPI == kEpiGate ? kSmallBN / 2 : kSmallBN;
  CUtensorMap a[2], b[2];
  for (int i = 0; i < 2; ++i) {
    const void *pa = p.a[i] ? p.a[i] : p.a[0], *pb = p.b[i] ? p.b[i] : p.b[0];
    if (!(A_MN ? matrix_map(&a[i], pa, p.K, p.M, kBK) : matrix_map(&a[i], pa, p.M, p.K, kSmallBM)) ||
        !(B_MN ? matrix_map(&b[i], pb, p.K, p.N, kBK) : matrix_map(&b[i], pb, p.N, p.K, kSmallBN)))
      return PSA_ERR_CUDA;
  }
  prm.M = int32_t(p.M);
  prm.N = int32_t(p.N);
  prm.k_tiles = int32_t((p.K + kBK - 1) / kBK);
  prm.k_pairs = p.k_pairs;
  prm.n_tiles = int32_t((p.N + kTileN - 1) / kTileN);
  prm.n_outputs = p.n_outputs;
  prm.splits = EPI == kEpiOut ? split_count(p.M, p.N, p.K, p.k_pairs, p.n_outputs) : 1;
  auto kernel = ffn_small_kernel<A_MN, B_MN, EPI>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmem) != cudaSuccess) return PSA_ERR_CUDA;
  const dim3 grid(unsigned((p.M + kSmallBM - 1) / kSmallBM), unsigned(prm.n_tiles * p.n_outputs), unsigned(prm.splits));
  kernel<<<grid, kSmallThreads, kSmallSmem, stream>>>(a[0], a[1], b[0], b[1], prm);
  if (prm.splits > 1) {
    const int64_t n = p.M * p.N;
    ffn_sum_kernel<<<dim3(unsigned((n + 2047) / 2048), unsigned(p.n_outputs)), 256, 0, stream>>>(prm.partial, prm.out[0], prm.out[1],
                                                                                                 n, prm.splits);
  }
  return check_last_cuda_error("psa_ffn launch");
}

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

struct FfnWorkspace {
  size_t h, d_gate, d_up, partial, total;
};

FfnWorkspace workspace_layout(int64_t T, int64_t D, int64_t F, bool backward) {
  FfnWorkspace w{};
  const size_t act = aligned(size_t(T) * F * 2);
  size_t at = act;   // h
  if (backward) {
    w.d_gate = at; at += act;
    w.d_up = at; at += act;
  }
  w.partial = at;
  int64_t part = backward ? std::max({partial_bytes(T, D, F, 2, 1), partial_bytes(D, F, T, 1, 2), partial_bytes(F, D, T, 1, 1)})
                          : partial_bytes(T, D, F, 1, 1);
  w.total = at + aligned(size_t(part));
  return w;
}

psa_status_t check_sizes(int64_t T, int32_t D, int32_t F) {
  if (T < 0 || D <= 0 || F <= 0) return PSA_ERR_INVALID_ARG;
  if (D % 8 || F % 8 || D > (1 << 20) || F > (1 << 20) || T > 0x7fffff00LL) return PSA_ERR_UNSUPPORTED;
  return PSA_OK;
}

bool all_set(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs) if (!p) return false;
  return true;
}
bool all_aligned(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs) if (reinterpret_cast<uintptr_t>(p) & 15) return false;
  return true;
}

}  // namespace
}  // namespace psa

extern "C" size_t psa_ffn_workspace_bytes(int64_t n_tokens, int32_t hidden, int32_t ffn, int32_t backward) {
  if (psa::check_sizes(n_tokens, hidden, ffn) != PSA_OK) return 0;
  return psa::workspace_layout(n_tokens, hidden, ffn, backward != 0).total;
}

extern "C" psa_status_t psa_ffn(const void* x, const void* w_gate, const void* w_up, const void* w_down, int64_t n_tokens,
                                int32_t hidden, int32_t ffn, void* out, void* gate, void* up, void* workspace,
                                int32_t* device_status, void* stream) {
  using namespace psa;
  const psa_status_t sizes = check_sizes(n_tokens, hidden, ffn);
  if (sizes != PSA_OK) return sizes;
  if ((gate == nullptr) != (up == nullptr)) return PSA_ERR_INVALID_ARG;
  if (n_tokens == 0) return PSA_OK;
  if (!all_set({x, w_gate, w_up, w_down, out, workspace})) return PSA_ERR_INVALID_ARG;
  if (!all_aligned({x, w_gate, w_up, w_down, out, gate, up, workspace})) return PSA_ERR_ALIGNMENT;
  const FfnWorkspace w = workspace_layout(n_tokens, hidden, ffn, false);
  char* ws = static_cast<char*>(workspace);
  __nv_bfloat16* h = reinterpret_cast<__nv_bfloat16*>(ws + w.h);
  cudaStream_t st = cudaStream_t(stream);

  GemmParams prm{};
  prm.status = device_status;
  prm.out[0] = static_cast<__nv_bfloat16*>(gate);
  prm.out[1] = static_cast<__nv_bfloat16*>(up);
  prm.h = h;
  Product first{n_tokens, ffn, hidden};
  first.a[0] = x;
  first.b[0] = w_gate;
  first.b[1] = w_up;
  psa_status_t rc = launch_product<false, true, kEpiGate>(first, prm, st);
  if (rc != PSA_OK) return rc;

  prm.out[0] = static_cast<__nv_bfloat16*>(out);
  prm.out[1] = nullptr;
  prm.partial = reinterpret_cast<float*>(ws + w.partial);
  Product second{n_tokens, hidden, ffn};
  second.a[0] = h;
  second.b[0] = w_down;
  return launch_product<false, true, kEpiOut>(second, prm, st);
}

extern "C" psa_status_t psa_ffn_bwd(const void* d_out, const void* x, const void* w_gate, const void* w_up, const void* w_down,
                                    const void* gate, const void* up, int64_t n_tokens, int32_t hidden, int32_t ffn, void* dx,
                                    void* dw_gate, void* dw_up, void* dw_down, void* workspace, int32_t* device_status,
                                    void* stream) {
  using namespace psa;
  const psa_status_t sizes = check_sizes(n_tokens, hidden, ffn);
  if (sizes != PSA_OK) return sizes;
  cudaStream_t st = cudaStream_t(stream);
  if (!all_set({dw_gate, dw_up, dw_down})) return PSA_ERR_INVALID_ARG;
  if (n_tokens == 0) {   // sums over no tokens
    const size_t bytes = size_t(hidden) * ffn * 2;
    for (void* p : {dw_gate, dw_up, dw_down})
      if (cudaMemsetAsync(p, 0, bytes, st) != cudaSuccess) {
        check_last_cuda_error("psa_ffn_bwd clear");
        return PSA_ERR_CUDA;
      }
    return PSA_OK;
  }
  if (!all_set({d_out, x, w_gate, w_up, w_down, gate, up, dx, workspace})) return PSA_ERR_INVALID_ARG;
  if (!all_aligned({d_out, x, w_gate, w_up, w_down, gate, up, dx, dw_gate, dw_up, dw_down, workspace})) return PSA_ERR_ALIGNMENT;
  const FfnWorkspace w = workspace_layout(n_tokens, hidden, ffn, true);
  char* ws = static_cast<char*>(workspace);
  auto bf = [](void* p) { return static_cast<__nv_bfloat16*>(p); };
  __nv_bfloat16 *h = bf(ws + w.h), *d_gate = bf(ws + w.d_gate), *d_up = bf(ws + w.d_up);

  GemmParams prm{};
  prm.status = device_status;
  prm.partial = reinterpret_cast<float*>(ws + w.partial);
  prm.out[0] = d_gate;
  prm.out[1] = d_up;
  prm.h = h;
  prm.gate = static_cast<const __nv_bfloat16*>(gate);
  prm.up = static_cast<const __nv_bfloat16*>(up);
  Product dh{n_tokens, ffn, hidden};   // dH = dY Wd^T: Wd has K (hidden) innermost
  dh.a[0] = d_out;
  dh.b[0] = w_down;
  psa_status_t rc = launch_product<false, false, kEpiGateBwd>(dh, prm, st);
  if (rc != PSA_OK) return rc;

  Product in{n_tokens, hidden, ffn};   // dX = dG Wg^T + dU Wu^T
  in.a[0] = d_gate;
  in.a[1] = d_up;
  in.b[0] = w_gate;
  in.b[1] = w_up;
  in.k_pairs = 2;
  prm.out[0] = bf(dx);
  prm.out[1] = nullptr;
  rc = launch_product<false, false, kEpiOut>(in, prm, st);
  if (rc != PSA_OK) return rc;

  Product gu{hidden, ffn, n_tokens};   // dWg = X^T dG and dWu = X^T dU
  gu.a[0] = x;
  gu.b[0] = d_gate;
  gu.b[1] = d_up;
  gu.n_outputs = 2;
  prm.out[0] = bf(dw_gate);
  prm.out[1] = bf(dw_up);
  rc = launch_product<true, true, kEpiOut>(gu, prm, st);
  if (rc != PSA_OK) return rc;

  Product down{ffn, hidden, n_tokens};   // dWd = H^T dY
  down.a[0] = h;
  down.b[0] = d_out;
  prm.out[0] = bf(dw_down);
  prm.out[1] = nullptr;
  return launch_product<true, true, kEpiOut>(down, prm, st);
}
