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
// Rounded to bf16, once each: what enters a product (H, dG, dU), as tcgen05.mma takes bf16, and G and U where a backward keeps
// them (in fp32 they would be 4 T F bytes more to write and to read; their part of a gradient's error is no larger than dG's own:
// in all 0.0035 of the gradient in the 2-norm, 0.0017 with only the result rounded).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "psa.h"
#include "psa_device.cuh"
#include "psa_internal.h"
#include "psa_launch.cuh"
#include "psa_product.cuh"
#include "psa_tensormap.h"

namespace psa {
namespace {

using namespace dev;

constexpr int kSmCount = 148;
constexpr int kMaxProducts = 3;

enum Epilogue {
  kEpiOut,        // C rounded to bf16
  kEpiGate,       // a tile holds G and U of the same features
  kEpiGateBwd,    // C is dH
};

struct ProductMaps {
  OperandMaps a[2], b[2];      // two pairs along K, or a second B for a second output (kEpiGate: Wg, Wu)
  CUtensorMap store[2];        // boxes of 32 rows of the outputs
};
struct Product {
  __nv_bfloat16* out[2];
  int32_t M, N;                // rows and columns of one output
  int32_t k_tiles, k_pairs;    // stages of one pair of operands; pairs that are summed
  int32_t m_tiles, n_tiles;    // tiles of one output
  int32_t n_outputs;           // outputs side by side
  int32_t first;               // the product's first tile in the launch
  int32_t a_mn, b_mn;          // which way the operands lie
  int32_t early;               // B may be loaded before behind_wait(): see Wanted::early
};
struct ProductList {
  ProductMaps maps[kMaxProducts];
  Product p[kMaxProducts];
  CUtensorMap in[2], store_h;  // kEpiGateBwd: G, U;  H
  const __nv_bfloat16 *gate, *up;
  __nv_bfloat16* h;
  int32_t n_products, n_work, splits, a_rows;
  int32_t* status;
};

// Output tile `tile` of the launch: its product and place.  The products' sizes are looked up in shared memory (`products`,
// copied there by copy_products): read from the kernel's parameters by a running index they cost a trip to memory each, and
// between two tiles the loads of the next one wait for them.
struct Place {
  int k, m0, n0, sel;
};
__device__ __forceinline__ void copy_products(const ProductList& list, Product* products) {
  constexpr int kWords = sizeof(Product) / 4;
  if (int(threadIdx.x) < kWords * kMaxProducts)
    reinterpret_cast<uint32_t*>(products)[threadIdx.x] = reinterpret_cast<const uint32_t*>(list.p)[threadIdx.x];
}
// Tiles run down kGroup rows of tiles (0: all) before they move one column on, so that the tiles in flight share strips of A
// and of B in L2.
template <int kBM, int kTileN, int kGroup>
__device__ __forceinline__ Place place_of(const Product* products, int n_products, int tile) {
  int k = 0;
  while (k + 1 < n_products && tile >= products[k + 1].first) ++k;
  const Product& p = products[k];
  const int m_tiles = p.m_tiles, n_tiles = p.n_tiles, n_all = n_tiles * p.n_outputs, at = tile - p.first;
  const int per_group = (kGroup ? kGroup : m_tiles) * n_all, group = at / per_group, first = group * kGroup;
  const int rows = kGroup ? min(kGroup, m_tiles - first) : m_tiles, in = at - group * per_group, n = in / rows;
  return Place{k, (first + in % rows) * kBM, (n % n_tiles) * kTileN, n / n_tiles};
}

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

__device__ __forceinline__ void unpack8(const uint4& w, float* v) {
  v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
  v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
}

// ---------------------------------------------------------------- one CTA per tile of 128 x 128
// For launches of few tiles.  Where they are fewer than the SMs can hold, a cluster of 2, 4 or 8 CTAs shares a tile's K: each
// leaves its sums in its shared memory, and all of them add the parts, in the CTAs' order, and finish a share of the tile.
// Warps 0-7: end of the tile (TMEM lane = row of the tile, half of its columns each), warp 8: TMA, warp 9: UMMA.
// Up to 64 tokens, a stage holds no more of A's rows than there are (rounded up to 8), and more stages fit; what the UMMA takes
// for the tile's other rows is whatever lies behind them, and goes to rows that nobody reads.
constexpr int kSmallBM = 128, kSmallBN = 128, kSmallMaxStages = 6, kSmallThreads = 320;
constexpr uint32_t kSmallRing = 96 * 1024, kSmallBBytes = kSmallBN * kBK * 2;
constexpr uint32_t kSmallSmem = kSmallRing + 1024 + 256;
constexpr int kPartPitch = kSmallBN + 4;      // floats per row of a part: rows start four banks apart
static_assert(kSmallBM * kPartPitch * 4 <= kSmallRing, "a part takes the place of the stages");
__host__ __device__ constexpr int small_rows(int64_t M) { return M <= 64 ? int(M + 7) / 8 * 8 : kSmallBM; }

// Eight neighbouring elements of a tile: their sums (kEpiGate: x of G, y of U) become outputs.
template <int EPI>
__device__ __forceinline__ void finish8(const ProductList& list, const Product& p, int sel, int row, int col, const float* x,
                                        const float* y, const uint4& gate, const uint4& up) {
  const int64_t to = int64_t(row) * p.N + col;
  if (!PSA_IN_BOUNDS(to + 7, int64_t(p.M) * p.N, list.status)) return;
  if (EPI == kEpiOut) {
    *reinterpret_cast<uint4*>(p.out[sel] + to) = pack8(x);
  } else if (EPI == kEpiGate) {
    float h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = x[i] * sigmoid(x[i]) * y[i];
    if (p.out[0]) {
      *reinterpret_cast<uint4*>(p.out[0] + to) = pack8(x);
      *reinterpret_cast<uint4*>(p.out[1] + to) = pack8(y);
    }
    *reinterpret_cast<uint4*>(list.h + to) = pack8(h);
  } else {
    float g[8], u[8], h[8];
    unpack8(gate, g);
    unpack8(up, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) gate_bwd(x[i], g[i], u[i], h[i]);
    *reinterpret_cast<uint4*>(p.out[0] + to) = pack8(g);
    *reinterpret_cast<uint4*>(p.out[1] + to) = pack8(u);
    *reinterpret_cast<uint4*>(list.h + to) = pack8(h);
  }
}

// The sums of eight elements over a cluster's CTAs, in their order.  All reads are on their way before the first is needed: one
// after the other, a trip to another SM each, they took more time than the product at a hundred tokens.
__device__ __forceinline__ void add_parts(uint32_t from, int splits, float (&x)[8]) {
  uint4 v[8][2];
#pragma unroll
  for (int s = 0; s < 8; ++s)
    if (s < splits) {
      const uint32_t addr = cluster_map(from, uint32_t(s));
      v[s][0] = ld_cluster_v4(addr);
      v[s][1] = ld_cluster_v4(addr + 16);
    }
#pragma unroll
  for (int s = 0; s < 8; ++s)
    if (s < splits) {
      const uint32_t w[8] = {v[s][0].x, v[s][0].y, v[s][0].z, v[s][0].w, v[s][1].x, v[s][1].y, v[s][1].z, v[s][1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += __uint_as_float(w[i]);
    }
}

template <int EPI>
__global__ void __launch_bounds__(kSmallThreads, 2)
ffn_small_kernel(const __grid_constant__ ProductList list) {
  constexpr int kBN = kSmallBN;
  constexpr int kTileN = EPI == kEpiGate ? kBN / 2 : kBN;      // features per tile
  const uint32_t a_bytes = uint32_t(list.a_rows) * kBK * 2, stage_bytes = a_bytes + kSmallBBytes;
  const int stages = min(kSmallMaxStages, int(kSmallRing / stage_bytes));
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + kSmallRing;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (kSmallMaxStages + s); };
  const uint32_t done = bars + 16u * kSmallMaxStages;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + kSmallRing + 128);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_base + kSmallRing + 136);
  const WaitCtx wctx{abort_flag, list.status, kWaitLimitClocks};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  __shared__ Product products[kMaxProducts];
  copy_products(list, products);
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(done, 1);
    fence_mbar_init();
  }
  if (warp == 9) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kBN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int splits = list.splits, part = int(blockIdx.x) % splits;
  const Place at = place_of<kSmallBM, kTileN, 0>(products, list.n_products, int(blockIdx.x) / splits);
  const Product& p = products[at.k];
  const int total = p.k_tiles * p.k_pairs;
  const int it0 = int(int64_t(total) * part / splits), it1 = int(int64_t(total) * (part + 1) / splits);
  if (warp != 8) {
    behind_wait();
    behind_go();
  }

  // Rows of this thread, for the warps that finish a tile from TMEM.
  const int quarter = warp & 3, row = at.m0 + quarter * 32 + lane, half = warp >> 2;
  const uint32_t lanes = tmem + (uint32_t(quarter * 32) << 16);
  constexpr int kHalfN = kTileN / 2;
  auto load_gate = [&](int r, int col, uint4& g, uint4& u) {
    if (EPI != kEpiGateBwd || r >= p.M || col >= p.N) return;
    const int64_t from = int64_t(r) * p.N + col;
    if (!PSA_IN_BOUNDS(from + 7, int64_t(p.M) * p.N, list.status)) return;
    g = *reinterpret_cast<const uint4*>(list.gate + from);
    u = *reinterpret_cast<const uint4*>(list.up + from);
  };

  if (warp == 8) {
    const uint32_t issuer = elect_one();
    const ProductMaps& maps = list.maps[at.k];
    const Strip a(maps.a, p.a_mn, at.m0, p.M), b(maps.b, p.b_mn, at.n0, p.N);
    const int k_tiles = p.k_tiles, sel = at.sel;
    auto load_a = [&](int it, int s) {
      const bool second = it >= k_tiles;
      const uint32_t bar = full(s);
      a.load(second, (second ? it - k_tiles : it) * kBK, base + s * stage_bytes,
             [&](uint32_t dst, const CUtensorMap* m, int c0, int c1, int c2) { tma_load_3d_w(dst, m, c0, c1, c2, bar, issuer); });
    };
    auto load_b = [&](int it, int s) {
      const bool second = it >= k_tiles;
      const int k0 = (second ? it - k_tiles : it) * kBK;
      const uint32_t sb = base + s * stage_bytes + a_bytes, bar = full(s);
      auto load = [&](uint32_t dst, const CUtensorMap* m, int c0, int c1, int c2) { tma_load_3d_w(dst, m, c0, c1, c2, bar, issuer); };
      mbar_expect_tx_w(bar, stage_bytes, issuer);
      if (EPI == kEpiGate) {   // the same features of two weights
        load(sb, &b.m[0].flat, at.n0, 0, k0);
        load(sb + kSub, &b.m[1].flat, at.n0, 0, k0);
      } else {
        b.load(second || sel, k0, sb, load);
      }
    };
    // Weights that the kernel before does not write may come before it has ended.
    const int ahead = p.early ? min(stages, it1 - it0) : 0;
    for (int i = 0; i < ahead; ++i) load_b(it0 + i, i);
    behind_wait();
    behind_go();
    int n = 0, s = 0, turn = 0;   // stages filled; the next one and its turn of the ring
    for (int it = it0; it < it1; ++it, ++n) {
      if (turn) mbar_wait(empty(s), (turn - 1) & 1, wctx);
      if (*abort_flag) break;
      if (n >= ahead) load_b(it, s);
      load_a(it, s);
      if (++s == stages) { s = 0; ++turn; }
    }
    if (*abort_flag) {   // shared memory must outlive the copies in flight
      const long long t0 = clock64();
      for (int i = n > stages ? n - stages : 0; i < n; ++i)      // (the first wait can only expire after `ahead` stages)
        while (!mbar_try_wait(full(i % stages), (i / stages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
    }
    __syncwarp();
  } else if (warp == 9) {
    const uint32_t issuer = elect_one();
    const bool a_mn = p.a_mn, b_mn = p.b_mn;
    const uint32_t idesc = umma_idesc_bf16(kSmallBM, kBN, false, false) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16);
    const uint32_t a_step = (a_mn ? 2048 : 32) >> 4, b_step = (b_mn ? 2048 : 32) >> 4;
    int s = 0, turn = 0;
    for (int it = it0; it < it1; ++it) {
      mbar_wait(full(s), turn & 1, wctx);
      tc_fence_after();
      const uint32_t sa = base + s * stage_bytes;
      const uint32_t a = smem_desc_lo(sa, a_mn ? kSub : 16), b = smem_desc_lo(sa + a_bytes, b_mn ? kSub : 16);
#pragma unroll
      for (int kk = 0; kk < kBK / 16; ++kk) umma_ss_w(tmem, a + kk * a_step, b + kk * b_step, idesc, it > it0 || kk > 0, issuer);
      umma_commit_w(empty(s), issuer);
      if (++s == stages) { s = 0; ++turn; }
    }
    umma_commit_w(done, issuer);
    __syncwarp();
  } else {
    uint4 g[4], u[4];
    if (splits == 1)
#pragma unroll
      for (int j = 0; j < 4; ++j) load_gate(row, at.n0 + half * kHalfN + 8 * j, g[j], u[j]);
    mbar_wait(done, 0, wctx);
    tc_fence_after();
    const bool live = row < p.M && !*abort_flag;
#pragma unroll 1
    for (int c = half * kHalfN; c < (half + 1) * kHalfN; c += 32) {
      uint32_t v[32], w[32];
      tmem_ld32_wait(lanes + c, v);
      if (EPI == kEpiGate) tmem_ld32_wait(lanes + kTileN + c, w);
      const float *x = reinterpret_cast<const float*>(v), *y = reinterpret_cast<const float*>(w);
      if (splits > 1) {   // (every UMMA that reads the stages has completed)
        if (it0 == it1)        // a short K leaves some of the CTAs nothing to add
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = w[j] = 0u;
        const uint32_t to = base + uint32_t(quarter * 32 + lane) * kPartPitch * 4 + c * 4;
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          st_shared_v4(to + 4 * j, v[j], v[j + 1], v[j + 2], v[j + 3]);
          if (EPI == kEpiGate) st_shared_v4(to + 4 * (kTileN + j), w[j], w[j + 1], w[j + 2], w[j + 3]);
        }
        continue;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = at.n0 + c + 8 * j;
        const uint4 g0 = g[j], u0 = u[j];
        if (c + 32 < (half + 1) * kHalfN) load_gate(row, col + 32, g[j], u[j]);
        if (live && col < p.N) finish8<EPI>(list, p, at.sel, row, col, x + 8 * j, y + 8 * j, g0, u0);
      }
    }
  }
  if (splits > 1) {
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    const int rows = min(kSmallBM, p.M - at.m0), n_eights = rows * (kTileN / 8);
    for (int i = part * kSmallThreads + int(threadIdx.x); i < n_eights && !*abort_flag; i += splits * kSmallThreads) {
      const int r = i / (kTileN / 8), c = (i % (kTileN / 8)) * 8, col = at.n0 + c;
      if (col >= p.N) continue;
      uint4 g, u;
      load_gate(at.m0 + r, col, g, u);
      float x[8] = {}, y[8] = {};
      const uint32_t from = base + uint32_t(r * kPartPitch + c) * 4;
      add_parts(from, splits, x);
      if (EPI == kEpiGate) add_parts(from + kTileN * 4, splits, y);
      finish8<EPI>(list, p, at.sel, at.m0 + r, col, x, y, g, u);
    }
    cluster_arrive();
    cluster_wait();     // the other CTAs have read this one's part
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, kBN);
  }
}

// ---------------------------------------------------------------- two CTAs per tile of 256 x 256
// A persistent kernel: 74 clusters of two CTAs take every 74th tile of the launch.  A tile's product is one UMMA stream of the
// pair (M = 256, N = 256): each CTA loads its 128 rows of A and 128 of the tile's 256 columns of B, so a stage brings 32 KB to
// each SM for the work of which a CTA alone would need 48.  The accumulator takes half of TMEM: while the end of one tile
// drains it, the next tile's UMMAs fill the other half.
// Warps: 0 TMA, 1 UMMA (in the CTA of rank 0), 2 TMEM, 4-7 the end of a tile, each for 32 rows of its CTA.
// Results leave by TMA stores from buffers that each warp owns: no barrier but the warp's own, and the tensor map clips what
// lies behind the last row or column.
constexpr int kBigBM = 256, kBigBN = 256, kBigStages = 5, kBigThreads = 256, kBigBufs = 4, kBigGroup = 16;
constexpr uint32_t kBigHalf = 128 * kBK * 2;                       // one operand's half of a stage
constexpr uint32_t kBigStageBytes = 2 * kBigHalf;
constexpr uint32_t kBufBytes = 32 * 64 * 2;
constexpr uint32_t kBigBufsAt = kBigStages * kBigStageBytes;
constexpr uint32_t kBigBarsAt = kBigBufsAt + 4 * kBigBufs * kBufBytes;
constexpr uint32_t kBigSmem = kBigBarsAt + 256 + 1024;
static_assert(kBigSmem <= 227 * 1024, "shared memory of one CTA");
// kEpiGateBwd: boxes of 32 rows x 32 columns.  G and U arrive in three sets of two buffers, up to two boxes ahead, and leave
// from them as dG and dU; H leaves from two buffers of its own.  Its five tensors take 640 KB of a tile's way through shared
// memory beside the 8 MB of 64 stages, which fill the 128 bytes a clock that shared memory has: at 4096 x 9472 x 4096 the
// product takes 231 us, without them 190.  G and U by ordinary loads into registers, each lane its row: 251 us; a fourth
// set and H by ordinary stores: 236; separate buffers for what arrives and what leaves: 236.
constexpr uint32_t kBoxBytes = 32 * 32 * 2;
constexpr int kBoxSets = 3, kBoxesPerTile = kBigBN / 32;
static_assert((2 * kBoxSets + 2) * kBoxBytes <= kBigBufs * kBufBytes, "a warp's buffers");

template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kBigThreads, 1)
ffn_big_kernel(const __grid_constant__ ProductList list) {
  constexpr int kTileN = EPI == kEpiGate ? kBigBN / 2 : kBigBN;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + kBigBarsAt;
  auto full = [&](int s) { return bars + 8u * s; };                    // of rank 0: both CTAs' loads
  auto empty = [&](int s) { return bars + 8u * (kBigStages + s); };
  auto acc_full = [&](int i) { return bars + 8u * (2 * kBigStages + i); };
  auto acc_empty = [&](int i) { return bars + 8u * (2 * kBigStages + 2 + i); };   // of rank 0: both CTAs' warps
  auto in_full = [&](int w, int set) { return bars + 8u * (2 * kBigStages + 4 + kBoxSets * w + set); };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + kBigBarsAt + 240);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_base + kBigBarsAt + 248);
  static_assert(8 * (2 * kBigStages + 4 + 4 * kBoxSets) <= 240, "barriers");
  const WaitCtx wctx{abort_flag, list.status, kWaitLimitClocks};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int cluster = int(blockIdx.x) >> 1, n_clusters = int(gridDim.x) >> 1, n_work = list.n_work;
  __shared__ Product products[kMaxProducts];
  copy_products(list, products);
  auto place = [&](int tile) { return place_of<kBigBM, kTileN, kBigGroup>(products, list.n_products, tile); };

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kBigStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(acc_full(i), 1); mbar_init(acc_empty(i), 8); }
    for (int w = 0; w < 4; ++w)
      for (int s = 0; s < kBoxSets; ++s) mbar_init(in_full(w, s), 1);
    fence_mbar_init();
  }
  if (warp == 2) tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();     // the other CTA's barriers are there
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  behind_wait();
  behind_go();

  if (warp == 0) {
    const uint32_t issuer = elect_one();
    int n = 0;
    for (int tile = cluster; tile < n_work && !*abort_flag; tile += n_clusters) {
      const Place at = place(tile);
      const Product& p = products[at.k];
      const ProductMaps& maps = list.maps[at.k];
      // kEpiGate: rank 0 loads the tile's features of Wg, rank 1 the same features of Wu.
      const Strip a(maps.a, p.a_mn, at.m0 + 128 * int(rank), p.M), b(maps.b, p.b_mn, EPI == kEpiGate ? at.n0 : at.n0 + 128 * int(rank), p.N);
      const int k_tiles = p.k_tiles, total = k_tiles * p.k_pairs, sel = EPI == kEpiGate ? int(rank) : at.sel;
      for (int it = 0; it < total; ++it, ++n) {
        const int s = n % kBigStages;
        if (n >= kBigStages) mbar_wait(empty(s), (n / kBigStages - 1) & 1, wctx);
        if (*abort_flag) break;
        const bool second = it >= k_tiles;
        const int k0 = (second ? it - k_tiles : it) * kBK;
        const uint32_t sa = base + s * kBigStageBytes, bar = cluster_map(full(s), 0);
        auto load = [&](uint32_t dst, const CUtensorMap* m, int c0, int c1, int c2) { tma_load_3d_pair_w(dst, m, c0, c1, c2, bar, issuer); };
        mbar_expect_tx_w(full(s), 2 * kBigStageBytes, rank == 0 ? issuer : 0u);
        a.load(second, k0, sa, load);
        b.load(second || sel, k0, sa + kBigHalf, load);
      }
    }
    if (*abort_flag) {   // shared memory must outlive the copies in flight (the cluster's last barrier holds the other CTA)
      const long long t0 = clock64();
      if (rank == 0)
        for (int i = n > kBigStages ? n - kBigStages : 0; i < n; ++i)
          while (!mbar_try_wait(full(i % kBigStages), (i / kBigStages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
      while (clock64() - t0 < 1000000) {}
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t issuer = elect_one();
      int n = 0, i = 0;
      for (int tile = cluster; tile < n_work && !*abort_flag; tile += n_clusters, ++i) {
        const Product& p = products[place(tile).k];
        const bool a_mn = p.a_mn, b_mn = p.b_mn;
        const uint32_t idesc = umma_idesc_bf16(kBigBM, kBigBN, false, false) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16);
        const uint32_t a_step = (a_mn ? 2048 : 32) >> 4, b_step = (b_mn ? 2048 : 32) >> 4;
        const int total = p.k_tiles * p.k_pairs;
        const uint32_t acc = tmem + uint32_t(i & 1) * 256;
        mbar_wait_cluster(acc_empty(i & 1), ((i >> 1) & 1) ^ 1, wctx);
        tc_fence_after();
        for (int it = 0; it < total; ++it, ++n) {
          const int s = n % kBigStages;
          mbar_wait_cluster(full(s), (n / kBigStages) & 1, wctx);
          if (*abort_flag) break;
          tc_fence_after();
          const uint32_t sa = base + s * kBigStageBytes;
          const uint32_t a = smem_desc_lo(sa, a_mn ? kSub : 16), b = smem_desc_lo(sa + kBigHalf, b_mn ? kSub : 16);
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk)
            umma_ss_pair_w(acc, a + kk * a_step, b + kk * b_step, idesc, it > 0 || kk > 0, issuer);
          umma_commit_pair_w(empty(s), issuer);
        }
        umma_commit_pair_w(acc_full(i & 1), issuer);
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    const int w = warp - 4;
    const uint32_t issuer = elect_one();     // the lane that owns the warp's copies and groups of stores
    const uint32_t bufs = base + kBigBufsAt + uint32_t(w) * kBigBufs * kBufBytes;
    auto drained = [&](int i) {      // this warp has read the accumulator
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(cluster_map(acc_empty(i & 1), 0));
    };
    if (EPI != kEpiGateBwd) {
      auto buf = [&](uint32_t use) { return bufs + (use % kBigBufs) * kBufBytes; };
      // 16 bytes (8 columns) of this thread's row in a buffer, in the 128-byte-swizzled layout of the tensor maps
      auto cell = [&](uint32_t b, int eight) { return b + uint32_t(lane) * 128 + ((uint32_t(eight) ^ uint32_t(lane & 7)) << 4); };
      uint32_t use = 0;      // buffers used so far; each is one group of stores
      int i = 0;
      for (int tile = cluster; tile < n_work && !*abort_flag; tile += n_clusters, ++i) {
        const Place at = place(tile);
        const Product& p = products[at.k];
        const ProductMaps& maps = list.maps[at.k];
        const int row0 = at.m0 + 128 * int(rank) + 32 * w;
        const uint32_t lanes = tmem + uint32_t(i & 1) * 256 + (uint32_t(w * 32) << 16);
        const int M = p.M, N = p.N;
        auto store = [&](const CUtensorMap* m, uint32_t b, int col) {    // after the warp's writes
          tma_store_3d_w(m, b, col, 0, row0, row0 < M && col < N ? issuer : 0u);
          if (issuer) tma_commit_group();
        };
        mbar_wait(acc_full(i & 1), (i >> 1) & 1, wctx);
        tc_fence_after();
        if (*abort_flag) break;
        if (EPI == kEpiOut) {
#pragma unroll 1
          for (int c = 0; c < kBigBN / 64; ++c, ++use) {
            uint32_t v[64];
            tmem_ld64_wait(lanes + c * 64, v);
            if (c == kBigBN / 64 - 1) drained(i);
            if (issuer) tma_wait_group_read<kBigBufs - 1>();
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint4 q = pack8(reinterpret_cast<const float*>(v) + 8 * j);
              st_shared_v4(cell(buf(use), j), q.x, q.y, q.z, q.w);
            }
            fence_proxy_async_smem();
            __syncwarp();
            store(&maps.store[at.sel], buf(use), at.n0 + c * 64);
          }
        } else {
          const bool keep = p.out[0] != nullptr;
          const int n_bufs = keep ? 3 : 1;
#pragma unroll 1
          for (int c = 0; c < kTileN / 64; ++c, use += n_bufs) {
            if (issuer) {
              if (keep) tma_wait_group_read<kBigBufs - 3>(); else tma_wait_group_read<kBigBufs - 1>();
            }
            __syncwarp();
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
              uint32_t g[32], u[32];
              tmem_ld32_wait(lanes + c * 64 + half * 32, g);
              tmem_ld32_wait(lanes + kTileN + c * 64 + half * 32, u);
              if (c == kTileN / 64 - 1 && half) drained(i);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float *gf = reinterpret_cast<const float*>(g) + 8 * j, *uf = reinterpret_cast<const float*>(u) + 8 * j;
                float h[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) h[k] = gf[k] * sigmoid(gf[k]) * uf[k];
                const int at8 = half * 4 + j;
                uint4 q = pack8(h);
                st_shared_v4(cell(buf(use), at8), q.x, q.y, q.z, q.w);
                if (keep) {
                  q = pack8(gf);
                  st_shared_v4(cell(buf(use + 1), at8), q.x, q.y, q.z, q.w);
                  q = pack8(uf);
                  st_shared_v4(cell(buf(use + 2), at8), q.x, q.y, q.z, q.w);
                }
              }
            }
            fence_proxy_async_smem();
            __syncwarp();
            store(&list.store_h, buf(use), at.n0 + c * 64);
            if (keep) {
              store(&maps.store[0], buf(use + 1), at.n0 + c * 64);
              store(&maps.store[1], buf(use + 2), at.n0 + c * 64);
            }
          }
        }
      }
    } else {
      // Box q of the warp: box q % 8 of its (q / 8)-th tile.
      const int n_tiles = cluster < n_work ? (n_work - cluster + n_clusters - 1) / n_clusters : 0, n_boxes = n_tiles * kBoxesPerTile;
      const int M = products[0].M, N = products[0].N, row_of = 128 * int(rank) + 32 * w;
      const ProductMaps& maps = list.maps[0];
      auto set_buf = [&](int q, int k) { return bufs + uint32_t(2 * (q % kBoxSets) + k) * kBoxBytes; };
      auto h_buf = [&](int q) { return bufs + uint32_t(2 * kBoxSets + (q & 1)) * kBoxBytes; };
      // as above, 64-byte-swizzled
      auto cell = [&](uint32_t b, int eight) { return b + uint32_t(lane) * 64 + ((uint32_t(eight) ^ uint32_t((lane >> 1) & 3)) << 4); };
      int asked = 0;
      Place ahead{};
      auto ask = [&]() {     // requests G and U of the next box
        if (asked >= n_boxes) return;
        const int c = asked % kBoxesPerTile;
        if (c == 0) ahead = place(cluster + asked / kBoxesPerTile * n_clusters);
        const uint32_t bar = in_full(w, asked % kBoxSets);
        mbar_expect_tx_w(bar, 2 * kBoxBytes, issuer);
        tma_load_3d_w(set_buf(asked, 0), &list.in[0], ahead.n0 + c * 32, 0, ahead.m0 + row_of, bar, issuer);
        tma_load_3d_w(set_buf(asked, 1), &list.in[1], ahead.n0 + c * 32, 0, ahead.m0 + row_of, bar, issuer);
        ++asked;
      };
      ask();
      ask();
      Place at{};
#pragma unroll 1
      for (int q = 0; q < n_boxes && !*abort_flag; ++q) {
        const int i = q / kBoxesPerTile, c = q % kBoxesPerTile;
        if (c == 0) {
          at = place(cluster + i * n_clusters);
          mbar_wait(acc_full(i & 1), (i >> 1) & 1, wctx);
          tc_fence_after();
        }
        mbar_wait(in_full(w, q % kBoxSets), (q / kBoxSets) & 1, wctx);
        __syncwarp();
        if (*abort_flag) break;
        uint32_t v[32];
        tmem_ld32_wait(tmem + uint32_t(i & 1) * 256 + (uint32_t(w * 32) << 16) + c * 32, v);
        if (c == kBoxesPerTile - 1) drained(i);
        const int row = at.m0 + row_of, col = at.n0 + c * 32;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float* x = reinterpret_cast<const float*>(v) + 8 * j;
          float g[8], u[8], h[8];
          unpack8(ld_shared_v4(cell(set_buf(q, 0), j)), g);
          unpack8(ld_shared_v4(cell(set_buf(q, 1), j)), u);
#pragma unroll
          for (int k = 0; k < 8; ++k) gate_bwd(x[k], g[k], u[k], h[k]);
          uint4 o = pack8(g);
          st_shared_v4(cell(set_buf(q, 0), j), o.x, o.y, o.z, o.w);
          o = pack8(u);
          st_shared_v4(cell(set_buf(q, 1), j), o.x, o.y, o.z, o.w);
          o = pack8(h);
          st_shared_v4(cell(h_buf(q), j), o.x, o.y, o.z, o.w);
        }
        fence_proxy_async_smem();
        __syncwarp();
        const uint32_t inside = row < M && col < N ? issuer : 0u;
        tma_store_3d_w(&maps.store[0], set_buf(q, 0), col, 0, row, inside);
        tma_store_3d_w(&maps.store[1], set_buf(q, 1), col, 0, row, inside);
        tma_store_3d_w(&list.store_h, h_buf(q), col, 0, row, inside);
        if (issuer) {
          tma_commit_group();
          tma_wait_group_read<1>();    // the set of the box before this one is free
        }
        __syncwarp();
        ask();
      }
      if (*abort_flag) {   // loads of G and U in flight
        const long long t0 = clock64();
        for (int q = asked > kBoxSets ? asked - kBoxSets : 0; q < asked; ++q)
          while (!mbar_try_wait(in_full(w, q % kBoxSets), (q / kBoxSets) & 1) && clock64() - t0 < kWaitLimitClocks) {}
      }
    }
    if (issuer) tma_wait_group_read<0>();   // shared memory must outlive the stores' reads
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

// ---------------------------------------------------------------- host
struct Matrix {
  const void* p;
  bool mn_major;
};
// C[M, N] = sum of A B over K, for up to two pairs of operands or two outputs.
struct Wanted {
  int64_t M, N, K;
  Matrix a[2], b[2];
  __nv_bfloat16* out[2];
  int k_pairs, n_outputs;
  // B may be loaded while the kernel before this one runs.  Only where that kernel is one of the same call, which waits before it
  // lets this one start (so what came before the call is complete), and writes no B of this one.
  bool early;
};

int64_t tiles_of(const Wanted& w, int edge_m, int edge_n) {
  return (w.M + edge_m - 1) / edge_m * ((w.N + edge_n - 1) / edge_n) * w.n_outputs;
}
int64_t stages_of(const Wanted& w) { return (w.K + kBK - 1) / kBK * w.k_pairs; }

template <typename... Params, typename... Args>
psa_status_t launch(void (*kernel)(Params...), int64_t grid, unsigned threads, uint32_t smem, int cluster, cudaStream_t stream,
                    const Args&... args) {
  if (smem && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess) return PSA_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(grid));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {unsigned(cluster), 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = cluster ? 2 : 1;      // (0: the kernel says it itself)
  cudaLaunchKernelEx(&cfg, kernel, args...);
  return check_last_cuda_error("psa_ffn launch");
}

// Estimates in us that choose between the two kernels and the parts of K, fitted to both at 36 sizes (16 to 2500 tokens,
// 512 x 1408 to 4096 x 14336, L2 cold: of 216 chosen launches 85 % are within 15 % of their estimate, 97 % within 20 %, and the
// choice took 2.4 % longer than the fastest one in the mean).  A pair's stage takes 0.37 with all SMs at work, 0.31 with few, the
// end of a tile 2.4 and more where it is not hidden behind the next tile's stages.  A stage of a CTA alone takes 0.38 (0.25 with
// few tokens), of an SM's two CTAs together 0.56; the parts of a split K cross between the SMs of their cluster at 1 TB/s
// (2816 features, K = 1024, 128 tokens in 8 parts: 23 MB, 45 us instead of 16).  Where they differ most: 1815 x 2048,
// K = 5632: 40 us by pairs, 53 without; 129 tokens, dX = 1024, K = 2 x 2816: 36 by pairs, 22 in 4 parts of K.
double dram_us(const Wanted* w, int n, int epilogue) {
  double bytes = 0;
  for (int i = 0; i < n; ++i)
    bytes += 2.0 * (double(w[i].M) * w[i].K * w[i].k_pairs + double(w[i].K) * w[i].N * (w[i].b[1].p ? 2 : 1) +
                    double(w[i].M) * w[i].N * w[i].n_outputs * (epilogue == kEpiOut ? 1 : 3));
  return bytes / 6.0e6;
}
double pairs_us(const Wanted* w, int n, int epilogue) {
  const int tile_n = epilogue == kEpiGate ? kBigBN / 2 : kBigBN;
  const double clusters = kSmCount / 2;
  double sum = 0, longest = 0, tiles = 0;
  for (int i = 0; i < n; ++i) tiles += double(tiles_of(w[i], kBigBM, tile_n));
  const double stage = tiles <= clusters / 2 ? 0.31 : 0.37;
  for (int i = 0; i < n; ++i) {
    const double stages = double(stages_of(w[i])), end = epilogue == kEpiGate ? 7.5 : epilogue == kEpiGateBwd ? 14 : 2.4 + 0.2 * stages;
    const double each = std::max(stage * stages, end);
    sum += each * double(tiles_of(w[i], kBigBM, tile_n));
    longest = std::max(longest, each);
  }
  const double work = n == 1 ? std::ceil(tiles / clusters) * longest : std::max(longest, sum / clusters + longest / 2);
  return 9 + (epilogue == kEpiOut ? 0 : 4) + std::max(work, dram_us(w, n, epilogue));
}
double small_us(const Wanted* w, int n, int epilogue, int splits) {
  const int tile_n = epilogue == kEpiGate ? kSmallBN / 2 : kSmallBN;
  const double sms = kSmCount;
  double work = 0, join = 0, longest = 0;
  for (int i = 0; i < n; ++i) {
    const bool few = w[i].M <= 64;
    const double stages = std::ceil(double(stages_of(w[i])) / splits), tiles = double(tiles_of(w[i], kSmallBM, tile_n));
    const double alone = std::max((few ? 0.25 : 0.38) * stages, 3.0), both = std::max((few ? 0.36 : 0.56) * stages, 6.0);   // a CTA, two of an SM
    const double ctas = tiles * splits, waves = std::floor(ctas / (2 * sms)), rest = ctas - waves * 2 * sms, second = std::max(0.0, rest / sms - 1);
    // what a tile's end adds where one CTA does all of it
    const double end_alone = splits > 1 || epilogue == kEpiOut ? 0 : epilogue == kEpiGate ? 4 : 7, end_both = end_alone == 7 ? 24 : end_alone;
    if (n == 1)
      work = waves * (both + end_both) + (rest > 0 ? alone + end_alone + second * (both - alone + end_both - end_alone) : 0);
    else
      work += ctas / (2 * sms) * both;
    longest = std::max(longest, alone);
    join += tiles * (splits - 1) * double(std::min<int64_t>(w[i].M, kSmallBM)) * (4 * kSmallBN) / 1.0e6;
  }
  return 10 + (splits > 1 ? 2 : 0) + join + std::max({n == 1 ? work : work + longest / 2, longest, dram_us(w, n, epilogue)});
}
int best_splits(const Wanted* w, int n, int epilogue) {
  int best = 1;
  for (int s = 2; s <= 8; s *= 2)
    if (small_us(w, n, epilogue, s) < small_us(w, n, epilogue, best)) best = s;
  return best;
}
double best_us(const Wanted* w, int n, int epilogue) {
  return std::min(pairs_us(w, n, epilogue), small_us(w, n, epilogue, best_splits(w, n, epilogue)));
}

// Products that do not depend on one another, in one launch.
template <int EPI>
psa_status_t run(const Wanted* wanted, int n, ProductList list, cudaStream_t stream) {
  constexpr int kBigN = EPI == kEpiGate ? kBigBN / 2 : kBigBN, kSmallN = EPI == kEpiGate ? kSmallBN / 2 : kSmallBN;
  list.splits = best_splits(wanted, n, EPI);
  const bool pairs = pairs_us(wanted, n, EPI) < small_us(wanted, n, EPI, list.splits);
  const int edge_m = pairs ? kBigBM : kSmallBM, edge_n = pairs ? kBigN : kSmallN;
  list.n_products = n;
  list.a_rows = pairs || n > 1 || wanted[0].a[0].mn_major ? 128 : small_rows(wanted[0].M);
  int64_t first = 0;
  for (int i = 0; i < n; ++i) {
    const Wanted& w = wanted[i];
    Product& p = list.p[i];
    ProductMaps& maps = list.maps[i];
    for (int k = 0; k < 2; ++k) {
      if (w.a[k].p && !operand_maps(&maps.a[k], w.a[k].p, w.a[k].mn_major, w.M, w.K, list.a_rows)) return PSA_ERR_CUDA;
      if (w.b[k].p && !operand_maps(&maps.b[k], w.b[k].p, w.b[k].mn_major, w.N, w.K, 128)) return PSA_ERR_CUDA;
      p.out[k] = w.out[k];
      if (pairs && w.out[k] && !matrix_map(&maps.store[k], w.out[k], w.M, w.N, 32, EPI == kEpiGateBwd ? 32 : 64)) return PSA_ERR_CUDA;
    }
    p.M = int32_t(w.M);
    p.N = int32_t(w.N);
    p.k_tiles = int32_t((w.K + kBK - 1) / kBK);
    p.k_pairs = w.k_pairs;
    p.m_tiles = int32_t((w.M + edge_m - 1) / edge_m);
    p.n_tiles = int32_t((w.N + edge_n - 1) / edge_n);
    p.n_outputs = w.n_outputs;
    p.first = int32_t(first);
    p.a_mn = w.a[0].mn_major;
    p.b_mn = w.b[0].mn_major;
    p.early = w.early;
    first += tiles_of(w, edge_m, edge_n);
  }
  if (first > 0x7fffffff / 8) return PSA_ERR_UNSUPPORTED;
  list.n_work = int32_t(first);
  if (pairs) {
    const Wanted& w = wanted[0];
    if (EPI != kEpiOut && !matrix_map(&list.store_h, list.h, w.M, w.N, 32, EPI == kEpiGateBwd ? 32 : 64)) return PSA_ERR_CUDA;
    if (EPI == kEpiGateBwd && (!matrix_map(&list.in[0], list.gate, w.M, w.N, 32, 32) || !matrix_map(&list.in[1], list.up, w.M, w.N, 32, 32)))
      return PSA_ERR_CUDA;
    return launch(ffn_big_kernel<EPI>, 2 * std::min<int64_t>(first, kSmCount / 2), kBigThreads, kBigSmem, 0, stream, list);
  }
  return launch(ffn_small_kernel<EPI>, first * list.splits, kSmallThreads, kSmallSmem, list.splits, stream, list);
}

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

struct FfnWorkspace {
  size_t h, d_gate, d_up, total;
};
FfnWorkspace workspace_layout(int64_t T, int64_t F, bool backward) {
  const size_t act = aligned(size_t(T) * F * 2);
  return backward ? FfnWorkspace{0, act, 2 * act, 3 * act} : FfnWorkspace{0, 0, 0, act};
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
__nv_bfloat16* bf(void* p) { return static_cast<__nv_bfloat16*>(p); }

}  // namespace
}  // namespace psa

extern "C" size_t psa_ffn_workspace_bytes(int64_t n_tokens, int32_t hidden, int32_t ffn, int32_t backward) {
  if (psa::check_sizes(n_tokens, hidden, ffn) != PSA_OK) return 0;
  return psa::workspace_layout(n_tokens, ffn, backward != 0).total;
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
  cudaStream_t st = cudaStream_t(stream);
  ProductList list{};
  list.status = device_status;
  list.h = bf(workspace);
  const Wanted first{n_tokens, ffn, hidden, {{x, false}}, {{w_gate, true}, {w_up, true}}, {bf(gate), bf(up)}, 1, 1, false};
  const psa_status_t rc = run<kEpiGate>(&first, 1, list, st);
  if (rc != PSA_OK) return rc;
  const Wanted second{n_tokens, hidden, ffn, {{list.h, false}}, {{w_down, true}}, {bf(out)}, 1, 1, true};
  return run<kEpiOut>(&second, 1, list, st);
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
  const FfnWorkspace w = workspace_layout(n_tokens, ffn, true);
  char* ws = static_cast<char*>(workspace);
  __nv_bfloat16 *h = bf(ws + w.h), *d_gate = bf(ws + w.d_gate), *d_up = bf(ws + w.d_up);
  ProductList list{};
  list.status = device_status;
  list.h = h;
  list.gate = static_cast<const __nv_bfloat16*>(gate);
  list.up = static_cast<const __nv_bfloat16*>(up);
  // dH = dY Wd^T: Wd has K (hidden) innermost
  const Wanted dh{n_tokens, ffn, hidden, {{d_out, false}}, {{w_down, false}}, {d_gate, d_up}, 1, 1, false};
  const psa_status_t rc = run<kEpiGateBwd>(&dh, 1, list, st);
  if (rc != PSA_OK) return rc;
  const Wanted last[3] = {
      // dX = dG Wg^T + dU Wu^T
      {n_tokens, hidden, ffn, {{d_gate, false}, {d_up, false}}, {{w_gate, false}, {w_up, false}}, {bf(dx)}, 2, 1, true},
      // dWg = X^T dG and dWu = X^T dU
      {hidden, ffn, n_tokens, {{x, true}}, {{d_gate, true}, {d_up, true}}, {bf(dw_gate), bf(dw_up)}, 1, 2, false},
      // dWd = H^T dY
      {ffn, hidden, n_tokens, {{h, true}}, {{d_out, true}}, {bf(dw_down)}, 1, 1, true}};
  // One launch, unless dX, with its long K in few tiles, does better alone (less 4 us: the second starts behind the first).
  if (best_us(last, 3, kEpiOut) <= best_us(last, 1, kEpiOut) + best_us(last + 1, 2, kEpiOut) - 4) return run<kEpiOut>(last, 3, list, st);
  const psa_status_t first = run<kEpiOut>(last, 1, list, st);
  return first != PSA_OK ? first : run<kEpiOut>(last + 1, 2, list, st);
}
