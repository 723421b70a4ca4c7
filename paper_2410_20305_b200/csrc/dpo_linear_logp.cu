// dpo_linear_logp / dpo_linear_logp_bwd: the log-probabilities of dpo_logp, and their gradient, from the hidden states h and the
// output table W, without the logits in between:
//     z[t, v] = scale * <h[t], W[v]>,   lse[t] = log sum_v exp(z[t, v]),   out[g] = sum over labels (t, y, g) of z[t, y] - lse[t],
//     dz[t, v] = scale * sum over labels (t, y, g) of coef[g] * (1[v = y] - exp(z[t, v] - lse[t])),
//     dh[t] = sum_v dz[t, v] W[v],   dW[v] = sum_t dz[t, v] h[t].
// Labels first: one kernel lists them (a row's own label, then the forks), so that each is a row of its own of the products, and
// a second copies their hidden rows side by side.  Rows that score nothing (the prompts) take part in nothing behind that.
// Forward: a tile of 256 labels x 256 tokens of the vocabulary is summed in TMEM and leaves as each row's maximum and sum of
// exponentials, the label's own left out; a last kernel joins the parts of a row.  With z the label's logit, a product of its own, its
// term is -log(1 + sum over the other tokens of exp(z[t, v] - z)): nothing near 1 is rounded and subtracted where the label is nearly certain.
// Backward: the logits once more, in pieces of the vocabulary; their tile leaves as dz, rounded to bf16 as tcgen05.mma takes it
// (2^-8 of each element at most, independent of one another), and both gradients are products with it.  dh is summed over
// pieces in fp32, and gets back what the label's element has lost; a piece of dW is complete.
// Bound by the tensor cores: 2 n V D operations forward and 6 n V D backward for n labels; with few labels by the table's bytes.
// Measured: 8499 labels of 16215 rows, 128256 x 4096, forward and backward 26.5 to 27.8 ms (1.28 to 1.35 PFLOP/s under the power cap);
// 988 of 15154, forward, 655 to 667 us alone (1.57 PFLOP/s) and 800 to 848 under repetition; one label 207 to 228 us (the table at 6 TB/s in the
// product); 1145 labels, 50257 x 1032, both 570 to 583 us; 206 labels, 1024 x 256, both 52 to 55 us (nine launches).
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
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

// tcgen05 cuts off what an addition of fp32 rounds.  Of a logit, a sum of terms of both signs, that takes 2^-30 of itself for each of its terms in the
// mean (2^-30 is 0.93e-9; measured 0.94e-9 at 1024 and 2048 columns, 0.98, 1.02 and 1.03e-9 at 4096, 8192 and 16384; sums of one sign lose 1.7 to 5 times as
// much), which the scale gives back: a log-probability of 128256 x 4096 was off by 1.2e-6 of itself and is by 2e-8 to 8e-8.
// A label's own product, by fp32 additions, takes the scale without it.
constexpr double cut_off(int32_t width) { return 1.0 + width * 0x1p-30; }

// ---------------------------------------------------------------- labels
// What the kernels of a call share, at the head of its workspace.
struct Shared {
  int32_t n_own, n_labels;      // labels of rows themselves; all labels
  int32_t finished;             // CTAs of the last kernel that have added their terms
};
struct Labels {
  Shared* shared;
  int32_t *row, *target, *segment;   // of each label: own labels in the rows' order, then the forks'
  // Of each row of hidden: its own label + 1 (0 without one), and the label of a fork that names it + 1 (0 without one), from which `next`
  // (backward) leads to the others, in no order.
  int2* state;
  int32_t* next;
  unsigned long long* best;          // forward, of each row that a fork names: the largest of its labels' ranked()
};
// A label's logit and the row's lse as it finds it, so that the largest is that of the likeliest label (or a NaN).  That label's logit is
// a product of its own in its lse, the row's other labels' are not: theirs weigh least.
__device__ __forceinline__ uint32_t rising(float v) {      // in the order of floats
  const uint32_t bits = __float_as_uint(v);
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ unsigned long long ranked(float logit, float lse) {
  return static_cast<unsigned long long>(rising(logit)) << 32 | rising(lse);
}
__device__ __forceinline__ float lse_of(unsigned long long rank) {
  const uint32_t bits = uint32_t(rank);
  return __uint_as_float(bits & 0x80000000u ? bits & 0x7fffffffu : ~bits);
}

// The sum of a response's terms as whole numbers, which do not depend on their order: floor(term), a term taken as -2^38 where it is below
// (2^25 labels, the most that there may be, then stay within 64 bits), and its rest in units of 2^-40.  From 2^24 labels on the rests may pass
// 2^64 units: the addition that sees them do so adds 2^24 to the whole numbers.
struct Sum {
  long long whole;
  unsigned long long rest;
  uint32_t odd, pad;                 // 1: a NaN was added, 2: an infinity
};
__device__ __forceinline__ void add_term(Sum* sum, double term) {
  if (!(fabs(term) <= 1.0e300)) {
    atomicOr(&sum->odd, term == term ? 2u : 1u);
    return;
  }
  term = fmin(fmax(term, -274877906944.0), 0.0);      // (a probability that rounding has put above 1 counts as 1)
  const double floored = floor(term);
  const unsigned long long rest = static_cast<unsigned long long>((term - floored) * 1099511627776.0 + 0.5);
  const unsigned long long before = atomicAdd(&sum->rest, rest);
  const long long whole = static_cast<long long>(floored) + (before + rest < before ? 1 << 24 : 0);
  atomicAdd(reinterpret_cast<unsigned long long*>(&sum->whole), static_cast<unsigned long long>(whole));
}
__device__ __forceinline__ float sum_of(const Sum& s) {
  if (s.odd & 1) return __uint_as_float(0x7fc00000u);
  if (s.odd & 2) return -INFINITY;
  return float(double(s.whole) + double(s.rest) * (1.0 / 1099511627776.0));
}

// One CTA lists the labels: rows are looked at 8192 at a time, and a label's place is the number of labels in front of it.
constexpr int kListThreads = 1024, kListEach = 8;
__global__ void __launch_bounds__(kListThreads)
logp_list_kernel(const int32_t* targets, const int32_t* segment_ids, const int32_t* fork_rows, const int32_t* fork_targets,
                 const int32_t* fork_segments, int32_t n_rows, int32_t n_forks, int32_t n_segments, int32_t vocab, Labels labels,
                 Sum* sums, int32_t* status) {
  constexpr int kWarps = kListThreads / 32, kCounts = kListEach * kWarps;
  __shared__ int32_t s_count[kCounts], s_warp[kCounts / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  behind_wait();
  behind_go();
  for (int g = threadIdx.x; sums && g < n_segments; g += kListThreads) sums[g] = Sum{0, 0, 0, 0};
  int32_t base = 0, n_own = 0;
  for (int list = 0; list < 2; ++list) {
    const int32_t n = list ? n_forks : n_rows;
    const int32_t *y_of = list ? fork_targets : targets, *g_of = list ? fork_segments : segment_ids;
    for (int32_t first = 0; first < n; first += kListThreads * kListEach) {
      int32_t row[kListEach], y[kListEach], g[kListEach];
      uint32_t mine[kListEach];
#pragma unroll
      for (int j = 0; j < kListEach; ++j) {
        const int32_t i = first + j * kListThreads + int32_t(threadIdx.x);
        const bool in = i < n;
        row[j] = !in ? -1 : list ? fork_rows[i] : i;
        y[j] = in ? y_of[i] : 0;
        g[j] = in ? g_of[i] : -1;
      }
#pragma unroll
      for (int j = 0; j < kListEach; ++j) {
        bool valid = g[j] >= 0 && row[j] >= 0 && row[j] < n_rows;      // (a fork that names no row is none)
        if (valid && g[j] >= n_segments) {
          if (status) atomicOr(status, PSA_DEVSTAT_BAD_SEGMENT);
          valid = false;
        }
        if (valid && (y[j] < 0 || y[j] >= vocab)) {
          if (status) atomicOr(status, PSA_DEVSTAT_BAD_TARGET);
          valid = false;
        }
        mine[j] = __ballot_sync(0xffffffffu, valid);
        if (lane == 0) s_count[j * kWarps + warp] = __popc(mine[j]);
      }
      __syncthreads();
      // counts become places: 32 of them by each of the first warps, then those of the warps in front are added
      int32_t v = 0, up = 0;
      if (warp < kCounts / 32) {
        v = up = s_count[threadIdx.x];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const int32_t w = __shfl_up_sync(0xffffffffu, up, o);
          if (lane >= o) up += w;
        }
        if (lane == 31) s_warp[warp] = up;
      }
      __syncthreads();
      if (warp < kCounts / 32) {
        int32_t in_front = base;
        for (int w = 0; w < warp; ++w) in_front += s_warp[w];
        s_count[threadIdx.x] = in_front + up - v;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kListEach; ++j) {
        const bool valid = (mine[j] >> lane) & 1;
        const int32_t place = s_count[j * kWarps + warp] + __popc(mine[j] & ((1u << lane) - 1));
        if (valid) {
          labels.row[place] = row[j];
          labels.target[place] = y[j];
          labels.segment[place] = g[j];
        }
        if (!list && row[j] >= 0) labels.state[row[j]] = make_int2(valid ? place + 1 : 0, 0);
        if (list && valid) {
          const int32_t other = atomicExch(&labels.state[row[j]].y, place + 1);
          if (labels.next) labels.next[place] = other;
          if (labels.best) labels.best[row[j]] = 0;
        }
      }
#pragma unroll
      for (int w = 0; w < kCounts / 32; ++w) base += s_warp[w];
      __syncthreads();
    }
    if (!list) n_own = base;
  }
  if (threadIdx.x == 0) *labels.shared = Shared{n_own, base, 0};
}

__host__ __device__ constexpr int64_t padded(int64_t n) { return (n + 255) / 256 * 256; }

// The hidden rows of the labels side by side, zeros behind the last one to the next multiple of 256 (and in the first 256 where
// there is no label), and the label's own product, by fp32 additions that round: what is left of a nearly certain label's
// probability is off, relative to itself, by the errors of the logits that it is taken from, and its own is the largest.  For the backward
// pass what a label's row of dz takes: coef * scale, lse in units of log 2, and its element at the label, coef * scale * (1 - p) from the
// product that the forward took lse from (from tcgen05's, d_hidden was off by 1.8 of its norm at 1 - p = 1e-4 and a logit of 16).
// kWarps of a CTA's 8 take a row: all of them in a small call, where a row's trips to memory one after the other are what counts.  The
// border lies at 2048 labels: forward at width 1024, vocabulary 8192, with one warp and with eight, 256 labels 32.7 and 30.7 us, 1024 38.5
// and 36.5, 2048 50.8 and 50.8, 4096 70.7 and 71.7, 8192 117 and 122; at width 4096 57.3 and 49.2, 79.5 and 72.7, 122.5 and 118.4, 194.5 and 191, 372 and 367.
template <int kWarps>
__global__ void __launch_bounds__(256)
logp_gather_kernel(const uint4* hidden, const uint4* table, Labels labels, int32_t vectors, int32_t pitch, uint4* rows, const float* coef, const float* lse,
                   float scale, double label_scale, float2* of_label, float* label_value) {
  constexpr int kThreads = 32 * kWarps;
  __shared__ float s_sum[8];
  const int tid = int(threadIdx.x) % kThreads, lane = threadIdx.x & 31;
  const int64_t i = int64_t(blockIdx.x) * (8 / kWarps) + int(threadIdx.x) / kThreads;
  behind_wait();
  behind_go();
  const int32_t n = labels.shared->n_labels;
  if (i >= max(padded(n), int64_t(256))) return;
  uint4* to = rows + i * pitch;
  if (i >= n) {
    for (int c = tid; c < vectors; c += kThreads) to[c] = make_uint4(0, 0, 0, 0);
    return;
  }
  const int32_t t = labels.row[i];
  const bool ends = tid == 0 && coef;      // (what it needs then, requested now)
  const float factor = ends ? coef[labels.segment[i]] * scale : 0.f, of_row = ends ? lse[t] : 0.f;
  const uint4* from = hidden + int64_t(t) * vectors;
  const uint4* weight = table + int64_t(labels.target[i]) * vectors;
  float sum[8] = {};
#pragma unroll 4
  for (int c = tid; c < vectors; c += kThreads) {
    const uint4 h = from[c], w = weight[c];
    to[c] = h;
    const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sum[2 * j] = fmaf(__uint_as_float(hw[j] << 16), __uint_as_float(ww[j] << 16), sum[2 * j]);
      sum[2 * j + 1] = fmaf(__uint_as_float(hw[j] & 0xffff0000u), __uint_as_float(ww[j] & 0xffff0000u), sum[2 * j + 1]);
    }
  }
  float all = ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
#pragma unroll
  for (int o = 16; o; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  if (kWarps > 1) {      // (a row a CTA: all threads are here)
    if (lane == 0) s_sum[tid >> 5] = all;
    __syncthreads();
    all = ((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3])) + ((s_sum[4] + s_sum[5]) + (s_sum[6] + s_sum[7]));
  }
  if (tid == 0 && !coef) label_value[i] = all;
  if (!ends) return;
  // (as the forward scales it; where fp32 does not tell it from lse, p is 1)
  const double z = double(all) * label_scale * kLn2;
  const float logp = float(z) == of_row ? 0.f : float(z - double(of_row));
  of_label[i] = make_float2(factor, of_row * kLog2e);
  label_value[i] = -factor * expm1f(logp > 0.f ? 0.f : logp);      // (NaN stays)
}

// ---------------------------------------------------------------- products
// A persistent kernel: 74 clusters of two CTAs take tiles of 256 x 256.  A tile's product is one UMMA stream of the pair: each
// CTA loads its 128 rows of A and 128 of the tile's 256 columns of B.  (Narrower tiles of the vocabulary, to fill the last round over
// the clusters, took longer: the loads, 64 bytes a clock and SM, bind as soon as a tile is: 988 labels x 128256 x 4096 677 -> 689 us
// with 240 columns, 1145 x 50257 x 1032 107 -> 128.)  The accumulator takes half of TMEM: while the end of one
// tile drains it, the next tile's UMMAs fill the other half.
// Warps: 0 TMA, 1 UMMA (in the CTA of rank 0), 2 TMEM, 4-7 the end of a tile, each for 32 rows of its CTA.
enum Epilogue {
  kEpiStats,      // logits -> each row's maximum and sum of exponentials
  kEpiGrad,       // logits -> dz
  kEpiOut,        // two products: parts of dh (fp32), dW (bf16)
};
constexpr int kTile = 256, kThreads = 256, kBufs = 4;
constexpr uint32_t kHalf = 128 * kBK * 2;                       // one operand's half of a stage
constexpr uint32_t kStageBytes = 2 * kHalf;
constexpr uint32_t kBufBytes = 32 * 128;                        // 32 rows of 128 bytes
template <int EPI>
__host__ __device__ constexpr int stages_of() { return EPI == kEpiStats ? 6 : 5; }
template <int EPI>
__host__ __device__ constexpr uint32_t bars_at() { return stages_of<EPI>() * kStageBytes + (EPI == kEpiStats ? 0 : 4 * kBufs * kBufBytes); }
template <int EPI>
__host__ __device__ constexpr uint32_t smem_of() { return bars_at<EPI>() + 256 + 1024; }
static_assert(smem_of<kEpiStats>() <= 227 * 1024 && smem_of<kEpiOut>() <= 227 * 1024, "shared memory of one CTA");

struct Operands {
  OperandMaps a, b;
  CUtensorMap store;      // boxes of 32 rows x 128 bytes of the output
};
struct ProductArgs {
  Operands of[2];         // kEpiOut: dh, dW;  else the logits (of[0])
  const Shared* shared;
  const int32_t* target;
  const float2* of_label;
  const float* label_dz;
  float2* stats;          // [tiles of the vocabulary][l_pad]: maximum and sum of exponentials, in units of log 2, without the label's own
  int64_t l_pad;
  int32_t hidden, columns, first_column;     // columns of this piece of the vocabulary, and where it starts
  int32_t splits;         // parts of dh's K, each with rows of its own of the output
  int32_t add;            // dh is added to what is there
  int32_t with_table;     // dW is wanted
  float scale_log2;       // scale / log 2, with what the sums have lost
  int32_t* status;
};

// A tile of a launch: which product, where, and its stages of K.
struct Tile {
  int which, m0, n0, part, k0, k1;
};
// What a tile of dW costs beside its stages (0.37 us each): its end, 3.3 us with the tile's bytes on their way to memory, where there are
// few stages, and a part of that where there are more.  (Counted by their stages alone, 1 to 64 labels of 128256 x 4096 took 1288 us
// instead of 480, 256 took 784 instead of 577, 512 940 instead of 850: clusters without a heavy tile took too many of them.  The whole
// backward with 3, 6, 9 and 14: 64 labels of that table 831, 659, 667 and 676 us, 256 of it 882, 832, 749 and 766, 64 of 50257 x 1032 139, 125, 120 and
// 124, 300 of 50257 x 768 141, 131, 124 and 128, 2 of 32000 x 4096 273, 209, 202 and 209.)
constexpr int kEndStages = 9;

// The tiles that a cluster takes.  Those of the first product (`heavy`) go round the clusters one by one; of the second, clusters
// that have one heavy tile less take as many more as fit into its time, and the rest goes round again.
struct Schedule {
  int c, n, heavy, light, mine, rest, extra, from;
  __device__ __forceinline__ Schedule(int cluster, int clusters, int heavy_, int light_, int cost_heavy, int cost_light)
      : c(cluster), n(clusters), heavy(heavy_), light(light_) {
    const int q = heavy / n;
    rest = heavy % n;                     // clusters below it have q + 1
    mine = q + (c < rest);
    extra = rest ? min(cost_heavy / cost_light, light / (n - rest)) : 0;
    from = extra * (n - rest);            // the first light tile that goes round
  }
  // The cluster's i-th tile: a heavy one's index, or heavy + a light one's; -1 behind the last.
  __device__ __forceinline__ int at(int i) const {
    if (i < mine) return i * n + c;
    i -= mine;
    int k;
    if (rest && c >= rest) {
      if (i < extra) return heavy + i * (n - rest) + c - rest;
      k = from + (i - extra) * n + c;
    } else {
      k = from + i * n + c;
    }
    return k < light ? heavy + k : -1;
  }
};
// Tiles run down `group` rows of tiles before they move one column on, so that the tiles in flight share strips of A and of B in L2.  The logits'
// 16: with 8, 8499 labels of 128256 x 4096 took 6.60 ms instead of 6.35, with 32 as long.  dh's 9: with 4, 5 and 16, backward passes of 1145 to 8499
// labels and widths of 1024 to 4096 came out within what repetitions of the same differ by (up to 8 %, under
// the power cap).
__device__ __forceinline__ void place(int at, int m_tiles, int n_tiles, int group, Tile* t) {
  const int per_group = group * n_tiles, g = at / per_group, first = g * group, rows = min(group, m_tiles - first), in = at - g * per_group;
  t->m0 = (first + in % rows) * kTile;
  t->n0 = in / rows * kTile;
}

template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
logp_product_kernel(const __grid_constant__ ProductArgs args) {
  constexpr int kStages = stages_of<EPI>();
  constexpr uint32_t kBarsAt = bars_at<EPI>(), kBufsAt = kStages * kStageBytes;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + kBarsAt;
  auto full = [&](int s) { return bars + 8u * s; };                    // of rank 0: both CTAs' loads
  auto empty = [&](int s) { return bars + 8u * (kStages + s); };
  auto acc_full = [&](int i) { return bars + 8u * (2 * kStages + i); };
  auto acc_empty = [&](int i) { return bars + 8u * (2 * kStages + 2 + i); };   // of rank 0: both CTAs' warps
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_base + kBarsAt + 240);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_base + kBarsAt + 248);
  static_assert(8 * (2 * kStages + 4) <= 240, "barriers");
  const WaitCtx wctx{abort_flag, args.status, kWaitLimitClocks};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(acc_full(i), 1); mbar_init(acc_empty(i), 8); }
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

  const int n_labels = args.shared->n_labels;
  // (without labels the gradients are those of 256 rows of zeros)
  const int m_tiles = EPI == kEpiStats ? (n_labels + kTile - 1) / kTile : max(1, (n_labels + kTile - 1) / kTile);
  const int v_tiles = (args.columns + kTile - 1) / kTile, d_tiles = (args.hidden + kTile - 1) / kTile;
  const int d_stages = (args.hidden + kBK - 1) / kBK, v_stages = (args.columns + kBK - 1) / kBK, l_stages = max(1, (n_labels + kBK - 1) / kBK);
  const int n_heavy = EPI == kEpiOut ? m_tiles * d_tiles * args.splits : 0, n_light = EPI == kEpiOut ? (args.with_table ? v_tiles * d_tiles : 0) : m_tiles * v_tiles;
  // dW: as many rows of tiles as let the tiles in flight write whole rows of the table
  const int dw_group = max(1, min(16, (int(gridDim.x) >> 1) / d_tiles));
  const Schedule schedule(int(blockIdx.x) >> 1, int(gridDim.x) >> 1, n_heavy, n_light, v_stages / args.splits, max(kEndStages, l_stages + kEndStages / 2));
  auto tile_at = [&](int i, Tile* t) {
    int at = schedule.at(i);
    if (at < 0) return false;
    if (EPI != kEpiOut) {
      place(at, m_tiles, v_tiles, 16, t);
      t->which = t->part = t->k0 = 0;
      t->k1 = d_stages;
    } else if (at < n_heavy) {
      t->part = at / (m_tiles * d_tiles);
      place(at - t->part * m_tiles * d_tiles, m_tiles, d_tiles, 9, t);
      t->which = 0;
      t->k0 = int(int64_t(v_stages) * t->part / args.splits);
      t->k1 = int(int64_t(v_stages) * (t->part + 1) / args.splits);
    } else {
      place(at - n_heavy, v_tiles, d_tiles, dw_group, t);
      t->which = 1;
      t->part = t->k0 = 0;
      t->k1 = l_stages;
    }
    return true;
  };
  // Which way the operands lie: logits A = h, B = W, both K-major; dh: A = dz K-major, B = W MN-major; dW: both MN-major.
  auto a_mn_of = [&](const Tile& t) { return EPI == kEpiOut && t.which == 1; };
  constexpr bool b_mn = EPI == kEpiOut;

  if (warp == 0) {
    const uint32_t issuer = elect_one();
    int n = 0;
    Tile t;
    for (int i = 0; !*abort_flag && tile_at(i, &t); ++i) {
      const Operands& of = args.of[t.which];
      const int m_end = t.which == 1 ? args.columns : int(args.l_pad), n_end = EPI == kEpiOut ? args.hidden : args.columns;
      const Strip a(&of.a, a_mn_of(t), t.m0 + 128 * int(rank), m_end), b(&of.b, b_mn, t.n0 + 128 * int(rank), n_end);
      for (int it = t.k0; it < t.k1; ++it, ++n) {
        const int s = n % kStages;
        if (n >= kStages) mbar_wait(empty(s), (n / kStages - 1) & 1, wctx);
        if (*abort_flag) break;
        const uint32_t sa = base + s * kStageBytes, bar = cluster_map(full(s), 0);
        auto load = [&](uint32_t dst, const CUtensorMap* m, int c0, int c1, int c2) { tma_load_3d_pair_w(dst, m, c0, c1, c2, bar, issuer); };
        mbar_expect_tx_w(full(s), 2 * kStageBytes, rank == 0 ? issuer : 0u);
        a.load(0, it * kBK, sa, load);
        b.load(0, it * kBK, sa + kHalf, load);
      }
    }
    if (*abort_flag) {   // shared memory must outlive the copies in flight (the cluster's last barrier holds the other CTA)
      const long long t0 = clock64();
      if (rank == 0)
        for (int i = n > kStages ? n - kStages : 0; i < n; ++i)
          while (!mbar_try_wait(full(i % kStages), (i / kStages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
      while (clock64() - t0 < 1000000) {}
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t issuer = elect_one();
      int n = 0;
      Tile t;
      for (int i = 0; !*abort_flag && tile_at(i, &t); ++i) {
        const bool a_mn = a_mn_of(t);
        const uint32_t idesc = umma_idesc_bf16(kTile, kTile, false, false) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16);
        const uint32_t a_step = (a_mn ? 2048 : 32) >> 4, b_step = (b_mn ? 2048 : 32) >> 4;
        const uint32_t acc = tmem + uint32_t(i & 1) * 256;
        mbar_wait_cluster(acc_empty(i & 1), ((i >> 1) & 1) ^ 1, wctx);
        tc_fence_after();
        for (int it = t.k0; it < t.k1; ++it, ++n) {
          const int s = n % kStages;
          mbar_wait_cluster(full(s), (n / kStages) & 1, wctx);
          if (*abort_flag) break;
          tc_fence_after();
          const uint32_t sa = base + s * kStageBytes;
          const uint32_t a = smem_desc_lo(sa, a_mn ? kSub : 16), b = smem_desc_lo(sa + kHalf, b_mn ? kSub : 16);
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk)
            umma_ss_pair_w(acc, a + kk * a_step, b + kk * b_step, idesc, it > t.k0 || kk > 0, issuer);
          umma_commit_pair_w(empty(s), issuer);
        }
        umma_commit_pair_w(acc_full(i & 1), issuer);
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    const int w = warp - 4;
    const uint32_t issuer = elect_one();     // the lane that owns the warp's groups of stores
    const uint32_t bufs = base + kBufsAt + uint32_t(w) * kBufs * kBufBytes;
    auto buf = [&](uint32_t use) { return bufs + (use % kBufs) * kBufBytes; };
    // 16 bytes of this thread's row in a buffer, in the 128-byte-swizzled layout of the tensor maps
    auto cell = [&](uint32_t b, int sixteen) { return b + uint32_t(lane) * 128 + ((uint32_t(sixteen) ^ uint32_t(lane & 7)) << 4); };
    uint32_t use = 0;      // buffers used so far; each is one group of stores
    auto room = [&]() {    // a buffer's last store has read it
      if (issuer) tma_wait_group_read<kBufs - 1>();
      __syncwarp();
    };
    auto drained = [&](int i) {      // this warp has read the accumulator
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(cluster_map(acc_empty(i & 1), 0));
    };
    Tile t;
    for (int i = 0; !*abort_flag && tile_at(i, &t); ++i) {
      const int row0 = t.m0 + 128 * int(rank) + 32 * w, row = row0 + lane;
      const uint32_t lanes = tmem + uint32_t(i & 1) * 256 + (uint32_t(w * 32) << 16);
      const bool live = row < n_labels;
      int y = -1;
      float2 own = make_float2(0.f, 0.f);
      float own_dz = 0.f;
      if (EPI != kEpiOut && live && PSA_IN_BOUNDS(row, args.l_pad, args.status)) {
        y = args.target[row] - args.first_column - t.n0;      // the label's column in the tile
        if (EPI == kEpiGrad) {
          own = args.of_label[row];
          own_dz = args.label_dz[row];
        }
      }
      mbar_wait(acc_full(i & 1), (i >> 1) & 1, wctx);
      tc_fence_after();
      if (*abort_flag) break;
      if (EPI == kEpiStats) {
        const int n_columns = args.columns - t.n0;       // of the vocabulary, from this tile on
        float m = -INFINITY, sum = 0.f;
#pragma unroll 1
        for (int c = 0; c < kTile; c += 64) {
          uint32_t v[64];
          tmem_ld64_wait(lanes + c, v);
          if (c == kTile - 64) drained(i);
          float* z = reinterpret_cast<float*>(v);
          if (c + 64 > n_columns)
#pragma unroll
            for (int j = 0; j < 64; ++j) z[j] = c + j < n_columns ? z[j] : -INFINITY;
          const int at = y - c;
          if (__any_sync(0xffffffffu, at >= 0 && at < 64)) {
#pragma unroll
            for (int j = 0; j < 64; ++j) z[j] = j == at ? -INFINITY : z[j];
          }
          float top[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
          for (int j = 4; j < 64; j += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) top[k] = max3(top[k], z[j + k], z[min(j + 4 + k, 63)]);
          const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * args.scale_log2;
          const float mn = fmaxf(m, mx);
          // (logits that are all -inf so far are taken against 0, so that (-inf) - (-inf) never forms)
          const float shift = mn == -INFINITY ? 0.f : mn;
          float s[4] = {sum * ex2_approx(m - shift), 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 64; ++j) s[j & 3] += ex2_approx(fmaf(z[j], args.scale_log2, -shift));
          sum = (s[0] + s[1]) + (s[2] + s[3]);
          m = mn;
        }
        if (live && PSA_IN_BOUNDS(row, args.l_pad, args.status)) args.stats[int64_t(t.n0 / kTile) * args.l_pad + row] = make_float2(m, sum);
      } else if (EPI == kEpiGrad) {
#pragma unroll 1
        for (int c = 0; c < kTile; c += 64, ++use) {
          uint32_t v[64];
          tmem_ld64_wait(lanes + c, v);
          if (c == kTile - 64) drained(i);
          float* z = reinterpret_cast<float*>(v);
#pragma unroll
          for (int j = 0; j < 64; ++j) z[j] = -own.x * ex2_approx(fmaf(z[j], args.scale_log2, -own.y));
          const int at = y - c;
          if (__any_sync(0xffffffffu, at >= 0 && at < 64)) {
#pragma unroll
            for (int j = 0; j < 64; ++j) z[j] = j == at ? own_dz : z[j];
          }
          if (!live)      // zeros, whatever the table holds
#pragma unroll
            for (int j = 0; j < 64; ++j) z[j] = 0.f;
          room();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint4 q = pack8(z + 8 * j);
            st_shared_v4(cell(buf(use), j), q.x, q.y, q.z, q.w);
          }
          fence_proxy_async_smem();
          __syncwarp();
          tma_store_3d_w(&args.of[0].store, buf(use), t.n0 + c, 0, row0, t.n0 + c < args.columns ? issuer : 0u);
          if (issuer) tma_commit_group();
        }
      } else if (t.which == 0) {      // dh: boxes of 32 columns of fp32
        const int64_t to_row = int64_t(t.part) * args.l_pad + row0;
#pragma unroll 1
        for (int c = 0; c < kTile; c += 32, ++use) {
          uint32_t v[32];
          tmem_ld32_wait(lanes + c, v);
          if (c == kTile - 32) drained(i);
          room();
#pragma unroll
          for (int j = 0; j < 8; ++j) st_shared_v4(cell(buf(use), j), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          fence_proxy_async_smem();
          __syncwarp();
          if (issuer && row0 < n_labels && t.n0 + c < args.hidden) {
            if (args.add) tma_reduce_add_3d(&args.of[0].store, buf(use), t.n0 + c, 0, int(to_row));
            else tma_store_3d(&args.of[0].store, buf(use), t.n0 + c, 0, int(to_row));
          }
          if (issuer) tma_commit_group();
          __syncwarp();
        }
      } else {                        // dW: boxes of 64 columns of bf16
#pragma unroll 1
        for (int c = 0; c < kTile; c += 64, ++use) {
          uint32_t v[64];
          tmem_ld64_wait(lanes + c, v);
          if (c == kTile - 64) drained(i);
          room();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint4 q = pack8(reinterpret_cast<const float*>(v) + 8 * j);
            st_shared_v4(cell(buf(use), j), q.x, q.y, q.z, q.w);
          }
          fence_proxy_async_smem();
          __syncwarp();
          tma_store_3d_w(&args.of[1].store, buf(use), t.n0 + c, 0, row0, row0 < args.columns && t.n0 + c < args.hidden ? issuer : 0u);
          if (issuer) tma_commit_group();
        }
      }
    }
    if (issuer) tma_wait_group<0>();   // shared memory must outlive the stores' reads, and the next kernel sees their writes
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

// ---------------------------------------------------------------- ends
// Joins the parts of 32 labels' rows (a lane each, the warps share the vocabulary's tiles), adds their terms to the responses'
// sums and writes lse; the last CTA turns the sums into out, and writes lse of the rows that forks name.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps)
logp_join_kernel(const float2* stats, const float* label_logit, Labels labels, int64_t l_pad, int32_t v_tiles, int32_t n_rows, int32_t n_segments,
                 double label_scale, Sum* sums, float* out, float* lse) {
  __shared__ float2 s_part[kJoinWarps][32];
  __shared__ bool s_last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  behind_wait();
  behind_go();
  const int32_t n = labels.shared->n_labels, i = int32_t(blockIdx.x) * 32 + lane;
  // rows that score nothing
  for (int64_t t = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; t < n_rows; t += int64_t(gridDim.x) * blockDim.x)
    if ((labels.state[t].x | labels.state[t].y) == 0) lse[t] = 0.f;
  if (int32_t(blockIdx.x) * 32 < n) {
    float m = -INFINITY, s = 0.f;
    auto merge = [&](float2 p) {
      const float mn = fmaxf(m, p.x);
      if (mn == -INFINITY) {      // nothing finite on either side: both sums are 0, or NaN where a logit was
        s += p.y;
        return;
      }
      s = s * ex2_approx(m - mn) + p.y * ex2_approx(p.x - mn);
      m = mn;
    };
    if (i < n) {
      int v = warp;
      for (; v + 7 * kJoinWarps < v_tiles; v += 8 * kJoinWarps) {
        float2 p[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) p[k] = stats[int64_t(v + k * kJoinWarps) * l_pad + i];
#pragma unroll
        for (int k = 0; k < 8; ++k) merge(p[k]);
      }
#pragma unroll 4
      for (; v < v_tiles; v += kJoinWarps) merge(stats[int64_t(v) * l_pad + i]);
    }
    s_part[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (warp == 0 && i < n) {
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int k = 0; k < kJoinWarps; ++k) top[k & 1] = fmaxf(top[k & 1], s_part[k][lane].x);
      m = fmaxf(top[0], top[1]);
      const float shift = m == -INFINITY ? 0.f : m;      // (nothing finite: all sums are 0, or NaN where a logit was)
      float all[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kJoinWarps; ++k) all[k & 1] += s_part[k][lane].y * ex2_approx(s_part[k][lane].x - shift);
      s = all[0] + all[1];
      // The other tokens' sum, s 2^m, against the label's own exponential; where that is far below it, the label's share of the row's sum is
      // lost in any case.
      const double label = double(label_logit[i]) * label_scale, apart = label - double(m);
      double term, row_lse;
      if (apart > -512.0) {
        const double others = log1p(double(s) * exp2(-apart));
        term = -others;
        row_lse = label * kLn2 + others;
      } else {
        const double log2s = log2(double(s));
        term = (apart - log2s) * kLn2;
        row_lse = (double(m) + log2s) * kLn2;
      }
      // (a label of +inf is not finite, and beside others of -inf alone one of -inf has nothing to be compared with)
      if (!(label < INFINITY) || apart != apart) term = row_lse = NAN;
      add_term(sums + labels.segment[i], term);
      const int32_t t = labels.row[i];
      if (labels.state[t].y) atomicMax(labels.best + t, ranked(label_logit[i], float(row_lse)));      // (several labels may score it)
      else lse[t] = float(row_lse);
    }
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) s_last = atomicAdd(&labels.shared->finished, 1) == int32_t(gridDim.x) - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  for (int g = threadIdx.x; g < n_segments; g += blockDim.x) {
    const Sum s{__ldcg(&sums[g].whole), __ldcg(&sums[g].rest), __ldcg(&sums[g].odd), 0};
    out[g] = sum_of(s);
  }
  for (int32_t k = labels.shared->n_own + int32_t(threadIdx.x); k < n; k += blockDim.x) {
    const int32_t t = labels.row[k];
    lse[t] = lse_of(__ldcg(labels.best + t));
  }
}

// dh of every row of hidden: the sum over its own label and the forks that name it, each the sum of its parts; zeros where it scores nothing.
// The label's element is most of a row of dz: what its rounding to bf16 has taken joins here, times its row of the table (dh's error in the 2-norm,
// the result's own rounding of 0.0017 with it, 0.0024 to 0.0026 -> 0.0017).
// Two labels are added as they come.  More, which are listed in no order, as whole numbers: the largest magnitude of a column gives a unit in which
// all of them stay within 62 bits and lose what is 2^-35 of it at most, so that their sum depends on no order.
__global__ void __launch_bounds__(256)
logp_scatter_kernel(const float* parts, const float* label_dz, const uint32_t* table, Labels labels, int32_t n_rows, int32_t hidden, int64_t l_pad,
                    int32_t splits, uint4* d_hidden) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t t = int64_t(blockIdx.x) * 8 + warp;
  behind_wait();
  behind_go();
  if (t >= n_rows) return;
  const int2 state = labels.state[t];
  const int c = int(blockIdx.y) * 32 + lane, vectors = hidden / 8;
  if (c >= vectors) return;
  auto part = [&](int32_t label, int p, int at) { return parts + (p * l_pad + label) * int64_t(hidden) + at; };
  auto row_of_table = [&](int32_t label, int at) { return table + (int64_t(labels.target[label]) * hidden + at) / 2; };
  auto taken = [&](int32_t label) {
    const float dz = label_dz[label];
    const float e = dz - __bfloat162float(__float2bfloat16(dz));
    return fabsf(e) < INFINITY ? e : 0.f;      // (beyond bf16's range the product has an infinity)
  };
  // (a table entry that is not finite has reached the product)
  auto give = [](float& to, float e, float w) { to += fabsf(w) < INFINITY ? e * w : 0.f; };
  if (!state.y || !labels.next[state.y - 1]) {
    float sum[8] = {};
    auto add = [&](int32_t label) {
      float v[8] = {};
      for (int p = 0; p < splits; ++p) {
        const float4* from = reinterpret_cast<const float4*>(part(label, p, 8 * c));
        const float4 a = from[0], b = from[1];
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
        v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
      }
      const float e = taken(label);
      const uint4 w = *reinterpret_cast<const uint4*>(row_of_table(label, 8 * c));
      const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        give(v[2 * j], e, __uint_as_float(words[j] << 16));
        give(v[2 * j + 1], e, __uint_as_float(words[j] & 0xffff0000u));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j];
    };
    if (state.x) add(state.x - 1);
    if (state.y) add(state.y - 1);
    d_hidden[t * vectors + c] = pack8(sum);
    return;
  }
#pragma unroll 1
  for (int at = 8 * c; at < 8 * c + 8; at += 2) {
    auto all = [&](auto&& take) {      // calls take() with the two columns of each label; the number of labels
      uint32_t n = 0;
      for (int32_t i = state.x, k = state.y; i || k; ++n) {
        const int32_t label = (i ? i : k) - 1;
        if (i) i = 0;
        else k = labels.next[label];
        float v[2] = {};
        for (int p = 0; p < splits; ++p) {
          const float2 f = *reinterpret_cast<const float2*>(part(label, p, at));
          v[0] += f.x;
          v[1] += f.y;
        }
        const uint32_t w = *row_of_table(label, at);
        give(v[0], taken(label), __uint_as_float(w << 16));
        give(v[1], taken(label), __uint_as_float(w & 0xffff0000u));
        take(v);
      }
      return n;
    };
    float top[2] = {}, sum[2] = {};      // sum: what is not finite
    const uint32_t n = all([&](const float (&v)[2]) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (fabsf(v[j]) < INFINITY) top[j] = fmaxf(top[j], fabsf(v[j]));
        else sum[j] += v[j];
      }
    });
    int shift[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) shift[j] = top[j] > 0.f ? 61 - (32 - __clz(n)) - ilogbf(top[j]) : 0;
    long long whole[2] = {};
    all([&](const float (&v)[2]) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (fabsf(v[j]) < INFINITY) whole[j] += __double2ll_rn(scalbn(double(v[j]), shift[j]));
    });
#pragma unroll
    for (int j = 0; j < 2; ++j) sum[j] += float(scalbn(double(whole[j]), -shift[j]));
    reinterpret_cast<uint32_t*>(d_hidden + t * vectors + c)[(at >> 1) & 3] = pack_bf16x2(sum[0], sum[1]);
  }
}

// ---------------------------------------------------------------- host
// dz of a piece of the vocabulary takes this much of the workspace at most (256 columns' worth where those are more already).
constexpr int64_t kPieceBytes = int64_t(1) << 30;

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

struct Workspace {
  int64_t l_pad;
  int64_t piece;                 // columns of a piece of the vocabulary
  int64_t pitch;                 // of the labels' rows: whole lines of 128 bytes
  int32_t splits;
  size_t row, target, segment, state, next, best, sums, rows, stats, label_value, of_label, dz, parts, total;
  Workspace(int64_t n_rows, int64_t n_forks, int64_t n_segments, int64_t vocab, int64_t hidden, bool backward) {
    l_pad = std::max<int64_t>(256, padded(n_rows + n_forks));
    const int64_t most = std::max<int64_t>(256, kPieceBytes / (2 * l_pad) / 256 * 256), pieces = (vocab + most - 1) / most;
    piece = padded((vocab + pieces - 1) / pieces);
    // K of dh is cut into parts, each with its own sums, where its tiles alone would leave clusters without work
    const int64_t tiles = l_pad / kTile * ((hidden + kTile - 1) / kTile), last = vocab - (vocab - 1) / piece * piece;
    splits = int32_t(std::max<int64_t>(1, std::min<int64_t>({16, kSmCount / 2 / tiles, (last + kBK - 1) / kBK / 4})));
    size_t at = 256;
    auto take = [&](size_t bytes) { const size_t here = at; at += aligned(bytes); return here; };
    row = take(l_pad * 4);
    target = take(l_pad * 4);
    segment = take(l_pad * 4);
    state = take(n_rows * 8);
    pitch = (hidden + 63) / 64 * 64;
    rows = take(l_pad * pitch * 2);
    label_value = take(l_pad * 4);
    next = best = sums = stats = of_label = dz = parts = 0;
    if (backward) {
      next = take(l_pad * 4);
      of_label = take(l_pad * sizeof(float2));
      dz = take(l_pad * piece * 2);
      parts = take(size_t(splits) * l_pad * hidden * 4);
    } else {
      best = take(n_rows * 8);
      sums = take(n_segments * sizeof(Sum));
      stats = take(size_t((vocab + kTile - 1) / kTile) * l_pad * sizeof(float2));
    }
    total = at;
  }
  Labels labels(char* ws) const {
    auto ints = [&](size_t at) { return reinterpret_cast<int32_t*>(ws + at); };
    return Labels{reinterpret_cast<Shared*>(ws), ints(row), ints(target), ints(segment), reinterpret_cast<int2*>(ws + state), next ? ints(next) : nullptr,
                  best ? reinterpret_cast<unsigned long long*>(ws + best) : nullptr};
  }
};

// The arguments that both passes share.
struct Call {
  const void *hidden, *table;
  int64_t n_rows, vocab;
  int32_t width;
  float scale;
  const int32_t *targets, *segment_ids, *fork_rows, *fork_targets, *fork_segments;
  int32_t n_forks, n_segments;
  char* ws;
  int32_t* status;
  cudaStream_t stream;
};

psa_status_t check_sizes(int64_t n_rows, int64_t n_forks, int64_t n_segments, int64_t vocab, int64_t width) {
  if (n_rows < 0 || n_forks < 0 || n_segments < 0 || vocab <= 0 || width <= 0) return PSA_ERR_INVALID_ARG;
  constexpr int64_t kMost = 1 << 24;
  if (width % 8 || width > (1 << 20) || n_rows > kMost || n_forks > kMost || n_segments > kMost || vocab > kMost) return PSA_ERR_UNSUPPORTED;
  if ((n_rows + n_forks) * vocab > (int64_t(1) << 45)) return PSA_ERR_UNSUPPORTED;      // fewer than 2^30 tiles: they are counted in 32 bits
  return PSA_OK;
}
psa_status_t check(const Call& c, std::initializer_list<const void*> outputs) {
  const psa_status_t sizes = check_sizes(c.n_rows, c.n_forks, c.n_segments, c.vocab, c.width);
  if (sizes != PSA_OK) return sizes;
  if (!(c.scale > 0.f) || !std::isfinite(c.scale)) return PSA_ERR_INVALID_ARG;
  if (!c.table || !c.ws || (c.n_rows > 0 && (!c.hidden || !c.targets || !c.segment_ids))) return PSA_ERR_INVALID_ARG;
  if (c.n_forks > 0 && (!c.fork_rows || !c.fork_targets || !c.fork_segments)) return PSA_ERR_INVALID_ARG;
  auto misaligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; };
  if (misaligned(c.hidden) || misaligned(c.table) || misaligned(c.ws)) return PSA_ERR_ALIGNMENT;
  for (const void* p : outputs)
    if (misaligned(p)) return PSA_ERR_ALIGNMENT;
  return PSA_OK;
}

// In units of log 2, of the logits from the tiles and of the labels' own: the same rounding in both.
float tile_scale(const Call& c) { return float(double(c.scale) / kLn2 * cut_off(c.width)); }
double label_scale(const Call& c) { return double(tile_scale(c)) / cut_off(c.width); }

// Lists the labels and copies their rows.
bool launch_labels(const Call& c, const Workspace& w, bool backward, const float* coef, const float* lse) {
  const Labels labels = w.labels(c.ws);
  if (launch_behind(true, logp_list_kernel, dim3(1), kListThreads, 0, c.stream, c.targets, c.segment_ids, c.fork_rows, c.fork_targets,
                    c.fork_segments, int32_t(c.n_rows), c.n_forks, c.n_segments, int32_t(c.vocab), labels,
                    backward ? nullptr : reinterpret_cast<Sum*>(c.ws + w.sums), c.status) != cudaSuccess)
    return false;
  const bool few = w.l_pad <= 2048;
  return launch_behind(true, few ? logp_gather_kernel<8> : logp_gather_kernel<1>, dim3(unsigned(few ? w.l_pad : w.l_pad / 8)), 256, 0, c.stream, static_cast<const uint4*>(c.hidden),
                       static_cast<const uint4*>(c.table), labels, c.width / 8, int32_t(w.pitch / 8), reinterpret_cast<uint4*>(c.ws + w.rows), coef, lse, c.scale, label_scale(c),
                       backward ? reinterpret_cast<float2*>(c.ws + w.of_label) : nullptr,
                       reinterpret_cast<float*>(c.ws + w.label_value)) == cudaSuccess;
}

template <int EPI>
bool launch_product(const ProductArgs& args, int64_t tiles, cudaStream_t stream) {
  constexpr uint32_t kSmem = smem_of<EPI>();
  if (cudaFuncSetAttribute(logp_product_kernel<EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmem)) != cudaSuccess) return false;
  const unsigned clusters = unsigned(std::min<int64_t>(kSmCount / 2, std::max<int64_t>(1, tiles)));
  return launch_behind(true, logp_product_kernel<EPI>, dim3(2 * clusters), kThreads, kSmem, stream, args) == cudaSuccess;
}

// Boxes of 32 rows of 32 columns of fp32.
bool f32_store_map(CUtensorMap* m, const void* p, int64_t rows, int64_t cols) {
  return encode(m, p, cols, 1, rows, cols * 4, cols * 4, 32, 1, 32, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_DATA_TYPE_FLOAT32);
}

ProductArgs common_args(const Call& c, const Workspace& w) {
  ProductArgs a{};
  const Labels labels = w.labels(c.ws);
  a.shared = labels.shared;
  a.target = labels.target;
  a.l_pad = w.l_pad;
  a.hidden = c.width;
  a.splits = 1;
  a.scale_log2 = tile_scale(c);
  a.status = c.status;
  return a;
}

psa_status_t forward(const Call& c, float* out, float* lse) {
  const Workspace w(c.n_rows, c.n_forks, c.n_segments, c.vocab, c.width, false);
  if (!launch_labels(c, w, false, nullptr, nullptr)) return failed_launch("dpo_linear_logp labels");
  ProductArgs a = common_args(c, w);
  a.columns = int32_t(c.vocab);
  a.stats = reinterpret_cast<float2*>(c.ws + w.stats);
  if (!operand_maps(&a.of[0].a, c.ws + w.rows, false, w.l_pad, c.width, 128, w.pitch) ||
      !operand_maps(&a.of[0].b, c.table, false, c.vocab, c.width, 128))
    return PSA_ERR_CUDA;
  const int64_t v_tiles = (c.vocab + kTile - 1) / kTile;
  if (!launch_product<kEpiStats>(a, w.l_pad / kTile * v_tiles, c.stream)) return failed_launch("dpo_linear_logp product");
  launch_behind(true, logp_join_kernel, dim3(unsigned(w.l_pad / 32)), 32 * kJoinWarps, 0, c.stream, a.stats,
                reinterpret_cast<const float*>(c.ws + w.label_value), w.labels(c.ws), w.l_pad,
                int32_t(v_tiles), int32_t(c.n_rows), c.n_segments, label_scale(c), reinterpret_cast<Sum*>(c.ws + w.sums), out, lse);
  return check_last_cuda_error("dpo_linear_logp launch");
}

psa_status_t backward(const Call& c, const float* coef, const float* lse, void* d_hidden, void* d_table) {
  const Workspace w(c.n_rows, c.n_forks, c.n_segments, c.vocab, c.width, true);
  if (!launch_labels(c, w, true, coef, lse)) return failed_launch("dpo_linear_logp_bwd labels");
  const int64_t d_tiles = (c.width + kTile - 1) / kTile;
  float* parts = reinterpret_cast<float*>(c.ws + w.parts);
  for (int64_t first = 0; first < c.vocab; first += w.piece) {
    const int64_t columns = std::min(w.piece, c.vocab - first), v_tiles = (columns + kTile - 1) / kTile;
    const char* table = static_cast<const char*>(c.table) + first * c.width * 2;
    ProductArgs a = common_args(c, w);
    a.columns = int32_t(columns);
    a.first_column = int32_t(first);
    a.of_label = reinterpret_cast<float2*>(c.ws + w.of_label);
    a.label_dz = reinterpret_cast<float*>(c.ws + w.label_value);
    if (!operand_maps(&a.of[0].a, c.ws + w.rows, false, w.l_pad, c.width, 128, w.pitch) ||
        !operand_maps(&a.of[0].b, table, false, columns, c.width, 128) ||
        !matrix_map(&a.of[0].store, c.ws + w.dz, w.l_pad, columns, 32, 64, w.piece))
      return PSA_ERR_CUDA;
    if (!launch_product<kEpiGrad>(a, w.l_pad / kTile * v_tiles, c.stream)) return failed_launch("dpo_linear_logp_bwd logits");
    a = common_args(c, w);
    a.columns = int32_t(columns);
    a.splits = w.splits;
    a.add = first > 0;
    a.with_table = d_table != nullptr;
    // dh = dz W: K runs along the vocabulary
    if (!operand_maps(&a.of[0].a, c.ws + w.dz, false, w.l_pad, columns, 128, w.piece) ||
        !operand_maps(&a.of[0].b, table, true, c.width, columns, 128) ||
        !f32_store_map(&a.of[0].store, parts, w.splits * w.l_pad, c.width))
      return PSA_ERR_CUDA;
    // dW = dz^T h: K runs along the labels
    if (d_table && (!operand_maps(&a.of[1].a, c.ws + w.dz, true, columns, w.l_pad, 128, w.piece) ||
                    !operand_maps(&a.of[1].b, c.ws + w.rows, true, c.width, w.l_pad, 128, w.pitch) ||
                    !matrix_map(&a.of[1].store, static_cast<char*>(d_table) + first * c.width * 2, columns, c.width, 32)))
      return PSA_ERR_CUDA;
    if (!launch_product<kEpiOut>(a, (w.l_pad / kTile * w.splits + (d_table ? v_tiles : 0)) * d_tiles, c.stream))
      return failed_launch("dpo_linear_logp_bwd products");
  }
  if (c.n_rows > 0)
    launch_behind(true, logp_scatter_kernel, dim3(unsigned((c.n_rows + 7) / 8), unsigned((c.width + 255) / 256)), 256, 0, c.stream, parts,
                  reinterpret_cast<const float*>(c.ws + w.label_value), static_cast<const uint32_t*>(c.table), w.labels(c.ws),
                  int32_t(c.n_rows), c.width, w.l_pad, w.splits, static_cast<uint4*>(d_hidden));
  return check_last_cuda_error("dpo_linear_logp_bwd launch");
}

}  // namespace
}  // namespace psa

extern "C" size_t dpo_linear_logp_workspace_bytes(int64_t n_rows, int32_t n_forks, int32_t n_segments, int64_t vocab, int32_t width,
                                                  int32_t backward) {
  if (psa::check_sizes(n_rows, n_forks, n_segments, vocab, width) != PSA_OK) return 0;
  return psa::Workspace(n_rows, n_forks, n_segments, vocab, width, backward != 0).total;
}

extern "C" psa_status_t dpo_linear_logp(const void* hidden, const void* table, int64_t n_rows, int64_t vocab, int32_t width,
                                        float scale, const int32_t* targets, const int32_t* segment_ids, const int32_t* fork_rows,
                                        const int32_t* fork_targets, const int32_t* fork_segments, int32_t n_forks,
                                        int32_t n_segments, float* out, float* lse, void* workspace, int32_t* device_status,
                                        void* stream) {
  const psa::Call c{hidden, table, n_rows, vocab, width, scale, targets, segment_ids, fork_rows, fork_targets, fork_segments,
                    n_forks, n_segments, static_cast<char*>(workspace), device_status, cudaStream_t(stream)};
  if ((n_segments > 0 && !out) || (n_rows > 0 && !lse)) return PSA_ERR_INVALID_ARG;
  const psa_status_t rc = psa::check(c, {});
  return rc != PSA_OK ? rc : psa::forward(c, out, lse);
}

extern "C" psa_status_t dpo_linear_logp_bwd(const float* coef, const void* hidden, const void* table, const float* lse,
                                            int64_t n_rows, int64_t vocab, int32_t width, float scale, const int32_t* targets,
                                            const int32_t* segment_ids, const int32_t* fork_rows, const int32_t* fork_targets,
                                            const int32_t* fork_segments, int32_t n_forks, int32_t n_segments, void* d_hidden,
                                            void* d_table, void* workspace, int32_t* device_status, void* stream) {
  const psa::Call c{hidden, table, n_rows, vocab, width, scale, targets, segment_ids, fork_rows, fork_targets, fork_segments,
                    n_forks, n_segments, static_cast<char*>(workspace), device_status, cudaStream_t(stream)};
  if ((n_segments > 0 && !coef) || (n_rows > 0 && (!lse || !d_hidden))) return PSA_ERR_INVALID_ARG;
  const psa_status_t rc = psa::check(c, {d_hidden, d_table});
  return rc != PSA_OK ? rc : psa::backward(c, coef, lse, d_hidden, d_table);
}
