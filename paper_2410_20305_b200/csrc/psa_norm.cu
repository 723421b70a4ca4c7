// psa_norm / psa_norm_bwd: normalisation of each token's row, with the residual add in front of it:
//     s = x + residual (rounded to x's type; s = x without one),
//     m = mean(s) (0 in the RMS form),  r = 1 / sqrt(mean((s - m)^2) + eps),  y = (s - m) * r * w + b,
// and its gradient, with u = (s - m) * r and g = dy * w:
//     ds = r * (g - u * mean(g u) - mean(g)) + d_total      (no mean(g) in the RMS form),
//     dw = sum over tokens of dy * u,   db = sum over tokens of dy.
// Bound by HBM: a row is read once into registers, its sums are taken from there (the variance after the mean, so a row far
// from 0 loses nothing), and it is written once.  Sums are fp32.  Rows of any width are moved 16 bytes at a time (psa_vector.cuh).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "psa.h"
#include "psa_device.cuh"
#include "psa_internal.h"
#include "psa_launch.cuh"
#include "psa_vector.cuh"

namespace psa {
namespace {

using namespace dev;

constexpr int kSmCount = 148;
constexpr int kMaxHidden = 16384;
constexpr int kRowsPerCta = 8;      // rows of a CTA where a warp holds a row
constexpr int kMaxGroups = 8;       // of the backward

// The most threads that divide() and divide_bwd() below give a CTA.
template <typename XT, int NV, bool kWarp, bool kRagged>
constexpr int max_threads() {
  return kWarp ? 32 * kRowsPerCta : NV == 1 && kRagged ? 544 : NV < 4 ? 256 : std::min(1024, kMaxHidden / (16 / int(sizeof(XT)) * NV) + 32);
}
// The forward's CTAs take several rows each; an SM then holds 1024 threads of them.
template <int NV, bool kWarp>
__host__ __device__ constexpr bool holds() { return NV == 1 && !kWarp; }
template <typename XT, int NV, bool kWarp, bool kRagged>
constexpr int fwd_ctas() {
  return holds<NV, kWarp>() ? 1088 / max_threads<XT, NV, kWarp, kRagged>() : 1;
}
template <typename XT, int NV, bool kWarp>
constexpr int bwd_threads() {
  return kWarp ? 32 * kRowsPerCta : NV * 16 / int(sizeof(XT)) < 32 ? 512 : 544;
}

// Sum over the threads that share a row: a warp (kWarp) or `n_warps`, for which sync() is a barrier.  `slot` alternates, so that one barrier is enough.
template <bool kWarp, int N, typename Sync>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*s_part)[32], int slot, int tid, int n_warps, Sync&& sync) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  if (kWarp) return;
  const int lane = tid & 31;
  if (lane == 0)
    for (int i = 0; i < N; ++i) s_part[slot * 2 + i][tid >> 5] = v[i];
  sync();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < n_warps ? s_part[slot * 2 + i][lane] : 0.f);
}

// A thread's columns in a row that starts `a` elements behind an aligned one: window k holds the columns [k V - a, (k + 1) V - a).
// `stride` rows lie between the rows that a warp or CTA takes, a multiple of V where it takes several: `a`, and with it every
// column of a thread, is the same in all of them.  Where a thread has one or two windows (kHold) it keeps its weights in
// registers and requests the next row ahead of the sums of this one; with a CTA for each row these kernels took more instructions,
// the weights' shift among them (bf16 layer norm with residual, one call between two events, cold in L2: 5465 x 1237 26.6 us, so 20.5;
// 4000 x 4095 49.2 and 36.9; 8000 x 1025 34.8 and 26.6).  At 1237 columns 66 % of the issue slots are taken, 41 % of DRAM's time and
// 40 % of the warps.
template <typename XT, typename WT, int NV, bool kWarp, bool kRagged>
__global__ void __launch_bounds__(max_threads<XT, NV, kWarp, kRagged>(), fwd_ctas<XT, NV, kWarp, kRagged>())
norm_kernel(const XT* x, const XT* residual, const WT* weight, const WT* bias, int64_t n_tokens, int64_t stride, int32_t hidden,
            float eps, int32_t rms, XT* out, XT* total, float* stats) {
  constexpr int V = 16 / int(sizeof(XT));
  constexpr bool kHold = holds<NV, kWarp>();
  using Weight = Span<WT, V, kRagged>;
  __shared__ float s_part[4][32];
  const int group = kWarp ? 32 : int(blockDim.x), tid = kWarp ? int(threadIdx.x) & 31 : int(threadIdx.x), n_warps = int(blockDim.x) >> 5;
  int64_t row = kWarp ? int64_t(blockIdx.x) * kRowsPerCta + (threadIdx.x >> 5) : int64_t(blockIdx.x);
  behind_wait();
  behind_go();
  if (kWarp && row >= n_tokens) return;
  const int64_t all = n_tokens * hidden;
  const int a = kRagged ? int(row * hidden & (V - 1)) : 0;
  // (A division by the width costs the kernels that instructions bind 1 us of 13 and 8 of 62 at 4000 x 7001; the others hide it,
  // and lost 7 us of 160 at 31041 x 4096 with the registers that the reciprocal takes.)
  const float inv = 1.0f / float(hidden);
  auto mean_of = [&](float v) { return kHold || kRagged ? v * inv : v / float(hidden); };
  uint4 rx[NV], rr[NV];
  auto fetch = [&](int64_t at) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V - a;
      if (col >= hidden) continue;
      rx[i] = kRagged ? load_window(x, at + col, all) : *reinterpret_cast<const uint4*>(x + at + col);
      if (residual) rr[i] = kRagged ? load_window(residual, at + col, all) : *reinterpret_cast<const uint4*>(residual + at + col);
    }
  };
  fetch(row * hidden);
  Vec<WT, V> hw[kHold ? NV : 1], hb[kHold ? NV : 1];
  if (kHold) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V - a;
      if (col >= hidden) continue;
      Weight v;
      v.load(weight, col, hidden);
      hw[kHold ? i : 0] = v.at(col);
      if (!bias) continue;
      v.load(bias, col, hidden);
      hb[kHold ? i : 0] = v.at(col);
    }
  }
  for (int slot = 0;; slot ^= 1) {
    const int64_t at = row * hidden;
    float s[NV][V], sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V - a;
#pragma unroll
      for (int j = 0; j < V; ++j) s[i][j] = 0.f;
      if (col >= hidden) continue;
      Vec<XT, V> v;
      memcpy(&v, &rx[i], 16);
      v.get(s[i]);
      if (residual) {
        float r[V];
        memcpy(&v, &rr[i], 16);
        v.get(r);
#pragma unroll
        for (int j = 0; j < V; ++j) s[i][j] += r[j];
        v.set(s[i]);     // what is normalised is what the residual stream holds
        v.get(s[i]);
        store_window(total, at + col, s[i], -col, hidden - col);
      }
      if (kRagged && (col < 0 || col + V > hidden))
#pragma unroll
        for (int j = 0; j < V; ++j) s[i][j] = col + j >= 0 && col + j < hidden ? s[i][j] : 0.f;
      if (!rms)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += s[i][j];
    }
    const int64_t next = row + stride;
    if (kHold && next < n_tokens) fetch(next * hidden);
    float mean = 0.f;
    if (!rms) {
      row_sum<kWarp>(sum, s_part, 0, tid, n_warps, [] { __syncthreads(); });
      mean = mean_of(sum[0]);
    }
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V - a;
      if (col >= hidden) continue;
      if (kRagged && (col < 0 || col + V > hidden)) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (col + j >= 0 && col + j < hidden) sq[0] += (s[i][j] - mean) * (s[i][j] - mean);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) sq[0] += (s[i][j] - mean) * (s[i][j] - mean);
      }
    }
    row_sum<kWarp>(sq, s_part, rms ? slot : 1, tid, n_warps, [] { __syncthreads(); });      // (a place that nobody still reads)
    const float rstd = 1.0f / sqrtf(mean_of(sq[0]) + eps);
    if (tid == 0) {
      stats[row] = mean;
      stats[n_tokens + row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V - a;
      if (col >= hidden) continue;
      float w[V], b[V], y[V];
      if (kHold) {
        hw[kHold ? i : 0].get(w);
        hb[kHold ? i : 0].get(b);
      } else {
        Weight ww, wb;
        ww.load(weight, col, hidden);
        if (bias) wb.load(bias, col, hidden);
        ww.at(col).get(w);
        wb.at(col).get(b);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = (s[i][j] - mean) * rstd * w[j] + (bias ? b[j] : 0.f);
      store_window(out, at + col, y, -col, hidden - col);
    }
    if (!kHold || next >= n_tokens) return;
    row = next;
  }
}

// V elements in shared memory from an address on that lies `a` elements behind a 16-byte boundary.
template <typename T, int V, bool kRagged>
__device__ __forceinline__ Vec<T, V> shared_vec(uint32_t addr, int a) {
  constexpr int kE = int(sizeof(T)), P = V * kE / 16;
  uint4 q[P + 1], w[P];
  if (kRagged) addr -= uint32_t(a * kE);
#pragma unroll
  for (int k = 0; k < (kRagged ? P + 1 : P); ++k) q[k] = ld_shared_v4(addr + 16 * k);
#pragma unroll
  for (int k = 0; k < P; ++k) w[k] = kRagged ? shift_pair<kE>(q[k], q[k + 1], a) : q[k];
  Vec<T, V> v;
  memcpy(&v, w, sizeof(w));
  return v;
}
template <typename T, int V>
__device__ __forceinline__ void zero_behind(Vec<T, V>& v, int n) {
  float f[V];
  v.get(f);
#pragma unroll
  for (int j = 0; j < V; ++j) f[j] = j < n ? f[j] : 0.f;
  v.set(f);
}
// The backward.  A CTA's threads are up to 8 groups, each with a ring and a barrier of its own; a group takes every n-th tile of rows:
// one row for all its threads, or (then the only one), of narrow rows, some for each of its warps.  (As CTAs of their own the groups
// wrote a part of the sums each: 24.0 us at 5465 x 1240, 22.3 so, 20.9 and 19.8 at 4000 x 1536.  Two groups of
// more threads are two CTAs: 179 us at 31041 x 4096, 193 as one.)  Tiles are contiguous in memory and come by bulk copies into a ring
// of stages, so that several are in flight whatever the arithmetic waits for (31041 x 4096 bf16 with d_total: 346 us with loads where
// the values are used, 253 with the next row's in registers, 187 so at first).  For the sums over tokens a thread keeps its columns [k V, (k + 1) V) throughout; of dx it
// writes window k of each row (the same columns where rows are aligned).  partial: [gridDim.x][2][part_pitch].
// A part's rows of sums start at 16 bytes.
__host__ __device__ constexpr int part_pitch(int hidden) { return (hidden + 3) / 4 * 4; }

struct BwdShape {
  int32_t rows, stages;                   // rows of a tile; tiles in flight
  int32_t groups;
  int32_t staged;                         // tensors that come by the ring: x, d_out and, where there is room, d_total
  uint32_t slot_bytes, w_bytes;           // of a tile of one tensor; of the weight with zeros around it
};
constexpr uint32_t kWeightPad = 64;       // zeros in front of the weight and behind it

template <typename XT, typename WT, int NV, bool kWarp, bool kRagged, bool kGrouped>
__global__ void __launch_bounds__(bwd_threads<XT, NV, kWarp>(), 1)
norm_bwd_kernel(const XT* d_out, const XT* x, const WT* weight, const float* stats, const XT* d_total, int64_t n_tokens,
                int32_t hidden, int32_t rms, XT* dx, float* partial, BwdShape shape, int32_t* status) {
  constexpr int V = 16 / int(sizeof(XT)), kE = int(sizeof(XT)), kW = int(sizeof(WT));
  constexpr bool kKeep = !kRagged && NV * V <= 16;
  extern __shared__ uint8_t smem_raw[];        // [stages][2 or 3 tensors][slot], weight;  at the end the warps' sums
  __shared__ float s_parts[kGrouped ? kMaxGroups : 1][4][32];
  __shared__ uint64_t s_bars[kGrouped ? kMaxGroups : 1][8], s_weight_bar;
  __shared__ int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int groups = kGrouped ? shape.groups : 1;
  const int width = int(blockDim.x) / groups, mine = kGrouped ? int(threadIdx.x) / width : 0;     // a group's threads; its number
  const int place = int(threadIdx.x) - mine * width;                                              // in the group
  const int group = kWarp ? 32 : width, tid = kWarp ? lane : place;                   // threads of a row
  const uint32_t n_tensors = uint32_t(shape.staged), ring_bytes = uint32_t(shape.stages) * n_tensors * shape.slot_bytes;
  const uint32_t base0 = (smem_u32(smem_raw) + 15u) & ~15u, base = base0 + uint32_t(mine) * ring_bytes;
  uint8_t* ring0 = smem_raw + (base0 - smem_u32(smem_raw));
  uint8_t* ring = ring0 + uint32_t(mine) * ring_bytes;
  uint8_t* s_weight = ring0 + uint32_t(groups) * ring_bytes + kWeightPad;
  const uint32_t sw = base0 + uint32_t(groups) * ring_bytes + kWeightPad;
  uint64_t* s_bar = s_bars[mine];
  float(*s_part)[32] = s_parts[mine];
  const int64_t start = int64_t(blockIdx.x) * groups + mine, stride = int64_t(gridDim.x) * groups;
  auto sync = [&] {
    if (!kGrouped) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(width) : "memory");
  };
  const WaitCtx wctx{&s_abort, status, kWaitLimitClocks};
  const int64_t all = n_tokens * hidden, tile_elems = int64_t(shape.rows) * hidden, n_tiles = (n_tokens + shape.rows - 1) / shape.rows;

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int g = 0; g < groups; ++g)
      for (int s = 0; s < shape.stages; ++s) mbar_init(smem_u32(&s_bars[g][s]), 1);
    mbar_init(smem_u32(&s_weight_bar), 1);
    fence_mbar_init();
  }
  if (kGrouped) __syncthreads();      // (the first threads of all groups use their barriers)
  behind_wait();
  behind_go();

  // One thread of a group requests a tile: from the 16-byte boundary at or before its first element to the one at or behind its last; the
  // tensor's last elements, if no boundary follows them within it, by hand.
  auto request = [&](int64_t tile, int stage) {
    const int64_t first = tile * tile_elems, from = first & ~int64_t(V - 1);
    if (!kRagged) {      // whole rows are whole vectors
      const uint32_t n = uint32_t(min(tile_elems, all - first)) * kE, bar = smem_u32(&s_bar[stage]);
      uint32_t to = base + uint32_t(stage) * n_tensors * shape.slot_bytes;
      mbar_expect_tx(bar, n_tensors * n);
      bulk_load(to, x + first, n, bar);
      bulk_load(to + shape.slot_bytes, d_out + first, n, bar);
      if (n_tensors == 3) bulk_load(to + 2 * shape.slot_bytes, d_total + first, n, bar);
      return;
    }
    const int64_t end = min(all, first + tile_elems), last = all & ~int64_t(V - 1), to = min(last, (end + V - 1) & ~int64_t(V - 1));
    const uint32_t bytes = uint32_t(to - from) * kE, bar = smem_u32(&s_bar[stage]), at = base + uint32_t(stage) * n_tensors * shape.slot_bytes;
    if (end > last)
      for (uint32_t t = 0; t < n_tensors; ++t) {
        const XT* src = t == 0 ? x : t == 1 ? d_out : d_total;
        XT* slot = reinterpret_cast<XT*>(ring + (uint32_t(stage) * n_tensors + t) * shape.slot_bytes);
        for (int64_t e = max(last, from); e < end; ++e) slot[e - from] = src[e];
      }
    mbar_expect_tx(bar, n_tensors * bytes);
    if (bytes == 0) return;
    bulk_load(at, x + from, bytes, bar);
    bulk_load(at + shape.slot_bytes, d_out + from, bytes, bar);
    if (n_tensors == 3) bulk_load(at + 2 * shape.slot_bytes, d_total + from, bytes, bar);
  };
  int64_t asked = start;     // the next tile to request, and how many have been (the first thread's)
  int n_asked = 0;
  if (place == 0)
    for (int s = 0; s < shape.stages && asked < n_tiles; ++s, asked += stride, ++n_asked) request(asked, s);
  // The weight, behind the first tiles (32.7 us instead of 38.0 element by element ahead of them at 4000 x 2048 fp32): whole vectors by
  // a copy, the rest and the zeros around it by hand.
  const int whole = hidden * kW & ~15;
  if (threadIdx.x == 0) {
    mbar_expect_tx(smem_u32(&s_weight_bar), uint32_t(whole));
    if (whole) bulk_load(sw, weight, uint32_t(whole), smem_u32(&s_weight_bar));
  }
  for (int i = threadIdx.x; i < int(kWeightPad); i += blockDim.x) s_weight[i - int(kWeightPad)] = 0;
  for (int i = whole / kW + int(threadIdx.x); i < int(shape.w_bytes - kWeightPad) / kW; i += blockDim.x)
    reinterpret_cast<WT*>(s_weight)[i] = i < hidden ? weight[i] : WT(0.f);
  __syncthreads();

  float dw[NV][V], db[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[i][j] = db[i][j] = 0.f;
  const float inv = 1.0f / float(hidden);
  int stage = 0, turn = 0, slot = 0, before = -1;     // before: the stage that the last tile was in
  float next_mean = 0.f, next_rstd = 0.f;             // of the row after this one
  auto fetch_stats = [&](int64_t row) {
    if (row >= n_tokens) return;
    next_mean = stats[row];
    next_rstd = stats[n_tokens + row];
  };
  const int first_r = kWarp ? warp : 0;
  fetch_stats(start * shape.rows + first_r);
  mbar_wait(smem_u32(&s_weight_bar), 0, wctx);
  for (int64_t tile = start; tile < n_tiles; tile += stride) {
    mbar_wait(smem_u32(&s_bar[stage]), turn & 1, wctx);
    const uint32_t tx = base + uint32_t(stage) * n_tensors * shape.slot_bytes;
    const int64_t row0 = tile * shape.rows;
    const int n_rows = int(min(int64_t(shape.rows), n_tokens - row0));
    const int lead = kRagged ? int(row0 * hidden & (V - 1)) : 0;      // elements in front of the tile in its slot
    for (int r = first_r; r < n_rows; r += kWarp ? kRowsPerCta : 1, slot ^= 1) {
      const int64_t row = row0 + r, at = row * hidden;
      const int o = lead + r * hidden, a = kRagged ? o & (V - 1) : 0;
      const uint32_t sx = tx + uint32_t(o * kE), sg = sx + shape.slot_bytes, sd = sg + shape.slot_bytes;
      const float mean = next_mean, rstd = next_rstd;
      fetch_stats(kWarp && r + kRowsPerCta < n_rows ? row + kRowsPerCta : (tile + stride) * shape.rows + first_r);
      const float shift = -mean * rstd;         // u = x rstd + shift
      float sum[2] = {0.f, 0.f};
      float ku[kKeep ? NV : 1][V], kg[kKeep ? NV : 1][V];     // u and g w, where there are registers for them
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = (i * group + tid) * V;
        if (col >= hidden) continue;
        Vec<XT, V> px = shared_vec<XT, V, kRagged>(sx + col * kE, a), pg = shared_vec<XT, V, kRagged>(sg + col * kE, a);
        if (kRagged && col + V > hidden) {    // what follows the row
          zero_behind(px, hidden - col);
          zero_behind(pg, hidden - col);
        }
        float u[V], g[V], w[V];
        px.get(u);
        pg.get(g);
        shared_vec<WT, V, false>(sw + col * kW, 0).get(w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          u[j] = u[j] * rstd + shift;
          dw[i][j] += g[j] * u[j];
          db[i][j] += g[j];
          g[j] *= w[j];
          sum[0] += g[j] * u[j];
          sum[1] += g[j];
          if (kKeep) {
            ku[kKeep ? i : 0][j] = u[j];
            kg[kKeep ? i : 0][j] = g[j];
          }
        }
      }
      row_sum<kWarp>(sum, s_part, slot, tid, width >> 5, sync);
      // (a row for all threads: they have left the tile before this one)
      if (!kWarp && before >= 0 && place == 0 && asked < n_tiles && !s_abort) {
        request(asked, before);
        asked += stride;
        ++n_asked;
      }
      // dx = (g w - u c_u - c_1) rstd + d_total
      const float c_u = -sum[0] * inv * rstd, c_1 = rms ? 0.f : -sum[1] * inv * rstd;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = (i * group + tid) * V - a;
        if (col >= hidden) continue;
        float u[V], g[V], d[V];
        if (kKeep) {
#pragma unroll
          for (int j = 0; j < V; ++j) { u[j] = ku[kKeep ? i : 0][j]; g[j] = kg[kKeep ? i : 0][j]; }
        } else {
          float w[V];
          shared_vec<XT, V, false>(sx + col * kE, 0).get(u);
          shared_vec<XT, V, false>(sg + col * kE, 0).get(g);
          shared_vec<WT, V, kRagged>(sw + col * kW, -a & (16 / kW - 1)).get(w);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            u[j] = u[j] * rstd + shift;
            g[j] *= w[j];
          }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = g[j] * rstd + (u[j] * c_u + c_1);
        if (d_total) {
          float t[V];
          if (n_tensors == 3) {
            shared_vec<XT, V, false>(sd + col * kE, 0).get(t);
          } else {
            const uint4 q = load_window(d_total, at + col, all);
            Vec<XT, V> v;
            memcpy(&v, &q, 16);
            v.get(t);
          }
#pragma unroll
          for (int j = 0; j < V; ++j) d[j] += t[j];
        }
        store_window(dx, at + col, d, -col, hidden - col);
      }
    }
    if (kWarp || shape.stages == 1) {     // all warps have left the tile
      sync();
      if (place == 0 && asked < n_tiles && !s_abort) {
        request(asked, stage);
        asked += stride;
        ++n_asked;
      }
    } else {
      before = stage;
    }
    if (++stage == shape.stages) { stage = 0; ++turn; }
  }
  if (s_abort && place == 0) {      // shared memory must outlive the copies in flight
    const long long t0 = clock64();
    while (!mbar_try_wait(smem_u32(&s_weight_bar), 0) && clock64() - t0 < kWaitLimitClocks) {}
    for (int q = max(0, n_asked - shape.stages); q < n_asked; ++q)
      while (!mbar_try_wait(smem_u32(&s_bar[q % shape.stages]), (q / shape.stages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
  }
  __syncthreads();
  // The sums of a CTA's warps or groups, each in a place of its own over the rings, are added in their order.
  const int pitch = part_pitch(hidden);
  float* mine_dw = partial + int64_t(blockIdx.x) * 2 * pitch;
  const int n_sums = kWarp ? kRowsPerCta : groups;
  float* to = n_sums > 1 ? reinterpret_cast<float*>(ring0) + (kWarp ? warp : mine) * 2 * pitch : mine_dw;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V;
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      if (col + j >= pitch) continue;
      *reinterpret_cast<float4*>(to + col + j) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
      *reinterpret_cast<float4*>(to + pitch + col + j) = make_float4(db[i][j], db[i][j + 1], db[i][j + 2], db[i][j + 3]);
    }
  }
  if (n_sums > 1) {
    __syncthreads();
    const float* sums = reinterpret_cast<const float*>(ring0);
    for (int c = threadIdx.x; c < 2 * pitch; c += blockDim.x) {
      float v = 0.f;
#pragma unroll 8
      for (int k = 0; k < n_sums; ++k) v += sums[k * 2 * pitch + c];
      mine_dw[c] = v;
    }
  }
}

// dw (blockIdx.y = 0) and db (1): the parts of all CTAs, added in a fixed order.
// (32 warps are faster from 400 parts on, of which there are none: two CTAs of the backward an SM at most.)
constexpr int kSumWarps = 16;
template <typename WT>
__global__ void __launch_bounds__(32 * kSumWarps)
norm_sum_kernel(const float* partial, int32_t n_parts, int32_t hidden, WT* dweight, WT* dbias) {
  __shared__ float s[kSumWarps][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  behind_wait();
  behind_go();
  const int pitch = part_pitch(hidden);
  float v = 0.f;
  if (col < hidden) {
    int p = part;
    for (; p + 7 * kSumWarps < n_parts; p += 8 * kSumWarps) {
      float w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = partial[(int64_t(p + k * kSumWarps) * 2 + blockIdx.y) * pitch + col];
#pragma unroll
      for (int k = 0; k < 8; ++k) v += w[k];
    }
    for (; p < n_parts; p += kSumWarps) v += partial[(int64_t(p) * 2 + blockIdx.y) * pitch + col];
  }
  s[part][lane] = v;
  __syncthreads();
  if (part == 0 && col < hidden) {
    for (int p = 1; p < kSumWarps; ++p) v += s[p][lane];
    set_element((blockIdx.y ? dbias : dweight) + col, v);
  }
}

// How a row is divided: NV vectors of 16 bytes a thread, `threads` threads (32: a warp).  Rows that start anywhere reach into
// one vector more.
struct Division {
  int nv, threads;
};
int vectors(int32_t hidden, int elem_bytes) {
  const int bytes = hidden * elem_bytes;
  return bytes % 16 ? (bytes + 16 - elem_bytes + 15) / 16 : bytes / 16;     // (16 - elem_bytes in front of it at most)
}
Division divide(int32_t hidden, int elem_bytes) {
  const int n = vectors(hidden, elem_bytes);
  if (n <= 128) return {n <= 32 ? 1 : n <= 64 ? 2 : 4, 32};
  const int nv = n <= (hidden * elem_bytes % 16 ? 544 : 256) ? 1 : n <= 512 ? 2 : n <= 4096 ? 4 : 8;
  return {nv, ((n + nv - 1) / nv + 31) / 32 * 32};
}
// The backward: a warp a row of up to 1024 columns, else 16 columns a thread for up to 512 threads, else 32.
Division divide_bwd(int32_t hidden, int elem_bytes) {
  const int n = vectors(hidden, elem_bytes), wide = elem_bytes / 2;     // 8 columns: `wide` vectors
  if (n <= 128 * wide) return {n <= 32 * wide ? wide : n <= 64 * wide ? 2 * wide : 4 * wide, 32};
  const int nv = n <= 1024 * wide ? 2 * wide : 4 * wide;
  return {nv, ((n + nv - 1) / nv + 31) / 32 * 32};
}

// CTAs of the backward for an SM (512 threads of 128 registers), and the groups of one: as many as tiles can fill.
bool grouped(const Division& d) { return d.threads > 32 && d.threads <= 160; }
int ctas_per_sm(const Division& d) { return d.threads == 32 ? 2 : grouped(d) ? 1 : std::max(1, 512 / d.threads); }
int groups_of(const Division& d, int64_t tiles) {
  return grouped(d) ? int(std::max<int64_t>(1, std::min<int64_t>({(tiles + kSmCount - 1) / kSmCount, 512 / d.threads, kMaxGroups}))) : 1;
}
// Rows of a tile: one, or one for each of a CTA's 8 warps, whatever their size (16 KB of a tensor at 1024 columns of bf16, 32 KB of
// fp32); up to 8 for each warp where a tensor's tile stays within 8 KB and there are tiles enough to fill the SMs.
int tile_rows(const Division& d, int64_t n_tokens, int32_t hidden, int elem_bytes) {
  if (d.threads != 32) return 1;
  int rows = kRowsPerCta;
  while (rows < 8 * kRowsPerCta && 2 * rows * hidden * elem_bytes <= 8192 && n_tokens >= 4 * int64_t(rows) * kSmCount) rows *= 2;
  return rows;
}
int64_t part_count(const Division& d, int64_t n_tokens, int rows) {
  const int64_t tiles = std::max<int64_t>(1, (n_tokens + rows - 1) / rows), groups = groups_of(d, tiles), most = int64_t(kSmCount) * ctas_per_sm(d) * groups;
  const int64_t each = (tiles + most - 1) / most;      // and no more than it takes for the busiest one's number of tiles
  return ((tiles + each - 1) / each + groups - 1) / groups;
}

template <typename F>
psa_status_t with_division(const Division& d, bool ragged, F&& f) {
  const bool warp = d.threads == 32;
#define PSA_NORM(NV) (warp ? (ragged ? f.template run<NV, true, true>() : f.template run<NV, true, false>()) \
                           : (ragged ? f.template run<NV, false, true>() : f.template run<NV, false, false>()))
  return d.nv == 1 ? PSA_NORM(1) : d.nv == 2 ? PSA_NORM(2) : d.nv == 4 ? PSA_NORM(4) : PSA_NORM(8);
#undef PSA_NORM
}

template <typename XT, typename WT>
struct Forward {
  const void *x, *residual, *weight, *bias;
  int64_t n_tokens;
  int32_t hidden;
  float eps;
  int32_t rms;
  void *out, *total;
  float* stats;
  int threads;
  cudaStream_t stream;
  template <int NV, bool kWarp, bool kRagged>
  psa_status_t run() {
    if constexpr (NV == 8 && (sizeof(XT) == 2 || kWarp || !kRagged)) return PSA_ERR_UNSUPPORTED;     // (divide() does not say so)
    else return go<NV, kWarp, kRagged>();
  }
  template <int NV, bool kWarp, bool kRagged>
  psa_status_t go() {
    int64_t grid = kWarp ? (n_tokens + kRowsPerCta - 1) / kRowsPerCta : n_tokens;
    if (holds<NV, kWarp>()) grid = std::min<int64_t>(grid, kSmCount * (1088 / threads) & ~7);      // (a multiple of V)
    const int64_t stride = kWarp ? grid * kRowsPerCta : grid;
    launch_behind(true, norm_kernel<XT, WT, NV, kWarp, kRagged>, dim3(unsigned(grid)), kWarp ? 32 * kRowsPerCta : threads, 0, stream,
        static_cast<const XT*>(x), static_cast<const XT*>(residual), static_cast<const WT*>(weight), static_cast<const WT*>(bias),
        n_tokens, stride, hidden, eps, rms, static_cast<XT*>(out), static_cast<XT*>(total), stats);
    return check_last_cuda_error("psa_norm launch");
  }
};

template <typename XT, typename WT>
struct Backward {
  const void *d_out, *x, *weight;
  const float* stats;
  const void* d_total;
  int64_t n_tokens;
  int32_t hidden, rms;
  void *dx, *dweight, *dbias;
  float* partial;
  Division d;
  int32_t* status;
  cudaStream_t stream;
  template <int NV, bool kWarp, bool kRagged>
  psa_status_t run() {
    constexpr int kWide = int(sizeof(XT)) / 2;
    if constexpr (NV < kWide || NV > 4 * kWide || (!kWarp && NV < 2 * kWide)) return PSA_ERR_UNSUPPORTED;   // (divide_bwd() does not say so)
    else return go<NV, kWarp, kRagged>();
  }
  template <int NV, bool kWarp, bool kRagged>
  psa_status_t go() {
    constexpr int kWide = int(sizeof(XT)) / 2;
    BwdShape shape{};
    shape.rows = tile_rows(d, n_tokens, hidden, int(sizeof(XT)));
    shape.groups = groups_of(d, (n_tokens + shape.rows - 1) / shape.rows);
    shape.slot_bytes = uint32_t((int64_t(shape.rows) * hidden * int(sizeof(XT)) + 47) / 16 * 16);    // and a vector around it
    shape.w_bytes = uint32_t((hidden * int(sizeof(WT)) + 15) / 16 * 16) + 2 * kWeightPad;
    const uint32_t room = (224 * 1024 / ctas_per_sm(d) - (grouped(d) ? 8192 : 1024) - shape.w_bytes) / uint32_t(shape.groups);     // of a group, less the static arrays
    shape.staged = d_total && 3 * shape.slot_bytes <= room ? 3 : 2;
    const uint32_t stage = uint32_t(shape.staged) * shape.slot_bytes;
    shape.stages = int(std::max(1u, std::min(8u, std::min(room / stage, 1 + 196608 / uint32_t(ctas_per_sm(d) * shape.groups) / stage))));
    const uint32_t sums = uint32_t((kWarp ? kRowsPerCta : shape.groups) * 2 * 4 * part_pitch(hidden));
    const uint32_t smem = std::max(shape.groups * shape.stages * stage + shape.w_bytes, sums) + 16;
    const int64_t parts = part_count(d, n_tokens, shape.rows);
    auto kernel = norm_bwd_kernel<XT, WT, NV, kWarp, kRagged, false>;
    if constexpr (!kWarp && NV == 2 * kWide)
      if (grouped(d)) kernel = norm_bwd_kernel<XT, WT, NV, kWarp, kRagged, true>;
    // (The limit is the kernel's, for all host threads: the same in every call, or a call could lower it under another one's launch.)
    const int limit = 227 * 1024 - (grouped(d) ? 8192 : 1024);      // of an SM's 228 KB, less the CTA's own and the static arrays
    if (smem > uint32_t(limit)) return PSA_ERR_UNSUPPORTED;         // (no shape asks for more)
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, limit) != cudaSuccess) return PSA_ERR_CUDA;
    if (launch_behind(true, kernel, dim3(unsigned(parts)), kWarp ? 32 * kRowsPerCta : d.threads * shape.groups, smem, stream,
                      static_cast<const XT*>(d_out), static_cast<const XT*>(x), static_cast<const WT*>(weight), stats,
                      static_cast<const XT*>(d_total), n_tokens, hidden, rms, static_cast<XT*>(dx), partial, shape,
                      status) != cudaSuccess)
      return failed_launch("psa_norm_bwd launch");      // (no sums of parts that are not written)
    launch_behind(true, norm_sum_kernel<WT>, dim3(unsigned((hidden + 31) / 32), dbias ? 2 : 1), 32 * kSumWarps, 0, stream, partial,
                  int32_t(parts), hidden, static_cast<WT*>(dweight), static_cast<WT*>(dbias));
    return check_last_cuda_error("psa_norm_bwd launch");
  }
};

bool bad_types(int32_t dtype, int32_t weight_dtype) {
  return !((dtype == PSA_DTYPE_BF16 && (weight_dtype == PSA_DTYPE_BF16 || weight_dtype == PSA_DTYPE_F32)) ||
           (dtype == PSA_DTYPE_F32 && weight_dtype == PSA_DTYPE_F32));
}
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

psa_status_t check_sizes(int64_t n_tokens, int32_t hidden, int32_t dtype, int32_t weight_dtype) {
  if (n_tokens < 0 || hidden <= 0) return PSA_ERR_INVALID_ARG;
  if (bad_types(dtype, weight_dtype)) return PSA_ERR_INVALID_ARG;
  if (hidden > kMaxHidden || n_tokens > 0x7fffffffLL) return PSA_ERR_UNSUPPORTED;
  return PSA_OK;
}

}  // namespace
}  // namespace psa

extern "C" psa_status_t psa_norm(const void* x, const void* residual, const void* weight, const void* bias, int32_t dtype,
                                 int32_t weight_dtype, int64_t n_tokens, int32_t hidden, float eps, int32_t rms, void* out,
                                 void* total, float* stats, void* stream) {
  using namespace psa;
  const psa_status_t sizes = check_sizes(n_tokens, hidden, dtype, weight_dtype);
  if (sizes != PSA_OK) return sizes;
  if (!(eps >= 0.f) || (rms && bias) || ((residual == nullptr) != (total == nullptr))) return PSA_ERR_INVALID_ARG;
  if (n_tokens == 0) return PSA_OK;
  if (!x || !weight || !out || !stats) return PSA_ERR_INVALID_ARG;
  for (const void* p : {x, residual, weight, bias, static_cast<const void*>(out), static_cast<const void*>(total),
                        static_cast<const void*>(stats)})
    if (misaligned(p, 16)) return PSA_ERR_ALIGNMENT;
  const int e = dtype == PSA_DTYPE_F32 ? 4 : 2;
  const Division d = divide(hidden, e);
  cudaStream_t st = cudaStream_t(stream);
  if (dtype == PSA_DTYPE_F32)
    return with_division(d, hidden * e % 16 != 0, Forward<float, float>{x, residual, weight, bias, n_tokens, hidden, eps, rms, out, total, stats, d.threads, st});
  if (weight_dtype == PSA_DTYPE_F32)
    return with_division(d, hidden * e % 16 != 0, Forward<__nv_bfloat16, float>{x, residual, weight, bias, n_tokens, hidden, eps, rms, out, total, stats, d.threads, st});
  return with_division(d, hidden * e % 16 != 0, Forward<__nv_bfloat16, __nv_bfloat16>{x, residual, weight, bias, n_tokens, hidden, eps, rms, out, total, stats, d.threads, st});
}

extern "C" size_t psa_norm_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden) {
  if (n_tokens < 0 || hidden <= 0 || hidden > psa::kMaxHidden) return 0;
  size_t parts = 0;
  for (int e : {2, 4}) {
    const psa::Division d = psa::divide_bwd(hidden, e);
    parts = std::max(parts, size_t(psa::part_count(d, n_tokens, psa::tile_rows(d, n_tokens, hidden, e))));
  }
  return parts * 2 * size_t(psa::part_pitch(hidden)) * 4;
}

extern "C" psa_status_t psa_norm_bwd(const void* d_out, const void* x, const void* weight, const float* stats,
                                     const void* d_total, int32_t dtype, int32_t weight_dtype, int64_t n_tokens, int32_t hidden,
                                     int32_t rms, void* dx, void* dweight, void* dbias, void* workspace, int32_t* device_status,
                                     void* stream) {
  using namespace psa;
  const psa_status_t sizes = check_sizes(n_tokens, hidden, dtype, weight_dtype);
  if (sizes != PSA_OK) return sizes;
  if (!weight || !dweight || !workspace || (rms && dbias)) return PSA_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!d_out || !x || !stats || !dx)) return PSA_ERR_INVALID_ARG;
  for (const void* p : {d_out, x, weight, static_cast<const void*>(stats), d_total, static_cast<const void*>(dx),
                        static_cast<const void*>(dweight), static_cast<const void*>(dbias), static_cast<const void*>(workspace)})
    if (misaligned(p, 16)) return PSA_ERR_ALIGNMENT;
  const int e = dtype == PSA_DTYPE_F32 ? 4 : 2;
  const Division d = divide_bwd(hidden, e);
  cudaStream_t st = cudaStream_t(stream);
  float* part = static_cast<float*>(workspace);
  if (dtype == PSA_DTYPE_F32)
    return with_division(d, hidden * e % 16 != 0, Backward<float, float>{d_out, x, weight, stats, d_total, n_tokens, hidden, rms, dx, dweight, dbias, part, d, device_status, st});
  if (weight_dtype == PSA_DTYPE_F32)
    return with_division(d, hidden * e % 16 != 0, Backward<__nv_bfloat16, float>{d_out, x, weight, stats, d_total, n_tokens, hidden, rms, dx, dweight, dbias, part, d, device_status, st});
  return with_division(d, hidden * e % 16 != 0, Backward<__nv_bfloat16, __nv_bfloat16>{d_out, x, weight, stats, d_total, n_tokens, hidden, rms, dx, dweight, dbias, part, d, device_status, st});
}
