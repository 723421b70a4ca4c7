// psa_block_norm / psa_block_norm_bwd: the step between two sublayers of a decoder whose output is normalised before it joins
// the residual stream.  For each token's row,
//     u1 = (x - m1) r1,   y = u1 pw + pb           (y = x without a norm behind the block)
//     s = a residual + gate y, rounded to x's type,   u2 = (s - m2) r2,   out = u2 w + b
// with m the mean (0 in the RMS form) and r = 1 / sqrt(mean((. - m)^2) + eps); and the gradient, with g = d_out w,
//     ds = r2 (g - u2 mean(g u2) - mean(g)) + d_total,            d_residual = a ds,
//     q = ds gate pw,   dx = r1 (q - u1 mean(q u1) - mean(q))     (dx = ds gate without a norm; no mean(g), mean(q) if RMS)
//     dw = sum d_out u2,  db = sum d_out,  A = sum ds u1 (ds x without a norm),  C = sum ds   over the tokens,
//     dpw = gate A,  dpb = gate C,  dgate = pw A + pb C           (dgate = A without a norm).
// Bound by HBM: forward two rows are read and two written, backward four and two.  Both norms of a row are taken while it is in
// registers.  Sums are fp32, the variance after the mean.
// Rows of any width are moved 16 bytes at a time (psa_vector.cuh): a row that starts `a` elements behind an aligned one is
// taken as windows, window k holding the columns [k V - a, (k + 1) V - a).
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

struct Args {
  const void *x, *residual, *weight, *bias, *post_weight, *post_bias, *gate;
  void *out, *total;
  float* stats;
  const void *d_out, *d_total;      // backward; total is read
  void *dx, *d_residual, *d_weight, *d_bias, *d_post_weight, *d_post_bias, *d_gate;
  float* partial;
  int64_t n_tokens;
  int32_t hidden, rms;
  float residual_scale, eps;
  int32_t* status;
};

// ---------------------------------------------------------------- forward
template <typename XT, int NV, bool kWarp>
constexpr int fwd_threads() {
  return kWarp ? 32 * kRowsPerCta : NV == 1 ? 544 : NV == 2 ? 288 : std::min(1024, kMaxHidden / (16 / int(sizeof(XT)) * NV) + 32);
}

template <typename XT, typename WT, int NV, bool kWarp, bool kRagged>
__global__ void __launch_bounds__(fwd_threads<XT, NV, kWarp>())
block_norm_kernel(const Args args) {
  constexpr int V = 16 / int(sizeof(XT));
  using Weight = Span<WT, V, kRagged>;
  __shared__ float s_part[8][32];
  const int group = kWarp ? 32 : int(blockDim.x), tid = kWarp ? int(threadIdx.x) & 31 : int(threadIdx.x), n_warps = int(blockDim.x) >> 5;
  const int64_t row = kWarp ? int64_t(blockIdx.x) * kRowsPerCta + (threadIdx.x >> 5) : int64_t(blockIdx.x);
  const int32_t hidden = args.hidden;
  const int64_t n_tokens = args.n_tokens;
  behind_wait();
  behind_go();
  if (kWarp && row >= n_tokens) return;
  const int64_t all = n_tokens * hidden, at = row * hidden;
  const int a = kRagged ? int(at & (V - 1)) : 0;
  const float inv = 1.0f / float(hidden);
  const XT *x = static_cast<const XT*>(args.x), *residual = static_cast<const XT*>(args.residual);
  auto fetch = [&](const XT* p, int64_t i) { return kRagged ? load_window(p, i, all) : *reinterpret_cast<const uint4*>(p + i); };
  auto load_weight = [&](const void* p, int col, float (&v)[V]) {
    Weight w;
    w.load(static_cast<const WT*>(p), col, hidden);
    w.at(col).get(v);
  };
  auto edge = [&](int col) { return kRagged && (col < 0 || col + V > hidden); };     // a window that reaches into another row
  uint4 rx[NV], rr[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V - a;
    if (col >= hidden) continue;
    rx[i] = fetch(x, at + col);
    rr[i] = fetch(residual, at + col);
  }
  float s[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V - a;
    if (col >= hidden) continue;
    Vec<XT, V> v;
    memcpy(&v, &rx[i], 16);
    v.get(s[i]);
  }
  // Mean and reciprocal deviation of the row in s.
  auto statistics = [&](int slot, float& mean, float& rstd) {
    mean = 0.f;
    if (!args.rms) {
      float sum[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = (i * group + tid) * V - a;
        if (col >= hidden) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += edge(col) && (col + j < 0 || col + j >= hidden) ? 0.f : s[i][j];
      }
      row_sum<kWarp>(sum, s_part, slot, tid, n_warps, [] { __syncthreads(); });
      mean = sum[0] * inv;
    }
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V - a;
      if (col >= hidden) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float c = edge(col) && (col + j < 0 || col + j >= hidden) ? 0.f : s[i][j] - mean;
        sq[0] += c * c;
      }
    }
    row_sum<kWarp>(sq, s_part, slot + 1, tid, n_warps, [] { __syncthreads(); });
    rstd = 1.0f / sqrtf(sq[0] * inv + args.eps);
  };
  float m1 = 0.f, r1 = 1.f, m2, r2;
  if (args.post_weight) statistics(0, m1, r1);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V - a;
    if (col >= hidden) continue;
    float p[V];
    if (args.post_weight) {
      load_weight(args.post_weight, col, p);
#pragma unroll
      for (int j = 0; j < V; ++j) s[i][j] = (s[i][j] - m1) * r1 * p[j];
      if (args.post_bias) {
        load_weight(args.post_bias, col, p);
#pragma unroll
        for (int j = 0; j < V; ++j) s[i][j] += p[j];
      }
    }
    if (args.gate) {
      load_weight(args.gate, col, p);
#pragma unroll
      for (int j = 0; j < V; ++j) s[i][j] *= p[j];
    }
    Vec<XT, V> v;
    memcpy(&v, &rr[i], 16);
    v.get(p);
#pragma unroll
    for (int j = 0; j < V; ++j) s[i][j] = fmaf(p[j], args.residual_scale, s[i][j]);
    v.set(s[i]);     // what is normalised is what the residual stream holds
    v.get(s[i]);
    store_window(static_cast<XT*>(args.total), at + col, s[i], -col, hidden - col);
  }
  statistics(2, m2, r2);
  if (tid == 0) {
    args.stats[row] = m1;
    args.stats[n_tokens + row] = r1;
    args.stats[2 * n_tokens + row] = m2;
    args.stats[3 * n_tokens + row] = r2;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V - a;
    if (col >= hidden) continue;
    float w[V], b[V];
    load_weight(args.weight, col, w);
    if (args.bias) load_weight(args.bias, col, b);
#pragma unroll
    for (int j = 0; j < V; ++j) s[i][j] = (s[i][j] - m2) * r2 * w[j] + (args.bias ? b[j] : 0.f);
    store_window(static_cast<XT*>(args.out), at + col, s[i], -col, hidden - col);
  }
}

// ---------------------------------------------------------------- backward
// A CTA's warps form groups of 1 to 32 warps, 16 columns a thread (24 beyond 8192); a group takes rows one after the other from a ring of its own, which
// bulk copies fill with the four tensors' rows, so that several rows are in flight whatever the arithmetic waits for.  (Beyond
// 8192 columns, where a ring of whole rows has no room, a CTA of 1024 threads loads from where the values lie.)  All
// rows of a CTA start equally far behind an aligned element (where rows start anywhere, they lie a multiple of V rows apart),
// so a thread's columns, and with them its sums over tokens, are the same in all of them.
// partial: [CTA][2 or 4 sums][pitch].
__host__ __device__ constexpr int columns_of(int threads) { return threads <= 512 ? 16 : 24; }      // of a thread
constexpr uint32_t kMaxStages = 8;
__host__ __device__ constexpr int part_pitch(int hidden) { return (hidden + 3) / 4 * 4; }

struct Shape {
  int32_t width;                    // threads of a group
  int32_t rows;                     // rows of a tile (1 where rows start anywhere)
  int32_t stages;
  uint32_t slot_bytes;              // of a tile of one tensor
};

template <typename XT, typename WT, bool kRagged, bool kRms, int kThreads>
__global__ void __launch_bounds__(kThreads, 1)
block_norm_bwd_kernel(const Args args, const Shape shape) {
  constexpr int V = 16 / int(sizeof(XT)), kE = int(sizeof(XT)), NV = columns_of(kThreads) / V, kSums = kRms ? 2 : 4;
  constexpr bool kRing = kThreads <= 512;      // else a row for all threads, from global memory
  constexpr int kMaxGroups = kRing ? kThreads / 32 : 1;
  extern __shared__ uint8_t smem_raw[];        // weight and post weight times gate as fp32 by window; the groups' rings; at the end their sums
  __shared__ float s_parts[kMaxGroups][4][32];
  __shared__ uint64_t s_bars[kMaxGroups][kMaxStages];
  __shared__ int s_abort;
  const int width = shape.width, mine = int(threadIdx.x) / width, tid = int(threadIdx.x) - mine * width, groups = kThreads / width;
  const int32_t hidden = args.hidden;
  const int64_t n_tokens = args.n_tokens, all = n_tokens * hidden;
  const int windows = width * NV, n_weights = windows * V;
  const uint32_t base = (smem_u32(smem_raw) + 15u) & ~15u;
  float* s_weight = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)));
  float* s_post = s_weight + n_weights;
  const uint32_t n_tensors = !kRing ? 0 : args.d_total ? 4 : 3, ring_bytes = uint32_t(shape.stages) * n_tensors * shape.slot_bytes;
  uint8_t* ring = reinterpret_cast<uint8_t*>(s_post + n_weights) + uint32_t(mine) * ring_bytes;
  const uint32_t ring_at = base + 8u * uint32_t(n_weights) + uint32_t(mine) * ring_bytes;
  uint64_t* s_bar = s_bars[mine];
  float(*s_part)[32] = s_parts[mine];
  auto sync = [&] { asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(width) : "memory"); };
  const WaitCtx wctx{&s_abort, args.status, kWaitLimitClocks};
  // Tiles of this group: first, first + stride, ..  A CTA's tiles are those of one residue modulo V where rows start anywhere.
  const int64_t n_tiles = (n_tokens + shape.rows - 1) / shape.rows, tile_elems = int64_t(shape.rows) * hidden;
  const int classes = kRagged ? V : 1, residue = int(blockIdx.x) % classes;
  const int64_t start = residue + (int64_t(blockIdx.x) / classes * groups + mine) * classes, stride = int64_t(gridDim.x) * groups;
  const int a = kRagged ? int(int64_t(residue) * hidden & (V - 1)) : 0;

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int g = 0; kRing && g < groups; ++g)
      for (int s = 0; s < shape.stages; ++s) mbar_init(smem_u32(&s_bars[g][s]), 1);
    fence_mbar_init();
  }
  __syncthreads();
  behind_wait();
  behind_go();

  const XT* const tensors[4] = {static_cast<const XT*>(args.d_out), static_cast<const XT*>(args.total), static_cast<const XT*>(args.x),
                                static_cast<const XT*>(args.d_total)};
  // One thread requests a tile: from the 16-byte boundary at or before its first element to the one at or behind its last; the
  // tensor's last elements, if no boundary follows them within it, by hand.
  auto request = [&](int64_t tile, int stage) {
    const int64_t first = tile * tile_elems, from = first & ~int64_t(V - 1), end = min(all, first + tile_elems);
    const int64_t last = all & ~int64_t(V - 1), to = min(last, (end + V - 1) & ~int64_t(V - 1));
    const uint32_t bytes = to > from ? uint32_t(to - from) * kE : 0, bar = smem_u32(&s_bar[stage]);
    const uint32_t at = uint32_t(stage) * n_tensors * shape.slot_bytes;
    if (end > last)
      for (uint32_t t = 0; t < n_tensors; ++t) {
        XT* slot = reinterpret_cast<XT*>(ring + at + t * shape.slot_bytes);
        for (int64_t e = max(last, from); e < end; ++e) slot[e - from] = tensors[t][e];
      }
    mbar_expect_tx(bar, n_tensors * bytes);
    if (bytes)
      for (uint32_t t = 0; t < n_tensors; ++t) bulk_load(ring_at + at + t * shape.slot_bytes, tensors[t] + from, bytes, bar);
  };
  int64_t asked = start;
  int n_asked = 0;
  if (kRing && tid == 0)
    for (int s = 0; s < shape.stages && asked < n_tiles; ++s, asked += stride, ++n_asked) request(asked, s);
  for (int k = threadIdx.x; k < n_weights; k += kThreads) {
    const int col = k - a;
    const bool in = col >= 0 && col < hidden;
    s_weight[k] = in ? float(static_cast<const WT*>(args.weight)[col]) : 0.f;
    float p = in ? 1.f : 0.f;
    if (in && args.post_weight) p *= float(static_cast<const WT*>(args.post_weight)[col]);
    if (in && args.gate) p *= float(static_cast<const WT*>(args.gate)[col]);
    s_post[k] = p;
  }
  __syncthreads();

  float sums[kSums][NV][V];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) sums[k][i][j] = 0.f;
  const float inv = 1.0f / float(hidden);
  const bool post = args.post_weight != nullptr;
  int stage = 0, turn = 0, slot = 0, before = -1;
  for (int64_t tile = start; tile < n_tiles; tile += stride) {
    if (kRing) mbar_wait(smem_u32(&s_bar[stage]), turn & 1, wctx);
    const uint32_t tile_at = ring_at + uint32_t(stage) * n_tensors * shape.slot_bytes;
    const int64_t row0 = tile * shape.rows;
    const int n_rows = int(min(int64_t(shape.rows), n_tokens - row0));
    for (int r = 0; r < n_rows; ++r, slot ^= 1) {
      const int64_t row = row0 + r, at = row * hidden;
      const uint32_t in_slot = tile_at + uint32_t(r * hidden * kE);      // (of window 0; r = 0 where rows start anywhere)
      const float m1 = args.stats[row], r1 = args.stats[n_tokens + row], m2 = args.stats[2 * n_tokens + row], r2 = args.stats[3 * n_tokens + row];
      const float shift1 = -m1 * r1, shift2 = -m2 * r2;
      auto load = [&](int t, int col, float (&v)[V]) {
        const uint4 q = kRing ? ld_shared_v4(in_slot + uint32_t(t) * shape.slot_bytes + uint32_t((col + a) * kE))
                        : kRagged ? load_window(tensors[t], at + col, all) : *reinterpret_cast<const uint4*>(tensors[t] + at + col);
        Vec<XT, V> w;
        memcpy(&w, &q, 16);
        w.get(v);
        if (kRagged && (col < 0 || col + V > hidden))
#pragma unroll
          for (int j = 0; j < V; ++j) v[j] = col + j >= 0 && col + j < hidden ? v[j] : 0.f;
      };
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = (i * width + tid) * V, col = k - a;
        if (col >= hidden) continue;
        float g[V], v[V];
        load(0, col, g);
        load(1, col, v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          v[j] = v[j] * r2 + shift2;
          sums[0][i][j] += g[j] * v[j];
          if (!kRms) sums[kSums - 2][i][j] += g[j];
          g[j] *= s_weight[k + j];
          sum[0] += g[j] * v[j];
          if (!kRms) sum[1] += g[j];
        }
      }
      if (width == 32) row_sum<true>(sum, s_part, slot, tid, 1, [] {});
      else row_sum<false>(sum, s_part, 0, tid, width >> 5, sync);
      // (all threads have left the tile before this one)
      if (kRing && before >= 0) {
        if (width == 32) __syncwarp();
        if (tid == 0 && asked < n_tiles && !s_abort) {
          request(asked, before);
          asked += stride;
          ++n_asked;
        }
        before = -1;
      }
      const float c_u = -sum[0] * inv * r2, c_1 = kRms ? 0.f : -sum[1] * inv * r2;
      float q[NV][V];
      sum[0] = sum[1] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = (i * width + tid) * V, col = k - a;
        if (col >= hidden) continue;
        float g[V], v[V], d[V];
        load(0, col, g);
        load(1, col, v);
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = g[j] * s_weight[k + j] * r2 + ((v[j] * r2 + shift2) * c_u + c_1);
        if (args.d_total) {
          load(3, col, g);
#pragma unroll
          for (int j = 0; j < V; ++j) d[j] += g[j];
        }
        if (kRagged && (col < 0 || col + V > hidden))
#pragma unroll
          for (int j = 0; j < V; ++j) d[j] = col + j >= 0 && col + j < hidden ? d[j] : 0.f;
        load(2, col, v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float u = v[j] * r1 + shift1;
          sums[1][i][j] += d[j] * u;
          if (!kRms) sums[kSums - 1][i][j] += d[j];
          q[i][j] = d[j] * s_post[k + j];
          sum[0] += q[i][j] * u;
          if (!kRms) sum[1] += q[i][j];
          d[j] *= args.residual_scale;
        }
        store_window(static_cast<XT*>(args.d_residual), at + col, d, -col, hidden - col);
      }
      float f = 1.f, e_u = 0.f, e_1 = 0.f;
      if (post) {
        if (width == 32) row_sum<true>(sum, s_part, 1, tid, 1, [] {});
        else row_sum<false>(sum, s_part, 1, tid, width >> 5, sync);
        f = r1;
        e_u = -sum[0] * inv * r1;
        e_1 = kRms ? 0.f : -sum[1] * inv * r1;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = (i * width + tid) * V, col = k - a;
        if (col >= hidden) continue;
        if (post) {
          float v[V];
          load(2, col, v);
#pragma unroll
          for (int j = 0; j < V; ++j) q[i][j] = q[i][j] * f + ((v[j] * r1 + shift1) * e_u + e_1);
        }
        store_window(static_cast<XT*>(args.dx), at + col, q[i], -col, hidden - col);
      }
      if (!post && width > 32) sync();       // (the next row's sums take the place of this one's)
    }
    if (!kRing) continue;
    before = stage;
    if (shape.stages == 1) {
      if (width == 32) __syncwarp(); else sync();
      if (tid == 0 && asked < n_tiles && !s_abort) {
        request(asked, stage);
        asked += stride;
        ++n_asked;
      }
      before = -1;
    }
    if (++stage == shape.stages) { stage = 0; ++turn; }
  }
  if (kRing && s_abort && tid == 0) {      // shared memory must outlive the copies in flight
    const long long t0 = clock64();
    for (int n = max(0, n_asked - shape.stages); n < n_asked; ++n)
      while (!mbar_try_wait(smem_u32(&s_bar[n % shape.stages]), (n / shape.stages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
  }
  __syncthreads();
  // The sums of a CTA's groups, each in a place of its own over the rings, are added in their order.
  float* const at_end = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)));
  const int pitch = part_pitch(hidden);
#pragma unroll
  for (int s = 0; s < kSums; ++s) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int k = (i * width + tid) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) at_end[mine * n_weights + k + j] = sums[s][i][j];
    }
    __syncthreads();
    for (int col = threadIdx.x; col < hidden; col += kThreads) {
      float v = 0.f;
      for (int g = 0; g < groups; ++g) v += at_end[g * n_weights + col + a];
      args.partial[(int64_t(blockIdx.x) * kSums + s) * pitch + col] = v;
    }
    __syncthreads();
  }
}

// The parts of all CTAs, added in a fixed order, and the parameters' gradients from the sums.
constexpr int kSumWarps = 16;
template <typename WT>
__global__ void __launch_bounds__(32 * kSumWarps)
block_norm_sum_kernel(const Args args, int32_t n_parts) {
  __shared__ float s[kSumWarps][4][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  behind_wait();
  behind_go();
  const int n_sums = args.rms ? 2 : 4, pitch = part_pitch(args.hidden);
  float v[4] = {};
  if (col < args.hidden) {
#pragma unroll 4
    for (int p = part; p < n_parts; p += kSumWarps)
      for (int k = 0; k < n_sums; ++k) v[k] += args.partial[(int64_t(p) * n_sums + k) * pitch + col];
  }
  for (int k = 0; k < 4; ++k) s[part][k][lane] = v[k];
  __syncthreads();
  if (part != 0 || col >= args.hidden) return;
  for (int p = 1; p < kSumWarps; ++p)
    for (int k = 0; k < 4; ++k) v[k] += s[p][k][lane];
  // dw, A, db, C
  auto put = [&](void* to, float f) {
    if (to) set_element(static_cast<WT*>(to) + col, f);
  };
  auto param = [&](const void* from, float other) { return from ? float(static_cast<const WT*>(from)[col]) : other; };
  put(args.d_weight, v[0]);
  put(args.d_bias, v[2]);
  const float gate = param(args.gate, 1.f);
  put(args.d_post_weight, gate * v[1]);
  put(args.d_post_bias, gate * v[3]);
  put(args.d_gate, param(args.post_weight, 1.f) * v[1] + param(args.post_bias, 0.f) * v[3]);
}

// ---------------------------------------------------------------- host
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
  const int nv = n <= 256 ? 1 : n <= 512 ? 2 : n <= 4096 ? 4 : 8;
  return {nv, ((n + nv - 1) / nv + 31) / 32 * 32};
}

template <typename XT, typename WT, int NV, bool kWarp, bool kRagged>
psa_status_t run_forward(const Args& args, int threads, cudaStream_t stream) {
  const int64_t grid = kWarp ? (args.n_tokens + kRowsPerCta - 1) / kRowsPerCta : args.n_tokens;
  launch_behind(true, block_norm_kernel<XT, WT, NV, kWarp, kRagged>, dim3(unsigned(grid)), kWarp ? 32 * kRowsPerCta : threads, 0, stream, args);
  return check_last_cuda_error("psa_block_norm launch");
}
template <typename XT, typename WT>
psa_status_t forward(const Args& args, cudaStream_t stream) {
  const Division d = divide(args.hidden, int(sizeof(XT)));
  const bool ragged = args.hidden * int(sizeof(XT)) % 16 != 0, warp = d.threads == 32;
#define PSA_BLOCK(NV) (warp ? (ragged ? run_forward<XT, WT, NV, true, true>(args, d.threads, stream) : run_forward<XT, WT, NV, true, false>(args, d.threads, stream)) \
                            : (ragged ? run_forward<XT, WT, NV, false, true>(args, d.threads, stream) : run_forward<XT, WT, NV, false, false>(args, d.threads, stream)))
  if (d.nv == 1) return PSA_BLOCK(1);
  if (d.nv == 2) return PSA_BLOCK(2);
  if (d.nv == 4) return PSA_BLOCK(4);
  if constexpr (sizeof(XT) == 4)      // rows of fp32 that reach into 4097 vectors
    return run_forward<XT, WT, 8, false, true>(args, d.threads, stream);
  return PSA_ERR_UNSUPPORTED;
#undef PSA_BLOCK
}

// The backward: a group of warps for a row, 16 columns a thread, in CTAs of 512 threads (1024 where a row needs more).
struct Launch {
  Shape shape;
  int32_t threads, ctas;
  uint32_t smem;
};
Launch plan_backward(int64_t n_tokens, int32_t hidden, int elem_bytes, int n_tensors) {
  Launch l{};
  const int V = 16 / elem_bytes, n = vectors(hidden, elem_bytes);
  const bool ragged = hidden * elem_bytes % 16 != 0;
  int warps = 1;
  while (warps < 32 && warps * 32 * (columns_of(512) / V) < n) warps *= 2;
  l.threads = warps > 16 ? 1024 : 512;
  const int columns = columns_of(l.threads);
  Shape& s = l.shape;
  s.width = 32 * warps;
  const int groups = l.threads / s.width;
  s.rows = 1;
  // several narrow rows a tile, as long as the tiles fill the groups
  while (!ragged && s.rows < 16 && 2 * s.rows * hidden * elem_bytes <= 2048 && n_tokens >= 4 * int64_t(s.rows) * groups * kSmCount) s.rows *= 2;
  s.slot_bytes = uint32_t((int64_t(s.rows) * hidden * elem_bytes + 47) / 16 * 16);
  if (warps > 16) n_tensors = 0;      // no ring
  const uint32_t weights = 2 * 4 * uint32_t(s.width * columns), room = 208 * 1024 - weights;
  s.stages = n_tensors ? int32_t(std::max(1u, std::min(kMaxStages, room / (uint32_t(groups) * n_tensors * s.slot_bytes)))) : 0;
  l.smem = weights + uint32_t(groups * s.stages * n_tensors) * s.slot_bytes + 16;
  l.smem = std::max(l.smem, uint32_t(groups * s.width * columns * 4) + 16);      // the groups' sums
  const int64_t tiles = std::max<int64_t>(1, (n_tokens + s.rows - 1) / s.rows);
  const int classes = ragged ? V : 1;
  int64_t ctas = std::min<int64_t>((tiles + groups - 1) / groups, kSmCount);
  if (ragged) ctas = ctas < classes ? classes : ctas / classes * classes;      // (the same number for every residue)
  l.ctas = int32_t(ctas);
  return l;
}

template <typename XT, typename WT>
psa_status_t backward(const Args& args, cudaStream_t stream) {
  const int e = int(sizeof(XT));
  const Launch l = plan_backward(args.n_tokens, args.hidden, e, args.d_total ? 4 : 3);
  const bool ragged = args.hidden * e % 16 != 0;
  auto go = [&](auto kernel) {
    constexpr int kLimit = 216 * 1024;      // (the kernel's, for all host threads: the same in every call)
    if (l.smem > uint32_t(kLimit)) return PSA_ERR_UNSUPPORTED;      // (no shape asks for more)
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLimit) != cudaSuccess) return PSA_ERR_CUDA;
    if (launch_behind(true, kernel, dim3(unsigned(l.ctas)), unsigned(l.threads), l.smem, stream, args, l.shape) != cudaSuccess)
      return failed_launch("psa_block_norm_bwd launch");      // (no sums of parts that are not written)
    launch_behind(true, block_norm_sum_kernel<WT>, dim3(unsigned((args.hidden + 31) / 32)), 32 * kSumWarps, 0, stream, args, l.ctas);
    return check_last_cuda_error("psa_block_norm_bwd launch");
  };
#define PSA_BLOCK(RAGGED, RMS) (l.threads == 512 ? go(block_norm_bwd_kernel<XT, WT, RAGGED, RMS, 512>) : go(block_norm_bwd_kernel<XT, WT, RAGGED, RMS, 1024>))
  return ragged ? (args.rms ? PSA_BLOCK(true, true) : PSA_BLOCK(true, false)) : (args.rms ? PSA_BLOCK(false, true) : PSA_BLOCK(false, false));
#undef PSA_BLOCK
}

psa_status_t check(const Args& a, int32_t dtype, int32_t weight_dtype) {
  if (a.n_tokens < 0 || a.hidden <= 0) return PSA_ERR_INVALID_ARG;
  if (!((dtype == PSA_DTYPE_BF16 && (weight_dtype == PSA_DTYPE_BF16 || weight_dtype == PSA_DTYPE_F32)) ||
        (dtype == PSA_DTYPE_F32 && weight_dtype == PSA_DTYPE_F32)))
    return PSA_ERR_INVALID_ARG;
  if (a.hidden > kMaxHidden || a.n_tokens > 0x7fffffffLL) return PSA_ERR_UNSUPPORTED;
  // biases go with layer norms, and a bias of the block's own norm with that norm
  if ((a.rms && (a.bias || a.post_bias || a.d_bias || a.d_post_bias)) || ((a.post_bias || a.d_post_bias) && !a.post_weight)) return PSA_ERR_INVALID_ARG;
  for (const void* p : {a.x, a.residual, a.weight, a.bias, a.post_weight, a.post_bias, a.gate, a.d_out, a.d_total,
                        static_cast<const void*>(a.out), static_cast<const void*>(a.total), static_cast<const void*>(a.stats),
                        static_cast<const void*>(a.dx), static_cast<const void*>(a.d_residual), static_cast<const void*>(a.d_weight),
                        static_cast<const void*>(a.d_bias), static_cast<const void*>(a.d_post_weight),
                        static_cast<const void*>(a.d_post_bias), static_cast<const void*>(a.d_gate), static_cast<const void*>(a.partial)})
    if (reinterpret_cast<uintptr_t>(p) & 15) return PSA_ERR_ALIGNMENT;
  return PSA_OK;
}

}  // namespace
}  // namespace psa

extern "C" psa_status_t psa_block_norm(const void* x, const void* residual, const void* weight, const void* bias,
                                       const void* post_weight, const void* post_bias, const void* gate, float residual_scale,
                                       int32_t dtype, int32_t weight_dtype, int64_t n_tokens, int32_t hidden, float eps, int32_t rms,
                                       void* out, void* total, float* stats, void* stream) {
  psa::Args a{};
  a.x = x; a.residual = residual; a.weight = weight; a.bias = bias; a.post_weight = post_weight; a.post_bias = post_bias; a.gate = gate;
  a.out = out; a.total = total; a.stats = stats;
  a.n_tokens = n_tokens; a.hidden = hidden; a.rms = rms; a.residual_scale = residual_scale; a.eps = eps;
  const psa_status_t rc = psa::check(a, dtype, weight_dtype);
  if (rc != PSA_OK) return rc;
  if (!(eps >= 0.f)) return PSA_ERR_INVALID_ARG;
  if (n_tokens == 0) return PSA_OK;
  if (!x || !residual || !weight || !out || !total || !stats) return PSA_ERR_INVALID_ARG;
  cudaStream_t st = cudaStream_t(stream);
  if (dtype == PSA_DTYPE_F32) return psa::forward<float, float>(a, st);
  return weight_dtype == PSA_DTYPE_F32 ? psa::forward<__nv_bfloat16, float>(a, st) : psa::forward<__nv_bfloat16, __nv_bfloat16>(a, st);
}

extern "C" size_t psa_block_norm_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden) {
  if (n_tokens < 0 || hidden <= 0 || hidden > psa::kMaxHidden) return 0;
  size_t parts = 0;
  for (int e : {2, 4})
    for (int tensors : {3, 4}) parts = std::max(parts, size_t(psa::plan_backward(n_tokens, hidden, e, tensors).ctas));
  return parts * 4 * size_t(psa::part_pitch(hidden)) * 4;
}

extern "C" psa_status_t psa_block_norm_bwd(const void* d_out, const void* x, const void* total, const void* weight,
                                           const void* post_weight, const void* post_bias, const void* gate, float residual_scale,
                                           const float* stats, const void* d_total, int32_t dtype, int32_t weight_dtype,
                                           int64_t n_tokens, int32_t hidden, int32_t rms, void* dx, void* d_residual, void* d_weight,
                                           void* d_bias, void* d_post_weight, void* d_post_bias, void* d_gate, void* workspace,
                                           int32_t* device_status, void* stream) {
  psa::Args a{};
  a.x = x; a.weight = weight; a.post_weight = post_weight; a.post_bias = post_bias; a.gate = gate;
  a.total = const_cast<void*>(total); a.stats = const_cast<float*>(stats); a.d_out = d_out; a.d_total = d_total;
  a.dx = dx; a.d_residual = d_residual; a.d_weight = d_weight; a.d_bias = d_bias; a.d_post_weight = d_post_weight;
  a.d_post_bias = d_post_bias; a.d_gate = d_gate; a.partial = static_cast<float*>(workspace);
  a.n_tokens = n_tokens; a.hidden = hidden; a.rms = rms; a.residual_scale = residual_scale; a.status = device_status;
  const psa_status_t rc = psa::check(a, dtype, weight_dtype);
  if (rc != PSA_OK) return rc;
  if (!weight || !d_weight || !workspace || (post_weight == nullptr) != (d_post_weight == nullptr) || (gate == nullptr) != (d_gate == nullptr))
    return PSA_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!d_out || !x || !total || !stats || !dx || !d_residual)) return PSA_ERR_INVALID_ARG;
  cudaStream_t st = cudaStream_t(stream);
  if (dtype == PSA_DTYPE_F32) return psa::backward<float, float>(a, st);
  return weight_dtype == PSA_DTYPE_F32 ? psa::backward<__nv_bfloat16, float>(a, st) : psa::backward<__nv_bfloat16, __nv_bfloat16>(a, st);
}
