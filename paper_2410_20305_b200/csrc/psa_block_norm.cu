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
// Measured: 16215 x 4096 bf16 RMS forward 93 to 95 us (5.7 TB/s), one token 7.6 to 8.2; 31041 x 4096 layer norm with gate backward 377 us (4.0 TB/s: two
// barriers for two rows, with as many warps as registers allow), RMS 329; 5465 x 1237 forward and backward 60.
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

// ---------------------------------------------------------------- pairs of fp32
// Two neighbouring columns in a 64-bit register: one instruction for both (half of these kernels' issue slots were arithmetic).
template <typename T, int V>
__device__ __forceinline__ void to_pairs(const Vec<T, V>& w, uint64_t (&v)[V / 2]) {
  float f[V];
  w.get(f);
#pragma unroll
  for (int j = 0; j < V / 2; ++j) v[j] = pack_f32x2(f[2 * j], f[2 * j + 1]);
}
template <int V>
__device__ __forceinline__ void to_floats(const uint64_t (&v)[V / 2], float (&f)[V]) {
#pragma unroll
  for (int j = 0; j < V / 2; ++j) unpack_f32x2(v[j], f[2 * j], f[2 * j + 1]);
}
__device__ __forceinline__ uint64_t both(float v) { return pack_f32x2(v, v); }
__device__ __forceinline__ float across(uint64_t v) {
  float lo, hi;
  unpack_f32x2(v, lo, hi);
  return lo + hi;
}
// Zeros in the columns of a window, which starts at column `col`, that belong to other rows.
template <int V>
__device__ __forceinline__ void clip(uint64_t (&v)[V / 2], int col, int hidden) {
  float f[V];
  to_floats<V>(v, f);
#pragma unroll
  for (int j = 0; j < V / 2; ++j)
    v[j] = pack_f32x2(col + 2 * j >= 0 && col + 2 * j < hidden ? f[2 * j] : 0.f, col + 2 * j + 1 >= 0 && col + 2 * j + 1 < hidden ? f[2 * j + 1] : 0.f);
}

// Sums over the warps of a row: each warp's by shuffles, then all of them read by everybody, 16 bytes at a time, in the warps'
// order.  parts: 32 floats a sum, zeros behind the last warp's.  One barrier; the caller alternates the place.
template <int N, typename Sync>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*parts)[32], int warp, int n_warps, Sync&& sync) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  if (n_warps == 1) return;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) parts[i][warp] = v[i];
  sync();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float sum = 0.f;
    for (int w = 0; w < n_warps; w += 4) {
      const float4 p = *reinterpret_cast<const float4*>(&parts[i][w]);
      sum += (p.x + p.y) + (p.z + p.w);
    }
    v[i] = sum;
  }
}

// ---------------------------------------------------------------- forward
template <typename XT, int NV, bool kWarp>
constexpr int fwd_threads() {
  return kWarp ? 32 * kRowsPerCta : NV <= 2 ? 256 : std::min(1024, kMaxHidden / (16 / int(sizeof(XT)) * NV) + 32);
}

template <typename XT, typename WT, int NV, bool kWarp, bool kRagged, bool kRms>
__global__ void __launch_bounds__(fwd_threads<XT, NV, kWarp>())
block_norm_kernel(const Args args) {
  constexpr int V = 16 / int(sizeof(XT)), H = V / 2;
  using Weight = Span<WT, V, kRagged>;
  __shared__ __align__(16) float s_part[4][32];
  const int group = kWarp ? 32 : int(blockDim.x), tid = kWarp ? int(threadIdx.x) & 31 : int(threadIdx.x), n_warps = kWarp ? 1 : int(blockDim.x) >> 5;
  const int64_t row = kWarp ? int64_t(blockIdx.x) * kRowsPerCta + (threadIdx.x >> 5) : int64_t(blockIdx.x);
  const int32_t hidden = args.hidden;
  const int64_t n_tokens = args.n_tokens;
  if (!kWarp && threadIdx.x < 128) s_part[threadIdx.x >> 5][threadIdx.x & 31] = 0.f;
  behind_wait();
  behind_go();
  if (kWarp && row >= n_tokens) return;
  const int64_t all = n_tokens * hidden, at = row * hidden;
  const int a = kRagged ? int(at & (V - 1)) : 0;
  const float inv = 1.0f / float(hidden);
  const XT *x = static_cast<const XT*>(args.x), *residual = static_cast<const XT*>(args.residual);
  // Threads behind a row's last window: in aligned rows they hold zeros throughout, so that only their loads and stores are left out (8000
  // rows of 2048: 42.7 -> 39.3 us; 16215 of 4096: 97.6 -> 93.4); in ragged ones, where edge windows branch anyway, they skip every step (8000 rows
  // of 1237: 31.2 us, with zeros 32.8).
  auto column = [&](int i) { return (i * group + tid) * V - a; };
  auto skips = [&](int i) { return kRagged && column(i) >= hidden; };
  auto fetch = [&](const XT* p, int col) {
    if (col >= hidden) return make_uint4(0, 0, 0, 0);
    return kRagged ? load_window(p, at + col, all) : *reinterpret_cast<const uint4*>(p + at + col);
  };
  auto load_weight = [&](const void* p, int col, uint64_t (&v)[H]) {
    Vec<WT, V> x;
    x.clear();
    if (col < hidden) {
      Weight w;
      w.load(static_cast<const WT*>(p), col, hidden);
      x = w.at(col);
    }
    to_pairs(x, v);
  };
  auto pairs_of = [&](const uint4& raw, uint64_t (&v)[H]) {
    Vec<XT, V> w;
    memcpy(&w, &raw, 16);
    to_pairs(w, v);
  };
  auto edge = [&](int col) { return kRagged && (col < 0 || col + V > hidden); };     // a window that reaches into another row
  auto put = [&](void* p, int col, const float (&f)[V]) {
    if (col < hidden) store_window(static_cast<XT*>(p), at + col, f, -col, hidden - col);
  };
  uint4 rx[NV], rr[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (skips(i)) continue;
    rx[i] = fetch(x, column(i));
    rr[i] = fetch(residual, column(i));
  }
  if (!kWarp) __syncthreads();      // the zeros are there
  uint64_t s[NV][H];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (!skips(i)) pairs_of(rx[i], s[i]);
  // Mean and reciprocal deviation of the row in s.
  auto statistics = [&](int slot, float& mean, float& rstd) {
    mean = 0.f;
    if (!kRms) {
      uint64_t sum2 = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (skips(i)) continue;
        uint64_t v[H];
#pragma unroll
        for (int j = 0; j < H; ++j) v[j] = s[i][j];
        if (edge(column(i))) clip<V>(v, column(i), hidden);
#pragma unroll
        for (int j = 0; j < H; ++j) sum2 = add_f32x2(sum2, v[j]);
      }
      float sum[1] = {across(sum2)};
      row_sums(sum, s_part + slot, int(threadIdx.x) >> 5, n_warps, [] { __syncthreads(); });
      mean = sum[0] * inv;
    }
    uint64_t sq2 = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (skips(i)) continue;
      const uint64_t shift = both(column(i) < hidden ? -mean : 0.f);
      uint64_t v[H];
#pragma unroll
      for (int j = 0; j < H; ++j) v[j] = kRms ? s[i][j] : add_f32x2(s[i][j], shift);
      if (edge(column(i))) clip<V>(v, column(i), hidden);
#pragma unroll
      for (int j = 0; j < H; ++j) sq2 = fma_f32x2(v[j], v[j], sq2);
    }
    float sq[1] = {across(sq2)};
    row_sums(sq, s_part + slot + 1, int(threadIdx.x) >> 5, n_warps, [] { __syncthreads(); });
    rstd = 1.0f / sqrtf(sq[0] * inv + args.eps);
  };
  float m1 = 0.f, r1 = 1.f, m2, r2;
  if (args.post_weight) statistics(0, m1, r1);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (skips(i)) continue;
    const int col = column(i);
    uint64_t p[H];
    if (args.post_weight) {
      load_weight(args.post_weight, col, p);
#pragma unroll
      for (int j = 0; j < H; ++j) s[i][j] = mul_f32x2(mul_f32x2(kRms ? s[i][j] : add_f32x2(s[i][j], both(-m1)), both(r1)), p[j]);
      if (!kRms && args.post_bias) {
        load_weight(args.post_bias, col, p);
#pragma unroll
        for (int j = 0; j < H; ++j) s[i][j] = add_f32x2(s[i][j], p[j]);
      }
    }
    if (args.gate) {
      load_weight(args.gate, col, p);
#pragma unroll
      for (int j = 0; j < H; ++j) s[i][j] = mul_f32x2(s[i][j], p[j]);
    }
    pairs_of(rr[i], p);
    float f[V];
    // The product is rounded before the sum: of a scale that fp32 does not hold, like 0.7, what was added to it goes with that.  (One fma kept it, and
    // 6e-4 of all sums, which lie on a tie of bf16 as written, went the other way.  Products of pairs are made one fma with the sum, too.)
    if (args.residual_scale != 1.f) {
#pragma unroll
      for (int j = 0; j < H; ++j) {
        float lo, hi;
        unpack_f32x2(p[j], lo, hi);
        p[j] = pack_f32x2(__fmul_rn(lo, args.residual_scale), __fmul_rn(hi, args.residual_scale));
      }
    }
#pragma unroll
    for (int j = 0; j < H; ++j) s[i][j] = add_f32x2(p[j], s[i][j]);
    to_floats<V>(s[i], f);
    put(args.total, col, f);
    Vec<XT, V> v;     // what is normalised is what the residual stream holds
    v.set(f);
    to_pairs(v, s[i]);
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
    if (skips(i)) continue;
    const int col = column(i);
    uint64_t w[H];
    load_weight(args.weight, col, w);
#pragma unroll
    for (int j = 0; j < H; ++j) s[i][j] = mul_f32x2(mul_f32x2(kRms ? s[i][j] : add_f32x2(s[i][j], both(-m2)), both(r2)), w[j]);
    if (!kRms && args.bias) {
      load_weight(args.bias, col, w);
#pragma unroll
      for (int j = 0; j < H; ++j) s[i][j] = add_f32x2(s[i][j], w[j]);
    }
    float f[V];
    to_floats<V>(s[i], f);
    put(args.out, col, f);
  }
}

// ---------------------------------------------------------------- backward
// A CTA's warps form groups that take rows one after the other, 8 columns a thread (16 beyond 4096), each from a ring of its own, which bulk copies
// fill with the four tensors' rows, so that several rows are in flight whatever the arithmetic waits for.
// (Beyond 8192 columns, where no ring of whole rows has room, 1024 threads take a row, 24 columns each, from where it lies, and spill 1 to 2 KB
// a thread.)
// The two norms of a row need its sums one after the other; a group takes two rows at a time
// (of up to 4096 columns), whose sums cross a barrier together.
// All rows of a CTA start equally far behind an aligned element (where rows start anywhere, they lie a multiple of V rows
// apart), so a thread's columns, and with them its sums over tokens, are the same in all of them.
// partial: [CTA][2 or 4 sums][pitch].
constexpr int kRingThreads = 512, kWideThreads = 1024;
constexpr int kMaxGroups = 16;                          // (15 of several warps: each needs a barrier)
constexpr uint32_t kMaxStages = 8;
// Shared memory of weights and rings.  (208 KB leave L1 no room for what the compiler spills, up to 276 bytes of stores a thread in layer
// norms, stacks of 8 to 104: 385 us instead of 371 at 31041 x 4096.)
constexpr uint32_t kRoom = 176 * 1024;
constexpr int kRingColumns = 16, kWideColumns = 24;      // of a thread, at most
__host__ __device__ constexpr int part_pitch(int hidden) { return (hidden + 3) / 4 * 4; }

struct Shape {
  int32_t width, groups;            // threads of a group; groups of a CTA
  int32_t rows;                     // rows of a tile (1 where rows start anywhere)
  int32_t stages;
  uint32_t slot_bytes;              // of a tile of one tensor
};

// Sums of N values (2 or 4) over a group's threads, in all of them.  A warp's: in each step the lanes that do not keep a value send it
// to those that do, until each lane holds one; the group's: the same lanes add the sums of kWarps warps, which they find in
// `parts` (zeros where there are fewer warps).
template <int N, int kWarps, typename Sync>
__device__ __forceinline__ void group_sums(float (&v)[N], float* parts, int warp, int n_warps, Sync&& sync) {
  constexpr int kLanes = 32 / N;      // of a value
  const int lane = threadIdx.x & 31, which = lane / kLanes, place = lane % kLanes;
  const bool high = lane & 16, odd = lane & 8;
  float mine;
  if (N == 4) {
    float k[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) k[i] = (high ? v[N / 2 + i] : v[i]) + __shfl_xor_sync(0xffffffffu, high ? v[i] : v[N / 2 + i], 16);
    mine = (odd ? k[1] : k[0]) + __shfl_xor_sync(0xffffffffu, odd ? k[0] : k[1], 8);
  } else {
    mine = (high ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, high ? v[0] : v[1], 16);
  }
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if (n_warps > 1) {
    if (place == 0) parts[warp * N + which] = mine;
    sync();
    mine = parts[place * N + which];
#pragma unroll
    for (int w = kLanes; w < kWarps; w += kLanes) mine += parts[(w + place) * N + which];
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, mine, i * kLanes);
}

template <typename XT, typename WT, bool kRagged, bool kRms, int kColumns>
__global__ void __launch_bounds__(kColumns <= kRingColumns ? kRingThreads : kWideThreads, 1)
block_norm_bwd_kernel(const Args args, const Shape shape) {
  constexpr bool kRing = kColumns <= kRingColumns;
  constexpr int V = 16 / int(sizeof(XT)), H = V / 2, kE = int(sizeof(XT)), NV = kColumns / V, kSums = kRms ? 2 : 4;
  constexpr int kN = kColumns == 8 ? 2 : 1;      // rows at a time
  extern __shared__ uint8_t smem_raw[];        // weight and post weight times gate as fp32 by window; the groups' rings; at the end their sums
  __shared__ __align__(16) float s_parts[kMaxGroups][2][4 * 32];
  // of two rows: m1, r1, m2, r2;  those of the next two arrive while slow warps still finish the two before these
  __shared__ __align__(16) float s_stats[kMaxGroups][3][2][4];
  __shared__ uint64_t s_full[kMaxGroups][kMaxStages];
  __shared__ int s_abort;
  const int width = shape.width, groups = shape.groups, n_warps = width >> 5;
  const int32_t hidden = args.hidden;
  const int64_t n_tokens = args.n_tokens, all = n_tokens * hidden;
  const int n_weights = width * NV * V;
  const uint32_t base = (smem_u32(smem_raw) + 15u) & ~15u;
  float* s_weight = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)));
  const uint32_t n_tensors = !kRing ? 0 : args.d_total ? 4 : 3, ring_bytes = uint32_t(shape.stages) * n_tensors * shape.slot_bytes;
  const uint32_t rings = base + 8u * uint32_t(n_weights);
  const WaitCtx wctx{&s_abort, args.status, kWaitLimitClocks};
  // Tiles of group g: first(g), first(g) + stride, ..  A CTA's tiles are those of one residue modulo V where rows start anywhere.
  const int64_t n_tiles = (n_tokens + shape.rows - 1) / shape.rows, stride = int64_t(gridDim.x) * groups;
  const int classes = kRagged ? V : 1, residue = int(blockIdx.x) % classes;
  auto first_of = [&](int g) { return residue + (int64_t(blockIdx.x) / classes * groups + g) * classes; };
  const int a = kRagged ? int(int64_t(residue) * hidden & (V - 1)) : 0;

  for (int k = threadIdx.x; k < kMaxGroups * 2 * 4 * 32; k += blockDim.x) (&s_parts[0][0][0])[k] = 0.f;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int g = 0; kRing && g < groups; ++g)
      for (int s = 0; s < shape.stages; ++s) mbar_init(smem_u32(&s_full[g][s]), 1);
    fence_mbar_init();
  }
  __syncthreads();
  behind_wait();
  behind_go();
  for (int k = threadIdx.x; k < n_weights; k += blockDim.x) {
    const int col = k - a;
    const bool in = col >= 0 && col < hidden;
    s_weight[k] = in ? float(static_cast<const WT*>(args.weight)[col]) : 0.f;
    float p = in ? 1.f : 0.f;
    if (in && args.post_weight) p *= float(static_cast<const WT*>(args.post_weight)[col]);
    if (in && args.gate) p *= float(static_cast<const WT*>(args.gate)[col]);
    s_weight[n_weights + k] = p;
  }

  const int mine = int(threadIdx.x) / width, tid = int(threadIdx.x) - mine * width, warp = tid >> 5;
  const uint32_t ring = rings + uint32_t(mine) * ring_bytes, leader = kRing && warp == 0 ? elect_one() : 0;
  // The first warp of a group requests a tile: from the 16-byte boundary at or before its first element to the one at or behind its
  // last; the tensor's last elements, if no boundary follows them within it, by hand.
  auto request = [&](int64_t tile, int stage) {
    const int64_t begin = tile * shape.rows * hidden, from = begin & ~int64_t(V - 1), end = min(all, begin + int64_t(shape.rows) * hidden);
    const int64_t last = all & ~int64_t(V - 1), to = min(last, (end + V - 1) & ~int64_t(V - 1));
    const uint32_t bytes = to > from ? uint32_t(to - from) * kE : 0, bar = smem_u32(&s_full[mine][stage]);
    const uint32_t slot = ring + uint32_t(stage) * n_tensors * shape.slot_bytes;
    const void* const tensors[4] = {args.d_out, args.total, args.x, args.d_total};
    if (kRagged && end > last && leader)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < int(n_tensors))
          for (int64_t e = max(last, from); e < end; ++e)
            reinterpret_cast<XT*>(smem_raw + (slot + t * shape.slot_bytes - smem_u32(smem_raw)))[e - from] = static_cast<const XT*>(tensors[t])[e];
    mbar_expect_tx_w(bar, n_tensors * bytes, leader);
#pragma unroll
    for (int t = 0; t < 4; ++t)
      bulk_load_w(slot + t * shape.slot_bytes, static_cast<const XT*>(tensors[t]) + from, bytes, bar, t < int(n_tensors) && bytes ? leader : 0);
  };
  int64_t asked = first_of(mine);      // the next tile to request, and how many have been (the first warp's)
  int n_asked = 0;
  if (kRing && warp == 0 && mine < groups)
    for (int s = 0; s < shape.stages && asked < n_tiles; ++s, asked += stride, ++n_asked) request(asked, s);
  __syncthreads();      // the weights are there

  uint64_t sums[kSums][NV][H];      // of the columns of this thread: d_out u2, ds u1, and without RMS d_out, ds
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < H; ++j) sums[k][i][j] = 0;
  if (mine < groups && first_of(mine) < n_tiles) {
    auto sync = [&] { asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(width) : "memory"); };
    auto load_weight = [&](uint32_t from, uint64_t (&v)[H]) {
#pragma unroll
      for (int j = 0; j < H; j += 2)
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[j]), "=l"(v[j + 1]) : "r"(from + 8u * uint32_t(j)) : "memory");
    };
    const float inv = 1.0f / float(hidden);
    const bool post = args.post_weight != nullptr, with_total = args.d_total != nullptr;
    // Rows of an iteration lie in one tile, or in two where a tile is a row; alone where the ring has one stage.
    const int rows = shape.rows, per_tile = kN == 2 && rows > 1 ? 2 : 1, stages = shape.stages;
    const bool pairs = kN == 2 && (rows > 1 || stages > 1);
    const int tiles_each = rows == 1 && pairs ? 2 : 1;
    const uint32_t step = uint32_t(stride) * rows;   // rows between two tiles of the group
    const uint32_t stage_bytes = n_tensors * shape.slot_bytes, weights_at = base + uint32_t(tid) * V * 4u;
    // (Threads behind a row's last window write nothing and have weights of zero; from a ring they take the row's first window, from
    // memory, where it may have been written over by then, nothing.)
    uint32_t in_row[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) in_row[i] = (i * width + tid) * V - a < hidden ? uint32_t(i * width + tid) * 16u : 0u;
    uint32_t tile = uint32_t(first_of(mine)), row = tile * rows;
    int r = 0, stage = 0, turn = 0, n_done = 0;      // r: row of the tile; n_done: tiles that the group is done with
    struct Row {
      uint32_t row;
      uint32_t slot;
    };
    // The statistics of a row and of the one that goes with it, copied ahead: eight lanes of the group's first warp.
    auto second_of = [&](uint32_t first) { return tiles_each == 2 ? first + step : first + 1; };
    auto fetch_stats = [&](uint32_t first, int place) {
      const int k = threadIdx.x & 3;
      const uint32_t at = (tid & 4) ? second_of(first) : first;
      if (tid < 8 && at < n_tokens)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(&s_stats[mine][place][tid >> 2][k])), "l"(args.stats + k * n_tokens + at) : "memory");
    };
    auto stats_there = [&] {
      if (tid < 8) asm volatile("cp.async.wait_all;" ::: "memory");
    };
    int place = 0;
    fetch_stats(row, 0);
    stats_there();
    if (n_warps > 1) sync(); else __syncwarp();
    while (tile < uint32_t(n_tiles)) {
      Row two[kN];
      two[0].row = row;
      two[0].slot = ring + uint32_t(stage) * stage_bytes + uint32_t(r * hidden * kE);
      const int other = stage + 1 == stages ? 0 : stage + 1;
      const bool second = pairs && second_of(row) < n_tokens;
      if (kN == 2) {
        two[kN - 1].row = second_of(row);
        two[kN - 1].slot = tiles_each == 2 ? ring + uint32_t(other) * stage_bytes : two[0].slot + uint32_t(hidden * kE);
      }
      const bool more = r + per_tile < rows && row + per_tile < n_tokens;      // of this tile
      fetch_stats(more ? row + per_tile : row - r + step * tiles_each, place == 2 ? 0 : place + 1);
      if (kRing) {
        if (r == 0) mbar_wait(smem_u32(&s_full[mine][stage]), turn & 1, wctx);
        if (tiles_each == 2 && second) mbar_wait(smem_u32(&s_full[mine][other]), (other ? turn : turn + 1) & 1, wctx);
      }
      auto load = [&](const Row& x, int t, const void* p, int i, uint64_t (&v)[H]) {
        const XT* const from = static_cast<const XT*>(p);
        const int64_t at = int64_t(x.row) * hidden + int64_t(in_row[i] / 16u) * V - a;
        const uint4 raw = kRing ? ld_shared_v4(x.slot + uint32_t(t) * shape.slot_bytes + in_row[i])
                          : (i * width + tid) * V - a >= hidden ? make_uint4(0, 0, 0, 0)
                          : kRagged ? load_window(from, at, all) : *reinterpret_cast<const uint4*>(from + at);
        Vec<XT, V> w;
        memcpy(&w, &raw, 16);
        to_pairs(w, v);
        return raw;
      };
      auto put = [&](void* p, const Row& x, int i, const uint64_t (&v)[H]) {
        float f[V];
        to_floats<V>(v, f);
        const int col = (i * width + tid) * V - a;
        if (col >= hidden) return;
        XT* const to = static_cast<XT*>(p) + (int64_t(x.row) * hidden + col);
        if (kRagged) store_window(to, 0, f, -col, hidden - col);
        else store_vec<XT, V>(to, f);
      };
      auto edge = [&](int col) { return kRagged && (col < 0 || col + V > hidden); };
      auto scaled = [](const uint64_t& v, float r, float m) { return kRms ? mul_f32x2(v, both(r)) : fma_f32x2(v, both(r), both(-m * r)); };   // (v - m) r
      auto stats_of = [&](int n) { return *reinterpret_cast<const float4*>(s_stats[mine][place][n]); };      // m1, r1, m2, r2
      constexpr int kValues = kRms || kN == 1 ? 2 : 4, kMaxWarps = (kRing ? kRingThreads : kWideThreads) / 32;
      float value[kValues];
#pragma unroll
      for (int k = 0; k < kValues; ++k) value[k] = 0.f;
#pragma unroll
      for (int n = 0; n < kN; ++n) {
        if (n && !second) break;
        const Row& x = two[n];
        const float4 st = stats_of(n);
        uint64_t sum_u = 0, sum_1 = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int col = (i * width + tid) * V - a;
          uint64_t g[H], v[H], w[H];
          load(x, 0, args.d_out, i, g);
          load(x, 1, args.total, i, v);
          load_weight(weights_at + uint32_t(i * width * V) * 4u, w);
#pragma unroll
          for (int j = 0; j < H; ++j) v[j] = scaled(v[j], st.w, st.z);
          if (edge(col)) {
            clip<V>(g, col, hidden);
            clip<V>(v, col, hidden);
          }
#pragma unroll
          for (int j = 0; j < H; ++j) {
            sums[0][i][j] = fma_f32x2(g[j], v[j], sums[0][i][j]);
            if (!kRms) sums[kSums - 2][i][j] = add_f32x2(sums[kSums - 2][i][j], g[j]);
            g[j] = mul_f32x2(g[j], w[j]);
            sum_u = fma_f32x2(g[j], v[j], sum_u);
            if (!kRms) sum_1 = add_f32x2(sum_1, g[j]);
          }
        }
        value[n] = across(sum_u);
        if (!kRms) value[kRms ? 0 : kN + n] = across(sum_1);
      }
      group_sums<kValues, kMaxWarps>(value, s_parts[mine][0], warp, n_warps, sync);
      uint64_t q[kN][NV][H];
      uint4 raw_x[kN][NV];      // (kept, so that the rows' place can be filled again before the last step)
      float kept[kValues];
#pragma unroll
      for (int k = 0; k < kValues; ++k) kept[k] = value[k];
#pragma unroll
      for (int n = 0; n < kN; ++n) {
        if (n && !second) break;
        const Row& x = two[n];
        // ds = g r2 + (u2 c_u + c_1) with u2 = (s - m2) r2
        const float4 st = stats_of(n);
        const float c_u = -kept[n] * inv * st.w * st.w, c_1 = kRms ? 0.f : -kept[kRms ? 0 : kN + n] * inv * st.w - st.z * c_u;
        uint64_t sum_u = 0, sum_1 = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int col = (i * width + tid) * V - a;
          uint64_t g[H], v[H], d[H];
          load(x, 0, args.d_out, i, g);
          load_weight(weights_at + uint32_t(i * width * V) * 4u, d);
          load(x, 1, args.total, i, v);
#pragma unroll
          for (int j = 0; j < H; ++j) {
            v[j] = kRms ? mul_f32x2(v[j], both(c_u)) : fma_f32x2(v[j], both(c_u), both(c_1));
            d[j] = fma_f32x2(mul_f32x2(g[j], d[j]), both(st.w), v[j]);
          }
          if (with_total) {
            load(x, 3, args.d_total, i, g);
#pragma unroll
            for (int j = 0; j < H; ++j) d[j] = add_f32x2(d[j], g[j]);
          }
          raw_x[n][i] = load(x, 2, args.x, i, v);
          if (post)
#pragma unroll
            for (int j = 0; j < H; ++j) v[j] = scaled(v[j], st.y, st.x);
          if (edge(col)) {
            clip<V>(d, col, hidden);
            clip<V>(v, col, hidden);
          }
          load_weight(weights_at + uint32_t(n_weights + i * width * V) * 4u, g);
#pragma unroll
          for (int j = 0; j < H; ++j) {
            sums[1][i][j] = fma_f32x2(d[j], v[j], sums[1][i][j]);
            if (!kRms) sums[kSums - 1][i][j] = add_f32x2(sums[kSums - 1][i][j], d[j]);
            q[n][i][j] = mul_f32x2(d[j], g[j]);
            sum_u = fma_f32x2(q[n][i][j], v[j], sum_u);
            if (!kRms) sum_1 = add_f32x2(sum_1, q[n][i][j]);
            d[j] = mul_f32x2(d[j], both(args.residual_scale));
          }
          put(args.d_residual, x, i, d);
          if (!post) put(args.dx, x, i, q[n][i]);
        }
        value[n] = across(sum_u);
        if (!kRms) value[kRms ? 0 : kN + n] = across(sum_1);
      }
      stats_there();
      if (post) group_sums<kValues, kMaxWarps>(value, s_parts[mine][1], warp, n_warps, sync);
      else if (n_warps > 1) sync();      // (the next sums take the place of these)
      if (n_warps == 1) __syncwarp();
      // on to the next rows; all threads have read these
      r += per_tile;
      row += per_tile;
      if (r >= rows || row >= n_tokens) {
        row += step - r;
        r = 0;
        tile += stride;
        ++n_done;
        if (++stage >= stages) { stage = 0; ++turn; }
        if (tiles_each == 2) {
          row += step;
          tile += stride;
          ++n_done;
          if (++stage >= stages) { stage = 0; ++turn; }
        }
        if (kRing) {
          if (warp == 0 && !s_abort)
            for (; n_asked < n_done + stages && asked < n_tiles; asked += stride, ++n_asked) request(asked, n_asked % stages);
        }
      }
      const int here = place;
      place = place == 2 ? 0 : place + 1;
      if (!post) continue;
#pragma unroll
      for (int n = 0; n < kN; ++n) {
        if (n && !second) break;
        const Row& x = two[n];
        // dx = q r1 + (u1 e_u + e_1) with u1 = (x - m1) r1
        const float4 st = *reinterpret_cast<const float4*>(s_stats[mine][here][n]);
        const float e_u = -value[n] * inv * st.y * st.y, e_1 = kRms ? 0.f : -value[kRms ? 0 : kN + n] * inv * st.y - st.x * e_u;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          uint64_t v[H];
          Vec<XT, V> w;
          memcpy(&w, &raw_x[n][i], 16);
          to_pairs(w, v);
#pragma unroll
          for (int j = 0; j < H; ++j) {
            v[j] = kRms ? mul_f32x2(v[j], both(e_u)) : fma_f32x2(v[j], both(e_u), both(e_1));
            v[j] = fma_f32x2(q[n][i][j], both(st.y), v[j]);
          }
          put(args.dx, x, i, v);
        }
      }
    }
    if (kRing && s_abort && warp == 0) {      // shared memory must outlive the copies in flight
      const long long t0 = clock64();
      for (int i = max(0, n_asked - stages); i < n_asked; ++i)
        while (!mbar_try_wait(smem_u32(&s_full[mine][i % stages]), (i / stages) & 1) && clock64() - t0 < kWaitLimitClocks) {}
    }
  }
  __syncthreads();
  // The sums of a CTA's groups, each in a place of its own over the rings, are added in their order.
  const int pitch = part_pitch(hidden);
#pragma unroll
  for (int s = 0; s < kSums; ++s) {
    if (mine < groups)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const uint32_t to = base + 4u * uint32_t(mine * n_weights + (i * width + tid) * V);
#pragma unroll
        for (int j = 0; j < H; j += 2)
          st_shared_v4(to + 8 * j, uint32_t(sums[s][i][j]), uint32_t(sums[s][i][j] >> 32), uint32_t(sums[s][i][j + 1]), uint32_t(sums[s][i][j + 1] >> 32));
      }
    __syncthreads();
    for (int col = threadIdx.x; col < hidden; col += blockDim.x) {
      float v = 0.f;
      for (int g = 0; g < groups; ++g) v += s_weight[g * n_weights + col + a];
      args.partial[(int64_t(blockIdx.x) * kSums + s) * pitch + col] = v;
    }
    __syncthreads();
  }
}

// The parts of all CTAs, added in a fixed order, and the parameters' gradients from the sums.  (Warps of a sum each, 8 loads in
// flight instead of 16, took 3 us longer at 148 parts of 4096 columns.)
constexpr int kSumWarps = 16;
template <typename WT>
__global__ void __launch_bounds__(32 * kSumWarps)
block_norm_sum_kernel(const Args args, int32_t n_parts) {
  __shared__ float s[kSumWarps][4][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  behind_wait();
  behind_go();
  const int n_sums = args.rms ? 2 : 4, pitch = part_pitch(args.hidden);
  float v[4] = {};      // d_out u2, ds u1, d_out, ds
  if (col < args.hidden) {
    const float* from = args.partial + col;
#pragma unroll 4
    for (int p = part; p < n_parts; p += kSumWarps)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n_sums) v[k] += from[(int64_t(p) * n_sums + k) * pitch];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) s[part][k][lane] = v[k];
  __syncthreads();
  if (part != 0 || col >= args.hidden) return;
  for (int p = 1; p < kSumWarps; ++p)
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += s[p][k][lane];
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
  launch_behind(true, args.rms ? block_norm_kernel<XT, WT, NV, kWarp, kRagged, true> : block_norm_kernel<XT, WT, NV, kWarp, kRagged, false>,
                dim3(unsigned(grid)), kWarp ? 32 * kRowsPerCta : threads, 0, stream, args);
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

// The backward: as many warps to a group as its rows need, as many groups to a CTA as fit, a CTA an SM.
struct Launch {
  Shape shape;
  int32_t ctas, columns;
  uint32_t smem;
};
Launch plan_backward(int64_t n_tokens, int32_t hidden, int elem_bytes, int n_tensors) {
  Launch l{};
  const int V = 16 / elem_bytes, n = vectors(hidden, elem_bytes);
  const bool ragged = hidden * elem_bytes % 16 != 0;
  auto warps_of = [&](int columns) { return (n * V + 32 * columns - 1) / (32 * columns); };
  l.columns = warps_of(8) <= kRingThreads / 32 ? 8 : warps_of(kRingColumns) <= kRingThreads / 32 ? kRingColumns : kWideColumns;
  const int warps = warps_of(l.columns);
  const bool ring = l.columns <= kRingColumns;
  Shape& s = l.shape;
  s.width = ring ? 32 * warps : kWideThreads;
  s.groups = ring ? std::min(kRingThreads / s.width, warps > 1 ? kMaxGroups - 1 : kMaxGroups) : 1;
  // no more groups than there are rows for them
  s.groups = int32_t(std::max<int64_t>(1, std::min<int64_t>(s.groups, (n_tokens + kSmCount - 1) / kSmCount)));
  s.rows = 1;
  // several narrow rows a tile, as long as the tiles fill the groups
  while (!ragged && s.rows < 16 && 2 * s.rows * hidden * elem_bytes <= 1024 && n_tokens >= 4 * int64_t(s.rows) * s.groups * kSmCount) s.rows *= 2;
  s.slot_bytes = uint32_t((int64_t(s.rows) * hidden * elem_bytes + 47) / 16 * 16);
  const uint32_t columns = uint32_t(s.width * l.columns), weights = 2 * 4 * columns, room = kRoom - weights;
  s.stages = ring ? int32_t(std::max(1u, std::min(kMaxStages, room / (uint32_t(s.groups) * n_tensors * s.slot_bytes)))) : 0;
  l.smem = weights + uint32_t(s.groups * s.stages * n_tensors) * s.slot_bytes + 16;
  l.smem = std::max(l.smem, uint32_t(s.groups) * columns * 4 + 16);      // the groups' sums
  const int64_t tiles = std::max<int64_t>(1, (n_tokens + s.rows - 1) / s.rows);
  const int classes = ragged ? V : 1;
  int64_t ctas = std::min<int64_t>((tiles + s.groups - 1) / s.groups, kSmCount);
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
    constexpr int kLimit = 200 * 1024;      // (the kernel's, for all host threads: the same in every call)
    if (l.smem > uint32_t(kLimit)) return PSA_ERR_UNSUPPORTED;      // (no shape asks for more)
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLimit) != cudaSuccess) return PSA_ERR_CUDA;
    if (launch_behind(true, kernel, dim3(unsigned(l.ctas)), unsigned(l.shape.width * l.shape.groups), l.smem, stream, args, l.shape) != cudaSuccess)
      return failed_launch("psa_block_norm_bwd launch");      // (no sums of parts that are not written)
    launch_behind(true, block_norm_sum_kernel<WT>, dim3(unsigned((args.hidden + 31) / 32)), 32 * kSumWarps, 0, stream, args, l.ctas);
    return check_last_cuda_error("psa_block_norm_bwd launch");
  };
#define PSA_BLOCK(RAGGED, RMS) (l.columns == 8 ? go(block_norm_bwd_kernel<XT, WT, RAGGED, RMS, 8>) \
                                : l.columns == kRingColumns ? go(block_norm_bwd_kernel<XT, WT, RAGGED, RMS, kRingColumns>) \
                                                            : go(block_norm_bwd_kernel<XT, WT, RAGGED, RMS, kWideColumns>))
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
