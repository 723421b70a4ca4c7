// psa_embed / psa_embed_bwd: token embedding and the gradient of its table,
//     y[t] = scale * table[id[t]],        dtable[v] = scale * sum over t with id[t] = v of dy[t].
// Both are bound by HBM: the forward writes T rows, the backward reads T rows and writes the table's V rows once, zeros
// included.  The backward's sums are fp32 and in an order that the ids and the sizes fix, whatever the order in which CTAs run: the
// tokens are sorted by id first (stably), a CTA adds a fixed run of the sorted tokens in their order, and an id whose tokens
// spread over several runs has the runs' sums added by eight warps, every eighth of them each, and those of the warps in order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "psa.h"
#include "psa_internal.h"
#include "psa_launch.cuh"
#include "psa_vector.cuh"

namespace psa {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// ---------------------------------------------------------------- forward
// A CTA writes `rows` consecutive tokens' rows, 16 bytes at a time: `windows` of them hold a row wherever it starts.
template <typename T, bool kRagged>
__global__ void __launch_bounds__(kThreads)
embed_kernel(const int32_t* ids, const T* table, int64_t n_tokens, int64_t vocab, int32_t hidden, int32_t windows, int32_t rows,
             float scale, T* out, int32_t* status) {
  constexpr int V = 16 / int(sizeof(T));
  const int64_t t0 = int64_t(blockIdx.x) * rows;
  const int n = int(min(int64_t(rows), n_tokens - t0)) * windows;
  behind_wait();
  behind_go();
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int r = i / windows, k = i - r * windows;
    const int64_t at = (t0 + r) * hidden;
    const int col = k * V - (kRagged ? int(at & (V - 1)) : 0);
    if (col >= hidden) continue;
    const int32_t id = ids[t0 + r];
    float v[V] = {};
    if (id >= 0 && id < vocab) {
      const int64_t from = int64_t(id) * hidden + col;
      Span<T, V, kRagged> in;
      in.load(table, from, vocab * hidden);
      in.at(from).get(v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] *= scale;
    } else if (k == 0 && status) {   // reported; the row is zeros
      atomicOr(status, PSA_DEVSTAT_BAD_TARGET);
    }
    store_window(out, at + col, v, -col, hidden - col);
  }
}

// ---------------------------------------------------------------- tokens sorted by id
// CTA b of a power of two owns the ids that leave b: frequent tokens often have neighbouring ids, and a CTA with a range of
// them would have most of the work.  Its 32 warps walk 32 consecutive parts of the tokens: once to count every id of theirs
// (a count per warp) and the tokens of the CTAs before, and, when the counts have become places, once more to put the
// tokens down.  Tokens are met in their order, so equal ids keep it.  Every CTA reads all ids (from L2),
// kAhead loads of a warp at a time (2, 4, 8 and 16: 35.5, 35.7, 36.6 and 39.2 us of the gradient of 2000 tokens of 32000 x 2047; 85, 83,
// 82 and 84 at 31041 of 50257 x 1002).
constexpr int kIndexThreads = 1024, kMaxBins = 1024, kAhead = 4;

__global__ void __launch_bounds__(kIndexThreads)
embed_index_kernel(const int32_t* ids, int32_t n_tokens, int32_t vocab, int32_t bins, int32_t* start, int32_t* count,
                   int32_t* order, int32_t* sorted_id, int32_t* status) {
  extern __shared__ int32_t counts[];     // [32][bins]
  __shared__ int32_t s_warp[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rest = blockIdx.x, mask = gridDim.x - 1, n_ids = uint32_t(vocab);
  const int log2_ctas = 31 - __clz(int(gridDim.x));
  const int share = ((n_tokens + 31) / 32 + 31) / 32 * 32;
  const int64_t first = int64_t(warp) * share;
  const int begin = int(min(first, int64_t(n_tokens))), end = int(min(first + share, int64_t(n_tokens)));
  int32_t* mine = counts + warp * bins;
  for (int i = threadIdx.x; i < 32 * bins; i += kIndexThreads) counts[i] = 0;
  behind_wait();
  behind_go();
  __syncthreads();

  // (ids as unsigned numbers: a negative one is larger than all others)
  int below = 0;
  bool bad = false;
  for (int t = begin; t < end; t += 32 * kAhead) {
    uint32_t id[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) id[k] = t + k * 32 + lane < end ? uint32_t(ids[t + k * 32 + lane]) : 0xffffffffu;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (id[k] >= n_ids) continue;
      below += (id[k] & mask) < rest;
      if ((id[k] & mask) == rest) atomicAdd(mine + (id[k] >> log2_ctas), 1);
    }
    if (blockIdx.x == 0)
#pragma unroll
      for (int k = 0; k < kAhead; ++k) bad |= t + k * 32 + lane < end && id[k] >= n_ids;
  }
  if (bad && status) atomicOr(status, PSA_DEVSTAT_BAD_TARGET);
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) s_warp[warp] = below;
  __syncthreads();
  below = __reduce_add_sync(0xffffffffu, s_warp[lane]);
  __syncthreads();

  // Thread i owns bin i: its tokens in all, the bins before it, then the warps before each warp.
  const int id = (int(threadIdx.x) << log2_ctas) + int(rest);
  const bool owner = int(threadIdx.x) < bins && id < vocab;
  int total = 0;
  if (owner)
    for (int w = 0; w < 32; ++w) total += counts[w * bins + threadIdx.x];
  int scan = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += v;
  }
  if (lane == 31) s_warp[warp] = scan;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += s_warp[w];
  int at = below + before + scan - total;
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == kIndexThreads - 1) start[vocab] = at + total;     // tokens with a good id
  if (owner) {
    start[id] = at;
    count[id] = total;
    for (int w = 0; w < 32; ++w) {
      const int c = counts[w * bins + threadIdx.x];
      counts[w * bins + threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();

  for (int t = begin; t < end; t += 32 * kAhead) {
    uint32_t v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = t + k * 32 + lane < end ? uint32_t(ids[t + k * 32 + lane]) : 0xffffffffu;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool here = v[k] < n_ids && (v[k] & mask) == rest;
      const unsigned any = __ballot_sync(0xffffffffu, here);
      if (!any) continue;
      const uint32_t bin = v[k] >> log2_ctas;
      int place = 0;
      unsigned same = 0;
      if (here) {
        same = __match_any_sync(any, bin);
        place = mine[bin] + __popc(same & ((1u << lane) - 1u));
      }
      __syncwarp();
      if (here) {
        if (lane == __ffs(same) - 1) mine[bin] += __popc(same);
        order[place] = t + k * 32 + lane;
        sorted_id[place] = int(v[k]);
      }
      __syncwarp();
    }
  }
}

// ---------------------------------------------------------------- sums
// blockIdx.x < n_runs: the sorted tokens [r * run, (r + 1) * run).  An id that lies within the run is written; the part of
// one that began in an earlier run goes to slot 0 of the run, of one that only goes on in the next run to slot 1.
// The other CTAs clear the rows of ids that do not occur (dense gradients only).  Where rows start anywhere and take several
// slices, neighbouring ones are cleared as one range: row by row, their ends made it 288 us instead of 194 at 4000 tokens of
// 128256 x 4095, while at one slice (50257 x 1002) rows took 81 and ranges 86.  (Clearing all rows beside the index took longer, 90
// there: here it fills the time in which the sums wait for their rows.)  blockIdx.y: a slice of the columns.
constexpr int kZeroRows = 16;

// A thread holds one window of V columns: of the row of the table that it adds to, so that what it writes is aligned.
template <typename XT, typename GT, bool kRagged>
__global__ void __launch_bounds__(kThreads)
embed_sum_kernel(const XT* d_out, const int32_t* start, const int32_t* count, const int32_t* order, const int32_t* sorted_id, int32_t run, int32_t n_runs,
                 int64_t n_tokens, int32_t vocab, int32_t hidden, int32_t windows, float scale, int32_t accumulate, GT* dtable,
                 float* partial) {
  constexpr int V = 16 / int(sizeof(XT)), W = 16 / int(sizeof(GT)), kUnroll = kRagged ? 4 : 8;     // rows in flight
  const int k = int(blockIdx.y) * int(blockDim.x) + int(threadIdx.x);
  const int lane = threadIdx.x & 31;
  behind_wait();
  behind_go();
  // The thread's first column in the row of id v (may be negative: elements of the row before).
  auto column = [&](int64_t v) { return k * V - (kRagged ? int(v * hidden & (W - 1)) : 0); };
  if (int(blockIdx.x) >= n_runs) {
    const int64_t v0 = (int64_t(blockIdx.x) - n_runs) * kZeroRows;
    const float zero[V] = {};
    if (!kRagged || gridDim.y == 1) {
      for (int r = 0; r < kZeroRows && v0 + r < vocab; ++r) {
        const int col = column(v0 + r);
        if (count[v0 + r] == 0 && col < hidden) store_window(dtable, (v0 + r) * hidden + col, zero, -col, hidden - col);
      }
      return;
    }
    unsigned absent = __ballot_sync(0xffffffffu, lane < kZeroRows && v0 + lane < vocab && count[v0 + lane] == 0);
    while (absent) {
      const int r = __ffs(absent) - 1, m = __ffs(~(absent >> r)) - 1;      // rows r to r + m - 1
      absent &= ~(((1u << m) - 1u) << r);
      const int64_t begin = (v0 + r) * hidden, end = begin + int64_t(m) * hidden;
      const int64_t low = min(end, (begin + W - 1) & ~int64_t(W - 1)), high = max(low, end & ~int64_t(W - 1));
      for (int64_t i = low + int64_t(k) * W; i < high; i += int64_t(gridDim.y) * blockDim.x * W)
        *reinterpret_cast<uint4*>(dtable + i) = make_uint4(0, 0, 0, 0);
      if (k < low - begin) set_element(dtable + begin + k, 0.f);
      if (k < end - high) set_element(dtable + high + k, 0.f);
    }
    return;
  }
  const int n_valid = start[vocab], first = int(blockIdx.x) * run, n = min(run, n_valid - first);
  if (n <= 0) return;
  // Lane l holds the run's l-th token and its id; `ends`: the next token's id is another one.
  const int mine = first + lane;
  const int pos = lane < n ? order[mine] : 0, id = lane < n ? sorted_id[mine] : -1;
  const unsigned ends = __ballot_sync(0xffffffffu, lane < n && (mine + 1 >= n_valid || sorted_id[mine + 1] != id));
  bool began_here = first == 0 || sorted_id[first - 1] != __shfl_sync(0xffffffffu, id, 0);
  float acc[V] = {};
  for (int e0 = 0; e0 < n; e0 += kUnroll) {
    Span<XT, V, kRagged> raw[kUnroll];
    int64_t from[kUnroll];
    int col[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      col[u] = column(__shfl_sync(0xffffffffu, id, (e0 + u) & 31));
      from[u] = int64_t(__shfl_sync(0xffffffffu, pos, (e0 + u) & 31)) * hidden + col[u];
      if (e0 + u < n && col[u] < hidden) raw[u].load(d_out, from[u], n_tokens * hidden);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int e = e0 + u;
      if (e >= n) break;
      const int64_t v = __shfl_sync(0xffffffffu, id, e);
      if (col[u] < hidden) {
        float x[V];
        raw[u].at(from[u]).get(x);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += x[j];
      }
      const bool end = ends >> e & 1u;
      if (!end && e + 1 < n) continue;
      if (k < windows && col[u] < hidden) {
        if (end && began_here) {
          const int64_t to = v * hidden + col[u];
          if (accumulate) {
            Span<GT, V, kRagged> old;
            float o[V];
            old.load(dtable, to, int64_t(vocab) * hidden);
            old.at(to).get(o);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = o[j] + scale * acc[j];
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] *= scale;
          }
          store_window(dtable, to, acc, -col[u], hidden - col[u]);
        } else {
          store_vec<float, V>(partial + ((int64_t(blockIdx.x) * 2 + (began_here ? 1 : 0)) * windows + k) * V, acc);
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] = 0.f;
      began_here = true;
    }
  }
}

// The ids that spread over several runs: the CTAs of the run in which one begins add the runs' sums, each warp every eighth of
// them, then the warps' sums in their order (one thread all of them one after the other: 17 us at 16215 tokens, of which
// the most frequent id has a twelfth).  A CTA holds 32 windows.
constexpr int kJoinWarps = 8;

template <typename GT, int V, bool kRagged>
__global__ void __launch_bounds__(32 * kJoinWarps)
embed_join_kernel(const int32_t* start, const int32_t* count, const int32_t* sorted_id, int32_t length, int32_t vocab, int32_t hidden, int32_t windows, float scale,
                  int32_t accumulate, const float* partial, GT* dtable) {
  constexpr int W = 16 / int(sizeof(GT));
  __shared__ float s_sum[kJoinWarps][V][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = int(blockIdx.y) * 32 + lane;
  const int run = blockIdx.x, last = run * length + length - 1;
  behind_wait();
  behind_go();
  if (last >= start[vocab]) return;
  const int id = sorted_id[last], from = start[id], to = from + count[id];
  if (from < run * length || to <= last + 1) return;
  const int64_t row = int64_t(id) * hidden;
  const int col = k * V - (kRagged ? int(row & (W - 1)) : 0), n = (to - 1) / length - run + 1;
  const bool live = k < windows && col < hidden;
  float acc[V] = {};
  if (live) {
#pragma unroll 4
    for (int r = warp; r < n; r += kJoinWarps) {      // the run that the id begins in has its sum in slot 1, the others in slot 0
      float v[V];
      load_vec<float, V>(partial + ((int64_t(run + r) * 2 + (r == 0 ? 1 : 0)) * windows + k) * V).get(v);
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += v[j];
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) s_sum[warp][j][lane] = acc[j];
  __syncthreads();
  if (warp != 0 || !live) return;
#pragma unroll
  for (int w = 1; w < kJoinWarps; ++w)
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += s_sum[w][j][lane];
  float old[V] = {};
  if (accumulate) {
    Span<GT, V, kRagged> in;
    in.load(dtable, row + col, int64_t(vocab) * hidden);
    in.at(row + col).get(old);
  }
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = old[j] + scale * acc[j];
  store_window(dtable, row + col, acc, -col, hidden - col);
}

// ---------------------------------------------------------------- host
constexpr int64_t kMaxVocab = 1 << 24, kMaxTokens = 1 << 24;
constexpr int kMaxEmbed = 1 << 20;

// Tokens of a run: a run's rows are read one batch behind the other, so shorter runs end sooner where there are few (16 and 32: 15.9
// and 20.5 us at 567 tokens x 94, 12.4 and 15.1 at 2192 x 56, 24.5 and 25.5 at 7965 x 1024), and cost more parts' sums where there
// are many (35.3 and 33.6 at 16215 x 1024, 89 and 82 at 31041 x 1002).
int run_length(int64_t T, int64_t hidden) { return T * hidden <= 1 << 23 ? 16 : 32; }

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

struct EmbedWorkspace {
  size_t start, count, order, sorted_id, partial, total;
};
EmbedWorkspace workspace_layout(int64_t T, int64_t vocab, int64_t hidden) {
  EmbedWorkspace w{};
  size_t at = aligned(size_t(vocab + 1) * 4);
  w.count = at;
  at += aligned(size_t(vocab) * 4);
  w.order = at;
  at += aligned(size_t(T) * 4);
  w.sorted_id = at;
  at += aligned(size_t(T) * 4);
  w.partial = at;
  w.total = at + size_t((T + run_length(T, hidden) - 1) / run_length(T, hidden)) * 2 * size_t(hidden / 8 + 2) * 8 * 4;
  return w;
}

psa_status_t check_sizes(int64_t n_tokens, int64_t vocab, int32_t hidden) {
  if (n_tokens < 0 || vocab <= 0 || hidden <= 0) return PSA_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens || vocab > kMaxVocab || hidden > kMaxEmbed) return PSA_ERR_UNSUPPORTED;
  return PSA_OK;
}
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Windows of V columns that a row reaches into; where its width is no multiple of V, it starts up to `align` - 1 elements into
// the first one.
int windows_of(int32_t hidden, int V, int align) { return hidden % V ? (hidden + align - 1 + V - 1) / V : hidden / V; }

template <typename T, bool kRagged>
psa_status_t embed_fwd(const int32_t* ids, const void* table, int64_t n_tokens, int64_t vocab, int32_t hidden, float scale,
                       void* out, int32_t* status, cudaStream_t stream) {
  constexpr int V = 16 / int(sizeof(T));
  const int windows = windows_of(hidden, V, V), rows = std::max(1, 2 * kThreads / windows);    // two loads a thread
  launch_behind(true, embed_kernel<T, kRagged>, dim3(unsigned((n_tokens + rows - 1) / rows)), kThreads, 0, stream, ids,
                static_cast<const T*>(table), n_tokens, vocab, hidden, windows, rows, scale, static_cast<T*>(out), status);
  return check_last_cuda_error("psa_embed launch");
}

template <typename XT, typename GT, bool kRagged>
psa_status_t embed_bwd(const void* d_out, const int32_t* ids, int64_t n_tokens, int64_t vocab, int32_t hidden, float scale,
                       int32_t accumulate, void* dtable, char* ws, int32_t* status, cudaStream_t stream) {
  constexpr int V = 16 / int(sizeof(XT));
  const EmbedWorkspace w = workspace_layout(n_tokens, vocab, hidden);
  auto ints = [&](size_t off) { return reinterpret_cast<int32_t*>(ws + off); };
  int ctas = 128;
  while (vocab > int64_t(ctas) * kMaxBins) ctas *= 2;
  const int bins = int((vocab + ctas - 1) / ctas);
  if (cudaFuncSetAttribute(embed_index_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * kMaxBins * 4) != cudaSuccess)
    return PSA_ERR_CUDA;
  // (The sums take token numbers and ids from the index, so nothing is launched behind a refused launch.)
  if (launch_behind(true, embed_index_kernel, dim3(unsigned(ctas)), kIndexThreads, size_t(32) * bins * 4, stream, ids,
                    int32_t(n_tokens), int32_t(vocab), bins, ints(w.start), ints(w.count), ints(w.order), ints(w.sorted_id),
                    status) != cudaSuccess)
    return failed_launch("psa_embed_bwd launch");
  const int run = run_length(n_tokens, hidden), n_runs = int((n_tokens + run - 1) / run);
  const int windows = windows_of(hidden, V, 16 / int(sizeof(GT)));
  const unsigned slices = unsigned((windows + kThreads - 1) / kThreads);
  const unsigned threads = unsigned((windows + int(slices) * 32 - 1) / (int(slices) * 32)) * 32;     // even slices of whole warps
  const unsigned zero = accumulate ? 0u : unsigned((vocab + kZeroRows - 1) / kZeroRows);
  float* partial = reinterpret_cast<float*>(ws + w.partial);
  if (n_runs + zero > 0 &&
      launch_behind(true, embed_sum_kernel<XT, GT, kRagged>, dim3(unsigned(n_runs) + zero, slices), threads, 0, stream,
                    static_cast<const XT*>(d_out), ints(w.start), ints(w.count), ints(w.order), ints(w.sorted_id), run, n_runs, n_tokens, int32_t(vocab),
                    hidden, windows, scale, accumulate, static_cast<GT*>(dtable), partial) != cudaSuccess)
    return failed_launch("psa_embed_bwd launch");
  if (n_runs > 1)
    launch_behind(true, embed_join_kernel<GT, V, kRagged>, dim3(unsigned(n_runs), unsigned((windows + 31) / 32)), 32 * kJoinWarps, 0, stream, ints(w.start),
                  ints(w.count), ints(w.sorted_id), run, int32_t(vocab), hidden, windows, scale, accumulate, partial, static_cast<GT*>(dtable));
  return check_last_cuda_error("psa_embed_bwd launch");
}

}  // namespace
}  // namespace psa

extern "C" psa_status_t psa_embed(const int32_t* token_ids, const void* table, int32_t dtype, int64_t n_tokens, int64_t vocab,
                                  int32_t hidden, float scale, void* out, int32_t* device_status, void* stream) {
  using namespace psa;
  const psa_status_t sizes = check_sizes(n_tokens, vocab, hidden);
  if (sizes != PSA_OK) return sizes;
  if (dtype != PSA_DTYPE_F32 && dtype != PSA_DTYPE_BF16) return PSA_ERR_INVALID_ARG;
  if (n_tokens == 0) return PSA_OK;
  if (!token_ids || !table || !out) return PSA_ERR_INVALID_ARG;
  if (misaligned(table, 16) || misaligned(out, 16) || misaligned(token_ids, 4)) return PSA_ERR_ALIGNMENT;
  cudaStream_t st = cudaStream_t(stream);
  const bool f32 = dtype == PSA_DTYPE_F32, ragged = hidden * (f32 ? 4 : 2) % 16 != 0;
  auto run = f32 ? (ragged ? embed_fwd<float, true> : embed_fwd<float, false>)
                 : (ragged ? embed_fwd<__nv_bfloat16, true> : embed_fwd<__nv_bfloat16, false>);
  return run(token_ids, table, n_tokens, vocab, hidden, scale, out, device_status, st);
}

extern "C" size_t psa_embed_bwd_workspace_bytes(int64_t n_tokens, int64_t vocab, int32_t hidden) {
  if (psa::check_sizes(n_tokens, vocab, hidden) != PSA_OK) return 0;
  return psa::workspace_layout(n_tokens, vocab, hidden).total;
}

extern "C" psa_status_t psa_embed_bwd(const void* d_out, const int32_t* token_ids, int32_t dtype, int32_t grad_dtype,
                                      int64_t n_tokens, int64_t vocab, int32_t hidden, float scale, int32_t accumulate,
                                      void* dtable, void* workspace, int32_t* device_status, void* stream) {
  using namespace psa;
  const psa_status_t sizes = check_sizes(n_tokens, vocab, hidden);
  if (sizes != PSA_OK) return sizes;
  const bool f32 = dtype == PSA_DTYPE_F32, bf16 = dtype == PSA_DTYPE_BF16;
  if (!(f32 && grad_dtype == PSA_DTYPE_F32) && !(bf16 && (grad_dtype == PSA_DTYPE_F32 || grad_dtype == PSA_DTYPE_BF16)))
    return PSA_ERR_INVALID_ARG;
  if (!dtable || !workspace || (n_tokens > 0 && (!d_out || !token_ids))) return PSA_ERR_INVALID_ARG;
  if (misaligned(d_out, 16) || misaligned(dtable, 16) || misaligned(workspace, 16) || misaligned(token_ids, 4)) return PSA_ERR_ALIGNMENT;
  char* ws = static_cast<char*>(workspace);
  cudaStream_t st = cudaStream_t(stream);
  const bool to_f32 = grad_dtype == PSA_DTYPE_F32, ragged = hidden * (f32 ? 4 : 2) % 16 != 0;
  auto run = f32      ? (ragged ? embed_bwd<float, float, true> : embed_bwd<float, float, false>)
             : to_f32 ? (ragged ? embed_bwd<__nv_bfloat16, float, true> : embed_bwd<__nv_bfloat16, float, false>)
                      : (ragged ? embed_bwd<__nv_bfloat16, __nv_bfloat16, true> : embed_bwd<__nv_bfloat16, __nv_bfloat16, false>);
  return run(d_out, token_ids, n_tokens, vocab, hidden, scale, accumulate, dtable, ws, device_status, st);
}
