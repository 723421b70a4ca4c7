// psa_embed / psa_embed_bwd: token embedding and the gradient of its table,
//     y[t] = scale * table[id[t]],        dtable[v] = scale * sum over t with id[t] = v of dy[t].
// Both are bound by HBM: the forward writes T rows, the backward reads T rows and writes the table's V rows once, zeros
// included.  The backward's sums are fp32 and taken in the tokens' order, whatever the order in which CTAs run: the tokens are
// sorted by id first (stably), a CTA adds a fixed run of the sorted tokens, and an id whose tokens spread over several runs
// has the runs' sums added in their order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "psa.h"
#include "psa_internal.h"
#include "psa_vector.cuh"

namespace psa {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// ---------------------------------------------------------------- forward
// A CTA writes `rows` consecutive tokens' rows, V elements a load.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads)
embed_kernel(const int32_t* ids, const T* table, int64_t n_tokens, int64_t vocab, int32_t hidden, int32_t rows, float scale,
             T* out, int32_t* status) {
  const int64_t t0 = int64_t(blockIdx.x) * rows;
  const int n_vec = hidden / V, n = int(min(int64_t(rows), n_tokens - t0)) * n_vec;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int r = i / n_vec, c = (i - r * n_vec) * V;
    const int32_t id = ids[t0 + r];
    float v[V];
    if (id >= 0 && id < vocab) {
      load_vec<T, V>(table + int64_t(id) * hidden + c).get(v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] *= scale;
    } else {   // reported; the row is zeros
      if (c == 0 && status) atomicOr(status, PSA_DEVSTAT_BAD_TARGET);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = 0.f;
    }
    store_vec<T, V>(out + (t0 + r) * hidden + c, v);
  }
}

// ---------------------------------------------------------------- tokens sorted by id
// CTA b owns the ids of [b * bins, (b + 1) * bins).  Its 32 warps walk 32 consecutive parts of the tokens: once to count
// every bin (a count per warp) and the tokens of smaller ids, and, when the counts have become places, once more to put
// the tokens down.  Tokens are met in their order, so equal ids keep it.  Every CTA reads all ids (from L2).
constexpr int kIndexThreads = 1024, kMaxBins = 1024, kAhead = 8;

__global__ void __launch_bounds__(kIndexThreads)
embed_index_kernel(const int32_t* ids, int32_t n_tokens, int32_t vocab, int32_t bins, int32_t* start, int32_t* order,
                   int32_t* sorted_id, int32_t* status) {
  extern __shared__ int32_t counts[];     // [32][bins]
  __shared__ int32_t s_warp[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lo = int(blockIdx.x) * bins, n_bins = min(bins, vocab - lo);
  const int share = ((n_tokens + 31) / 32 + 31) / 32 * 32;
  const int64_t first = int64_t(warp) * share;
  const int begin = int(min(first, int64_t(n_tokens))), end = int(min(first + share, int64_t(n_tokens)));
  int32_t* mine = counts + warp * bins;
  for (int i = threadIdx.x; i < 32 * bins; i += kIndexThreads) counts[i] = 0;
  __syncthreads();

  int below = 0;
  bool bad = false;
  for (int t = begin; t < end; t += 32 * kAhead) {
    int32_t id[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) id[k] = t + k * 32 + lane < end ? ids[t + k * 32 + lane] : vocab;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (t + k * 32 + lane < end) bad |= id[k] < 0 || id[k] >= vocab;
      if (id[k] < 0 || id[k] >= lo + n_bins) continue;
      if (id[k] < lo) ++below;
      else atomicAdd(mine + (id[k] - lo), 1);
    }
  }
  if (bad && blockIdx.x == 0 && status) atomicOr(status, PSA_DEVSTAT_BAD_TARGET);
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) s_warp[warp] = below;
  __syncthreads();
  below = __reduce_add_sync(0xffffffffu, s_warp[lane]);
  __syncthreads();

  // Thread i owns bin i: its tokens in all, the bins before it, then the warps before each warp.
  int total = 0;
  if (threadIdx.x < n_bins)
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
  if (threadIdx.x < n_bins) {
    start[lo + threadIdx.x] = at;
    if (lo + int(threadIdx.x) == vocab - 1) start[vocab] = at + total;
    for (int w = 0; w < 32; ++w) {
      const int c = counts[w * bins + threadIdx.x];
      counts[w * bins + threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();

  for (int t = begin; t < end; t += 32 * kAhead) {
    int32_t id[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) id[k] = t + k * 32 + lane < end ? ids[t + k * 32 + lane] : vocab;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool here = id[k] >= lo && id[k] < lo + n_bins;
      const unsigned any = __ballot_sync(0xffffffffu, here);
      if (!any) continue;
      int place = 0;
      unsigned same = 0;
      if (here) {
        same = __match_any_sync(any, id[k]);
        place = mine[id[k] - lo] + __popc(same & ((1u << lane) - 1u));
      }
      __syncwarp();
      if (here) {
        if (lane == __ffs(same) - 1) mine[id[k] - lo] += __popc(same);
        order[place] = t + k * 32 + lane;
        sorted_id[place] = id[k];
      }
      __syncwarp();
    }
  }
}

// ---------------------------------------------------------------- sums
// blockIdx.x < n_runs: the sorted tokens [r * kRun, (r + 1) * kRun).  An id that lies within the run is written; the part of
// one that began in an earlier run goes to slot 0 of the run, of one that only goes on in the next run to slot 1.
// The other CTAs write the rows of ids that do not occur (dense gradients only).  blockIdx.y: a slice of the columns.
constexpr int kRun = 32, kZeroRows = 16, kUnroll = 4;

template <typename XT, typename GT, int V>
__global__ void __launch_bounds__(kThreads)
embed_sum_kernel(const XT* d_out, const int32_t* start, const int32_t* order, const int32_t* sorted_id, int32_t n_runs,
                 int32_t vocab, int32_t hidden, float scale, int32_t accumulate, GT* dtable, float* partial) {
  const int col = (int(blockIdx.y) * kThreads + int(threadIdx.x)) * V;
  if (int(blockIdx.x) >= n_runs) {
    if (col >= hidden) return;
    const int64_t v0 = (int64_t(blockIdx.x) - n_runs) * kZeroRows;
    float zero[V] = {};
    for (int k = 0; k < kZeroRows && v0 + k < vocab; ++k)
      if (start[v0 + k] == start[v0 + k + 1]) store_vec<GT, V>(dtable + (v0 + k) * hidden + col, zero);
    return;
  }
  __shared__ int32_t s_pos[kRun], s_id[kRun + 2];     // s_id: one before, the run, one after
  const int n_valid = start[vocab], first = int(blockIdx.x) * kRun, n = min(kRun, n_valid - first);
  if (n <= 0) return;
  if (threadIdx.x < kRun + 2) {
    const int i = first + int(threadIdx.x) - 1;
    s_id[threadIdx.x] = i >= 0 && i < n_valid ? sorted_id[i] : -1;
  }
  if (int(threadIdx.x) < n) s_pos[threadIdx.x] = order[first + threadIdx.x];
  __syncthreads();
  if (col >= hidden) return;
  float acc[V] = {};
  bool began_here = s_id[0] != s_id[1];
  for (int e0 = 0; e0 < n; e0 += kUnroll) {
    Vec<XT, V> raw[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
      if (e0 + k < n) raw[k] = load_vec<XT, V>(d_out + int64_t(s_pos[e0 + k]) * hidden + col);
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int e = e0 + k;
      if (e >= n) break;
      float x[V];
      raw[k].get(x);
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += x[j];
      const int id = s_id[e + 1];
      const bool ends = s_id[e + 2] != id;
      if (!ends && e + 1 < n) continue;
      if (ends && began_here) {
        GT* row = dtable + int64_t(id) * hidden + col;
        float old[V] = {};
        if (accumulate) load_vec<GT, V>(row).get(old);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = old[j] + scale * acc[j];
        store_vec<GT, V>(row, acc);
      } else {
        float* p = partial + (int64_t(blockIdx.x) * 2 + (began_here ? 1 : 0)) * hidden + col;
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = acc[j];
      }
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] = 0.f;
      began_here = true;
    }
  }
}

// The ids that spread over several runs: the CTA of the run in which one begins adds the runs' sums in their order.
template <typename GT, int V>
__global__ void __launch_bounds__(kThreads)
embed_join_kernel(const int32_t* start, const int32_t* sorted_id, int32_t vocab, int32_t hidden, float scale, int32_t accumulate,
                  const float* partial, GT* dtable) {
  const int col = (int(blockIdx.y) * kThreads + int(threadIdx.x)) * V;
  const int run = blockIdx.x, last = run * kRun + kRun - 1;
  if (last >= start[vocab]) return;
  const int id = sorted_id[last], from = start[id], to = start[id + 1];
  if (from < run * kRun || to <= last + 1 || col >= hidden) return;
  const int last_run = (to - 1) / kRun;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = partial[(int64_t(run) * 2 + 1) * hidden + col + j];
#pragma unroll 8
  for (int r = run + 1; r <= last_run; ++r)
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += partial[int64_t(r) * 2 * hidden + col + j];
  GT* row = dtable + int64_t(id) * hidden + col;
  float old[V] = {};
  if (accumulate) load_vec<GT, V>(row).get(old);
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = old[j] + scale * acc[j];
  store_vec<GT, V>(row, acc);
}

// ---------------------------------------------------------------- host
constexpr int64_t kMaxVocab = 1 << 24, kMaxTokens = 1 << 24;
constexpr int kMaxEmbed = 1 << 20;

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

struct EmbedWorkspace {
  size_t start, order, sorted_id, partial, total;
};
EmbedWorkspace workspace_layout(int64_t T, int64_t vocab, int64_t hidden) {
  EmbedWorkspace w{};
  size_t at = aligned(size_t(vocab + 1) * 4);
  w.order = at;
  at += aligned(size_t(T) * 4);
  w.sorted_id = at;
  at += aligned(size_t(T) * 4);
  w.partial = at;
  w.total = at + size_t((T + kRun - 1) / kRun) * 2 * size_t(hidden) * 4;
  return w;
}

psa_status_t check_sizes(int64_t n_tokens, int64_t vocab, int32_t hidden) {
  if (n_tokens < 0 || vocab <= 0 || hidden <= 0) return PSA_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens || vocab > kMaxVocab || hidden > kMaxEmbed) return PSA_ERR_UNSUPPORTED;
  return PSA_OK;
}
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

template <typename T, int V>
psa_status_t embed_fwd(const int32_t* ids, const void* table, int64_t n_tokens, int64_t vocab, int32_t hidden, float scale,
                       void* out, int32_t* status, cudaStream_t stream) {
  const int rows = std::max(1, 2 * kThreads / (hidden / V));    // two loads a thread
  embed_kernel<T, V><<<unsigned((n_tokens + rows - 1) / rows), kThreads, 0, stream>>>(
      ids, static_cast<const T*>(table), n_tokens, vocab, hidden, rows, scale, static_cast<T*>(out), status);
  return check_last_cuda_error("psa_embed launch");
}

template <typename XT, typename GT, int V>
psa_status_t embed_bwd(const void* d_out, const int32_t* ids, int64_t n_tokens, int64_t vocab, int32_t hidden, float scale,
                       int32_t accumulate, void* dtable, char* ws, int32_t* status, cudaStream_t stream) {
  const EmbedWorkspace w = workspace_layout(n_tokens, vocab, hidden);
  auto ints = [&](size_t off) { return reinterpret_cast<int32_t*>(ws + off); };
  // A range of ids per SM, of at least 32 and at most kMaxBins ids.
  const int bins = int(std::min<int64_t>(kMaxBins, std::max<int64_t>(32, (vocab + 147) / 148)));
  const int smem = 32 * bins * 4;
  if (cudaFuncSetAttribute(embed_index_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * kMaxBins * 4) != cudaSuccess)
    return PSA_ERR_CUDA;
  embed_index_kernel<<<unsigned((vocab + bins - 1) / bins), kIndexThreads, smem, stream>>>(
      ids, int32_t(n_tokens), int32_t(vocab), bins, ints(w.start), ints(w.order), ints(w.sorted_id), status);
  const int n_runs = int((n_tokens + kRun - 1) / kRun);
  const unsigned slices = unsigned((hidden + kThreads * V - 1) / (kThreads * V));
  const unsigned zero = accumulate ? 0u : unsigned((vocab + kZeroRows - 1) / kZeroRows);
  float* partial = reinterpret_cast<float*>(ws + w.partial);
  if (n_runs + zero > 0)
    embed_sum_kernel<XT, GT, V><<<dim3(unsigned(n_runs) + zero, slices), kThreads, 0, stream>>>(
        static_cast<const XT*>(d_out), ints(w.start), ints(w.order), ints(w.sorted_id), n_runs, int32_t(vocab), hidden, scale,
        accumulate, static_cast<GT*>(dtable), partial);
  if (n_runs > 1)
    embed_join_kernel<GT, V><<<dim3(unsigned(n_runs), slices), kThreads, 0, stream>>>(
        ints(w.start), ints(w.sorted_id), int32_t(vocab), hidden, scale, accumulate, partial, static_cast<GT*>(dtable));
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
  if (dtype == PSA_DTYPE_F32) {
    if (hidden % 4 == 0) return embed_fwd<float, 4>(token_ids, table, n_tokens, vocab, hidden, scale, out, device_status, st);
    if (hidden % 2 == 0) return embed_fwd<float, 2>(token_ids, table, n_tokens, vocab, hidden, scale, out, device_status, st);
    return embed_fwd<float, 1>(token_ids, table, n_tokens, vocab, hidden, scale, out, device_status, st);
  }
  if (hidden % 8 == 0) return embed_fwd<__nv_bfloat16, 8>(token_ids, table, n_tokens, vocab, hidden, scale, out, device_status, st);
  if (hidden % 2 == 0) return embed_fwd<__nv_bfloat16, 2>(token_ids, table, n_tokens, vocab, hidden, scale, out, device_status, st);
  return embed_fwd<__nv_bfloat16, 1>(token_ids, table, n_tokens, vocab, hidden, scale, out, device_status, st);
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
#define PSA_EMBED_BWD(XT, GT, V) embed_bwd<XT, GT, V>(d_out, token_ids, n_tokens, vocab, hidden, scale, accumulate, dtable, ws, device_status, st)
  if (f32) return hidden % 4 == 0 ? PSA_EMBED_BWD(float, float, 4) : hidden % 2 == 0 ? PSA_EMBED_BWD(float, float, 2) : PSA_EMBED_BWD(float, float, 1);
  if (grad_dtype == PSA_DTYPE_F32)
    return hidden % 8 == 0 ? PSA_EMBED_BWD(__nv_bfloat16, float, 8) : hidden % 2 == 0 ? PSA_EMBED_BWD(__nv_bfloat16, float, 2) : PSA_EMBED_BWD(__nv_bfloat16, float, 1);
  return hidden % 8 == 0 ? PSA_EMBED_BWD(__nv_bfloat16, __nv_bfloat16, 8) : hidden % 2 == 0 ? PSA_EMBED_BWD(__nv_bfloat16, __nv_bfloat16, 2) : PSA_EMBED_BWD(__nv_bfloat16, __nv_bfloat16, 1);
#undef PSA_EMBED_BWD
}
