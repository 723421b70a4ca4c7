// psa_norm / psa_norm_bwd: normalisation of each token's row, with the residual add in front of it:
//     s = x + residual (rounded to x's type; s = x without one),
//     m = mean(s) (0 in the RMS form),  r = 1 / sqrt(mean((s - m)^2) + eps),  y = (s - m) * r * w + b,
// and its gradient, with u = (s - m) * r and g = dy * w:
//     ds = r * (g - u * mean(g u) - mean(g)) + d_total      (no mean(g) in the RMS form),
//     dw = sum over tokens of dy * u,   db = sum over tokens of dy.
// Bound by HBM: a row is read once into registers, its sums are taken from there (the variance after the mean, so a row far
// from 0 loses nothing), and it is written once.  Sums are fp32.
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

constexpr int kSmCount = 148;
constexpr int kMaxHidden = 16384;
constexpr int kRowsPerCta = 8;      // rows of a CTA where a warp holds a row

// The most threads that divide() below gives a CTA, for the compiler's share of registers.
template <int V, int NV, bool kWarp>
constexpr int max_threads() {
  return kWarp ? 32 * kRowsPerCta : V == 1 ? 1024 : NV < 4 ? 256 : kMaxHidden / (V * NV);
}

// Sum over the threads that share a row: a warp (kWarp) or the CTA.  `slot` alternates, so that one barrier is enough.
template <bool kWarp, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*s_part)[32], int slot) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  if (kWarp) return;
  const int lane = threadIdx.x & 31, n_warps = blockDim.x >> 5;
  if (lane == 0)
    for (int i = 0; i < N; ++i) s_part[slot * 2 + i][threadIdx.x >> 5] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < n_warps ? s_part[slot * 2 + i][lane] : 0.f);
}

template <typename XT, typename WT, int V, int NV, bool kWarp>
__global__ void __launch_bounds__(max_threads<V, NV, kWarp>())
norm_kernel(const XT* x, const XT* residual, const WT* weight, const WT* bias, int64_t n_tokens, int32_t hidden, float eps,
            int32_t rms, XT* out, XT* total, float* stats) {
  __shared__ float s_part[4][32];
  const int group = kWarp ? 32 : int(blockDim.x), tid = kWarp ? int(threadIdx.x) & 31 : int(threadIdx.x);
  const int64_t row = kWarp ? int64_t(blockIdx.x) * kRowsPerCta + (threadIdx.x >> 5) : int64_t(blockIdx.x);
  if (kWarp && row >= n_tokens) return;
  const int64_t at = row * hidden;
  float s[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V;
    if (col < hidden) {
      load_vec<XT, V>(x + at + col).get(s[i]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) s[i][j] = 0.f;
    }
  }
  if (residual) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V;
      if (col >= hidden) continue;
      float r[V];
      load_vec<XT, V>(residual + at + col).get(r);
#pragma unroll
      for (int j = 0; j < V; ++j) s[i][j] += r[j];
      Vec<XT, V> w;     // what is normalised is what the residual stream holds
      w.set(s[i]);
      *reinterpret_cast<Vec<XT, V>*>(total + at + col) = w;
      w.get(s[i]);
    }
  }
  float mean = 0.f;
  if (!rms) {
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += s[i][j];
    row_sum<kWarp>(sum, s_part, 0);
    mean = sum[0] / float(hidden);
  }
  float sq[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if ((i * group + tid) * V >= hidden) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) sq[0] += (s[i][j] - mean) * (s[i][j] - mean);
  }
  row_sum<kWarp>(sq, s_part, 1);
  const float rstd = 1.0f / sqrtf(sq[0] / float(hidden) + eps);
  if (tid == 0) {
    stats[row] = mean;
    stats[n_tokens + row] = rstd;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V;
    if (col >= hidden) continue;
    float w[V], b[V], y[V];
    load_vec<WT, V>(weight + col).get(w);
    if (bias) load_vec<WT, V>(bias + col).get(b);
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = (s[i][j] - mean) * rstd * w[j] + (bias ? b[j] : 0.f);
    store_vec<XT, V>(out + at + col, y);
  }
}

// A CTA takes every gridDim.x-th row (or set of rows); a thread keeps its columns, and their parts of dw and db, throughout.
// partial: [gridDim.x][2][hidden].
template <typename XT, typename WT, int V, int NV, bool kWarp>
__global__ void __launch_bounds__(max_threads<V, NV, kWarp>())
norm_bwd_kernel(const XT* d_out, const XT* x, const WT* weight, const float* stats, const XT* d_total, int64_t n_tokens,
                int32_t hidden, int32_t rms, XT* dx, float* partial) {
  __shared__ float s_part[4][32];
  extern __shared__ float s_sum[];    // [2][hidden], kWarp only
  const int group = kWarp ? 32 : int(blockDim.x), tid = kWarp ? int(threadIdx.x) & 31 : int(threadIdx.x);
  const int rows = kWarp ? kRowsPerCta : 1, mine = kWarp ? int(threadIdx.x) >> 5 : 0;
  float dw[NV][V], db[NV][V], w[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * group + tid) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) dw[i][j] = db[i][j] = w[i][j] = 0.f;
    if (col < hidden) load_vec<WT, V>(weight + col).get(w[i]);
  }
  const float inv = 1.0f / float(hidden);
  int slot = 0;
  for (int64_t row = int64_t(blockIdx.x) * rows + mine; row < n_tokens; row += int64_t(gridDim.x) * rows, slot ^= 1) {
    const int64_t at = row * hidden;
    const float mean = stats[row], rstd = stats[n_tokens + row];
    float u[NV][V], g[NV][V], sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V;
      if (col < hidden) {
        load_vec<XT, V>(x + at + col).get(u[i]);
        load_vec<XT, V>(d_out + at + col).get(g[i]);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) { u[i][j] = mean; g[i][j] = 0.f; }
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        u[i][j] = (u[i][j] - mean) * rstd;
        dw[i][j] += g[i][j] * u[i][j];
        db[i][j] += g[i][j];
        g[i][j] *= w[i][j];
        sum[0] += g[i][j] * u[i][j];
        sum[1] += g[i][j];
      }
    row_sum<kWarp>(sum, s_part, slot);
    const float c_u = sum[0] * inv, c_1 = rms ? 0.f : sum[1] * inv;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V;
      if (col >= hidden) continue;
      float d[V];
#pragma unroll
      for (int j = 0; j < V; ++j) d[j] = (g[i][j] - u[i][j] * c_u - c_1) * rstd;
      if (d_total) {
        float t[V];
        load_vec<XT, V>(d_total + at + col).get(t);
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] += t[j];
      }
      store_vec<XT, V>(dx + at + col, d);
    }
  }
  float* mine_dw = partial + int64_t(blockIdx.x) * 2 * hidden;
  if (kWarp) {   // the rows of a CTA are added in their order
    for (int k = 0; k < kRowsPerCta; ++k) {
      if (k == mine) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int col = (i * group + tid) * V;
          if (col >= hidden) continue;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            s_sum[col + j] = (k ? s_sum[col + j] : 0.f) + dw[i][j];
            s_sum[hidden + col + j] = (k ? s_sum[hidden + col + j] : 0.f) + db[i][j];
          }
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * hidden; c += blockDim.x) mine_dw[c] = s_sum[c];
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * group + tid) * V;
      if (col >= hidden) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        mine_dw[col + j] = dw[i][j];
        mine_dw[hidden + col + j] = db[i][j];
      }
    }
  }
}

// dw (blockIdx.y = 0) and db (1): the parts of all CTAs, added in a fixed order.
constexpr int kSumRows = 16;
template <typename WT>
__global__ void __launch_bounds__(32 * kSumRows)
norm_sum_kernel(const float* partial, int32_t n_parts, int32_t hidden, WT* dweight, WT* dbias) {
  __shared__ float s[kSumRows][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (col < hidden)
    for (int p = part; p < n_parts; p += kSumRows) v += partial[(int64_t(p) * 2 + blockIdx.y) * hidden + col];
  s[part][lane] = v;
  __syncthreads();
  if (part == 0 && col < hidden) {
    for (int p = 1; p < kSumRows; ++p) v += s[p][lane];
    const float one[1] = {v};
    store_vec<WT, 1>((blockIdx.y ? dbias : dweight) + col, one);
  }
}

// How a row is divided: V elements a load, NV loads a thread, `threads` of them (32: a warp).
struct Division {
  int v, nv, threads;
};
Division divide(int32_t hidden, int elem_bytes) {
  const int v = 16 / elem_bytes;
  if (hidden % v == 0) {
    const int n = hidden / v;
    if (n <= 128) return {v, n <= 32 ? 1 : n <= 64 ? 2 : 4, 32};
    const int nv = n <= 256 ? 1 : n <= 512 ? 2 : 4;
    return {v, nv, ((n + nv - 1) / nv + 31) / 32 * 32};
  }
  if (hidden <= 128) return {1, 4, 32};
  const int nv = hidden <= 4096 ? 4 : 16;
  return {1, nv, ((hidden + nv - 1) / nv + 31) / 32 * 32};
}

int64_t part_count(int64_t n_tokens, int32_t hidden) {
  const int64_t most = hidden > 4096 ? kSmCount : 2 * kSmCount;
  return std::max<int64_t>(1, std::min(most, n_tokens));
}

template <typename F>
psa_status_t with_division(const Division& d, int elem_bytes, F&& f) {
  const bool warp = d.threads == 32;
  const int v = d.v == 1 ? 1 : 16 / elem_bytes;
  if (v != 1) {
    if (warp) return d.nv == 1 ? f.template run<0, 1, true>() : d.nv == 2 ? f.template run<0, 2, true>() : f.template run<0, 4, true>();
    return d.nv == 1 ? f.template run<0, 1, false>() : d.nv == 2 ? f.template run<0, 2, false>() : f.template run<0, 4, false>();
  }
  if (warp) return f.template run<1, 4, true>();
  return d.nv == 4 ? f.template run<1, 4, false>() : f.template run<1, 16, false>();
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
  template <int kScalar, int NV, bool kWarp>
  psa_status_t run() {
    constexpr int V = kScalar ? 1 : 16 / int(sizeof(XT));
    const int64_t grid = kWarp ? (n_tokens + kRowsPerCta - 1) / kRowsPerCta : n_tokens;
    norm_kernel<XT, WT, V, NV, kWarp><<<unsigned(grid), kWarp ? 32 * kRowsPerCta : threads, 0, stream>>>(
        static_cast<const XT*>(x), static_cast<const XT*>(residual), static_cast<const WT*>(weight), static_cast<const WT*>(bias),
        n_tokens, hidden, eps, rms, static_cast<XT*>(out), static_cast<XT*>(total), stats);
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
  int threads;
  cudaStream_t stream;
  template <int kScalar, int NV, bool kWarp>
  psa_status_t run() {
    constexpr int V = kScalar ? 1 : 16 / int(sizeof(XT));
    const int rows = kWarp ? kRowsPerCta : 1;
    const int64_t parts = std::min(part_count(n_tokens, hidden), std::max<int64_t>(1, (n_tokens + rows - 1) / rows));
    norm_bwd_kernel<XT, WT, V, NV, kWarp><<<unsigned(parts), kWarp ? 32 * kRowsPerCta : threads, kWarp ? 8 * hidden : 0, stream>>>(
        static_cast<const XT*>(d_out), static_cast<const XT*>(x), static_cast<const WT*>(weight), stats,
        static_cast<const XT*>(d_total), n_tokens, hidden, rms, static_cast<XT*>(dx), partial);
    norm_sum_kernel<WT><<<dim3(unsigned((hidden + 31) / 32), dbias ? 2 : 1), 32 * kSumRows, 0, stream>>>(
        partial, int32_t(parts), hidden, static_cast<WT*>(dweight), static_cast<WT*>(dbias));
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
    return with_division(d, e, Forward<float, float>{x, residual, weight, bias, n_tokens, hidden, eps, rms, out, total, stats, d.threads, st});
  if (weight_dtype == PSA_DTYPE_F32)
    return with_division(d, e, Forward<__nv_bfloat16, float>{x, residual, weight, bias, n_tokens, hidden, eps, rms, out, total, stats, d.threads, st});
  return with_division(d, e, Forward<__nv_bfloat16, __nv_bfloat16>{x, residual, weight, bias, n_tokens, hidden, eps, rms, out, total, stats, d.threads, st});
}

extern "C" size_t psa_norm_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden) {
  if (n_tokens < 0 || hidden <= 0 || hidden > psa::kMaxHidden) return 0;
  return size_t(psa::part_count(n_tokens, hidden)) * 2 * size_t(hidden) * 4;
}

extern "C" psa_status_t psa_norm_bwd(const void* d_out, const void* x, const void* weight, const float* stats,
                                     const void* d_total, int32_t dtype, int32_t weight_dtype, int64_t n_tokens, int32_t hidden,
                                     int32_t rms, void* dx, void* dweight, void* dbias, void* workspace, void* stream) {
  using namespace psa;
  const psa_status_t sizes = check_sizes(n_tokens, hidden, dtype, weight_dtype);
  if (sizes != PSA_OK) return sizes;
  if (!weight || !dweight || !workspace || (rms && dbias)) return PSA_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!d_out || !x || !stats || !dx)) return PSA_ERR_INVALID_ARG;
  for (const void* p : {d_out, x, weight, static_cast<const void*>(stats), d_total, static_cast<const void*>(dx),
                        static_cast<const void*>(dweight), static_cast<const void*>(dbias), static_cast<const void*>(workspace)})
    if (misaligned(p, 16)) return PSA_ERR_ALIGNMENT;
  const int e = dtype == PSA_DTYPE_F32 ? 4 : 2;
  const Division d = divide(hidden, e);
  cudaStream_t st = cudaStream_t(stream);
  float* part = static_cast<float*>(workspace);
  if (dtype == PSA_DTYPE_F32)
    return with_division(d, e, Backward<float, float>{d_out, x, weight, stats, d_total, n_tokens, hidden, rms, dx, dweight, dbias, part, d.threads, st});
  if (weight_dtype == PSA_DTYPE_F32)
    return with_division(d, e, Backward<__nv_bfloat16, float>{d_out, x, weight, stats, d_total, n_tokens, hidden, rms, dx, dweight, dbias, part, d.threads, st});
  return with_division(d, e, Backward<__nv_bfloat16, __nv_bfloat16>{d_out, x, weight, stats, d_total, n_tokens, hidden, rms, dx, dweight, dbias, part, d.threads, st});
}
