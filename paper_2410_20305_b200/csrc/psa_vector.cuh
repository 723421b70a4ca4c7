// Loads and stores of V neighbouring elements as fp32, for kernels that stream rows: 16 bytes at a time where rows allow it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

namespace psa {
namespace dev {

template <typename T, int V>
struct Vec;   // .raw: what one load brings;  V elements

template <>
struct Vec<__nv_bfloat16, 8> {
  uint4 raw;
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    raw = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void clear() { raw = make_uint4(0, 0, 0, 0); }
};
template <>
struct Vec<float, 8> {
  float4 raw[2];
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = raw[0].x; v[1] = raw[0].y; v[2] = raw[0].z; v[3] = raw[0].w;
    v[4] = raw[1].x; v[5] = raw[1].y; v[6] = raw[1].z; v[7] = raw[1].w;
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    raw[0] = make_float4(v[0], v[1], v[2], v[3]);
    raw[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
  __device__ __forceinline__ void clear() { raw[0] = raw[1] = make_float4(0.f, 0.f, 0.f, 0.f); }
};
template <>
struct Vec<float, 4> {
  float4 raw;
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = raw.x; v[1] = raw.y; v[2] = raw.z; v[3] = raw.w; }
  __device__ __forceinline__ void set(const float (&v)[4]) { raw = make_float4(v[0], v[1], v[2], v[3]); }
  __device__ __forceinline__ void clear() { raw = make_float4(0.f, 0.f, 0.f, 0.f); }
};
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T* p) { return *reinterpret_cast<const Vec<T, V>*>(p); }
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
  Vec<T, V> w;
  w.set(v);
  *reinterpret_cast<Vec<T, V>*>(p) = w;
}

__device__ __forceinline__ void set_element(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }
__device__ __forceinline__ void set_element(float* p, float v) { *p = v; }

// ---------------------------------------------------------------- rows of any width
// Rows of `width` elements lie one behind the other from a 16-byte boundary on: where width is no multiple of 16 bytes, a row
// starts anywhere.  A thread then writes one of the aligned vectors (`windows`) that the row reaches into, of which the first
// and the last may hold elements of the rows beside it, and shifts what it needs at other places (weights, other rows) into
// line with it.
//
// Elements [k, k + V) of the 2 V elements (lo, hi), V = 16 bytes of them, 0 <= k <= V; `k` is the same for all threads of a row.
template <int kBytes>   // of an element
__device__ __forceinline__ uint4 shift_pair(const uint4& lo, const uint4& hi, int k) {
  uint32_t w[9] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w, 0u};
  const int words = k * kBytes / 4;
  if (words & 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = w[i + 4];
  }
  if (words & 2) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (words & 1) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  if (kBytes == 2 && (k & 1)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One window: the aligned vector at element `first`, elements behind the tensor's end as zeros.
template <typename T>
__device__ __forceinline__ uint4 load_window(const T* p, int64_t first, int64_t all) {
  constexpr int W = 16 / int(sizeof(T));
  if (first + W <= all) return *reinterpret_cast<const uint4*>(p + first);
  T v[W];
#pragma unroll
  for (int j = 0; j < W; ++j) v[j] = first + j < all ? p[first + j] : T(0.f);
  uint4 r;
  memcpy(&r, v, 16);
  return r;
}

// V elements (a multiple of 16 bytes) from element `first` on of a tensor of `all` elements; those outside it read as zeros.
// kAny: from any element on, of which some may lie outside; else from a multiple of V within the tensor.
template <typename T, int V, bool kAny>
struct Span {
  static constexpr int W = 16 / int(sizeof(T)), P = V / W;
  uint4 r[kAny ? P + 1 : P];
  __device__ __forceinline__ void load(const T* p, int64_t first, int64_t all) {
    if (!kAny) {
#pragma unroll
      for (int k = 0; k < P; ++k) r[k] = *reinterpret_cast<const uint4*>(p + first + k * W);
      return;
    }
    const int64_t q = first & ~int64_t(W - 1);
#pragma unroll
    for (int k = 0; k <= P; ++k) {
      const int64_t at = q + k * W;
      r[kAny ? k : 0] = at < 0 || at >= all ? make_uint4(0, 0, 0, 0) : load_window(p, at, all);
    }
  }
  __device__ __forceinline__ Vec<T, V> at(int64_t first) const {
    uint4 w[P];
#pragma unroll
    for (int k = 0; k < P; ++k) w[k] = kAny ? shift_pair<int(sizeof(T))>(r[k], r[kAny ? k + 1 : 0], int(first & (W - 1))) : r[k];
    Vec<T, V> v;
    memcpy(&v, w, sizeof(w));
    return v;
  }
};
// Writes the elements [lo, hi) of V (a multiple of 16 bytes) that start at the aligned element `first`.
template <typename T, int V>
__device__ __forceinline__ void store_window(T* p, int64_t first, const float (&f)[V], int lo, int hi) {
  if (lo <= 0 && hi >= V) {
    store_vec<T, V>(p + first, f);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= lo && j < hi) set_element(p + first + j, f[j]);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace dev
}  // namespace psa
