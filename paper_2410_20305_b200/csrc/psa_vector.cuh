// Loads and stores of V neighbouring elements as fp32, for kernels that stream rows: 16 bytes at a time where rows allow it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

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
struct Vec<__nv_bfloat16, 2> {
  uint32_t raw;
  __device__ __forceinline__ void get(float (&v)[2]) const { v[0] = __uint_as_float(raw << 16); v[1] = __uint_as_float(raw & 0xffff0000u); }
  __device__ __forceinline__ void set(const float (&v)[2]) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(v[0], v[1]);
    raw = *reinterpret_cast<const uint32_t*>(&p);
  }
  __device__ __forceinline__ void clear() { raw = 0; }
};
template <>
struct Vec<__nv_bfloat16, 1> {
  __nv_bfloat16 raw;
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __bfloat162float(raw); }
  __device__ __forceinline__ void set(const float (&v)[1]) { raw = __float2bfloat16(v[0]); }
  __device__ __forceinline__ void clear() { raw = __float2bfloat16(0.f); }
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
template <>
struct Vec<float, 2> {
  float2 raw;
  __device__ __forceinline__ void get(float (&v)[2]) const { v[0] = raw.x; v[1] = raw.y; }
  __device__ __forceinline__ void set(const float (&v)[2]) { raw = make_float2(v[0], v[1]); }
  __device__ __forceinline__ void clear() { raw = make_float2(0.f, 0.f); }
};
template <>
struct Vec<float, 1> {
  float raw;
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = raw; }
  __device__ __forceinline__ void set(const float (&v)[1]) { raw = v[0]; }
  __device__ __forceinline__ void clear() { raw = 0.f; }
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T* p) { return *reinterpret_cast<const Vec<T, V>*>(p); }
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
  Vec<T, V> w;
  w.set(v);
  *reinterpret_cast<Vec<T, V>*>(p) = w;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace dev
}  // namespace psa
