// psa_rotary: rotary position embedding of the queries and keys of a layer in one launch, in the forms that psa_rope does not
// have: pairs of neighbours or of halves, a part of the head, frequencies scaled for long contexts, bf16 or fp32, any strides.
// With pair i of a head (a, b) = (x[2i], x[2i + 1]) or (x[i], x[i + r/2]) and w_i its frequency,
//     a' = m (a cos(p w_i) - b sin(p w_i)),   b' = m (b cos(p w_i) + a sin(p w_i));
// the gradient is the same with -sin.
// Angles: a frequency is kept in turns per position as a 64-bit fixed-point fraction, so that its product with the position,
// taken modulo 2^64, is the fraction of a turn exactly, for any position (an fp32 product p w is off by 0.06 rad at 10^6).
// Bound by HBM.  A thread owns a few pairs of a token, computes their sines once and turns them in several heads, which it requests ahead
// of the sines (with loads behind them 68.5 us instead of 54 in the first of these).  Measured: 16215 x 40 heads of 128 bf16, views of one
// projection, 51.5 to 55 us (6.0 to 6.4 TB/s); 7965 x 15 heads of 80 fp32, 36 of them turned, 13.2 to 13.5 us (5.7 TB/s); one token 5.6 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "psa.h"
#include "psa_internal.h"
#include "psa_launch.cuh"

namespace psa {
namespace {

constexpr int kThreads = 256;
constexpr int kSmCount = 148;
constexpr int kMaxHeadDim = 1024;

struct Side {
  const void* x;
  void* y;
  int64_t x_token, x_head, y_token, y_head;      // strides in elements
  int32_t heads, groups;                         // groups of `each` heads
};
struct Args {
  Side side[2];
  const int32_t* position_ids;
  const unsigned long long* turns;
  int64_t n_tokens;
  int32_t head_dim, rotary_dim, each;
  int32_t copies;         // vectors behind the rotary part that are copied (0 in place)
  float magnitude;
  int32_t inverse;
};

// W elements as one load brings them.
template <typename T, int W>
struct alignas(W * sizeof(T)) Pack {
  static constexpr int kWords = W * int(sizeof(T)) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void get(float (&v)[W]) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) {
        v[i] = __uint_as_float(w[i]);
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&v)[W]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) {
        w[i] = __float_as_uint(v[i]);
      } else {
        const __nv_bfloat162 pair = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&pair);
      }
    }
  }
};
template <>
struct Pack<__nv_bfloat16, 1> {
  __nv_bfloat16 w;
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __bfloat162float(w); }
  __device__ __forceinline__ void set(const float (&v)[1]) { w = __float2bfloat16(v[0]); }
};

// W elements a load.  Half layout: a thread holds W pairs, one vector of each half; interleaved: W / 2 pairs in one vector.
// All of a thread's heads are requested ahead of the sines; threads whose vector is only copied go the same way.
template <bool kInterleaved>
__host__ __device__ constexpr int most_heads() { return kInterleaved ? 8 : 4; }      // of a thread

template <typename T, int W, bool kInterleaved>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const Args args) {
  using P = Pack<T, W>;
  constexpr int kPairs = kInterleaved ? W / 2 : W, kHeads = most_heads<kInterleaved>();
  const int turned = args.rotary_dim / 2 / kPairs, per_group = turned + args.copies;
  const int groups = args.side[0].groups + args.side[1].groups, per_token = groups * per_group;
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x, token = i / per_token;
  behind_wait();
  behind_go();
  if (token >= args.n_tokens) return;
  const int at = int(i - token * per_token), group = at / per_group, v = at - group * per_group;
  const bool second = group >= args.side[0].groups, turns = v < turned;
  const Side& side = args.side[second];
  const int head0 = (second ? group - args.side[0].groups : group) * args.each, heads = min(args.each, side.heads - head0);
  const int first = kInterleaved || turns ? v * W : args.rotary_dim + (v - turned) * W, half = args.rotary_dim / 2;
  const T* x = static_cast<const T*>(side.x) + token * side.x_token + head0 * side.x_head + first;
  T* y = static_cast<T*>(side.y) + token * side.y_token + head0 * side.y_head + first;
  P p[kHeads], q[kInterleaved ? 1 : kHeads];
  const long long position = args.position_ids[token];
#pragma unroll
  for (int h = 0; h < kHeads; ++h)
    if (h < heads) {
      p[h] = *reinterpret_cast<const P*>(x + h * side.x_head);
      if (!kInterleaved && turns) q[kInterleaved ? 0 : h] = *reinterpret_cast<const P*>(x + h * side.x_head + half);
    }
  float cs[kPairs], sn[kPairs];
  if (turns) {
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      const unsigned long long angle = static_cast<unsigned long long>(position) * args.turns[v * kPairs + j];
      // the signed top 32 bits: -1/2 to 1/2 of a turn
      sincospif(float(int32_t(angle >> 32)) * 4.656612873077393e-10f, &sn[j], &cs[j]);
      cs[j] *= args.magnitude;
      sn[j] *= args.inverse ? -args.magnitude : args.magnitude;
    }
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if (h >= heads) break;
    P* to = reinterpret_cast<P*>(y + h * side.y_head);
    if (!turns) {
      *to = p[h];
      continue;
    }
    float a[W], b[W], r[W];
    p[h].get(a);
    if (kInterleaved) {
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        r[2 * k] = a[2 * k] * cs[k] - a[2 * k + 1] * sn[k];
        r[2 * k + 1] = a[2 * k + 1] * cs[k] + a[2 * k] * sn[k];
      }
      p[h].set(r);
      *to = p[h];
    } else {
      P& second_half = q[kInterleaved ? 0 : h];
      second_half.get(b);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) r[k] = a[k] * cs[k] - b[k] * sn[k];
      p[h].set(r);
      *to = p[h];
#pragma unroll
      for (int k = 0; k < kPairs; ++k) r[k] = b[k] * cs[k] + a[k] * sn[k];
      second_half.set(r);
      *reinterpret_cast<P*>(y + h * side.y_head + half) = second_half;
    }
  }
}

// The most elements (16 bytes at most) that every vector of a head can be loaded by: its addresses, and the places of the
// halves and of the part that is not turned, are multiples of them.
int width_of(const Args& a, int elem_bytes, bool interleaved) {
  int64_t all = interleaved ? a.rotary_dim : a.rotary_dim / 2;      // (any common divisor's powers of two)
  if (a.copies) all |= a.head_dim - a.rotary_dim;
  for (const Side& s : a.side) {
    if (s.heads == 0) continue;
    for (const void* p : {s.x, static_cast<const void*>(s.y)}) all |= int64_t(reinterpret_cast<uintptr_t>(p)) / elem_bytes;
    if (a.n_tokens > 1) all |= s.x_token | s.y_token;
    if (s.heads > 1) all |= s.x_head | s.y_head;
  }
  const int64_t low = all & -all;
  return int(std::min<int64_t>(low ? low : 16, 16 / elem_bytes));
}

template <typename T, int W, bool kInterleaved>
psa_status_t launch(Args a, cudaStream_t stream) {
  if constexpr (kInterleaved && W == 1) {
    return PSA_ERR_ALIGNMENT;      // (pairs of neighbours are loaded together)
  } else {
    if (a.copies) a.copies = (a.head_dim - a.rotary_dim) / W;
    const int per_group = a.rotary_dim / 2 / (kInterleaved ? W / 2 : W) + a.copies;
    // Heads a thread: as many as leave 1024 threads for each SM
    a.each = most_heads<kInterleaved>();
    auto threads = [&] {
      int64_t groups = 0;
      for (Side& s : a.side) groups += s.groups = (s.heads + a.each - 1) / a.each;
      return a.n_tokens * groups * per_group;
    };
    while (a.each > 1 && threads() < int64_t(kSmCount) * 1024) a.each /= 2;
    const int64_t blocks = (threads() + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return PSA_ERR_UNSUPPORTED;
    launch_behind(true, rotary_kernel<T, W, kInterleaved>, dim3(unsigned(blocks)), kThreads, 0, stream, a);
    return check_last_cuda_error("psa_rotary launch");
  }
}
template <typename T, bool kInterleaved>
psa_status_t launch(const Args& a, cudaStream_t stream) {
  switch (width_of(a, int(sizeof(T)), kInterleaved)) {
    case 8:
      if constexpr (sizeof(T) == 2) return launch<T, 8, kInterleaved>(a, stream);
    case 4: return launch<T, 4, kInterleaved>(a, stream);
    case 2: return launch<T, 2, kInterleaved>(a, stream);
    default: return launch<T, 1, kInterleaved>(a, stream);
  }
}

}  // namespace
}  // namespace psa

extern "C" psa_status_t psa_rotary_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor, double original_length,
                                               double low, double high, int64_t* turns, float* magnitude) {
  const int32_t r = rotary_dim;
  if (r <= 0 || r % 2 || r > psa::kMaxHeadDim || !(theta > 1.0) || !std::isfinite(theta) || !turns || !magnitude) return PSA_ERR_INVALID_ARG;
  if (scaling < PSA_ROTARY_PLAIN || scaling > PSA_ROTARY_RAMP) return PSA_ERR_INVALID_ARG;
  if (scaling != PSA_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return PSA_ERR_INVALID_ARG;
  const bool by_length = scaling == PSA_ROTARY_WAVELENGTH || scaling == PSA_ROTARY_RAMP;
  if (by_length && (!(original_length >= 1.0) || !std::isfinite(original_length) || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
    return PSA_ERR_INVALID_ARG;
  if (scaling == PSA_ROTARY_BASE && r == 2) return PSA_ERR_INVALID_ARG;      // (its only pair keeps its frequency whatever the base)
  const double two_pi = 6.283185307179586476925286766559;
  if (scaling == PSA_ROTARY_BASE) theta *= std::pow(factor, double(r) / double(r - 2));
  double first = 0, last = 0;
  if (scaling == PSA_ROTARY_RAMP) {
    // the pair that turns so many times over the original length
    auto pair_of = [&](double times) { return r * std::log(original_length / (times * two_pi)) / (2 * std::log(theta)); };
    first = std::max(std::floor(pair_of(high)), 0.0);
    last = std::min(std::ceil(pair_of(low)), double(r - 1));
  }
  *magnitude = scaling == PSA_ROTARY_RAMP ? float(0.1 * std::log(factor) + 1.0) : 1.0f;
  for (int32_t i = 0; i < r / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / r);
    if (scaling == PSA_ROTARY_LINEAR) f /= factor;
    if (by_length) {
      const double times = original_length * f / two_pi;      // turns over the original length
      const double keep = scaling == PSA_ROTARY_WAVELENGTH ? (times - low) / (high - low) : 1.0 - (i - first) / std::max(last - first, 0.001);
      const double k = std::min(std::max(keep, 0.0), 1.0);
      f = f * k + f / factor * (1.0 - k);
    }
    turns[i] = static_cast<int64_t>(static_cast<uint64_t>(f / two_pi * 18446744073709551616.0 + 0.5));      // (f <= 1: below 2^62)
  }
  return PSA_OK;
}

extern "C" psa_status_t psa_rotary(const void* q, const void* k, void* q_out, void* k_out, const int32_t* position_ids,
                                   const int64_t* turns, int32_t dtype, int64_t n_tokens, int32_t n_q_heads, int32_t n_k_heads,
                                   int32_t head_dim, int32_t rotary_dim, const int64_t* strides, int32_t interleaved, int32_t inverse,
                                   float magnitude, void* stream) {
  if (n_tokens < 0 || n_q_heads <= 0 || n_k_heads < 0 || head_dim <= 0 || rotary_dim <= 0 || rotary_dim % 2 || rotary_dim > head_dim)
    return PSA_ERR_INVALID_ARG;
  if (dtype != PSA_DTYPE_F32 && dtype != PSA_DTYPE_BF16) return PSA_ERR_INVALID_ARG;
  if (head_dim > psa::kMaxHeadDim || n_tokens > 0x7fffffffLL || int64_t(n_q_heads) + n_k_heads > 65536) return PSA_ERR_UNSUPPORTED;
  if (n_tokens == 0) return PSA_OK;
  if (!q || !q_out || !position_ids || !turns || (n_k_heads > 0 && (!k || !k_out))) return PSA_ERR_INVALID_ARG;
  const int e = dtype == PSA_DTYPE_F32 ? 4 : 2;
  for (const void* p : {q, k, static_cast<const void*>(q_out), static_cast<const void*>(k_out)})
    if (reinterpret_cast<uintptr_t>(p) % e) return PSA_ERR_ALIGNMENT;
  psa::Args a{};
  auto side = [&](const void* x, void* y, int32_t heads, const int64_t* s) {
    const int64_t row = int64_t(heads) * head_dim;
    return s ? psa::Side{x, y, s[0], s[1], s[2], s[3], heads, 0} : psa::Side{x, y, row, head_dim, row, head_dim, heads, 0};
  };
  a.side[0] = side(q, q_out, n_q_heads, strides);
  a.side[1] = side(n_k_heads ? k : nullptr, n_k_heads ? k_out : nullptr, n_k_heads, strides ? strides + 4 : nullptr);
  a.position_ids = position_ids;
  a.turns = reinterpret_cast<const unsigned long long*>(turns);
  a.n_tokens = n_tokens;
  a.head_dim = head_dim;
  a.rotary_dim = rotary_dim;
  a.magnitude = magnitude;
  a.inverse = inverse;
  const bool in_place = q == q_out && (n_k_heads == 0 || k == k_out);
  a.copies = rotary_dim < head_dim && !in_place;
  cudaStream_t st = cudaStream_t(stream);
  if (dtype == PSA_DTYPE_F32) return interleaved ? psa::launch<float, true>(a, st) : psa::launch<float, false>(a, st);
  return interleaved ? psa::launch<__nv_bfloat16, true>(a, st) : psa::launch<__nv_bfloat16, false>(a, st);
}
