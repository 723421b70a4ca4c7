// Operands of products C[M, N] = sum over K of A B with bf16 operands that tcgen05.mma reads from 128-byte-swizzled tiles of
// shared memory: how they lie in memory, and the copies that bring them.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "psa_device.cuh"
#include "psa_tensormap.h"

namespace psa {

constexpr int kBK = 64;                // K per stage: one 128-byte swizzle row of bf16
constexpr int kChunk = 64;             // columns of an MN-major sub-tile
constexpr uint32_t kSub = kChunk * kBK * 2;

// An operand in memory: rows x cols, cols innermost.  MN-major (cols along M or N): `flat` brings 64 columns of 64 rows,
// `pair` 128 columns of 64 rows in one copy (two copies of half the size cost 10 % of a large product's time), as long as
// they lie within the last whole 64 columns.  K-major: `flat` brings 64 columns of 128 rows.
struct OperandMaps {
  CUtensorMap flat, pair;
};

// The 128 rows of A, or columns of B, that a CTA loads for a tile.
struct Strip {
  const OperandMaps* m;
  int mn0, way;         // way: 0 K-major, 1 MN-major in one copy, 2 in two
  __device__ __forceinline__ Strip(const OperandMaps* maps, bool mn_major, int at, int end)
      : m(maps), mn0(at), way(mn_major ? (at + 2 * kChunk <= end ? 1 : 2) : 0) {}
  template <typename Load>
  __device__ __forceinline__ void load(int which, int k0, uint32_t dst, Load&& load) const {
    if (way == 2) {
      load(dst, &m[which].flat, mn0, 0, k0);
      load(dst + kSub, &m[which].flat, mn0 + kChunk, 0, k0);
    } else {
      const bool pair = way == 1;
      load(dst, pair ? &m[which].pair : &m[which].flat, pair ? 0 : k0, pair ? k0 : 0, pair ? mn0 / kChunk : mn0);
    }
  }
};

namespace dev {
// Eight fp32 values as 16 bytes of bf16.
__device__ __forceinline__ uint4 pack8(const float* v) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
}  // namespace dev

// ---------------------------------------------------------------- host
inline bool encode(CUtensorMap* m, const void* p, cuuint64_t d0, cuuint64_t d1, cuuint64_t d2, cuuint64_t s1, cuuint64_t s2,
                   cuuint32_t b0, cuuint32_t b1, cuuint32_t b2, CUtensorMapSwizzle swizzle,
                   CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16) {
  EncodeTiledFn fn = encode_tiled_fn();
  const cuuint64_t dims[3] = {d0, d1, d2}, strides[2] = {s1, s2};
  const cuuint32_t box[3] = {b0, b1, b2}, step[3] = {1, 1, 1};
  return fn && fn(m, type, 3, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Boxes of `box_rows` x `box_cols` of a row-major matrix whose rows lie `pitch` elements apart (0: cols); coordinates
// (column, 0, row).
inline bool matrix_map(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int box_rows, int box_cols = kBK, int64_t pitch = 0) {
  const cuuint64_t bytes = cuuint64_t(pitch ? pitch : cols) * 2;
  return encode(m, p, cols, 1, rows, bytes, bytes, box_cols, 1, box_rows,
                box_cols == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B);
}
// Boxes of two times 64 columns of 64 rows, the second behind the first; coordinates (0, row, column / 64).
inline bool pair_map(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int64_t pitch = 0) {
  return encode(m, p, kChunk, rows, cols / kChunk, (pitch ? pitch : cols) * 2, kChunk * 2, kChunk, kBK, 2, CU_TENSOR_MAP_SWIZZLE_128B);
}
inline bool operand_maps(OperandMaps* o, const void* p, bool mn_major, int64_t mn, int64_t k, int rows, int64_t pitch = 0) {
  if (!mn_major) return matrix_map(&o->flat, p, mn, k, rows, kBK, pitch);
  return matrix_map(&o->flat, p, k, mn, kBK, kBK, pitch) && (mn < 2 * kChunk || pair_map(&o->pair, p, k, mn, pitch));
}

}  // namespace psa
