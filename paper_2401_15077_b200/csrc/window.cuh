// What the two attention kernels with a window share (window.cu, window_rows.cu): fp16 operands, e4m3 codes, scales of blocks.
#pragma once
#include "chunk.cuh"
#include "tc.cuh"

namespace eagle {
namespace tc {

// Over codes the reference of the exponentials lies this much (log2 units) below the row's: probabilities then use the upper part of
// fp16's range (2^7 at the reference, 2^15 at the most before the accumulator is rescaled) and keep full precision down to 2^-21 of the largest
// one, steps of 2^-31 below.
constexpr float kHalfShift = 7.f;

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Four e4m3 codes as four fp16 numbers (exact).
__device__ __forceinline__ void half_of_codes(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(four));
}
__device__ __forceinline__ float fast_log2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float fast_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// What scores over codes are multiplied by: a block's scale times that of the softmax times what the row was divided by.  Masked scores are -infinity, so
// the product may not come out 0: the least normal number is added.  Factors from 2^-101 on do not change by it, and smaller ones leave scores of 2^-83
// at the most (the products are below 2^17).
__device__ __forceinline__ float score_factor(float a, float b) { return fmaf(a, b, 1.17549435e-38f); }

// Value scales that the arithmetic holds for: 2^-60 to 2^60, by their bits (NaN and negative numbers are outside).
__device__ __forceinline__ uint32_t beyond_range(float vs) { return __float_as_uint(vs) - (67u << 23); }
constexpr uint32_t kScaleRange = 120u << 23;

// Of a row whose largest |element| has the bits `top` (bf16, without the sign): 2^e with |element| < 2^(e + 1), and 2^-e by which the row is
// multiplied before it is rounded to fp16.  Rows of zeros and rows with infinities or NaN (whose output is NaN anyhow) stay as they are.
struct RowFactor {
  float up, down;
};
__device__ __forceinline__ RowFactor row_factor(uint32_t top) {
  const int e = static_cast<int>(top >> 7);
  if (top == 0 || e == 255) return {1.f, 1.f};
  const int k = min(max(e, 1), 253);                      // (2^-126 .. 2^126, both factors normal numbers)
  return {__uint_as_float(static_cast<uint32_t>(k) << 23), __uint_as_float(static_cast<uint32_t>(254 - k) << 23)};
}
// Largest magnitude of a word of two bf16 numbers, as bits.
__device__ __forceinline__ uint32_t magnitude_bits(uint32_t two) { return max(two & 0x7fffu, (two >> 16) & 0x7fffu); }
// A word of two bf16 numbers times `f`, as two fp16 numbers.
__device__ __forceinline__ uint32_t half_of_bf16(uint32_t two, float f) {
  return pack_half(__uint_as_float(two << 16) * f, __uint_as_float(two & 0xffff0000u) * f);
}

// A dense tensor of bytes [n2, n1, 128] read in boxes of b1 rows by `cols` columns (128 with the 128-byte swizzle, else without one).
inline bool map_codes_3d(CUtensorMap* map, const void* base, long long n1, long long n2, int cols, int b1, bool swizzled) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {128, static_cast<cuuint64_t>(n1), static_cast<cuuint64_t>(n2)};
  const cuuint64_t strides[2] = {128, static_cast<cuuint64_t>(n1) * 128};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(cols), static_cast<cuuint32_t>(b1), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace tc
}  // namespace eagle
