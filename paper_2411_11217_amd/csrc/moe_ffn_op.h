// The kinds of operands that the expert-FFN kernels and the linear map multiply, as a template argument.  Both MFMAs take 16 bytes of a
// row per lane, chunk lane / 16 of 64 bytes, and add up a 16 x 16 tile in four registers in the same number of cycles: a row of n bytes
// is n / 2 bf16 or n 8-bit integers, and tiles, pages, LDS images, loads and loops, which count in bytes, are the same for both.
#pragma once

#include <hip/hip_runtime.h>

namespace moe {

typedef int i32x4 __attribute__((ext_vector_type(4)));        // an MFMA operand: 16 bytes of a row
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kHalfTileBytes = 128 * 64;                     // half of a page tile's k: 32 bf16 or 64 integers of each row
constexpr int kTileBytes = 2 * kHalfTileBytes;

struct Bf16 {                                                 // v_mfma_f32_16x16x32_bf16: sums in float32
    static constexpr bool kScaled = false;
    typedef f32x4 Acc;
    typedef float Out;                                        // of a down product
    __device__ static __forceinline__ Acc mfma(const i32x4& a, const i32x4& b, const Acc& c) {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

// v_mfma_i32_16x16x64_i8: whole numbers, exact as long as 128 * 128 * k stays below 2^31 (the host refuses longer rows).  A sum becomes a float
// once, at the end, times its column's and its row's scale.
template <class OutT>
struct Int8 {
    static constexpr bool kScaled = true;
    typedef i32x4 Acc;
    typedef OutT Out;
    __device__ static __forceinline__ Acc mfma(const i32x4& a, const i32x4& b, const Acc& c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

}  // namespace moe
