// Shared by the kernels for products with 4-bit weights: parameters, and how codes and tokens become operands.
//
// A code c under zeros is a 16-bit floating-point number with 5 exponent bits: c * 2^-24, one of its subnormal numbers, and
// four bits higher up it is c * 2^-20, of equal spacing still.  So a word of 8 codes becomes four operand registers of two
// codes each by one shift and four ANDs, without any offset that would have to be taken out of the sums again.
// The tokens' values meet them in the same type: multiplied by the power of two that brings the largest of their group to
// 2^14 .. 2^15, where codes stand higher (every second column) by 2^-4 of it, so that it is at 2^10 at least.  A value keeps its
// 8 (bf16) or 11 bits as long as the last of them is 2^-24, the smallest number, or more: down to 2^-27 or 2^-24 of the largest
// (2^-31 and 2^-28 in the other columns).  Below, it is off by 2^-25, 2^-35 of the largest (2^-39), at most.  Products are exact, sums binary32.
#pragma once

#include "stom_internal.cuh"
#include "stom_kv.cuh"
#include "stom_w4.h"

#include <type_traits>

namespace stom {

struct W4Params {
    const uint8_t *codes;
    const void *scale, *zero;
    int32_t n, k, groups, meta_dtype;
    int64_t code_stride, meta_stride;
    const void *x;
    int64_t x_stride;
    const void *bias, *add;
    int64_t add_stride;
    void *y;
    int64_t y_stride;
    int32_t tokens;
    uint32_t *flags;
};

#ifdef __CUDACC__

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

// Of the largest magnitude of a group (the bits of a 16-bit number without its sign): what its values are multiplied by,
// and what sums of products with codes are multiplied by, less the factor kCodeUnit.  A largest value that is none (infinite,
// or none at all): not a number.
constexpr float kCodeUnit = 4096.f;   // 2^24 is shared between this factor and the rows' scales, so that neither overflows
template <typename T>
__device__ __forceinline__ void factors_of(uint32_t top_bits, float &before, float &after) {
    float top, unused;
    unpack2<T>(top_bits, top, unused);
    const int e = (int)(__float_as_uint(top) >> 23);                 // biased exponent
    const int m = min(253, 127 + 14 - (e - 127));                    // of 2^(14 - exponent)
    before = __uint_as_float((uint32_t)max(m, 1) << 23);
    after = e == 255 ? __uint_as_float(0x7fffffffu) : __uint_as_float((uint32_t)(254 - m + 12) << 23);
}

// Eight values of adjacent columns as operands, in pairs four columns apart, as the codes of a word
template <typename T>
__device__ __forceinline__ uint4 token_operand(const uint4 &v, float before) {
    float a[8];
    unpack2<T>(v.x, a[0], a[1]);
    unpack2<T>(v.y, a[2], a[3]);
    unpack2<T>(v.z, a[4], a[5]);
    unpack2<T>(v.w, a[6], a[7]);
    const float higher = before * 0.0625f;
    return make_uint4(pack2<__half>(a[0] * before, a[4] * before), pack2<__half>(a[1] * higher, a[5] * higher),
                      pack2<__half>(a[2] * before, a[6] * before), pack2<__half>(a[3] * higher, a[7] * higher));
}

#endif  // __CUDACC__

// Many tokens (stom_w4_many.cu)
template <typename T>
cudaError_t w4_many(const W4Params &p, int group, int sms, void *workspace, cudaStream_t s);
int64_t w4_many_workspace(int32_t k, int32_t group, int32_t tokens);

}  // namespace stom
