// Operands of the scan's products on the matrix cores.
//
// The matrix cores multiply bfloat16.  Operands that are wider are split into bfloat16 parts whose sum holds 8, 16 or 24
// bits, and the products of parts that matter are added up in 32 bits: bfloat16 inputs are exact in one part, float16 in two,
// float32 takes three, and so does what is computed on the way (states, scores), whatever the type: 24 bits, 2^-25 of a term.
// The matrix cores round their sums downwards, by some 2e-8 of a result; sums over a whole text of what has been multiplied by
// values that are mostly positive collect that.  So what goes into such sums is computed with odd channels negated, from
// their rows in LDS on: an error of either sign for every other channel, and nothing to pay but a sign.
//
// With g = lane / 16, a lane holds rows 4g..4g+3 of one column of a 16 x 16 result, and eight inner indexes of one row (or column)
// of an operand: any eight, as long as both operands hold the same.  They are 4g..4g+3 of each of two tiles of 16, so that two
// results stacked are an operand as they stand.
#ifndef SEMICRF_SSM_OPS_H
#define SEMICRF_SSM_OPS_H

#include "ssm.h"

namespace semicrf_enc {

typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

template <class T> struct Parts;  // of an input
template <> struct Parts<__bf16> { static constexpr int raw = 1; };
template <> struct Parts<_Float16> { static constexpr int raw = 2; };
template <> struct Parts<float> { static constexpr int raw = 3; };
constexpr int HELD = 3;           // of what is computed on the way

template <int n> struct Op { bf8 p[n]; };

// Two floats rounded to bfloat16 (to nearest even), the first in the lower half.
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t round2(float a, float b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    uint32_t o = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){a, b}, bf2));
    asm("" : "+v"(o));  // one conversion for the pair: without this each value is rounded again for its remainder
    return o;
}
// What rounding took from them: a product of the pair with (-1, 0), and with (0, -1), added to the value, which is exact and one
// instruction where widening and subtracting are two.  The factors come as registers: as literals they are read wrongly.
__device__ __forceinline__ void remainder2(uint32_t rounded, float &a, float &b)
{
    uint32_t first = 0x0000bf80u, second = 0xbf800000u;
    asm("" : "+s"(first), "+s"(second));
    const bf2 p = __builtin_bit_cast(bf2, rounded);
    a = __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf2, first), a, false);
    b = __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf2, second), b, false);
}

// n parts of 2 m values: v = p[0] + p[1] + ..
template <int n, int m> __device__ __forceinline__ void split_pairs(float (&v)[2 * m], uint32_t (&o)[n][m])
{
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
        for (int k = 0; k < m; ++k) {
            o[i][k] = round2(v[2 * k], v[2 * k + 1]);
            if (i + 1 < n) remainder2(o[i][k], v[2 * k], v[2 * k + 1]);
        }
}

template <int n> __device__ __forceinline__ Op<n> split(f8 v)
{
    float a[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    uint32_t p[n][4];
    split_pairs<n, 4>(a, p);
    Op<n> o;
#pragma unroll
    for (int i = 0; i < n; ++i) o.p[i] = __builtin_bit_cast(bf8, (u4){p[i][0], p[i][1], p[i][2], p[i][3]});
    return o;
}

// Of the products of parts those that matter: the rest is below what the operands' last parts have lost.  Two inputs of two parts
// each are multiplied out, which is exact.
template <int na, int nb> __device__ __forceinline__ f4 mma(f4 acc, const Op<na> &a, const Op<nb> &b)
{
    constexpr int most = na > nb ? na : nb;
#pragma unroll
    for (int i = na - 1; i >= 0; --i)
#pragma unroll
        for (int j = nb - 1; j >= 0; --j)
            if (i + j < most) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[j], acc, 0, 0, 0);
    return acc;
}
template <int n> __device__ __forceinline__ f4 mma_inputs(f4 acc, const Op<n> &a, const Op<n> &b)
{
    if constexpr (n == 2) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[1], b.p[1], acc, 0, 0, 0);
    return mma(acc, a, b);
}

}  // namespace semicrf_enc

#endif
