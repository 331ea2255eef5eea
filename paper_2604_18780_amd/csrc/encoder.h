// Shared by the encoder operators (embedding, short convolution, state space scan): storage types of activations,
// argument checks and the lengths rule.
#ifndef SEMICRF_ENCODER_H
#define SEMICRF_ENCODER_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "semicrf.h"

namespace semicrf_enc {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// Elements of a type in the 16 bytes a lane loads at once.
template <class T> constexpr int PER16 = 16 / (int)sizeof(T);

// n consecutive elements from / to memory that is aligned to their size, as float.  Narrowing rounds to nearest even.
template <class T, int n> __device__ __forceinline__ void load_n(const T *p, float (&o)[n])
{
    typedef T V __attribute__((ext_vector_type(n)));
    const V v = *(const V *)p;
#pragma unroll
    for (int e = 0; e < n; ++e) o[e] = (float)v[e];
}

template <class T, int n> __device__ __forceinline__ void store_n(T *p, const float (&o)[n])
{
    typedef T V __attribute__((ext_vector_type(n)));
    typedef float F __attribute__((ext_vector_type(n)));
    F f;
#pragma unroll
    for (int e = 0; e < n; ++e) f[e] = o[e];
    *(V *)p = __builtin_convertvector(f, V);
}

__device__ __forceinline__ int length_of(const int32_t *lengths, int b, int T)
{
    if (!lengths) return T;
    const int L = lengths[b];
    return L < 0 ? 0 : (L > T ? T : L);
}

// e^v to the rounding of its result (the hardware's power of two, with the rounding of its argument made good).
__device__ __forceinline__ float exp_of(float v)
{
    const float h = v * 1.44269504f, l = __builtin_fmaf(v, 1.44269504f, -h) + v * 1.92596299e-8f;
    const float e = __builtin_amdgcn_exp2f(h);
    return __builtin_fmaf(e, l * 0.693147181f, e);
}

// e^-|v|, no less than e^-100; not a number where v is none (a maximum would lose that).
__device__ __forceinline__ float exp_down(float v)
{
    const float a = -fabsf(v);
    return exp_of(a < -100.0f ? -100.0f : a);
}

// ln(1 + e^v) without overflow, and its derivative.  With e = e^-|v| and s = e / (2 + e) <= 1/3, ln(1 + e) = 2 artanh(s), of which
// seven terms hold 2^-26; the hardware's logarithm loses digits where 1 + e is near 1.
__device__ __forceinline__ float softplus(float v)
{
    const float e = exp_down(v), d = 2.0f + e;
    const float r = __builtin_amdgcn_rcpf(d), q = e * r, s = __builtin_fmaf(__builtin_fmaf(-q, d, e), r, q), z = s * s;
    float p = __builtin_fmaf(z, 1.0f / 13.0f, 1.0f / 11.0f);
    p = __builtin_fmaf(p, z, 1.0f / 9.0f);
    p = __builtin_fmaf(p, z, 1.0f / 7.0f);
    p = __builtin_fmaf(p, z, 0.2f);
    p = __builtin_fmaf(p, z, 1.0f / 3.0f);
    p = __builtin_fmaf(p * z, s, s);
    return __builtin_fmaf(2.0f, p, fmaxf(v, 0.0f));
}
__device__ __forceinline__ float sigmoid(float v)
{
    const float e = exp_down(v);
    return (v < 0.0f ? e : 1.0f) / (1.0f + e);
}

enum ActType { ACT_F32 = 0, ACT_F16 = 1, ACT_BF16 = 2 };

// The storage type a call's flags name, or -1 where they name two.
inline int act_type(unsigned flags)
{
    const unsigned t = flags & (SEMICRF_EMIS_F16 | SEMICRF_EMIS_BF16);
    return t == 0 ? ACT_F32 : t == SEMICRF_EMIS_F16 ? ACT_F16 : t == SEMICRF_EMIS_BF16 ? ACT_BF16 : -1;
}
inline int act_bytes(int type) { return type == ACT_F32 ? 4 : 2; }

// Rows that are read 16 bytes at a time: base and stride on a 16-byte boundary, at least `width` elements apart, and so little that
// 64 of them are within a 32-bit offset.
inline bool rows_ok(const void *p, int64_t row, int64_t width, int type)
{
    return p && ((uintptr_t)p & 15) == 0 && row >= width && row <= (1 << 22) && row * act_bytes(type) % 16 == 0;
}

inline int launched() { return hipGetLastError() == hipSuccess ? SEMICRF_OK : SEMICRF_ELAUNCH; }

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace semicrf_enc

#endif
