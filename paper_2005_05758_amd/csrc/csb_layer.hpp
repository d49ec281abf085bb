// What the kernels around a recurrent layer share (convolution, scan, norms): runs of eight elements of any type and alignment, and
// the functions of gates.
#pragma once

#include "csb_lm.hpp"

namespace csb {

#ifdef __HIPCC__
// A vector at the address of any element.  (By a copy: an alignment given to a vector type's alias in its declaration is not taken up, and of an address
// that is the same for all lanes the scalar unit then reads whole words, the low bits left out.)
template <typename V, typename T> __device__ __forceinline__ V load_any(const T *p) {
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <typename V, typename T> __device__ __forceinline__ void store_any(T *p, const V &v) { __builtin_memcpy(p, &v, sizeof(V)); }

// Eight elements from p[0] on, of which the first `there` are (the others are zeros, or are not stored); p at any element.
template <int VF> struct Run8 {
    using T = typename Elem<VF>::T;
    using T8 = T __attribute__((ext_vector_type(8)));
    T8 v;
    __device__ __forceinline__ void load(const T *p, int there) {
        if (there >= 8) v = load_any<T8>(p);
        else {
            v = T8{};
#pragma unroll
            for (int j = 0; j < 7; ++j) if (j < there) v[j] = p[j];
        }
    }
    __device__ __forceinline__ float operator[](int j) const { return (float)v[j]; }
    __device__ __forceinline__ void set(int j, float x) { v[j] = (T)x; }
    __device__ __forceinline__ void store(T *p, int there) const {
        if (there >= 8) store_any(p, v);
        else {
#pragma unroll
            for (int j = 0; j < 7; ++j) if (j < there) p[j] = v[j];
        }
    }
};

// e^x for x in [-104, 88], nearer ends taken for others (NaN too), to 2 units of 2^-24: the product with log2 e in two parts, as its rounding alone
// would be |x| units off.
__device__ __forceinline__ float exp_within(float x) {
    x = __builtin_amdgcn_fmed3f(x, -104.0f, 88.0f);
    const float p = x * 1.44269502162933349609375f;            // log2 e as the sum of two numbers
    const float rest = fmaf(x, 1.44269502162933349609375f, -p) + x * 1.925963033500011079e-08f;
    const float e = __builtin_amdgcn_exp2f(p);
    return fmaf(e, rest * 0.693147182464599609375f, e);
}
// 1 / (1 + e^-x), as e^x / (1 + e^x) below zero: it goes to zero there, so that the product with any finite x does.  (NaN gives a
// number: callers multiply by x, or look for it.)
__device__ __forceinline__ float sigmoid_within(float x) {
    const float e = exp_within(-fabsf(x));
    return (x < 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e);
}
// The same for results that are rounded to 16 bits: the argument of the exponential rounded once, 1.3 |x| units of 2^-24 off (2^-12 of a result's rounding for |x| up to 8),
// half as many instructions.
template <int VF> __device__ __forceinline__ float sigmoid_for(float x) {
    if constexpr (VF == CSB_VAL_F32) return sigmoid_within(x);
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269502162933349609375f));
}
template <int VF> __device__ __forceinline__ float silu(float x) { return x * sigmoid_for<VF>(x); }

// ln(1 + e^x) = max(x, 0) + ln(1 + e), e = e^-|x| in (0, 1]: 2 atanh(s), s = e / (2 + e), as 2 s (1 + w p(w)), w = s^2 <= 1/9, p through five of Chebyshev's points
// (2^-29): small steps keep all of their digits, which ln(1 + e) of a rounded sum would not.  From 16 bits the argument of the
// exponential is rounded once, 17 instructions' time instead of 24: 1.25 |x| units of 2^-24 of the result more (x below zero), a 2^12th and less of what the rounding of a 16-bit
// number as large as x makes.  States, which are binary32, keep that.
template <int VF> __device__ __forceinline__ float softplus_from(float x) {
    constexpr bool SHORT = VF != CSB_VAL_F32;
    const float e = SHORT ? __builtin_amdgcn_exp2f(fabsf(x) * -1.44269502162933349609375f) : exp_within(-fabsf(x));
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), w = s * s;
    float p = 0.11612164974212646f;
    p = fmaf(p, w, 0.1085328757762909f);
    p = fmaf(p, w, 0.142961785197258f);
    p = fmaf(p, w, 0.19999852776527405f);
    p = fmaf(p, w, 0.3333333432674408f);
    const float l = fmaf(s + s, w * p, s + s), y = fmaxf(x, 0.0f) + l;
    return SHORT || x == x ? y : x;                            // (without limits of the exponential's argument NaN stays)
}
#endif

}  // namespace csb
