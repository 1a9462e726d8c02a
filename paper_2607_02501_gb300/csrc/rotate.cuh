// Cosine and sine of an angle held as two floats, and the frequencies of a rotary embedding as
// two floats each: shared by the rotary kernels.
#pragma once

#include <cmath>

#include "common.cuh"

namespace emb {

// (c, s) = (cos, sin)(A + a). a is a small correction (|a| < 2^-11, to first order: a^2 / 2 < 7e-8 up to
// 2^-12 + 2^-13), or with LARGE any float.
template <bool LARGE>
__device__ __forceinline__ void sincos_two_float(float A, float a, float& c, float& s) {
    float sA, cA;
    sincosf(A, &sA, &cA);
    if constexpr (LARGE) {
        // sine and cosine of a by their series (error below 1e-10 up to 1/16), then the addition formulas
        const float a2 = __fmul_rn(a, a);
        float sa = __fmul_rn(a, fmaf(a2, fmaf(a2, 1.0f / 120.0f, -1.0f / 6.0f), 1.0f));
        float ca = fmaf(a2, fmaf(a2, 1.0f / 24.0f, -0.5f), 1.0f);
        if (fabsf(a) > 0.0625f) sincosf(a, &sa, &ca);
        c = fmaf(cA, ca, -__fmul_rn(sA, sa));
        s = fmaf(sA, ca, __fmul_rn(cA, sa));
    } else {
        c = fmaf(-a, sA, cA);
        s = fmaf(a, cA, sA);
    }
}

// hi[i] + lo[i] = unit * base^(-2i/d) for i < d / 2, as the product of two powers, i = 16 j + k: at most 32 calls
// of pow instead of one per pair, within three roundings of fp64. d <= 512.
inline void rotary_frequencies(double base, int64_t d, float* hi, float* lo, double unit = 1.0) {
    double coarse[16], fine[16];
    const int half = int(d / 2);
    for (int j = 0; 16 * j < half; ++j) coarse[j] = std::pow(base, -32.0 * double(j) / double(d));
    for (int k = 0; k < 16 && k < half; ++k) fine[k] = std::pow(base, -2.0 * double(k) / double(d));
    for (int i = 0; i < half; ++i) {
        const double v = unit * (coarse[i >> 4] * fine[i & 15]);
        hi[i] = float(v);
        lo[i] = float(v - double(hi[i]));
    }
}

}  // namespace emb
