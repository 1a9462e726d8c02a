// Declarations and the code arithmetic shared by the translation units of the 8-bit paged cache (not installed).
#pragma once

#include <cuda_fp16.h>

#include "paged_math.cuh"

namespace emb {

constexpr int kBlock8 = 16;      // places of a page that share an exponent
constexpr int kExpMost = 48;     // exponents are -48 .. 48
constexpr int kExpBias = 127;    // of the stored byte
constexpr float kCodeMost = 448.0f;

struct Store8Args {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const float* q_gamma;
    const float* k_gamma;
    const int32_t* positions;
    const uint8_t* axis_of_pair;
    const uint64_t* turns;
    const int64_t* slots;
    uint16_t* q_out;
    uint8_t* k_codes;
    uint8_t* v_codes;
    uint8_t* k_exp;
    uint8_t* v_exp;
    int64_t q_stride, k_stride, v_stride, pos_stride, n_tokens, n_slots;
    int n_heads, n_kv_heads, head_dim, rot_dim, n_axes;
    float eps, factor;
    bool neighbours;
};
cudaError_t launch_paged8_store(const Store8Args& a, cudaStream_t s);

struct Read8Args {
    const uint8_t* k_codes;
    const uint8_t* v_codes;
    const uint8_t* k_exp;
    const uint8_t* v_exp;
    const int64_t* slots;
    uint16_t* k_out;
    uint16_t* v_out;
    int64_t n_rows, n_slots;
    int n_kv_heads, head_dim;
};
cudaError_t launch_paged8_read(const Read8Args& a, cudaStream_t s);

// The cache pointers of `a` are the codes'.
struct Paged8AttnArgs {
    PagedAttnArgs a;
    const uint8_t* k_exp;
    const uint8_t* v_exp;
};
cudaError_t launch_paged8_attention(const Paged8AttnArgs& a, cudaStream_t s);

struct Paged8Params : PagedParams {
    const uint8_t* k_exp;
    const uint8_t* v_exp;
};
// Few query rows per request (paged8_few.cu) and many (paged8_many.cu).
cudaError_t launch_paged8_few(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s);
cudaError_t launch_paged8_many(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s);
// Codes as (head_dim, kv head, place in page, page), boxes of min(head_dim, 128) dims x `box` places, rows swizzled.
bool encode_codes(CUtensorMap* m, const void* base, const PagedAttnArgs& a, uint32_t box);

// 2^e, |e| < 127.
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ int exp_of_byte(uint32_t x) { return min(max(int(x) - kExpBias, -kExpMost), kExpMost); }

// Two codes (low byte first) as f16 (exact).
__device__ __forceinline__ uint32_t codes_to_f16x2(uint32_t two) {
    uint32_t h;
    asm("{\n\t.reg .b16 x;\n\tcvt.u16.u32 x, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(h) : "r"(two));
    return h;
}
__device__ __forceinline__ void codes_to_f16x4(uint32_t four, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(four));
}
// Two numbers of at most 448 in magnitude to codes, nearest, ties to even (NaN to NaN).
__device__ __forceinline__ uint32_t codes_of(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b16 x;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %2, %1;\n\tcvt.u32.u16 %0, x;\n\t}" : "=r"(r) : "f"(lo), "f"(hi));
    return r;
}
// The high bit of each byte that is a NaN code.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t without(uint32_t w, uint32_t bad) { return w & ~((bad >> 7) * 0xFFu); }

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The power of two that a row of queries of largest magnitude `top` is multiplied by before it is rounded to f16 (its elements
// then stay below 2^15, and those above 2^-28 of the largest are exact), and that power's inverse. Of a row with an infinity
// nothing is left but NaN, which its scores then are.
struct RowPower {
    float to, back;
};
__device__ __forceinline__ RowPower row_power(float top) {
    const int e = max(int(__float_as_uint(top) >> 23) - 127, -100);  // floor(log2(top))
    return RowPower{top == INFINITY ? NAN : pow2i(14 - e), pow2i(e - 14)};
}
// The factor of a row's raw products over a block is row power x block power, without a cap times the scale. Its part that is the
// row's may then pass fp32's range where the factor does not, so the block powers count from their least (2^48 larger, CAP == 0) and the
// row's part is as much smaller; what falls below the subnormal numbers here is below 2^-20 in a score, |scale| <= 2^50.
template <int CAP>
__device__ __forceinline__ float block_power(int e) { return pow2i(CAP ? e : e + kExpMost); }
__device__ __forceinline__ float row_factor(float back, float scale2) {
    const float least = pow2i(-kExpMost);
    return back >= 1.0f ? back * least * scale2 : back * scale2 * least;
}
// A block's factor of the raw products, held within fp32's range (a product of 0 stays 0 under the largest of them).
__device__ __forceinline__ float score_factor(float x) { return fminf(fmaxf(x, -3.0e38f), 3.0e38f); }

}  // namespace emb
