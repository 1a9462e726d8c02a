// Arithmetic shared by the paged attention's kernels, and the join of items that several CTAs share.
#pragma once

#include "paged_sched.cuh"

namespace emb {

// 2^x (results below the normal range become zero; -inf gives 0).
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// cap log2(e) tanh(y / 2), y = 2 scale q.k / cap with its base 2: tanh as 1 - 2 / (1 + e^y), within 2^-22 of 1
__device__ __forceinline__ float capped(float y, float cap2) { return fmaf(-2.0f * cap2, rcp_fast(1.0f + exp2_fast(y)), cap2); }

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_bf16x2(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ bool not_finite(uint32_t bf16_bits) { return (bf16_bits & 0x7F80u) == 0x7F80u; }

// Rows of O behind the last request's (padding of a recorded step): zeros.
__device__ __forceinline__ void zero_padding(const PagedParams& p, int D, int tid, int nt) {
    const int64_t used = min(max(int64_t(p.q_start[p.n_req]), int64_t(0)), p.n_tokens);
    const int64_t row16 = int64_t(p.H) * D / 8;
    uint4* o = reinterpret_cast<uint4*>(p.O);
    for (int64_t i = used * row16 + int64_t(blockIdx.x) * nt + tid; i < p.n_tokens * row16; i += int64_t(gridDim.x) * nt)
        o[i] = make_uint4(0, 0, 0, 0);
}

// Adds the partial results of an item that several CTAs shared and stores this CTA's part of its outputs.
// A partial result is ROWS maxima, ROWS sums and [ROWS][D] values, in CTA order (deterministic).
template <int D, int ROWS>
__device__ __forceinline__ void join_store(const PagedParams& p, const PagedJoin& J, const PagedReq& q, int me, int tid, int nt) {
    constexpr int64_t kSlot = int64_t(ROWS) * (D + 2);
    const int i0 = J.b * p.QB, rows = min(p.QB, q.n - i0) * p.G;
    for (int e = me * nt + tid; e < rows * (D / 4); e += J.count * nt) {
        const int row = e / (D / 4), c = (e - row * (D / 4)) * 4;
        float M = -INFINITY;
#pragma unroll 8
        for (int i = 0; i < J.count; ++i) M = fmaxf(M, __ldcg(p.part + part_slot(J.first + i, J.first) * kSlot + row));
        const float m0 = M == -INFINITY ? 0.0f : M;
        float L = 0.0f;
        float4 o = make_float4(0, 0, 0, 0);
#pragma unroll 8
        for (int i = 0; i < J.count; ++i) {
            const float* s = p.part + part_slot(J.first + i, J.first) * kSlot;
            const float4 v = __ldcg(reinterpret_cast<const float4*>(s + 2 * ROWS + row * D + c));
            // weight 0 of a partial without a finite score: its sums are 0, or NaN, which has to show
            const float w = exp2_fast(__ldcg(s + row) - m0);
            L = fmaf(__ldcg(s + ROWS + row), w, L);
            o.x = fmaf(v.x, w, o.x);
            o.y = fmaf(v.y, w, o.y);
            o.z = fmaf(v.z, w, o.z);
            o.w = fmaf(v.w, w, o.w);
        }
        const float inv = L == 0.0f ? 0.0f : __fdiv_rn(1.0f, L);
        uint2 u;
        u.x = pack_bf16x2(__fmul_rn(o.x, inv), __fmul_rn(o.y, inv));
        u.y = pack_bf16x2(__fmul_rn(o.z, inv), __fmul_rn(o.w, inv));
        const int64_t t = q.q0 + i0 + row / p.G;
        *reinterpret_cast<uint2*>(p.O + (t * p.H + J.g * p.G + row % p.G) * D + c) = u;
    }
}

}  // namespace emb
