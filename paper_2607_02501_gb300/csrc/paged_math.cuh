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
// Capped scores cap log2(e) tanh(x), x = scale q.k / cap, from q.k.
// capped_far: as 1 - 2 / (1 + e^2x), within 2^-22 of the cap: 2^-20 of the value from |x| = 0.35 on, and for caps up to 64 within
// the 2^-16 that the weights are held to. capped_near, below 0.35: the series x (1 - x^2 / 3 + 2 x^4 / 15 - 17 x^6 / 315 +
// 62 x^8 / 2835), whose next term is 2.4e-7 of it; the factor cap log2(e) x = q.k lin2 is formed without the cap, so it is right
// however far the cap lies above the scores.
// Kernels for caps of up to 64 have the first form for all scores, those for any cap have for each score its own. (us, the two:
// 2048 tokens of 32 heads of 128 over 8192 keys, a cap of 65 and scores up to it 435 and 528.)
constexpr float kNearCap = 2.0f * 1.4426950408889634f * 0.35f;  // |x| = 0.35 in units of |q.k scale2|
enum : int { kUncapped, kLowCap, kAnyCap };                     // a kernel's scores
constexpr float kMostLowCap = 64.0f;
__device__ __forceinline__ float2 capped_near2(float2 qk, const PagedParams& p, float2 plus) {
    auto k = [](float v) { return make_float2(v, v); };
    const float2 x = mul2(qk, k(p.scale2 * (0.5f / 1.4426950408889634f))), y = mul2(x, x);
    float2 t = fma2(y, k(62.0f / 2835.0f), k(-17.0f / 315.0f));
    t = fma2(t, y, k(2.0f / 15.0f));
    t = fma2(t, y, k(-1.0f / 3.0f));
    t = fma2(t, y, k(1.0f));
    return fma2(mul2(qk, k(p.lin2)), t, plus);
}
__device__ __forceinline__ float capped_far(float qk, const PagedParams& p) {
    return fmaf(p.cap2, -2.0f * rcp_fast(1.0f + exp2_fast(qk * p.scale2)), p.cap2);
}
template <int CAP>
__device__ __forceinline__ float2 capped2(float2 qk, const PagedParams& p) {
    const float2 far = make_float2(capped_far(qk.x, p), capped_far(qk.y, p));
    if constexpr (CAP == kLowCap) return far;
    const float2 near = capped_near2(qk, p, make_float2(0, 0));
    return make_float2(fabsf(qk.x * p.scale2) < kNearCap ? near.x : far.x, fabsf(qk.y * p.scale2) < kNearCap ? near.y : far.y);
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_bf16x2(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ bool not_finite(uint32_t bf16_bits) { return (bf16_bits & 0x7F80u) == 0x7F80u; }
// Bits 15 and 31: whether the low and the high bf16 of a word are not finite.
__device__ __forceinline__ uint32_t not_finite2(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }

// Rows of O behind the last request's (padding of a recorded step): zeros.
__device__ __forceinline__ void zero_padding(const PagedParams& p, int D, int tid, int nt) {
    const int64_t used = min(max(p.q_start[p.n_req], 0), p.n_tokens), row16 = int64_t(p.H) * D / 8;
    uint4* o = reinterpret_cast<uint4*>(p.O);
    for (int64_t i = used * row16 + int64_t(blockIdx.x) * nt + tid; i < int64_t(p.n_tokens) * row16; i += int64_t(gridDim.x) * nt)
        o[i] = make_uint4(0, 0, 0, 0);
}

// A partial result of an item, ROWS x D values not yet divided by their row's sum: ROWS maxima, ROWS sums, then the
// values as [D / 4][ROWS][4], so that neighbouring rows lie side by side.
template <int D, int ROWS>
struct PartLayout {
    static constexpr int64_t kFloats = int64_t(ROWS) * (D + 2);
    __device__ static float* value(float* part, int row, int c) { return part + 2 * ROWS + ((c >> 2) * ROWS + row) * 4 + (c & 3); }
};

// Counts this CTA's partial result in: one thread, after a barrier behind all that was written of it.
__device__ __forceinline__ void part_publish(uint32_t* flag) {
    __threadfence();
    atomicAdd(flag, 1u);
}
// Waits for all partial results of an item: one thread. The last CTA to pass hands the flag back at zero.
__device__ __forceinline__ bool part_wait(uint32_t* flag, int count, volatile int* abort, int* status, uint64_t limit_ns = kWaitLimitNs) {
    if (!join_wait(flag, uint32_t(count), abort, status, limit_ns)) return false;
    if (atomicAdd(flag, 1u) == 2u * uint32_t(count) - 1u) ptx::st_relaxed_gpu(flag, 0u);
    return true;
}

// Adds the partial results of an item that several CTAs shared, in CTA order (deterministic), and stores this CTA's
// share of the rows. One round of loads covers PARTS partial results of VALS groups of four values: the loads, not the
// arithmetic, take the time.
template <int D, int ROWS, int PARTS, int VALS>
__device__ __forceinline__ void join_store(const PagedParams& p, const PagedJoin& J, const PagedReq& q, int me, int tid, int nt) {
    using PL = PartLayout<D, ROWS>;
    const int i0 = J.b * p.QB, rows = min(p.QB, q.n - i0) * p.G;
    const int row0 = rows * me / J.count, mine = rows * (me + 1) / J.count - row0;
    if (mine <= 0) return;
    for (int e0 = tid; e0 < mine * (D / 4); e0 += nt * VALS) {
        float M[VALS], L[VALS];
        float4 o[VALS];
#pragma unroll
        for (int v = 0; v < VALS; ++v) {
            M[v] = -INFINITY;
            L[v] = 0.0f;
            o[v] = make_float4(0, 0, 0, 0);
        }
        for (int i0p = 0; i0p < J.count; i0p += PARTS) {
            float m[VALS][PARTS], l[VALS][PARTS];
            float4 x[VALS][PARTS];
#pragma unroll
            for (int v = 0; v < VALS; ++v) {
                const int e = e0 + v * nt;
                const int c4 = e / mine, row = row0 + e - c4 * mine;
#pragma unroll
                for (int k = 0; k < PARTS; ++k) {
                    m[v][k] = -INFINITY;
                    l[v][k] = 0.0f;
                    x[v][k] = make_float4(0, 0, 0, 0);
                    if (e < mine * (D / 4) && i0p + k < J.count) {
                        float* part = p.part + part_slot(J.first + i0p + k, J.first) * PL::kFloats;
                        m[v][k] = __ldcg(part + row);
                        l[v][k] = __ldcg(part + ROWS + row);
                        x[v][k] = __ldcg(reinterpret_cast<const float4*>(PL::value(part, row, c4 * 4)));
                    }
                }
            }
#pragma unroll
            for (int v = 0; v < VALS; ++v) {
                float top = M[v];
#pragma unroll
                for (int k = 0; k < PARTS; ++k) top = fmaxf(top, m[v][k]);
                const float z = top == -INFINITY ? 0.0f : top;
                const float f = exp2_fast(M[v] - z);
                M[v] = top;
                L[v] *= f;
                o[v] = make_float4(o[v].x * f, o[v].y * f, o[v].z * f, o[v].w * f);
#pragma unroll
                for (int k = 0; k < PARTS; ++k) {
                    // weight 0 of a partial without a finite score: its sums are 0, or NaN, which has to show
                    const float w = exp2_fast(m[v][k] - z);
                    L[v] = fmaf(l[v][k], w, L[v]);
                    o[v].x = fmaf(x[v][k].x, w, o[v].x);
                    o[v].y = fmaf(x[v][k].y, w, o[v].y);
                    o[v].z = fmaf(x[v][k].z, w, o[v].z);
                    o[v].w = fmaf(x[v][k].w, w, o[v].w);
                }
            }
        }
#pragma unroll
        for (int v = 0; v < VALS; ++v) {
            const int e = e0 + v * nt;
            if (e >= mine * (D / 4)) continue;
            const int c4 = e / mine, row = row0 + e - c4 * mine;
            const float inv = L[v] == 0.0f ? 0.0f : __fdiv_rn(1.0f, L[v]);
            uint2 u;
            u.x = pack_bf16x2(__fmul_rn(o[v].x, inv), __fmul_rn(o[v].y, inv));
            u.y = pack_bf16x2(__fmul_rn(o[v].z, inv), __fmul_rn(o[v].w, inv));
            const int64_t t = q.q0 + i0 + row / p.G;
            *reinterpret_cast<uint2*>(p.O + (t * p.H + J.g * p.G + row % p.G) * D + c4 * 4) = u;
        }
    }
}

}  // namespace emb
