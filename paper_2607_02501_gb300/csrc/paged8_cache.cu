// What fills the 8-bit paged cache and what reads rows of it back (definitions in include/emb_paged.h).
//
// Both kernels are launched with programmatic stream serialisation and read device memory only after
// griddepcontrol.wait, with ordinary loads.
#include <algorithm>

#include "paged8.cuh"

namespace emb {
namespace {

// ------------------------------------------------------------------ norm, rotation, store
// HBM bounds it. Every thread has eight elements of a row (a head of a token): the four pairs 4 u .. 4 u + 3, so the rotation
// stays within the thread and the sum of squares is a shuffle over the row's d / 8 lanes.
// A CTA (16 rows' threads) takes either queries of a few heads, or one key/value head of a window of 16 tokens. A block's exponent
// needs all tokens of the call that go into it, which stand within 16 of one another: the CTA takes those blocks whose first token
// is in its window, up to 15 tokens beyond it, and leaves those that began before. So no two CTAs meet in a block, nothing is
// exchanged between CTAs, and a token's rows stay in registers between the block's maximum and the rounding.
constexpr int kRows8 = 16;   // rows that a CTA has threads for
constexpr int kHeads8 = 4;   // heads that a thread takes of its token

struct Store8Params {
    Store8Args a;
    int q_ctas, kv_windows;
    int log_tokens, head_groups;  // queries: a CTA's tokens 2^n, CTAs to share a token's heads
};

// Cosine and sine of `factor` times a pair's angle. The product of position and turns wraps at 2^64, one turn, so the
// angle's fraction is exact; its upper 32 bits go to the hardware's sine and cosine in +-pi (error below 2^-21).
__device__ __forceinline__ void angle_of(int32_t at, uint64_t turns, float factor, float& c, float& s) {
    const uint64_t t = uint64_t(int64_t(at)) * turns;
    __sincosf(float(int32_t(uint32_t(t >> 32))) * (6.283185307179586f / 4294967296.0f), &s, &c);
    c *= factor;
    s *= factor;
}

// Where a thread's elements lie: two groups of four at e0 and e1. Halves: firsts and seconds of its pairs; elements behind the turned
// ones likewise. Neighbours: eight in a row.
template <int D, bool NB>
struct Place8 {
    int e0, e1;
    bool turned;
    __device__ __forceinline__ Place8(int u, int rot) {
        if constexpr (NB) {
            e0 = u * 8;
            e1 = e0 + 4;
            turned = e0 < rot;
        } else {
            const int half = rot / 2, units = half / 4;
            turned = u < units;
            e0 = turned ? u * 4 : rot + (u - units) * 4;
            e1 = turned ? half + u * 4 : e0 + (D - rot) / 2;
        }
    }
};

__device__ __forceinline__ void load4(const uint16_t* p, float* x) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    const float2 a = unpack_bf16x2(w.x), b = unpack_bf16x2(w.y);
    x[0] = a.x;
    x[1] = a.y;
    x[2] = b.x;
    x[3] = b.y;
}

// A row in place: norm (g: the thread's eight gains, or none) and rotation.
template <int D, bool NB>
__device__ __forceinline__ void norm_turn(float (&x)[8], bool norm, const float* g, float eps, bool turned, const float (&c)[4], const float (&s)[4]) {
    if (norm) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int o = D / 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float inv = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(ss * (1.0f / D), eps)));
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
    }
    if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float& a = x[NB ? 2 * i : i];
            float& b = x[NB ? 2 * i + 1 : 4 + i];
            const float y = fmaf(a, c[i], -b * s[i]);
            b = fmaf(b, c[i], a * s[i]);
            a = y;
        }
    }
}

template <int D, bool NB>
__global__ void __launch_bounds__(kRows8* D / 8) paged8_store_kernel(const __grid_constant__ Store8Params p) {
    constexpr int kLanes = D / 8;
    const Store8Args& a = p.a;
    const int tid = threadIdx.x, row = tid / kLanes, u = tid % kLanes;
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const Place8<D, NB> at(u, a.rot_dim);

    // the pairs' turns and axes
    uint64_t turns[4] = {0, 0, 0, 0};
    int axis[4] = {0, 0, 0, 0};
    if (at.turned)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            turns[i] = a.turns[u * 4 + i];
            if (a.axis_of_pair) axis[i] = min(int(a.axis_of_pair[u * 4 + i]), a.n_axes - 1);
        }
    auto angles = [&](int64_t t, float (&c)[4], float (&s)[4]) {
        if (!at.turned) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) angle_of(a.positions[axis[i] * a.pos_stride + t], turns[i], a.factor, c[i], s[i]);
    };
    auto gains = [&](const float* gamma, float (&g)[8]) {
        if (!gamma) return;
        *reinterpret_cast<float4*>(g) = *reinterpret_cast<const float4*>(gamma + at.e0);
        *reinterpret_cast<float4*>(g + 4) = *reinterpret_cast<const float4*>(gamma + at.e1);
    };

    const int kv_ctas = p.kv_windows * a.n_kv_heads;
    if (int(blockIdx.x) >= kv_ctas) {
        // ---------------------------------------------------------------------------- queries
        const int id = int(blockIdx.x) - kv_ctas, group = id % p.head_groups, hw = kRows8 >> p.log_tokens;
        const int64_t t = (int64_t(id / p.head_groups) << p.log_tokens) + (row & ((1 << p.log_tokens) - 1));
        const int h0 = group * hw * kHeads8 + (row >> p.log_tokens);
        const bool live = t < a.n_tokens;
        float x[kHeads8][8];
#pragma unroll
        for (int k = 0; k < kHeads8; ++k) {
            const int h = h0 + k * hw;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = 0.0f;
            if (live && h < a.n_heads) {
                const uint16_t* q = a.q + t * a.q_stride + h * D;
                load4(q + at.e0, x[k]);
                load4(q + at.e1, x[k] + 4);
            }
        }
        float c[4], s[4], g[8];
        if (live) angles(t, c, s);
        gains(a.q_gamma, g);
#pragma unroll
        for (int k = 0; k < kHeads8; ++k) {
            const int h = h0 + k * hw;
            norm_turn<D, NB>(x[k], a.q_gamma != nullptr, g, a.eps, at.turned, c, s);
            if (live && h < a.n_heads) {
                uint16_t* o = a.q_out + (t * a.n_heads + h) * D;
                *reinterpret_cast<uint2*>(o + at.e0) = make_uint2(pack_bf16x2(x[k][0], x[k][1]), pack_bf16x2(x[k][2], x[k][3]));
                *reinterpret_cast<uint2*>(o + at.e1) = make_uint2(pack_bf16x2(x[k][4], x[k][5]), pack_bf16x2(x[k][6], x[k][7]));
            }
        }
        return;
    }

    // ------------------------------------------------------------------------- keys and values
    __shared__ int64_t slot_of[32];
    __shared__ float top[2][32];          // of a token's key and value row
    __shared__ int exp_of[2][kRows8];     // of the run that token i of the window begins: its block's exponents,
    __shared__ int exp_was[2][kRows8];    // what they were,
    __shared__ uint32_t written[kRows8];  // and its places
    const int g = int(blockIdx.x) % a.n_kv_heads, Hk = a.n_kv_heads;
    const int64_t t0 = int64_t(int(blockIdx.x) / a.n_kv_heads) * kRows8;
    // Tokens t0 .. t0 + 31, a lane each in every warp: which share a block. A run, the tokens of a block, is this CTA's if the
    // first of them is in its window and none is in the window before.
    const int lane = tid & 31;
    auto slot_at = [&](int64_t t) {
        const int64_t s = t >= 0 && t < a.n_tokens ? a.slots[t] : -1;
        return s >= 0 && s < a.n_slots ? s : int64_t(-1);
    };
    auto block_of = [&](int64_t s) { return s >= 0 ? s / kBlock8 : -1 - int64_t(lane); };  // (no slot: a block by itself)
    const int64_t mine = slot_at(t0 + lane), shifted = slot_at(t0 - kRows8 + lane);
    const uint32_t members = __match_any_sync(0xffffffffu, block_of(mine));
    const uint32_t around = __match_any_sync(0xffffffffu, block_of(shifted));  // of tokens t0 - 16 .. t0 + 15
    const bool older = __shfl_sync(0xffffffffu, int((around & 0xFFFFu) != 0), (lane & 15) + 16) != 0;  // of token lane % 16
    const int head = __ffs(members) - 1;
    const uint32_t begun = __ballot_sync(0xffffffffu, mine >= 0 && head == lane && lane < kRows8 && !older);
    if (begun == 0) return;  // (the CTA as a whole)
    if (tid < 32) slot_of[lane] = mine;
    // the run that token j belongs to, by its first token, or -1: no slot, or not this CTA's
    const int own_run = mine >= 0 && (begun >> head & 1u) ? head : -1;

    // this thread's rows: tokens `row` and `row + 16` of the window
    float x[2][2][8];  // [key, value][token]
    int run[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        run[i] = __shfl_sync(0xffffffffu, own_run, row + i * kRows8);
        const int64_t t = t0 + row + i * kRows8;
        if (run[i] < 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[0][i][e] = x[1][i][e] = 0.0f;
            continue;
        }
        const uint16_t* k = a.k + t * a.k_stride + g * D;
        const uint16_t* v = a.v + t * a.v_stride + g * D;
        load4(k + at.e0, x[0][i]);
        load4(k + at.e1, x[0][i] + 4);
        load4(v + at.e0, x[1][i]);
        load4(v + at.e1, x[1][i] + 4);
    }
    // the exponents before, of the runs that begin here
    int was[2] = {0, 0};
    if (tid < 32 && (begun >> lane & 1u)) {
        const int64_t at8 = (mine / kBlock8) * Hk + g;
        was[0] = exp_of_byte(a.k_exp[at8]);
        was[1] = exp_of_byte(a.v_exp[at8]);
    }
    float gk[8];
    gains(a.k_gamma, gk);
    const float limit = kCodeMost * pow2i(kExpMost);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float c[4], s[4];
        if (run[i] >= 0) angles(t0 + row + i * kRows8, c, s);
        norm_turn<D, NB>(x[0][i], a.k_gamma != nullptr, gk, a.eps, at.turned, c, s);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = fabsf(x[kv][i][e]);
                m = v <= limit ? fmaxf(m, v) : m;
            }
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (u == 0) top[kv][row + i * kRows8] = m;
        }
    }
    __syncthreads();
    if (tid < 32 && (begun >> lane & 1u)) {
        const int64_t at8 = (mine / kBlock8) * Hk + g;
        uint32_t places = 0;
        for (uint32_t m = members; m != 0; m &= m - 1) places |= 1u << (slot_of[__ffs(m) - 1] & (kBlock8 - 1));
        written[lane] = places;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            float m = 0.0f;
            for (uint32_t left = members; left != 0; left &= left - 1) m = fmaxf(m, top[kv][__ffs(left) - 1]);
            // 448 = 1.75 * 2^8: the least e with m <= 448 * 2^e by m's exponent and mantissa
            const uint32_t bits = __float_as_uint(m);
            const int need = int(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
            const int e = max(places & 1u ? -kExpMost : was[kv], min(max(need, -kExpMost), kExpMost));
            exp_of[kv][lane] = e;
            exp_was[kv][lane] = was[kv];
            (kv ? a.v_exp : a.k_exp)[at8] = uint8_t(e + kExpBias);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (run[i] < 0) continue;
        const int64_t to = (slot_of[row + i * kRows8] * Hk + g) * D;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const float by = pow2i(-exp_of[kv][run[i]]);
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                uint32_t two = codes_of(x[kv][i][e] * by, x[kv][i][e + 1] * by);
                if (!(fabsf(x[kv][i][e]) <= limit)) two = (two & 0xFF00u) | 0x7Fu;
                if (!(fabsf(x[kv][i][e + 1]) <= limit)) two = (two & 0xFFu) | 0x7F00u;
                w[e / 2] = two;
            }
            uint8_t* codes = (kv ? a.v_codes : a.k_codes) + to;
            *reinterpret_cast<uint32_t*>(codes + at.e0) = w[0] | w[1] << 16;
            *reinterpret_cast<uint32_t*>(codes + at.e1) = w[2] | w[3] << 16;
        }
    }
    // the other places of the blocks: zeros in a block that starts anew, re-encoded where the exponent grew
    for (uint32_t left = begun; left != 0; left &= left - 1) {
        const int h = __ffs(left) - 1;
        const int64_t block = slot_of[h] & ~int64_t(kBlock8 - 1);
        const uint32_t places = written[h];
        if (places >> row & 1u) continue;
        const int64_t to = ((block + row) * Hk + g) * D + u * 8;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            uint2* codes = reinterpret_cast<uint2*>((kv ? a.v_codes : a.k_codes) + to);
            if (places & 1u) {
                *codes = make_uint2(0u, 0u);
            } else if (exp_of[kv][h] > exp_was[kv][h]) {
                const float by = pow2i(exp_was[kv][h] - exp_of[kv][h]);
                const uint2 old = *codes;
                uint32_t w[2] = {old.x, old.y};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t lo, hi;
                    codes_to_f16x4(w[i], lo, hi);
                    const float2 f0 = __half22float2(*reinterpret_cast<__half2*>(&lo)), f1 = __half22float2(*reinterpret_cast<__half2*>(&hi));
                    w[i] = codes_of(f0.x * by, f0.y * by) | codes_of(f1.x * by, f1.y * by) << 16;
                }
                *codes = make_uint2(w[0], w[1]);
            }
        }
    }
}

// ------------------------------------------------------------------ rows of the cache as bf16
// HBM bounds it. A thread takes 16 codes of a key row and of a value row: 32 bytes in, 64 out.
constexpr int kReadThreads = 256;
constexpr int kReadChunks = 1024;  // of 16 codes of a CTA, about

__device__ __forceinline__ void read16(const uint8_t* codes, const uint8_t* exp, int64_t slot, int Hk, int c, int log_d, uint4 (&out)[2]) {
    const int g = (c * 16) >> log_d;
    const uint4 w = *reinterpret_cast<const uint4*>(codes + ((slot * Hk) << log_d) + c * 16);
    const float by = pow2i(exp_of_byte(exp[(slot / kBlock8) * Hk + g]));
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t* o = reinterpret_cast<uint32_t*>(out);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t lo, hi;
        codes_to_f16x4(in[i], lo, hi);
        const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo)), b = __half22float2(*reinterpret_cast<__half2*>(&hi));
        o[2 * i] = pack_bf16x2(a.x * by, a.y * by);
        o[2 * i + 1] = pack_bf16x2(b.x * by, b.y * by);
    }
}

__global__ void __launch_bounds__(kReadThreads) paged8_read_kernel(const __grid_constant__ Read8Args p, int rows, int log_d) {
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int Hk = p.n_kv_heads, per = (Hk << log_d) / 16;  // chunks of a row
    const int64_t r0 = int64_t(blockIdx.x) * rows;
    const int n = int(min(int64_t(rows), p.n_rows - r0)) * per;
    for (int e = threadIdx.x; e < n; e += kReadThreads) {
        const int r = e / per, c = e - r * per;
        const int64_t slot = p.slots[r0 + r];
        uint4 k[2] = {}, v[2] = {};
        if (slot >= 0 && slot < p.n_slots) {
            read16(p.k_codes, p.k_exp, slot, Hk, c, log_d, k);
            read16(p.v_codes, p.v_exp, slot, Hk, c, log_d, v);
        }
        const int64_t to = (r0 + r) * per + c;
        uint4* ko = reinterpret_cast<uint4*>(p.k_out) + 2 * to;
        uint4* vo = reinterpret_cast<uint4*>(p.v_out) + 2 * to;
        ko[0] = k[0];
        ko[1] = k[1];
        vo[0] = v[0];
        vo[1] = v[1];
    }
}

template <int D>
const void* store_kernel(bool neighbours) {
    return neighbours ? reinterpret_cast<const void*>(paged8_store_kernel<D, true>) : reinterpret_cast<const void*>(paged8_store_kernel<D, false>);
}

}  // namespace

cudaError_t launch_paged8_store(const Store8Args& a, cudaStream_t s) {
    Store8Params p;
    p.a = a;
    p.kv_windows = int((a.n_tokens + kRows8 - 1) / kRows8);
    // a thread takes up to four heads of its token; few tokens leave rows for more heads at once
    p.log_tokens = 0;
    while (p.log_tokens < 4 && (int64_t(1) << p.log_tokens) < a.n_tokens) ++p.log_tokens;
    const int heads = (kRows8 >> p.log_tokens) * kHeads8;
    p.head_groups = (a.n_heads + heads - 1) / heads;
    const int64_t q_ctas = ((a.n_tokens - 1) >> p.log_tokens) * p.head_groups + p.head_groups;
    const int64_t grid = q_ctas + int64_t(p.kv_windows) * a.n_kv_heads;
    if (grid > 2147483647) return cudaErrorInvalidValue;
    p.q_ctas = int(q_ctas);
    void* args[] = {&p};
    const void* fn = a.head_dim == 64 ? store_kernel<64>(a.neighbours) : a.head_dim == 128 ? store_kernel<128>(a.neighbours) : store_kernel<256>(a.neighbours);
    return launch_serialised(fn, unsigned(grid), unsigned(kRows8 * a.head_dim / 8), 0, s, args);
}

cudaError_t launch_paged8_read(const Read8Args& a, cudaStream_t s) {
    Read8Args p = a;
    int log_d = 0;
    while ((1 << log_d) < a.head_dim) ++log_d;
    const int per = a.n_kv_heads * a.head_dim / 16;
    int rows = std::max(1, kReadChunks / per);
    const int64_t grid = (a.n_rows + rows - 1) / rows;
    void* args[] = {&p, &rows, &log_d};
    return launch_serialised(reinterpret_cast<const void*>(paged8_read_kernel), unsigned(grid), kReadThreads, 0, s, args);
}

}  // namespace emb
