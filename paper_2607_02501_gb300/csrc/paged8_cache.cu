// What fills the 8-bit paged cache and what reads rows of it back (definitions in include/emb_paged.h).
//
// Both kernels are launched with programmatic stream serialisation and read device memory only after
// griddepcontrol.wait, with ordinary loads.
#include <algorithm>
#include <type_traits>

#include "paged8.cuh"

namespace emb {
namespace {

// ------------------------------------------------------------------ norm, rotation, store
// HBM bounds it, and the instructions are not far behind. Every thread has E elements of a row (a head of a token): E / 2 pairs
// one after another, so the rotation stays within the thread and the sum of squares is a shuffle over the row's d / E lanes. E is 16
// where both halves of the turned elements are whole groups of eight, else 8.
// A CTA takes either queries of a few heads, or the keys or the values of one head of a window of 16 tokens. A block's exponent
// needs all tokens of the call that go into it, which stand within 16 of one another: the CTA takes those blocks whose first token
// is in its window, up to 15 tokens beyond it, and leaves those that began before. So no two CTAs meet in a block, nothing is
// exchanged between CTAs, and a token's rows stay in registers between the block's maximum and the rounding. Every warp works out
// the blocks of all 32 tokens by itself, a lane a token, so there is one barrier.
// Measured (us replayed): 15600 tokens of 10 heads of 256 (152 MB) 37.5, 0.60 of the measured copy rate; 256 decoded tokens of 48 heads of
// 128 4.9, one of 10 heads 3.2. With eight elements a thread and keys and values in one CTA 86, 8.7 and 4.5.
constexpr int kStoreThreads = 256;
constexpr int kWindow8 = 16;  // tokens
constexpr int kMostRounds = 8;  // heads that a thread takes of its token, at most

struct Store8Params {
    Store8Args a;
    int kv_ctas;                         // the first CTAs: keys and values
    int log_tokens, rounds, head_groups; // queries: a CTA's tokens 2^n, a thread's heads, CTAs to share a token's heads
};

// Cosine and sine of a pair's angle, times `factor`. The product of position and turns wraps at 2^64, one turn, so the angle's
// fraction is exact; of its upper 32 bits fp32 keeps 24. Queries, which bf16 rounds, take the hardware's sine and cosine in +-pi
// (error below 2^-21); keys exact ones: next to a border between two codes an error of fp32's size is an eighth of the value.
// (15600 tokens of 10 heads of 256: 38.9 us with the hardware's for keys too, 39.4 so.)
template <bool EXACT>
__device__ __forceinline__ void angle_of(int32_t at, uint64_t turns, float factor, float& c, float& s) {
    // (the upper half of the product modulo 2^64, from the 32-bit halves)
    const uint32_t lo = uint32_t(turns), hi = uint32_t(turns >> 32), p = uint32_t(at);
    const float half_turns = float(int32_t(__umulhi(p, lo) + p * hi - (at < 0 ? lo : 0u))) * (1.0f / 2147483648.0f);
    if constexpr (EXACT) sincospif(half_turns, &s, &c);
    else __sincosf(half_turns * 3.1415926535897931f, &s, &c);
    c *= factor;
    s *= factor;
}

// Where a thread's elements lie: two groups of E / 2 at e0 and e1. Halves: firsts and seconds of its pairs; elements behind the
// turned ones likewise. Neighbours: E in a row.
template <int D, bool NB, int E>
struct Place8 {
    int e0, e1;
    bool turned;
    __device__ __forceinline__ Place8(int u, int rot) {
        if constexpr (NB) {
            e0 = u * E;
            e1 = e0 + E / 2;
            turned = e0 < rot;
        } else {
            const int half = rot / 2, units = half / (E / 2);
            turned = u < units;
            e0 = turned ? u * (E / 2) : rot + (u - units) * (E / 2);
            e1 = turned ? half + u * (E / 2) : e0 + (D - rot) / 2;
        }
    }
};

// N bf16 numbers (4 or 8, aligned to their size) from and to memory.
template <int N>
struct alignas(2 * N) RawRow {
    uint32_t w[N / 2];
};
template <int N>
__device__ __forceinline__ void unpack_row(const RawRow<N>& r, float* x) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const float2 u = unpack_bf16x2(r.w[i]);
        x[2 * i] = u.x;
        x[2 * i + 1] = u.y;
    }
}
template <int N>
__device__ __forceinline__ void load_row(const uint16_t* p, float* x) {
    unpack_row<N>(*reinterpret_cast<const RawRow<N>*>(p), x);
}
template <int N>
__device__ __forceinline__ void store_row(uint16_t* p, const float* x) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(w);
    else *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(w);
}

// A row in place: norm (with the head's gains, or none) and rotation.
template <int D, bool NB, int E>
__device__ __forceinline__ void norm_turn(float (&x)[E], const float* gamma, float eps, const Place8<D, NB, E>& at, const float (&c)[E / 2], const float (&s)[E / 2]) {
    if (gamma) {
        float2 s2 = make_float2(0, 0);
#pragma unroll
        for (int e = 0; e < E; e += 2) s2 = fma2(make_float2(x[e], x[e + 1]), make_float2(x[e], x[e + 1]), s2);
        float ss = s2.x + s2.y;
#pragma unroll
        for (int o = D / E / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float inv = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(ss * (1.0f / D), eps)));
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const float4 g = *reinterpret_cast<const float4*>(gamma + (e < E / 2 ? at.e0 + e : at.e1 + e - E / 2));
            x[e] = x[e] * inv * g.x;
            x[e + 1] = x[e + 1] * inv * g.y;
            x[e + 2] = x[e + 2] * inv * g.z;
            x[e + 3] = x[e + 3] * inv * g.w;
        }
    }
    if (!at.turned) return;
    if constexpr (NB) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = fmaf(a, c[i], -b * s[i]);
            x[2 * i + 1] = fmaf(b, c[i], a * s[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; i += 2) {
            const float2 a = make_float2(x[i], x[i + 1]), b = make_float2(x[E / 2 + i], x[E / 2 + i + 1]);
            const float2 c2 = make_float2(c[i], c[i + 1]), s2 = make_float2(s[i], s[i + 1]), bs = mul2(b, s2);
            const float2 y = fma2(a, c2, make_float2(-bs.x, -bs.y)), z = fma2(b, c2, mul2(a, s2));
            x[i] = y.x;
            x[i + 1] = y.y;
            x[E / 2 + i] = z.x;
            x[E / 2 + i + 1] = z.y;
        }
    }
}

// (three CTAs per SM: without the bound two fit, and 15600 tokens of 10 heads of 256 with eight elements a thread took 79 us, so 60)
template <int D, bool NB, int E>
__global__ void __launch_bounds__(kStoreThreads, 3) paged_codes_store_kernel(const __grid_constant__ Store8Params p) {
    constexpr int kLanes = D / E, kRows = kStoreThreads / kLanes, kPasses = kRows < 2 * kWindow8 ? 2 * kWindow8 / kRows : 1;
    const Store8Args& a = p.a;
    // of the block that token i of the window begins: the bits of the largest magnitude and its places
    __shared__ uint32_t run_top[kWindow8], run_places[kWindow8];
    const int tid = threadIdx.x, row = tid / kLanes, u = tid % kLanes;
    if (tid < kWindow8) run_top[tid] = run_places[tid] = 0;
    ptx::griddep_launch_dependents();
    __syncthreads();
    ptx::griddep_wait();
    const Place8<D, NB, E> at(u, a.rot_dim);
    // (pos: the token's only position, or anything if there are several axes)
    auto angles = [&](auto exact, int64_t t, int32_t pos, float (&c)[E / 2], float (&s)[E / 2]) {
        constexpr bool kExact = decltype(exact)::value;
        if (!at.turned) return;
        const int pair = u * (E / 2);
        if (!a.axis_of_pair) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) angle_of<kExact>(pos, a.turns[pair + i], a.factor, c[i], s[i]);
        } else {
#pragma unroll
            for (int i = 0; i < E / 2; ++i)
                angle_of<kExact>(a.positions[min(int(a.axis_of_pair[pair + i]), a.n_axes - 1) * a.pos_stride + t], a.turns[pair + i], a.factor, c[i], s[i]);
        }
    };
    const unsigned all = 0xffffffffu;

    if (int(blockIdx.x) >= p.kv_ctas) {
        // -------------------------------------------------- queries: head after head of a token, the next two on their way
        const int id = int(blockIdx.x) - p.kv_ctas, group = id % p.head_groups, hw = kRows >> p.log_tokens;
        const int64_t t = (int64_t(id / p.head_groups) << p.log_tokens) + (row & ((1 << p.log_tokens) - 1));
        const int h0 = group * hw * p.rounds + (row >> p.log_tokens), h_end = t < a.n_tokens ? min(a.n_heads, h0 + hw * p.rounds) : 0;
        const uint16_t* q = a.q + t * a.q_stride;
        uint16_t* out = a.q_out + t * a.n_heads * D;
        RawRow<E / 2> raw[2][2];
        auto fetch = [&](int h, RawRow<E / 2> (&to)[2]) {
            if (h < h_end) {
                to[0] = *reinterpret_cast<const RawRow<E / 2>*>(q + h * D + at.e0);
                to[1] = *reinterpret_cast<const RawRow<E / 2>*>(q + h * D + at.e1);
            }
        };
        raw[0][0] = raw[0][1] = raw[1][0] = raw[1][1] = RawRow<E / 2>{};
        fetch(h0, raw[0]);
        fetch(h0 + hw, raw[1]);
        float c[E / 2], s[E / 2];
        if (h_end > 0) angles(std::false_type{}, t, a.positions[t], c, s);
        for (int r = 0; r < p.rounds; r += 2) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int h = h0 + (r + k) * hw;
                float x[E];
                unpack_row<E / 2>(raw[k][0], x);
                unpack_row<E / 2>(raw[k][1], x + E / 2);
                fetch(h + 2 * hw, raw[k]);
                norm_turn<D, NB, E>(x, a.q_gamma, a.eps, at, c, s);
                if (h < h_end) {
                    store_row<E / 2>(out + h * D + at.e0, x);
                    store_row<E / 2>(out + h * D + at.e1, x + E / 2);
                }
            }
        }
        return;
    }

    // ------------------------------------------------------------------------- keys or values
    const int Hk = a.n_kv_heads, lane = tid & 31;
    const bool is_k = int(blockIdx.x) % 2 == 0;
    const int g = int(blockIdx.x) / 2 % Hk;
    const int64_t t0 = int64_t(int(blockIdx.x) / 2 / Hk) * kWindow8;
    uint8_t* codes = is_k ? a.k_codes : a.v_codes;
    uint8_t* exps = is_k ? a.k_exp : a.v_exp;
    auto row_at = [&](int j) { return (is_k ? a.k + (t0 + j) * a.k_stride : a.v + (t0 + j) * a.v_stride) + g * D; };
    // the window's own rows and positions are on their way while it is found out whose blocks they are
    RawRow<E / 2> early[2] = {};
    int32_t early_pos = 0;
    if (row < kWindow8 && t0 + row < a.n_tokens) {
        early[0] = *reinterpret_cast<const RawRow<E / 2>*>(row_at(row) + at.e0);
        early[1] = *reinterpret_cast<const RawRow<E / 2>*>(row_at(row) + at.e1);
        if (is_k) early_pos = a.positions[t0 + row];
    }
    // Tokens t0 .. t0 + 31, a lane each. The first token of a token's block is the furthest of those up to 15 before it that share
    // the block; the block is this CTA's if that lies in the window. (By comparisons: matching 64-bit numbers over a
    // warp takes 2 us where each token has a block of its own.)
    __shared__ int64_t block_of[kStoreThreads / 32][3 * kWindow8];  // a warp's copy: of tokens t0 - 16 .. t0 + 31
    auto slot_at = [&](int64_t t) {
        const int64_t s = t >= 0 && t < a.n_tokens ? a.slots[t] : -1;
        return s >= 0 && s < a.n_slots ? s : int64_t(-1);
    };
    const int64_t mine = slot_at(t0 + lane), before = lane < kWindow8 ? slot_at(t0 - kWindow8 + lane) : -1;
    const int64_t block = mine >= 0 ? mine / kBlock8 : -1;
    int64_t* blocks = block_of[tid / 32] + kWindow8;
    blocks[lane] = block;
    if (lane < kWindow8) blocks[lane - kWindow8] = before >= 0 ? before / kBlock8 : -1;
    __syncwarp();
    int head = lane;
#pragma unroll
    for (int d = 1; d < kBlock8; ++d)
        if (blocks[lane - d] == block) head = lane - d;
    const uint32_t begun = __ballot_sync(all, mine >= 0 && head == lane && lane < kWindow8);
    if (begun == 0) return;  // (the CTA as a whole)
    const bool own = mine >= 0 && head >= 0 && head < kWindow8;
    const int64_t exp_at = block * Hk + g;
    const int was = own ? exp_of_byte(exps[exp_at]) : 0;
    const uint32_t owned = __ballot_sync(all, own);
    if (tid < 32 && own) atomicOr(&run_places[head], 1u << (mine & (kBlock8 - 1)));

    // this thread's rows: tokens `row` of each pass; a warp's rows of a pass that are none of the CTA's are left out together
    auto token = [&](int i) { return row + i * kRows; };
    auto is_own = [&](int i) { return token(i) < 2 * kWindow8 && (owned >> token(i) & 1u) != 0; };
    auto any_own = [&](int i) { return __any_sync(all, is_own(i)); };
    float x[kPasses][E];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        if (is_own(i) && token(i) < kWindow8 && i == 0) {
            unpack_row<E / 2>(early[0], x[i]);
            unpack_row<E / 2>(early[1], x[i] + E / 2);
        } else if (is_own(i)) {
            load_row<E / 2>(row_at(token(i)) + at.e0, x[i]);
            load_row<E / 2>(row_at(token(i)) + at.e1, x[i] + E / 2);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] = 0.0f;
        }
    }
    const float limit = kCodeMost * pow2i(kExpMost);
    bool odd[kPasses] = {};
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        if (!any_own(i)) continue;
        if (is_k) {
            float c[E / 2], s[E / 2];
            if (is_own(i)) angles(std::true_type{}, t0 + token(i), i == 0 && token(i) < kWindow8 ? early_pos : a.positions[t0 + token(i)], c, s);
            norm_turn<D, NB, E>(x[i], a.k_gamma, a.eps, at, c, s);
        }
        // (zero times an infinity or NaN is NaN: elements that become NaN codes are looked for one by one only then)
        float m = 0.0f;
        float2 zeros = make_float2(0, 0);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            m = fmaxf(m, fmaxf(fabsf(x[i][e]), fabsf(x[i][e + 1])));
            zeros = fma2(make_float2(x[i][e], x[i][e + 1]), make_float2(0, 0), zeros);
        }
        odd[i] = !(m <= limit) || zeros.x + zeros.y != 0.0f;
        if (odd[i]) {
            m = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) m = fabsf(x[i][e]) <= limit ? fmaxf(m, fabsf(x[i][e])) : m;
        }
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(all, m, o));
        const int h = __shfl_sync(all, head, token(i) & 31);
        if (u == 0 && is_own(i)) atomicMax(&run_top[h], __float_as_uint(m));  // (magnitudes compare as their bits do)
    }
    __syncthreads();
    // the blocks' exponents, in the lanes of their tokens
    const uint32_t bits = own ? run_top[head] : 0, places = own ? run_places[head] : 0;
    // 448 = 1.75 * 2^8: the least e with the maximum <= 448 * 2^e by its exponent and mantissa
    const int need = int(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    const int now = max(places & 1u ? -kExpMost : was, min(max(need, -kExpMost), kExpMost));
    if (tid < 32 && (begun >> lane & 1u)) exps[exp_at] = uint8_t(now + kExpBias);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        if (!any_own(i)) continue;
        const float unit = pow2i(-__shfl_sync(all, now, token(i) & 31));
        const int64_t slot = __shfl_sync(all, mine, token(i) & 31);
        if (!is_own(i)) continue;
        uint32_t w[E / 4];
        const float2 unit2 = make_float2(unit, unit);
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const float2 y = mul2(make_float2(x[i][e], x[i][e + 1]), unit2), z = mul2(make_float2(x[i][e + 2], x[i][e + 3]), unit2);
            w[e / 4] = codes_of(y.x, y.y) | codes_of(z.x, z.y) << 16;
        }
        if (odd[i]) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (!(fabsf(x[i][e]) <= limit)) w[e / 4] = (w[e / 4] & ~(0xFFu << (8 * (e & 3)))) | 0x7Fu << (8 * (e & 3));
        }
        uint8_t* to = codes + (slot * Hk + g) * D;
        if constexpr (E == 16) {
            *reinterpret_cast<uint2*>(to + at.e0) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2*>(to + at.e1) = make_uint2(w[2], w[3]);
        } else {
            *reinterpret_cast<uint32_t*>(to + at.e0) = w[0];
            *reinterpret_cast<uint32_t*>(to + at.e1) = w[1];
        }
    }
    // the other places of the blocks: zeros in a block that starts anew, re-encoded where the exponent grew
    __syncwarp();
    const bool more = (begun >> lane & 1u) && places != 0xFFFFu && ((places & 1u) || now > was);
    for (uint32_t left = __ballot_sync(all, more); left != 0; left &= left - 1) {
        const int h = __ffs(left) - 1;
        const int64_t first = __shfl_sync(all, block, h) * kBlock8;
        const uint32_t written = __shfl_sync(all, places, h);
        const float by = pow2i(max(__shfl_sync(all, was - now, h), -126));  // (of a block that starts anew it is not used)
        for (int place = row; place < kBlock8; place += kRows) {
            if (written >> place & 1u) continue;
            uint2* to = reinterpret_cast<uint2*>(codes + ((first + place) * Hk + g) * D + u * E);
#pragma unroll
            for (int k = 0; k < E / 8; ++k) {
                if (written & 1u) {
                    to[k] = make_uint2(0u, 0u);
                    continue;
                }
                uint32_t w[2] = {to[k].x, to[k].y};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t lo, hi;
                    codes_to_f16x4(w[i], lo, hi);
                    const float2 f0 = __half22float2(*reinterpret_cast<__half2*>(&lo)), f1 = __half22float2(*reinterpret_cast<__half2*>(&hi));
                    w[i] = codes_of(f0.x * by, f0.y * by) | codes_of(f1.x * by, f1.y * by) << 16;
                }
                to[k] = make_uint2(w[0], w[1]);
            }
        }
    }
}

// ------------------------------------------------------------------ rows of the cache as bf16
// HBM bounds it. A thread takes 16 codes of a key row and of a value row: 32 bytes in, 64 out.
constexpr int kReadThreads = 256;

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

__global__ void __launch_bounds__(kReadThreads) paged_codes_read_kernel(const __grid_constant__ Read8Args p, int rounds, int log_d) {
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int Hk = p.n_kv_heads, per = (Hk << log_d) / 16;  // chunks of a row
    const int64_t chunks = p.n_rows * per, c0 = int64_t(blockIdx.x) * (kReadThreads * rounds);
    // (a CTA's first row by a division of 64 bits, the rest by ones of 32)
    const int64_t r0 = c0 / per;
    const int first = int(c0 - r0 * per), n = int(min(int64_t(kReadThreads * rounds), chunks - c0));
    for (int i = threadIdx.x; i < n; i += kReadThreads) {
        const int r = (first + i) / per, c = first + i - r * per;
        const int64_t slot = p.slots[r0 + r];
        uint4 k[2] = {}, v[2] = {};
        if (slot >= 0 && slot < p.n_slots) {
            read16(p.k_codes, p.k_exp, slot, Hk, c, log_d, k);
            read16(p.v_codes, p.v_exp, slot, Hk, c, log_d, v);
        }
        uint4* ko = reinterpret_cast<uint4*>(p.k_out) + 2 * (c0 + i);
        uint4* vo = reinterpret_cast<uint4*>(p.v_out) + 2 * (c0 + i);
        ko[0] = k[0];
        ko[1] = k[1];
        vo[0] = v[0];
        vo[1] = v[1];
    }
}

template <int D, int E>
const void* store_kernel(bool neighbours) {
    return neighbours ? reinterpret_cast<const void*>(paged_codes_store_kernel<D, true, E>) : reinterpret_cast<const void*>(paged_codes_store_kernel<D, false, E>);
}

}  // namespace

cudaError_t launch_paged8_store(const Store8Args& a, cudaStream_t s) {
    Store8Params p;
    p.a = a;
    const int each = a.rot_dim % 16 == 0 ? 16 : 8, rows = kStoreThreads / (a.head_dim / each);
    const int64_t kv_ctas = (a.n_tokens + kWindow8 - 1) / kWindow8 * a.n_kv_heads * 2, sms = std::max(1, device_sm_count());
    // A thread takes up to eight heads of its token, so that its angles serve them all: fewer where that leaves SMs without work;
    // few tokens leave rows for more heads at once.
    p.log_tokens = 0;
    while ((2 << p.log_tokens) <= std::min(rows, 16) && (int64_t(1) << p.log_tokens) < a.n_tokens) ++p.log_tokens;
    const int64_t tokens = ((a.n_tokens - 1) >> p.log_tokens) + 1, side = rows >> p.log_tokens;  // heads side by side
    auto groups = [&](int64_t rounds) { return (a.n_heads + side * rounds - 1) / (side * rounds); };
    p.rounds = int(std::min<int64_t>(kMostRounds, (a.n_heads + side - 1) / side));
    while (p.rounds > 2 && tokens * groups(p.rounds) < 6 * sms) p.rounds = (p.rounds + 1) / 2;
    p.head_groups = int(groups(p.rounds));
    const int64_t q_ctas = tokens * p.head_groups;
    if (q_ctas + kv_ctas > 2147483647) return cudaErrorInvalidValue;
    p.kv_ctas = int(kv_ctas);
    void* args[] = {&p};
    const bool nb = a.neighbours;
    const void* fn = each == 16 ? (a.head_dim == 64 ? store_kernel<64, 16>(nb) : a.head_dim == 128 ? store_kernel<128, 16>(nb) : store_kernel<256, 16>(nb))
                                : (a.head_dim == 64 ? store_kernel<64, 8>(nb) : a.head_dim == 128 ? store_kernel<128, 8>(nb) : store_kernel<256, 8>(nb));
    return launch_serialised(fn, unsigned(q_ctas + kv_ctas), kStoreThreads, 0, s, args);
}

cudaError_t launch_paged8_read(const Read8Args& a, cudaStream_t s) {
    Read8Args p = a;
    int log_d = 0;
    while ((1 << log_d) < a.head_dim) ++log_d;
    const int64_t chunks = a.n_rows * (int64_t(a.n_kv_heads) * a.head_dim / 16);
    // several rounds where that leaves every SM its eight CTAs (25 MB 7 us, with four rounds 13; 830 MB 134 and 129)
    int rounds = chunks >= int64_t(kReadThreads) * 4 * 8 * std::max(1, device_sm_count()) ? 4 : 1;
    const int64_t each = int64_t(kReadThreads) * rounds, grid = (chunks + each - 1) / each;
    if (grid > 2147483647) return cudaErrorInvalidValue;
    void* args[] = {&p, &rounds, &log_d};
    return launch_serialised(reinterpret_cast<const void*>(paged_codes_read_kernel), unsigned(grid), kReadThreads, 0, s, args);
}

}  // namespace emb
