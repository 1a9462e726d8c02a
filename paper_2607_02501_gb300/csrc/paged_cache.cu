// What fills a paged key/value cache: the step's block table, slots and positions from the
// requests' lengths, and the pass that normalises and rotates queries and keys and stores keys and
// values in their slots.
//
// Both kernels are launched with programmatic stream serialisation and read device memory only
// after griddepcontrol.wait, with ordinary loads.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>

#include "paged.cuh"

namespace emb {
namespace {

// ------------------------------------------------------------------ block table, slots, positions
// One launch. A CTA takes 1024 tokens and a share of the requests. Its threads scan all the
// requests' new tokens and new pages (a thread a run of requests, then shuffles), so no CTA waits for
// another; a request that overlaps the CTA's tokens leaves its numbers in shared memory at its first token
// there, and a maximum scan over those marks gives every token its request. A new page's table entry is written by
// the token at the page's start, which is always new. Latency bounds it: two dependent loads, two scans (50 tokens of one
// request 2.9 to 3.2 us, 500 of 1000 requests 4.7 to 5.0, 417000 of 512 requests, 5 MB written, 6.5).
constexpr int kSlotTokens = 1024;

struct PageDiv {
    uint32_t size;
    int shift;  // log2(size), or -1
    __device__ uint32_t div(uint32_t x) const { return shift >= 0 ? x >> shift : x / size; }
};

__device__ __forceinline__ uint32_t warp_scan(uint32_t v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

template <int NT>  // threads
__global__ void __launch_bounds__(NT) paged_slots_kernel(const __grid_constant__ SlotArgs p, PageDiv pd) {
    constexpr int kPer = kSlotTokens / NT;  // consecutive tokens of a thread
    // of the request whose first token of this CTA is token i: (request, position - token, last token + 1,
    // pages it had, index of its page 0 in the free list)
    __shared__ int mark[kSlotTokens];
    __shared__ uint32_t s_req[kSlotTokens], s_base[kSlotTokens], s_end[kSlotTokens], s_have[kSlotTokens], s_first[kSlotTokens];
    __shared__ uint32_t sum_a[NT / 32], sum_n[NT / 32];
    __shared__ int top[NT / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    ptx::griddep_launch_dependents();
#pragma unroll
    for (int i = 0; i < kPer; ++i) mark[tid * kPer + i] = 0;
    ptx::griddep_wait();
    const uint32_t used = uint32_t(*p.used);

    const uint32_t max_pages = uint32_t(p.max_pages);
    auto pages = [&](uint32_t n) {  // pages of n tokens
        const uint32_t full = pd.div(n);
        return min(full + (full * pd.size != n), max_pages);
    };
    const int per = (p.n_req + NT - 1) / NT;
    const int r0 = min(p.n_req, tid * per), r1 = min(p.n_req, r0 + per);
    uint32_t a_sum = 0, n_sum = 0;
    for (int r = r0; r < r1; ++r) {
        const uint32_t c = uint32_t(max(0, p.cached[r])), a = uint32_t(max(0, p.added[r]));
        a_sum += a;
        n_sum += pages(c + a) - pages(c);
    }
    const uint32_t a_in = warp_scan(a_sum, lane), n_in = warp_scan(n_sum, lane);
    if (lane == 31) {
        sum_a[warp] = a_in;
        sum_n[warp] = n_in;
    }
    __syncthreads();
    uint32_t start = a_in - a_sum, first = used + n_in - n_sum;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w)
        if (w < warp) {
            start += sum_a[w];
            first += sum_n[w];
        }
    if (blockIdx.x == 0 && tid == NT - 1) {
        p.q_start[p.n_req] = int32_t(start + a_sum);
        *p.used_out = int32_t(first + n_sum);
    }

    const int64_t t0 = int64_t(blockIdx.x) * kSlotTokens;
    const int64_t t1 = min(p.n_tokens, t0 + kSlotTokens);
    const int w0 = int(int64_t(p.n_req) * blockIdx.x / gridDim.x), w1 = int(int64_t(p.n_req) * (blockIdx.x + 1) / gridDim.x);
    for (int r = r0; r < r1; ++r) {
        const uint32_t c = uint32_t(max(0, p.cached[r])), a = uint32_t(max(0, p.added[r]));
        const uint32_t have = pages(c), want = pages(c + a);
        if (r >= w0 && r < w1) {
            p.q_start[r] = int32_t(start);
            p.kv_len[r] = int32_t(c + a);
        }
        const int64_t end = int64_t(start) + a;
        if (a > 0 && start < t1 && end > t0) {
            const int at = start <= t0 ? 0 : int(start - t0);
            mark[at] = at + 1;
            s_req[at] = uint32_t(r);
            s_base[at] = c - start;
            s_end[at] = uint32_t(end);
            s_have[at] = have;
            s_first[at] = first - have;
        }
        start += a;
        first += want - have;
    }
    __syncthreads();

    int m[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        m[i] = mark[tid * kPer + i];
        if (i > 0) m[i] = max(m[i], m[i - 1]);
    }
    int incl = m[kPer - 1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl = max(incl, u);
    }
    if (lane == 31) top[warp] = incl;
    int before = __shfl_up_sync(0xffffffffu, incl, 1);
    if (lane == 0) before = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 32; ++w)
        if (w < warp) before = max(before, top[w]);

    int64_t slot[kPer];
    int32_t pos[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int64_t t = t0 + tid * kPer + i;
        const int at = max(m[i], before) - 1;
        slot[i] = -1;
        pos[i] = 0;
        if (t >= t1 || at < 0 || t >= int64_t(s_end[at])) continue;
        const uint32_t ps = s_base[at] + uint32_t(t);
        pos[i] = int32_t(ps);
        const uint32_t pg = pd.div(ps), in = ps - pg * pd.size;
        if (pg >= max_pages) continue;
        int32_t page;
        if (pg >= s_have[at]) {
            const uint32_t k = s_first[at] + pg;
            page = int64_t(k) < p.n_free ? p.free_pages[k] : -1;
            if (in == 0) p.table[int64_t(s_req[at]) * p.max_pages + pg] = page;
        } else {
            page = p.table[int64_t(s_req[at]) * p.max_pages + pg];
        }
        if (page >= 0) slot[i] = int64_t(page) * pd.size + in;
    }
    const int64_t t = t0 + tid * kPer;
    if constexpr (kPer == 4) {
        if (t + kPer <= t1 && ((uintptr_t(p.slots) | uintptr_t(p.positions)) & 15) == 0) {
            *reinterpret_cast<longlong2*>(p.slots + t) = make_longlong2(slot[0], slot[1]);
            *reinterpret_cast<longlong2*>(p.slots + t + 2) = make_longlong2(slot[2], slot[3]);
            *reinterpret_cast<int4*>(p.positions + t) = make_int4(pos[0], pos[1], pos[2], pos[3]);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (t + i < t1) {
            p.slots[t + i] = slot[i];
            p.positions[t + i] = pos[i];
        }
}

// ------------------------------------------------------------------ norm, rotation, cache write
// HBM bounds it: every element is read and written once. CTAs stay and take items in turn, an item being a run of rows
// (heads of queries, then of keys, then of values) of a few tokens. A ring of three items in shared memory is filled by
// bulk copies and written out by bulk copies, both by a warp of their own, so what is on its way needs no registers and
// holds nobody up; values pass through untouched. In between four warps turn the rows in place: 2^n lanes to a row, each with VEC elements of the first half and
// the VEC that they are paired with, so the rotation stays within the thread and the sum of squares takes n shuffles.
// Elements behind the rotated ones are paired likewise and turned by nothing. A token's cosines and sines are formed once
// for all heads.
// Angles are counted in turns: the host passes frequency / 2 pi as two floats, position times that is formed with one
// exact FMA residual, and its fraction goes to the hardware's sine and cosine, whose error in +-pi is below 2^-21.
// Measured (us): 16000 tokens of 10 heads of 256 (164 MB) 30.9, 78 % of the measured copy rate; 816 of 48 heads of 128
// (20 MB, three axes, norms) 7.5; one token of 10 heads of 128 2.8. Rows through registers, angles by sincosf for every CTA
// of a few tokens took 72, 11 and 2.8; with the copies issued by one of the computing warps 43 and 8.7; CTAs of eight
// computing warps and 24 KB items, two per SM, 33.5, 7.9 and 2.8.
constexpr int kQkWarps = 4;  // that compute; one more copies
constexpr int kQkCompute = 32 * kQkWarps, kQkThreads = kQkCompute + 32;
constexpr int kQkMaxPairs = 128;
constexpr int kQkMaxTokens = 16;  // of an item
constexpr int kQkStages = 3;
constexpr int kQkItemBytes = 12 * 1024;  // of rows, at most
constexpr int kQkCtas = 4;               // per SM

struct QkParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const float* q_gamma;
    const float* k_gamma;
    const int32_t* positions;
    const int64_t* slots;
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_cache;
    __nv_bfloat16* v_cache;
    int64_t q_stride, k_stride, v_stride, pos_stride, n_tokens, n_slots, items;
    int H, Hk, d, half;        // half: rotated pairs of a head
    int tokens, run, runs;     // an item's tokens and rows of a token; runs of a token
    int axes, log_lanes;       // a row's lanes are 2^log_lanes
    float eps;
    alignas(16) float turn_hi[kQkMaxPairs];  // frequency / 2 pi
    alignas(16) float turn_lo[kQkMaxPairs];
    alignas(16) uint8_t axis[kQkMaxPairs];
};
constexpr int kQkHeadBytes = 64 + kQkStages * kQkMaxTokens * (8 + 4 * 4) + 2 * kQkMaxPairs * 4 + kQkMaxPairs;  // 16-byte multiple

template <int VEC>
struct alignas(2 * VEC) QkVec {
    __nv_bfloat16 v[VEC];
};

// The fraction of at * (hi + lo) turns where the residual is turns by itself (far positions, a base below one). Called,
// not inlined: as predicated instructions the few fp64 operations cost every position.
__device__ __noinline__ float far_turn(int32_t at, float hi, float lo) {
    const double t = double(at) * (double(hi) + double(lo));
    return float(t - rint(t));
}
// Cosine and sine of 2 pi * at * (hi + lo).
__device__ __forceinline__ void turn_sincos(int32_t at, float hi, float lo, float& c, float& s) {
    const float pos = float(at), T = __fmul_rn(pos, hi);
    float frac;
    if (fabsf(T) < 1048576.0f && fabsf(pos) < 16777216.0f) {
        frac = (T - rintf(T)) + fmaf(pos, lo, fmaf(pos, hi, -T));
    } else {
        frac = far_turn(at, hi, lo);
    }
    __sincosf(frac * 6.283185307179586f, &s, &c);
}

__device__ __forceinline__ float2 pair_of(const QkVec<2>& v) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&v);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
// VEC numbers of unit u, kept as [VEC / 4][units][4]: neighbouring lanes' loads lie side by side.
template <int VEC>
__device__ __forceinline__ void load_unit(const float* p, int u, int units, float2 (&v)[VEC / 2]) {
#pragma unroll
    for (int e = 0; e < VEC; e += 4)
        *reinterpret_cast<float4*>(&v[e / 2]) = *reinterpret_cast<const float4*>(p + ((e >> 2) * units + u) * 4);
}
template <int VEC>
__device__ __forceinline__ int unit_place(int i, int units) {  // of number i in that order
    const int u = i / VEC, e = i % VEC;
    return ((e >> 2) * units + u) * 4 + (e & 3);
}

template <int VEC>
__global__ void __launch_bounds__(kQkThreads, kQkCtas) qk_norm_rope_kernel(const __grid_constant__ QkParams p, int* status) {
    extern __shared__ __align__(128) uint8_t sm[];
    uint64_t* full = reinterpret_cast<uint64_t*>(sm);                               // [stages]
    uint64_t* done = full + kQkStages;                                              // [stages]
    int* abort_flag = reinterpret_cast<int*>(done + kQkStages);
    int64_t* slot_of = reinterpret_cast<int64_t*>(sm + 64);                         // [stages][tokens]
    int32_t* pos_of = reinterpret_cast<int32_t*>(slot_of + kQkStages * kQkMaxTokens);  // [stages][4][tokens]
    float* turn_hi = reinterpret_cast<float*>(pos_of + kQkStages * 4 * kQkMaxTokens);
    float* turn_lo = turn_hi + kQkMaxPairs;
    uint8_t* axis_of = reinterpret_cast<uint8_t*>(turn_lo + kQkMaxPairs);
    float* gam = reinterpret_cast<float*>(sm + kQkHeadBytes);                       // [q, k][first, second of the pairs][d / 2]
    float* cs = gam + 2 * p.d;                                                      // [2][cos, sin][tokens][half]
    const int cs_size = p.tokens * p.half;
    uint8_t* ring = reinterpret_cast<uint8_t*>(cs + 4 * cs_size);
    const int tid = threadIdx.x;
    const uint32_t row_bytes = uint32_t(p.d) * 2, token_bytes = row_bytes * p.run, stage_bytes = token_bytes * p.tokens;

    if (tid < kQkMaxPairs / 4) {
        reinterpret_cast<float4*>(turn_hi)[tid] = reinterpret_cast<const float4*>(p.turn_hi)[tid];
        reinterpret_cast<uint32_t*>(axis_of)[tid] = reinterpret_cast<const uint32_t*>(p.axis)[tid];
    } else if (tid < kQkMaxPairs / 2) {
        const int i = tid - kQkMaxPairs / 4;
        reinterpret_cast<float4*>(turn_lo)[i] = reinterpret_cast<const float4*>(p.turn_lo)[i];
    } else if (tid == kQkCompute) {
        for (int i = 0; i < kQkStages; ++i) {
            ptx::mbar_init(&full[i], 1 + 32);  // the rows, and the copy warp's lanes with slots and positions
            ptx::mbar_init(&done[i], kQkWarps);
        }
        *abort_flag = 0;
        ptx::fence_mbar_init();
    }
    ptx::griddep_launch_dependents();
    __syncthreads();
    ptx::griddep_wait();

    // Item `item`: tokens t0 .. t0 + nt - 1, rows h0 .. h1 - 1 of each. A token's part in the ring is its rows in order.
    struct Item {
        int64_t t0;
        int nt, h0, h1;
    };
    auto item_at = [&](int64_t item) {
        Item I;
        const int64_t group = p.runs == 1 ? item : item / p.runs;
        I.t0 = group * p.tokens;
        I.nt = int(min(int64_t(p.tokens), p.n_tokens - I.t0));
        I.h0 = int(item - group * p.runs) * p.run;
        I.h1 = min(I.h0 + p.run, p.H + 2 * p.Hk);
        return I;
    };
    const int64_t step = gridDim.x;

    if (tid >= kQkCompute) {
        // -------------------------------------------------------------------------- copies, a lane a token
        const int lane = tid - kQkCompute;
        // an item's rows of queries, keys and values: [lo, hi) counted from the kind's first head
        struct Part {
            int lo, hi;
        };
        auto part = [&](const Item& I, int first, int count) { return Part{max(I.h0 - first, 0), min(I.h1 - first, count)}; };
        auto fill = [&](int64_t item, int st) {  // rows into a stage, and the token's slot and positions beside it
            const Item I = item_at(item);
            if (lane == 0) ptx::mbar_arrive_expect_tx(&full[st], uint32_t(I.nt * (I.h1 - I.h0)) * row_bytes);
            __syncwarp();
            if (lane < I.nt) {
                const int64_t t = I.t0 + lane;
                uint8_t* to = ring + st * stage_bytes + lane * token_bytes;
                const Part q = part(I, 0, p.H), k = part(I, p.H, p.Hk), v = part(I, p.H + p.Hk, p.Hk);
                if (q.lo < q.hi) ptx::bulk_load(to, p.q + t * p.q_stride + q.lo * p.d, uint32_t(q.hi - q.lo) * row_bytes, &full[st]);
                if (k.lo < k.hi)
                    ptx::bulk_load(to + (p.H + k.lo - I.h0) * row_bytes, p.k + t * p.k_stride + k.lo * p.d, uint32_t(k.hi - k.lo) * row_bytes, &full[st]);
                if (v.lo < v.hi)
                    ptx::bulk_load(to + (p.H + p.Hk + v.lo - I.h0) * row_bytes, p.v + t * p.v_stride + v.lo * p.d, uint32_t(v.hi - v.lo) * row_bytes, &full[st]);
                ptx::async_copy<8>(slot_of + st * kQkMaxTokens + lane, p.slots + t);
                for (int a = 0; a < p.axes; ++a)
                    ptx::async_copy<4>(pos_of + (st * 4 + a) * kQkMaxTokens + lane, p.positions + a * p.pos_stride + t);
            }
            ptx::async_copy_arrive(&full[st]);
        };
        auto drain = [&](const Item& I, int st) {  // and out of it
            if (lane < I.nt) {
                const int64_t t = I.t0 + lane, slot = slot_of[st * kQkMaxTokens + lane];
                const uint8_t* from = ring + st * stage_bytes + lane * token_bytes;
                const Part q = part(I, 0, p.H), k = part(I, p.H, p.Hk), v = part(I, p.H + p.Hk, p.Hk);
                if (q.lo < q.hi) ptx::bulk_store(p.q_out + (t * p.H + q.lo) * p.d, from, uint32_t(q.hi - q.lo) * row_bytes);
                if (slot >= 0 && slot < p.n_slots) {
                    if (k.lo < k.hi)
                        ptx::bulk_store(p.k_cache + (slot * p.Hk + k.lo) * p.d, from + (p.H + k.lo - I.h0) * row_bytes, uint32_t(k.hi - k.lo) * row_bytes);
                    if (v.lo < v.hi)
                        ptx::bulk_store(p.v_cache + (slot * p.Hk + v.lo) * p.d, from + (p.H + p.Hk + v.lo - I.h0) * row_bytes, uint32_t(v.hi - v.lo) * row_bytes);
                }
                ptx::bulk_commit();
            }
        };
        ptx::fence_proxy_async_global();  // (the rows were written by ordinary stores)
        uint32_t fills = 0;
        for (; fills < kQkStages && blockIdx.x + fills * step < p.items; ++fills) fill(blockIdx.x + fills * step, int(fills));
        uint32_t n = 0;
        for (int64_t item = blockIdx.x; item < p.items; item += step, ++n) {
            const int st = int(n % kQkStages);
            ptx::mbar_wait(&done[st], (n / kQkStages) & 1, abort_flag, status, kWaitLimitNs);
            __syncwarp();
            if (__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(abort_flag) != 0)) {
                // a wait gave up: what is still on its way into shared memory lands before the CTA leaves
                for (uint32_t i = n; i < fills; ++i)
                    ptx::mbar_wait(&full[i % kQkStages], (i / kQkStages) & 1, nullptr, status, kWaitLimitNs);
                break;
            }
            drain(item_at(item), st);
            // the item before this one has left its stage (its copies were given an item's time): it is filled again
            const int64_t ahead = item + (kQkStages - 1) * step;
            if (n > 0 && ahead < p.items) {
                ptx::bulk_wait_read<1>();
                __syncwarp();
                fill(ahead, int(fills++ % kQkStages));
            }
        }
        ptx::bulk_wait_all();
        return;
    }

    // ------------------------------------------------------------------------------ norm and rotation
    // (a wait that gave up sets the abort flag; the loop runs on, so that every barrier meets its threads)
    const int lanes = 1 << p.log_lanes, u = tid & (lanes - 1), pass = kQkCompute >> p.log_lanes;
    const int units = p.d / (2 * VEC);
    // the lane's elements: first and second of its pairs
    const int turned = p.half / VEC, rot = 2 * p.half;
    const int e0 = u < turned ? u * VEC : rot + (u - turned) * VEC;
    const int e1 = u < turned ? p.half + u * VEC : e0 + (p.d - rot) / 2;
    for (int i = tid; i < p.d; i += kQkCompute) {
        // element i is number `at` of the first or second halves of the pairs
        const int in = i < rot ? i : i - rot, len = i < rot ? p.half : (p.d - rot) / 2;
        const int second = in >= len, at = (i < rot ? 0 : p.half) + (second ? in - len : in);
        float* to = gam + second * (p.d / 2) + unit_place<VEC>(at, units);
        if (p.q_gamma) to[0] = p.q_gamma[i];
        if (p.k_gamma) to[p.d] = p.k_gamma[i];
    }
    uint32_t n = 0;
    for (int64_t item = blockIdx.x; item < p.items; item += step, ++n) {
        const int st = int(n % kQkStages);
        const Item I = item_at(item);
        float* cosv = cs + (n & 1) * 2 * cs_size;  // (used two items ago: a barrier lies between)
        float* sinv = cosv + cs_size;
        ptx::mbar_wait(&full[st], (n / kQkStages) & 1, abort_flag, status, kWaitLimitNs);
        const int per = min(I.h1, p.H + p.Hk) - I.h0, rows = max(per, 0) * I.nt;  // of queries and keys
        if (rows > 0)
            for (int i = tid; i < I.nt * p.half; i += kQkCompute) {
                const int tt = i / p.half, j = i - tt * p.half, to = tt * p.half + unit_place<VEC>(j, turned);
                turn_sincos(pos_of[(st * 4 + axis_of[j]) * kQkMaxTokens + tt], turn_hi[j], turn_lo[j], cosv[to], sinv[to]);
            }
        asm volatile("bar.sync 1, %0;" ::"n"(kQkCompute) : "memory");
        for (int base = 0; base < rows; base += pass) {
            const int row = base + (tid >> p.log_lanes);
            const bool live = row < rows && u < units;
            const int tt = live ? row / per : 0, h = live ? row - tt * per : 0;
            __nv_bfloat16* x = reinterpret_cast<__nv_bfloat16*>(ring + st * stage_bytes + tt * token_bytes + h * row_bytes);
            QkVec<VEC>* pa = reinterpret_cast<QkVec<VEC>*>(x + e0);
            QkVec<VEC>* pb = reinterpret_cast<QkVec<VEC>*>(x + e1);
            const bool is_q = I.h0 + h < p.H, norm = is_q ? p.q_gamma != nullptr : p.k_gamma != nullptr;
            float2 xa[VEC / 2], xb[VEC / 2];
            if (live) {
                const QkVec<VEC> a = *pa, b = *pb;
#pragma unroll
                for (int e = 0; e < VEC / 2; ++e) {
                    xa[e] = pair_of(reinterpret_cast<const QkVec<2>*>(&a)[e]);
                    xb[e] = pair_of(reinterpret_cast<const QkVec<2>*>(&b)[e]);
                }
            }
            if (p.q_gamma || p.k_gamma) {
                float ss = 0.0f;
                if (live) {
                    float2 s2 = make_float2(0, 0);
#pragma unroll
                    for (int e = 0; e < VEC / 2; ++e) s2 = fma2(xb[e], xb[e], fma2(xa[e], xa[e], s2));
                    ss = s2.x + s2.y;
                }
                __syncwarp();
                for (int o = lanes >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                if (live && norm) {
                    const float inv = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, float(p.d)), p.eps)));
                    const float2 inv2 = make_float2(inv, inv);
                    float2 ga[VEC / 2], gb[VEC / 2];
                    load_unit<VEC>(gam + (is_q ? 0 : p.d), u, units, ga);
                    load_unit<VEC>(gam + (is_q ? 0 : p.d) + p.d / 2, u, units, gb);
#pragma unroll
                    for (int e = 0; e < VEC / 2; ++e) {
                        xa[e] = mul2(mul2(xa[e], inv2), ga[e]);
                        xb[e] = mul2(mul2(xb[e], inv2), gb[e]);
                    }
                }
            }
            if (!live) continue;
            if (u < turned) {
                float2 c[VEC / 2], s[VEC / 2];
                load_unit<VEC>(cosv + tt * p.half, u, turned, c);
                load_unit<VEC>(sinv + tt * p.half, u, turned, s);
#pragma unroll
                for (int e = 0; e < VEC / 2; ++e) {
                    const float2 bs = mul2(xb[e], s[e]);
                    const float2 y = fma2(xa[e], c[e], make_float2(-bs.x, -bs.y));
                    xb[e] = fma2(xb[e], c[e], mul2(xa[e], s[e]));
                    xa[e] = y;
                }
            }
            QkVec<VEC> oa, ob;
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) {
                reinterpret_cast<__nv_bfloat162*>(&oa)[e] = __floats2bfloat162_rn(xa[e].x, xa[e].y);
                reinterpret_cast<__nv_bfloat162*>(&ob)[e] = __floats2bfloat162_rn(xb[e].x, xb[e].y);
            }
            *pa = oa;
            *pb = ob;
        }
        ptx::fence_proxy_async_smem();  // the rows, before they are copied out
        __syncwarp();
        if ((tid & 31) == 0) ptx::mbar_arrive(&done[st]);
    }
}

// The opt-in shared-memory size is a per-device function attribute.
template <int VEC>
cudaError_t qk_shared_memory() {
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
    e = cudaFuncSetAttribute(qk_norm_rope_kernel<VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, 110 * 1024);
    if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
    return e;
}

}  // namespace

cudaError_t launch_paged_slots(const SlotArgs& a, cudaStream_t s) {
    SlotArgs p = a;
    PageDiv pd{uint32_t(a.page_size), -1};
    for (int i = 0; i <= 16; ++i)
        if (a.page_size == 1 << i) pd.shift = i;
    void* args[] = {&p, &pd};
    const int64_t blocks = std::max<int64_t>(1, (a.n_tokens + kSlotTokens - 1) / kSlotTokens);
    // a thread a token while one CTA does, four in many CTAs
    if (blocks == 1 && (a.n_tokens > 256 || a.n_req > 256))
        return launch_serialised(reinterpret_cast<const void*>(paged_slots_kernel<1024>), 1, 1024, 0, s, args);
    return launch_serialised(reinterpret_cast<const void*>(paged_slots_kernel<256>), unsigned(blocks), 256, 0, s, args);
}

cudaError_t launch_qk_norm_rope(const QkArgs& a, cudaStream_t s) {
    QkParams p;
    p.q = reinterpret_cast<const __nv_bfloat16*>(a.q);
    p.k = reinterpret_cast<const __nv_bfloat16*>(a.k);
    p.v = reinterpret_cast<const __nv_bfloat16*>(a.v);
    p.q_gamma = a.q_gamma;
    p.k_gamma = a.k_gamma;
    p.positions = a.positions;
    p.slots = a.slots;
    p.q_out = reinterpret_cast<__nv_bfloat16*>(a.q_out);
    p.k_cache = reinterpret_cast<__nv_bfloat16*>(a.k_cache);
    p.v_cache = reinterpret_cast<__nv_bfloat16*>(a.v_cache);
    p.q_stride = a.q_stride;
    p.k_stride = a.k_stride;
    p.v_stride = a.v_stride;
    p.pos_stride = a.pos_stride;
    p.n_slots = a.n_slots;
    p.H = int(a.n_heads);
    p.Hk = int(a.n_kv_heads);
    p.d = int(a.head_dim);
    p.half = int(a.rot_dim / 2);
    p.eps = a.eps;
    std::memset(p.turn_hi, 0, sizeof(p.turn_hi) + sizeof(p.turn_lo) + sizeof(p.axis));
    if (p.half > 0) {
        // base^(-2i/d) / 2 pi, i = 16 j + k, from two powers by multiplication: within 32 roundings of fp64, which the two
        // floats (48 bits) do not see; a call of pow per pair takes longer than the launch
        const double fine = std::pow(double(a.base), -2.0 / double(a.rot_dim)), coarse = std::pow(double(a.base), -32.0 / double(a.rot_dim));
        double c = 1.0 / 6.283185307179586;
        for (int j = 0; 16 * j < p.half; ++j, c *= coarse) {
            double v = c;
            for (int i = 16 * j; i < std::min(16 * j + 16, p.half); ++i, v *= fine) {
                p.turn_hi[i] = float(v);
                p.turn_lo[i] = float(v - double(p.turn_hi[i]));
            }
        }
    }
    if (a.axis_of_pair) std::memcpy(p.axis, a.axis_of_pair, size_t(p.half));
    // 16-byte accesses where both halves of the pairs start on that boundary
    const int vec = p.half % 8 == 0 && (p.d - 2 * p.half) % 16 == 0 ? 8 : 4;
    const int units = p.d / (2 * vec);
    p.log_lanes = 0;
    while ((1 << p.log_lanes) < units) ++p.log_lanes;
    // as many rows and tokens to an item as its bytes allow, fewer tokens while that leaves SMs without one
    const int64_t heads = a.n_heads + 2 * a.n_kv_heads, row_bytes = a.head_dim * 2;
    const int64_t sms = std::max(1, device_sm_count()), rows = kQkItemBytes / row_bytes;
    p.run = int(std::min(heads, rows));
    p.runs = int((heads + p.run - 1) / p.run);
    p.run = int((heads + p.runs - 1) / p.runs);
    p.tokens = int(std::max<int64_t>(1, std::min<int64_t>({kQkMaxTokens, rows / p.run, a.n_tokens * p.runs / (sms * kQkCtas * 2)})));
    p.items = (a.n_tokens + p.tokens - 1) / p.tokens * p.runs;
    p.axes = int(a.n_axes);
    p.n_tokens = a.n_tokens;
    const size_t smem = kQkHeadBytes + (2 * size_t(p.d) + 4 * size_t(p.tokens) * p.half) * 4 +
                        size_t(kQkStages) * p.tokens * p.run * row_bytes;
    const void* fn = vec == 8 ? reinterpret_cast<const void*>(qk_norm_rope_kernel<8>) : reinterpret_cast<const void*>(qk_norm_rope_kernel<4>);
    const cudaError_t e = vec == 8 ? qk_shared_memory<8>() : qk_shared_memory<4>();
    if (e != cudaSuccess) return e;
    int* status = a.status;
    void* args[] = {&p, &status};
    return launch_serialised(fn, unsigned(std::min(p.items, sms * kQkCtas)), kQkThreads, smem, s, args);
}

}  // namespace emb
