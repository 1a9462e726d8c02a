// What fills a paged key/value cache: the step's block table, slots and positions from the
// requests' lengths, and the pass that normalises and rotates queries and keys and stores keys and
// values in their slots.
//
// Both kernels are launched with programmatic stream serialisation and read device memory only
// after griddepcontrol.wait, with ordinary loads.
#include <algorithm>

#include "paged.cuh"
#include "rotate.cuh"

namespace emb {
namespace {

// ------------------------------------------------------------------ block table, slots, positions
// One launch. A CTA takes 1024 tokens and a share of the requests. Its 256 threads scan all the
// requests' new tokens and new pages (a thread a run of requests, then shuffles), so no CTA waits for
// another; a request that overlaps the CTA's tokens leaves its numbers in shared memory at its first token
// there, and a maximum scan over those marks gives every token its request. A new page's table entry is written by
// the token at the page's start, which is always new. Latency bounds it: two dependent loads, two scans.
constexpr int kSlotThreads = 256;
constexpr int kSlotPer = 4;  // consecutive tokens of a thread
constexpr int kSlotTokens = kSlotThreads * kSlotPer;

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

__global__ void __launch_bounds__(kSlotThreads) paged_slots_kernel(const __grid_constant__ SlotArgs p, PageDiv pd) {
    // of the request whose first token of this CTA is token i: (request, position - token, last token + 1,
    // pages it had, index of its page 0 in the free list)
    __shared__ int mark[kSlotTokens];
    __shared__ uint32_t s_req[kSlotTokens], s_base[kSlotTokens], s_end[kSlotTokens], s_have[kSlotTokens], s_first[kSlotTokens];
    __shared__ uint32_t sum_a[kSlotThreads / 32], sum_n[kSlotThreads / 32];
    __shared__ int top[kSlotThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    ptx::griddep_launch_dependents();
#pragma unroll
    for (int i = 0; i < kSlotPer; ++i) mark[tid * kSlotPer + i] = 0;
    ptx::griddep_wait();
    const uint32_t used = uint32_t(*p.used);

    const uint32_t max_pages = uint32_t(p.max_pages);
    auto pages = [&](uint32_t n) {  // pages of n tokens
        const uint32_t full = pd.div(n);
        return min(full + (full * pd.size != n), max_pages);
    };
    const int per = (p.n_req + kSlotThreads - 1) / kSlotThreads;
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
    for (int w = 0; w < kSlotThreads / 32; ++w)
        if (w < warp) {
            start += sum_a[w];
            first += sum_n[w];
        }
    if (blockIdx.x == 0 && tid == kSlotThreads - 1) {
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

    int m[kSlotPer];
#pragma unroll
    for (int i = 0; i < kSlotPer; ++i) {
        m[i] = mark[tid * kSlotPer + i];
        if (i > 0) m[i] = max(m[i], m[i - 1]);
    }
    int incl = m[kSlotPer - 1];
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
    for (int w = 0; w < kSlotThreads / 32; ++w)
        if (w < warp) before = max(before, top[w]);

    int64_t slot[kSlotPer];
    int32_t pos[kSlotPer];
#pragma unroll
    for (int i = 0; i < kSlotPer; ++i) {
        const int64_t t = t0 + tid * kSlotPer + i;
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
    const int64_t t = t0 + tid * kSlotPer;
    if (t + kSlotPer <= t1 && ((uintptr_t(p.slots) | uintptr_t(p.positions)) & 15) == 0) {
        *reinterpret_cast<longlong2*>(p.slots + t) = make_longlong2(slot[0], slot[1]);
        *reinterpret_cast<longlong2*>(p.slots + t + 2) = make_longlong2(slot[2], slot[3]);
        *reinterpret_cast<int4*>(p.positions + t) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
        for (int i = 0; i < kSlotPer; ++i)
            if (t + i < t1) {
                p.slots[t + i] = slot[i];
                p.positions[t + i] = pos[i];
            }
    }
}

// ------------------------------------------------------------------ norm, rotation, cache write
// A CTA takes a few tokens: it forms their cosines and sines once, in shared memory, for all heads
// (a token's 40 heads share 64 of them), while the first rows are on their way. A row (one head of one token)
// belongs to 2^n lanes, each of which holds VEC elements of the row's first half and the VEC they are paired with, so
// the rotation stays within the thread and the sum of squares takes n shuffles. Elements behind the rotated ones
// are paired likewise and turned by nothing. Rows of values are copied the same way. HBM bounds it: every
// element is read and written once.
constexpr int kQkThreads = 256;
constexpr int kQkMaxPairs = 128;
constexpr int kQkMaxTokens = 16;  // of a CTA

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
    int64_t q_stride, k_stride, v_stride, pos_stride, n_tokens, n_slots;
    int H, Hk, d, half, tokens;  // half: rotated pairs of a head; tokens of a CTA
    int log_lanes;               // a row's lanes are 2^log_lanes
    float eps;
    float inv_hi[kQkMaxPairs], inv_lo[kQkMaxPairs];
    uint8_t axis[kQkMaxPairs];
};

template <int VEC>
struct alignas(2 * VEC) QkVec {
    __nv_bfloat16 v[VEC];
};

template <int VEC, int ROWS>  // ROWS: rows that a thread has in flight at once
__global__ void __launch_bounds__(kQkThreads) qk_norm_rope_kernel(const __grid_constant__ QkParams p) {
    extern __shared__ __align__(16) float sm[];
    float* gam = sm;                        // [2][d] of queries and keys
    float* cosv = gam + 2 * p.d;            // [tokens][half]
    float* sinv = cosv + p.tokens * p.half;
    float* fhi = sinv + p.tokens * p.half;  // [half]
    float* flo = fhi + p.half;
    int* axis = reinterpret_cast<int*>(flo + p.half);
    const int tid = threadIdx.x;
    ptx::griddep_launch_dependents();
    for (int i = tid; i < p.half; i += kQkThreads) {
        fhi[i] = p.inv_hi[i];
        flo[i] = p.inv_lo[i];
        axis[i] = p.axis[i];
    }
    __syncthreads();
    ptx::griddep_wait();

    const int64_t t0 = int64_t(blockIdx.x) * p.tokens;
    const int nt = int(min(int64_t(p.tokens), p.n_tokens - t0));
    const uint32_t heads = uint32_t(p.H + 2 * p.Hk), rows = heads * uint32_t(nt);
    const int lanes = 1 << p.log_lanes;
    const int u = tid & (lanes - 1), units = p.d / (2 * VEC), turned = p.half / VEC;
    const uint32_t row_in = uint32_t(tid) >> p.log_lanes, pass = uint32_t(kQkThreads) >> p.log_lanes;
    // the unit's elements: first and second of its pairs
    const int rot = 2 * p.half, tail = (p.d - rot) / 2;
    const int e0 = u < turned ? u * VEC : rot + (u - turned) * VEC;
    const int e1 = u < turned ? p.half + u * VEC : e0 + tail;

    QkVec<VEC> a[ROWS], b[ROWS];
    int64_t slot[ROWS];
    auto load = [&](uint32_t base) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const uint32_t row = base + row_in + i * pass;
            if (row >= rows || u >= units) continue;
            const uint32_t tt = row / heads, h = row - tt * heads;
            const int64_t t = t0 + tt;
            const __nv_bfloat16* x = h < uint32_t(p.H)          ? p.q + t * p.q_stride + int64_t(h) * p.d
                                     : h < uint32_t(p.H + p.Hk) ? p.k + t * p.k_stride + int64_t(h - p.H) * p.d
                                                                : p.v + t * p.v_stride + int64_t(h - p.H - p.Hk) * p.d;
            a[i] = *reinterpret_cast<const QkVec<VEC>*>(x + e0);
            b[i] = *reinterpret_cast<const QkVec<VEC>*>(x + e1);
            slot[i] = h < uint32_t(p.H) ? 0 : p.slots[t];
        }
    };
    load(0);
    for (int i = tid; i < p.d; i += kQkThreads) {
        if (p.q_gamma) gam[i] = p.q_gamma[i];
        if (p.k_gamma) gam[p.d + i] = p.k_gamma[i];
    }
    for (int i = tid; i < nt * p.half; i += kQkThreads) {
        const int tt = i / p.half, j = i - tt * p.half;
        const int32_t at = p.positions[int64_t(axis[j]) * p.pos_stride + t0 + tt];
        // at * (hi + lo) as A + a, with what a position beyond 2^24 loses in fp32
        const float pos = float(at), rest = float(int64_t(at) - int64_t(pos));
        const float A = __fmul_rn(pos, fhi[j]);
        const float r = fmaf(pos, flo[j], fmaf(pos, fhi[j], -A)) + rest * fhi[j];
        sincos_two_float<true>(A, r, cosv[i], sinv[i]);
    }
    __syncthreads();

    for (uint32_t base = 0; base < rows; base += ROWS * pass) {
        if (base > 0) load(base);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const uint32_t row = base + row_in + i * pass;
            const bool live = row < rows && u < units;
            const uint32_t tt = row / heads, h = row - tt * heads;
            const int64_t t = t0 + tt;
            const bool is_q = h < uint32_t(p.H), is_v = h >= uint32_t(p.H + p.Hk);
            float xa[VEC], xb[VEC], ss = 0.0f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                xa[e] = live ? __bfloat162float(a[i].v[e]) : 0.0f;
                xb[e] = live ? __bfloat162float(b[i].v[e]) : 0.0f;
                ss = fmaf(xa[e], xa[e], ss);
                ss = fmaf(xb[e], xb[e], ss);
            }
            if (p.q_gamma || p.k_gamma)
                for (int o = lanes >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            if (!live) continue;
            QkVec<VEC> oa = a[i], ob = b[i];
            if (!is_v) {
                if (is_q ? p.q_gamma != nullptr : p.k_gamma != nullptr) {
                    const float inv = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, float(p.d)), p.eps)));
                    const float* g = gam + (is_q ? 0 : p.d);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        xa[e] = __fmul_rn(__fmul_rn(xa[e], inv), g[e0 + e]);
                        xb[e] = __fmul_rn(__fmul_rn(xb[e], inv), g[e1 + e]);
                    }
                }
                if (u < turned) {
                    const float* c = cosv + tt * p.half + e0;
                    const float* s = sinv + tt * p.half + e0;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float ya = __fsub_rn(__fmul_rn(xa[e], c[e]), __fmul_rn(xb[e], s[e]));
                        xb[e] = __fadd_rn(__fmul_rn(xb[e], c[e]), __fmul_rn(xa[e], s[e]));
                        xa[e] = ya;
                    }
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    oa.v[e] = __float2bfloat16_rn(xa[e]);
                    ob.v[e] = __float2bfloat16_rn(xb[e]);
                }
            }
            __nv_bfloat16* y;
            if (is_q) {
                y = p.q_out + (t * p.H + h) * int64_t(p.d);
            } else {
                if (slot[i] < 0 || slot[i] >= p.n_slots) continue;
                y = is_v ? p.v_cache + (slot[i] * p.Hk + (h - p.H - p.Hk)) * int64_t(p.d)
                         : p.k_cache + (slot[i] * p.Hk + (h - p.H)) * int64_t(p.d);
            }
            *reinterpret_cast<QkVec<VEC>*>(y + e0) = oa;
            *reinterpret_cast<QkVec<VEC>*>(y + e1) = ob;
        }
    }
}

}  // namespace

cudaError_t launch_paged_slots(const SlotArgs& a, cudaStream_t s) {
    SlotArgs p = a;
    PageDiv pd{uint32_t(a.page_size), -1};
    for (int i = 0; i <= 16; ++i)
        if (a.page_size == 1 << i) pd.shift = i;
    void* args[] = {&p, &pd};
    const int64_t blocks = std::max<int64_t>(1, (a.n_tokens + kSlotTokens - 1) / kSlotTokens);
    return launch_serialised(reinterpret_cast<const void*>(paged_slots_kernel), unsigned(blocks), kSlotThreads, 0, s, args);
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
    p.n_tokens = a.n_tokens;
    p.n_slots = a.n_slots;
    p.H = int(a.n_heads);
    p.Hk = int(a.n_kv_heads);
    p.d = int(a.head_dim);
    p.half = int(a.rot_dim / 2);
    p.eps = a.eps;
    if (p.half > 0) rotary_frequencies(double(a.base), a.rot_dim, p.inv_hi, p.inv_lo);
    for (int i = 0; i < p.half; ++i) p.axis[i] = a.axis_of_pair ? a.axis_of_pair[i] : uint8_t(0);
    // 16-byte accesses where both halves of the pairs start on that boundary
    const int vec = p.half % 8 == 0 && (p.d - 2 * p.half) % 16 == 0 ? 8 : 4;
    const int units = p.d / (2 * vec);
    p.log_lanes = 0;
    while ((1 << p.log_lanes) < units) ++p.log_lanes;
    const int64_t pass = kQkThreads >> p.log_lanes, heads = a.n_heads + 2 * a.n_kv_heads;
    // as many tokens as give every thread four rows at once, one while that leaves SMs without a CTA
    int rows = 4;
    p.tokens = int(std::min<int64_t>(kQkMaxTokens, std::max<int64_t>(1, rows * pass / heads)));
    if ((a.n_tokens + p.tokens - 1) / p.tokens < 2 * 152) {
        rows = 1;
        p.tokens = int(std::min<int64_t>(kQkMaxTokens, std::max<int64_t>(1, pass / heads)));
    }
    const size_t smem = (2 * size_t(p.d) + 2 * size_t(p.tokens) * p.half + 3 * size_t(p.half)) * 4;
    const void* fn = vec == 8 ? (rows == 4 ? reinterpret_cast<const void*>(qk_norm_rope_kernel<8, 4>)
                                           : reinterpret_cast<const void*>(qk_norm_rope_kernel<8, 1>))
                              : (rows == 4 ? reinterpret_cast<const void*>(qk_norm_rope_kernel<4, 4>)
                                           : reinterpret_cast<const void*>(qk_norm_rope_kernel<4, 1>));
    void* args[] = {&p};
    return launch_serialised(fn, unsigned((a.n_tokens + p.tokens - 1) / p.tokens), kQkThreads, smem, s, args);
}

}  // namespace emb
