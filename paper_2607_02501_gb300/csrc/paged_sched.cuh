// Which keys a block of queries of a paged attention call sees, and how the call's work is shared
// out over the CTAs: used by its kernels alike.
//
// An item is a block of QB consecutive queries of one request with the query heads of one key/value
// head; its work is counted in tiles of KT keys, from the first that one of its queries sees to the last (one
// unit at least, so that a block without a key gets its zeros). The items in order (request, key/value head, block)
// are one line of units, of which every CTA takes an equal stretch: requests of any lengths keep all CTAs
// equally long at work. An item that a stretch's border cuts is joined through the workspace. Every CTA
// finds its stretch by itself from the lengths on the device: no plan to keep, and a recorded call follows its lengths.
#pragma once

#include <cuda.h>

#include "paged.cuh"

namespace emb {

constexpr int kMaxJoin = 64;  // CTAs that share one item, at most: the join reads all their partial results

struct PagedParams {
    CUtensorMap k_map, v_map;  // cache as (head_dim, kv head, place in page, page); boxes of 64 dims
    CUtensorMap q_map;         // Q as (head_dim, head, token)
    const __nv_bfloat16* Q;
    const __nv_bfloat16* K;
    const __nv_bfloat16* V;
    __nv_bfloat16* O;
    const int32_t* table;
    const int32_t* q_start;
    const int32_t* kv_len;
    const int32_t* prefix;
    uint32_t* flags;  // one per CTA: arrivals of the item that starts in it and goes on
    float* part;      // two partial results per CTA
    int* status;
    int64_t max_pages, n_tokens;
    int n_req, n_pages, page_shift, kv_limit, window;
    int H, Hk, G, QB, min_units;
    uint32_t grid_inv;  // ceil(2^32 / grid)
    float scale2;  // scores are kept in base 2: scale * log2(e); capped, 2 log2(e) scale / cap
    float cap2;    // cap * log2(e)
};

struct PagedReq {
    int q0, n, L, f;  // first token, queries, keys, fully visible prefix
};
__device__ __forceinline__ PagedReq paged_req(const PagedParams& p, int r) {
    const int64_t a = p.q_start[r], b = p.q_start[r + 1];
    const int len = p.kv_len[r], f = p.prefix ? p.prefix[r] : 0;
    PagedReq q;
    q.q0 = int(min(max(a, int64_t(0)), p.n_tokens));
    q.n = int(max(min(b, p.n_tokens) - q.q0, int64_t(0)));
    q.L = min(max(len, 0), p.kv_limit);
    q.f = min(max(f, 0), q.L);
    return q;
}

struct KeyRange {
    int lo, hi;
};
// Keys that query i of the request sees (lo >= hi: none).
__device__ __forceinline__ KeyRange query_keys(const PagedParams& p, const PagedReq& q, int i) {
    const int64_t at = int64_t(q.L) - q.n + i;
    KeyRange k;
    k.hi = int(min(int64_t(q.L), max(at + 1, int64_t(q.f))));
    k.lo = p.window > 0 ? int(max(int64_t(0), at - p.window + 1)) : 0;
    return k;
}

// The item (r, g, b): its queries, and the tiles of the keys that any of them sees.
struct PagedItem {
    int r, g, b;
    PagedReq q;
    int i0, nq;      // its queries of the request
    int lo, hi;      // keys that any of them sees
    int lo_all, hi_all;  // keys that all of them see
    int t0, nt, units;
};
template <int KT>
__device__ __forceinline__ void item_span(const PagedParams& p, const PagedReq& q, int b, PagedItem& it) {
    it.i0 = b * p.QB;
    it.nq = min(p.QB, q.n - it.i0);
    const KeyRange first = query_keys(p, q, it.i0), last = query_keys(p, q, it.i0 + it.nq - 1);
    it.lo = first.lo;  // both ends grow with the query
    it.hi = last.hi;
    it.lo_all = last.lo;
    it.hi_all = first.hi;
    it.t0 = it.lo / KT;
    it.nt = it.hi > it.lo ? (it.hi + KT - 1) / KT - it.t0 : 0;
    it.units = max(1, it.nt);
}
template <int KT>
__device__ __forceinline__ PagedItem paged_item(const PagedParams& p, int r, int g, int b) {
    PagedItem it;
    it.r = r;
    it.g = g;
    it.b = b;
    it.q = paged_req(p, r);
    item_span<KT>(p, it.q, b, it);
    return it;
}

// A CTA's stretch of units [x0, x1), and where x0 lies: unit `off` of item (r, g, b).
struct PagedStretch {
    uint32_t x0, x1, chunk;
    int r, g, b;
    uint32_t off;
};

// Units of a CTA's stretch: total / grid rounded up (or one more: any that is enough will do).
__device__ __forceinline__ uint32_t stretch_chunk(const PagedParams& p, uint32_t total, uint32_t biggest) {
    const uint32_t even = __umulhi(total + gridDim.x - 1, p.grid_inv);
    return max(max(even, (biggest + kMaxJoin - 2) / (kMaxJoin - 1)), uint32_t(p.min_units));
}

// For up to 64 requests of up to four blocks: every warp by itself, two requests a lane, without a barrier (one
// decoded token over 867 keys: 4350 cycles by the general way, a fifth of the call). False if there are more.
template <int KT>
__device__ __forceinline__ bool paged_stretch_few(const PagedParams& p, PagedStretch& st) {
    if (p.n_req > 64) return false;
    const int lane = threadIdx.x & 31;
    PagedReq q[2];
    uint32_t s[2], biggest = 0;
    bool fits = true;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        s[k] = 0;
        q[k] = PagedReq{0, 0, 0, 0};
        if (2 * lane + k < p.n_req) q[k] = paged_req(p, 2 * lane + k);
        fits = fits && q[k].n <= 4 * p.QB;
    }
    if (!__all_sync(0xffffffffu, fits)) return false;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        for (int b = 0; b * p.QB < q[k].n; ++b) {
            PagedItem it;
            item_span<KT>(p, q[k], b, it);
            s[k] += uint32_t(it.units);
            biggest = max(biggest, uint32_t(it.units));
        }
    __syncwarp();
    const uint32_t sum = (s[0] + s[1]) * uint32_t(p.Hk);
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    biggest = __reduce_max_sync(0xffffffffu, biggest);
    const uint32_t total = __shfl_sync(0xffffffffu, incl, 31);
    st.chunk = stretch_chunk(p, total, biggest);
    st.x0 = uint32_t(min(uint64_t(blockIdx.x) * st.chunk, uint64_t(total)));
    st.x1 = min(total, st.x0 + st.chunk);
    const bool here = st.x0 < st.x1 && st.x0 >= incl - sum && st.x0 < incl;
    st.r = st.g = st.b = 0;
    st.off = 0;
    if (here) {
        uint32_t rem = st.x0 - (incl - sum);
        const int k = rem >= s[0] * uint32_t(p.Hk) ? 1 : 0;
        if (k) rem -= s[0] * uint32_t(p.Hk);
        const uint32_t per = k ? s[1] : s[0];
        st.r = 2 * lane + k;
        st.g = p.Hk > 1 ? int(rem / per) : 0;
        rem -= uint32_t(st.g) * per;
        const PagedReq qk = k ? q[1] : q[0];
        for (;; ++st.b) {
            PagedItem it;
            item_span<KT>(p, qk, st.b, it);
            if (rem < uint32_t(it.units)) break;
            rem -= uint32_t(it.units);
        }
        st.off = rem;
    }
    const uint32_t found = __ballot_sync(0xffffffffu, here);
    const int src = found ? __ffs(found) - 1 : 0;
    st.r = __shfl_sync(0xffffffffu, st.r, src);
    st.g = __shfl_sync(0xffffffffu, st.g, src);
    st.b = __shfl_sync(0xffffffffu, st.b, src);
    st.off = __shfl_sync(0xffffffffu, st.off, src);
    return true;
}

// Found by all NT threads of the CTA (a multiple of 32, at most 512). Requests go to groups of 2^n lanes that
// share out a request's blocks; a block scan over the groups' units gives the total, so the stretch, and its group
// walks to x0.
template <int KT, int NT>
__device__ __noinline__ PagedStretch paged_stretch_all(const PagedParams& p) {
    __shared__ PagedStretch found;
    __shared__ uint32_t warp_sum[NT / 32], warp_max[NT / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int sub = 32;
    while (sub > 1 && NT / sub < p.n_req) sub >>= 1;
    const int groups = NT / sub, per = (p.n_req + groups - 1) / groups;
    const int l = tid & (sub - 1), r0 = (tid / sub) * per;
    const uint32_t gmask = sub == 32 ? 0xffffffffu : ((1u << sub) - 1u) << (lane & ~(sub - 1));
    uint32_t biggest = 0;
    auto units_of = [&](const PagedReq& q) {  // of one key/value head, summed over the group
        uint32_t s = 0;
        const int nb = (q.n + p.QB - 1) / p.QB;
        for (int b = l; b < nb; b += sub) {
            PagedItem it;
            item_span<KT>(p, q, b, it);
            s += uint32_t(it.units);
            biggest = max(biggest, uint32_t(it.units));
        }
        for (int o = sub >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(gmask, s, o);
        return s;
    };
    uint32_t sum = 0;
    for (int k = 0; k < per; ++k)
        if (r0 + k < p.n_req) sum += units_of(paged_req(p, r0 + k)) * uint32_t(p.Hk);
    __syncwarp();
    uint32_t incl = l == 0 ? sum : 0u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
        biggest = max(biggest, __shfl_xor_sync(0xffffffffu, biggest, o));
    }
    if (lane == 31) warp_sum[warp] = incl;
    if (lane == 0) warp_max[warp] = biggest;
    if (tid == 0) found.x0 = found.x1 = 0;
    __syncthreads();
    uint32_t total = 0, before = 0;
    biggest = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) before += warp_sum[w];
        total += warp_sum[w];
        biggest = max(biggest, warp_max[w]);
    }
    const uint32_t chunk = stretch_chunk(p, total, biggest);
    const uint32_t x0 = uint32_t(min(uint64_t(blockIdx.x) * chunk, uint64_t(total)));
    const uint32_t x1 = min(total, x0 + chunk);
    // (lane 0 of a group holds the sum up to and with its group)
    const uint32_t end = __shfl_sync(0xffffffffu, incl, lane & ~(sub - 1)) + before, begin = end - sum;
    if (x0 < x1 && x0 >= begin && x0 < end) {
        uint32_t rem = x0 - begin;
        for (int k = 0; k < per && r0 + k < p.n_req; ++k) {
            const PagedReq q = paged_req(p, r0 + k);
            const uint32_t s = units_of(q);
            if (rem >= s * uint32_t(p.Hk)) {
                rem -= s * uint32_t(p.Hk);
                continue;
            }
            const int g = int(rem / s);
            rem -= uint32_t(g) * s;
            const int nb = (q.n + p.QB - 1) / p.QB;
            for (int base = 0; base < nb; base += sub) {
                uint32_t u = 0;
                if (base + l < nb) {
                    PagedItem it;
                    item_span<KT>(p, q, base + l, it);
                    u = uint32_t(it.units);
                }
                uint32_t c = u;
                for (int o = 1; o < sub; o <<= 1) {
                    const uint32_t v = __shfl_up_sync(gmask, c, o, sub);
                    if (l >= o) c += v;
                }
                const uint32_t all = __shfl_sync(gmask, c, sub - 1, sub);
                if (rem < all) {
                    if (rem >= c - u && rem < c) found = PagedStretch{x0, x1, chunk, r0 + k, g, base + l, rem - (c - u)};
                    break;
                }
                rem -= all;
            }
            break;
        }
    }
    __syncthreads();
    return found;
}

template <int KT, int NT>
__device__ __forceinline__ PagedStretch paged_stretch(const PagedParams& p) {
    PagedStretch st;
    return paged_stretch_few<KT>(p, st) ? st : paged_stretch_all<KT, NT>(p);
}

// The item after (r, g, b): the next block, key/value head or request that has queries.
__device__ __forceinline__ void next_item(const PagedParams& p, int& r, int& g, int& b, int n_queries) {
    if (++b < (n_queries + p.QB - 1) / p.QB) return;
    b = 0;
    if (++g < p.Hk) return;
    g = 0;
    do ++r;
    while (r < p.n_req && paged_req(p, r).n == 0);
}

// An item that several CTAs share: CTAs first .. first + count - 1, each with one partial result.
struct PagedJoin {
    int r, g, b, first, count;
};
// The partial result of CTA c for an item that starts in CTA `first`: a CTA has at most one that started
// before it and one that goes on after it.
__device__ __forceinline__ int64_t part_slot(int c, int first) { return 2 * int64_t(c) + (c == first ? 1 : 0); }

// Waits until *flag >= count (acquire); gives up like ptx::mbar_wait.
__device__ __forceinline__ bool join_wait(const uint32_t* flag, uint32_t count, volatile int* abort, int* status) {
    if (ptx::ld_acquire_gpu(flag) >= count) return true;
    const uint64_t t0 = ptx::globaltimer();
    for (;;) {
        if (ptx::ld_acquire_gpu(flag) >= count) return true;
        if (*abort) return false;
        if (ptx::globaltimer() - t0 > kWaitLimitNs) {
            atomicOr(status, kStatusTimeout);
            *abort = 1;
            return false;
        }
        __nanosleep(32);
    }
}

// ------------------------------------------------------------------ host side
constexpr size_t kPagedFlagBytes = 4096;  // of the workspace

// A cache array as (head_dim, kv head, place in page, page), boxes of 64 dims x `box` places; Q as (head_dim, head,
// token), boxes of 64 dims x heads x tokens. Rows of 128 bytes, swizzled.
bool encode_cache(CUtensorMap* m, const void* base, const PagedAttnArgs& a, uint32_t box);
bool encode_queries(CUtensorMap* m, const PagedAttnArgs& a, uint32_t heads, uint32_t tokens);
// Units of work of a call, at most: every block of every request over a full block table.
double unit_bound(const PagedAttnArgs& a, int qb, int kt);
// What a launch of `grid` CTAs (two at least), with stretches of min_units at least, tells its kernel.
inline void set_grid(PagedParams& p, unsigned grid, int min_units) {
    p.min_units = min_units;
    p.grid_inv = uint32_t(((uint64_t(1) << 32) + grid - 1) / grid);
}
// The tcgen05 kernel (paged_many.cu).
cudaError_t launch_paged_many(PagedParams& p, const PagedAttnArgs& a, cudaStream_t s);

}  // namespace emb
