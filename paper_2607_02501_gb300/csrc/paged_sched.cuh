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
    int64_t max_pages;
    int n_tokens, n_req, n_pages, page_shift, kv_limit, window;
    int H, Hk, G, QB, QT;  // heads, those of one key/value head; queries of an item and of a row tile
    int cluster, side;     // few rows: CTAs of a cluster, or 0; clusters of a request's key/value head, for its blocks
    bool negate;           // the scale is negative: its magnitude is in scale2
    uint32_t join_units;  // units that joining a cut item costs
    uint32_t grid_inv;  // ceil(2^32 / grid)
    float scale2;  // scores are kept in base 2: scale * log2(e); capped, 2 log2(e) scale / cap
    float cap2;    // cap * log2(e)
    float lin2;    // scale * log2(e)
};

struct PagedReq {
    int q0, n, L, f;  // first token, queries, keys, fully visible prefix
};
__device__ __forceinline__ PagedReq paged_req(const PagedParams& p, int r) {
    const int a = p.q_start[r], b = p.q_start[r + 1], len = p.kv_len[r], f = p.prefix ? p.prefix[r] : 0, T = p.n_tokens;
    PagedReq q;
    q.q0 = min(max(a, 0), T);
    q.n = max(min(b, T), q.q0) - q.q0;
    q.L = min(max(len, 0), p.kv_limit);
    q.f = min(max(f, 0), q.L);
    return q;
}

struct KeyRange {
    int lo, hi;
};
// Keys that query i of the request sees (lo >= hi: none).
__device__ __forceinline__ KeyRange query_keys(const PagedParams& p, const PagedReq& q, int i) {
    const int at = q.L - q.n + i;  // its position, above -2^31
    KeyRange k;
    k.hi = min(q.L, max(at + 1, q.f));
    k.lo = p.window > 0 && at >= p.window ? at - p.window + 1 : 0;
    return k;
}

// The item (r, g, b): its queries, and the tiles of the keys that any of them sees. (Found by whole warps.)
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
    it.t0 = int(uint32_t(it.lo) / KT);
    it.nt = it.hi > it.lo ? int((uint32_t(it.hi) + KT - 1) / KT) - it.t0 : 0;
    it.units = max(1, it.nt);
}
template <int KT>
__device__ __forceinline__ PagedItem paged_item(const PagedParams& p, int r, int g, int b) {
    PagedItem it;
    it.r = r;
    it.g = g;
    it.b = b;
    const PagedReq q = paged_req(p, r);
    it.q = PagedReq{ptx::warp_uniform(q.q0), ptx::warp_uniform(q.n), ptx::warp_uniform(q.L), ptx::warp_uniform(q.f)};
    item_span<KT>(p, it.q, b, it);
    return it;
}

// A CTA's stretch of units [x0, x1), and where x0 lies: unit `off` of item (r, g, b).
struct PagedStretch {
    uint32_t x0, x1, chunk;
    int r, g, b;
    uint32_t off;
};
// Where a unit lies: unit `off` of item (r, g, b), which has `rest` units from there on.
struct PagedPlace {
    int r, g, b;
    uint32_t off, rest;
};
// The item after (r, g, b): the next block, key/value head or request that has queries.
__device__ __forceinline__ void next_item(const PagedParams& p, int& r, int& g, int& b, int n_queries) {
    if (++b < (n_queries + p.QB - 1) / p.QB) return;
    b = 0;
    if (++g < p.Hk) return;
    g = 0;
    do ++r;
    while (r < p.n_req && ptx::warp_uniform(paged_req(p, r).n) == 0);
}

// Units of a CTA's stretch: total / grid rounded up (or one more: any that is enough will do).
__device__ __forceinline__ uint32_t stretch_chunk(const PagedParams& p, uint32_t total, uint32_t biggest) {
    const uint32_t even = __umulhi(total + gridDim.x - 1, p.grid_inv);
    return max(even, (biggest + kMaxJoin - 2) / (kMaxJoin - 1));
}

// Whether no item is cut: a CTA's items, the longest as many as come to each, against equal stretches and a join.
__device__ __forceinline__ bool stretch_whole(const PagedParams& p, uint32_t chunk, uint32_t biggest, uint32_t items) {
    const uint32_t each = __umulhi(items + gridDim.x - 1, p.grid_inv);
    return each * uint64_t(biggest) < uint64_t(chunk) + p.join_units;
}

// This CTA's stretch of `total` units; find(x) tells where a unit lies. Where no item is cut, both ends move on to the
// next item's start.
template <typename Find>
__device__ __forceinline__ PagedStretch cut_stretch(const PagedParams& p, uint32_t total, uint32_t biggest, uint32_t items, Find find) {
    PagedStretch st{};
    st.chunk = stretch_chunk(p, total, biggest);
    st.x0 = uint32_t(min(uint64_t(blockIdx.x) * st.chunk, uint64_t(total)));
    st.x1 = min(total, st.x0 + st.chunk);
    if (st.x0 == st.x1) return st;
    const bool whole = stretch_whole(p, st.chunk, biggest, items);
    const PagedPlace a = find(st.x0);
    st.r = a.r;
    st.g = a.g;
    st.b = a.b;
    st.off = a.off;
    if (whole) {
        if (st.x1 < total) {
            const PagedPlace z = find(st.x1);
            if (z.off > 0) st.x1 += z.rest;
        }
        if (st.off > 0) {
            st.x0 += a.rest;
            st.off = 0;
            if (st.x0 < st.x1) next_item(p, st.r, st.g, st.b, paged_req(p, st.r).n);
        }
    }
    return st;
}

// The stretch, found by NT threads: a warp by itself (NT = 32), or all threads of the CTA (a multiple of 32, at most
// 512). Requests go to groups of 2^n lanes that share out a request's blocks; a scan over the groups' units gives the
// total, and a unit's group walks to it.
template <int KT, int NT, bool ONE = false>  // ONE: there is one request only
__device__ __forceinline__ PagedStretch paged_stretch_by(const PagedParams& p) {
    constexpr bool kBlock = NT > 32;
    constexpr int kWarps = NT / 32;
    __shared__ PagedPlace found;
    __shared__ uint32_t warp_sum[kWarps], warp_max[kWarps], warp_items[kWarps];
    __shared__ float warp_claim[kWarps];
    const int tid = kBlock ? int(threadIdx.x) : int(threadIdx.x & 31), lane = tid & 31, warp = tid >> 5;
    int sub = 32, per = 1;
    if constexpr (!ONE) {
        while (sub > 1 && NT / sub < p.n_req) sub >>= 1;
        const int groups = NT / sub;
        per = (p.n_req + groups - 1) / groups;
    }
    const int l = tid & (sub - 1), r0 = ONE ? 0 : (tid / sub) * per;
    const uint32_t gmask = sub == 32 ? 0xffffffffu : ((1u << sub) - 1u) << (lane & ~(sub - 1));
    uint32_t biggest = 0, items = 0;
    auto units_of = [&](const PagedReq& q) {  // of one key/value head, summed over the group
        uint32_t s = 0;
        for (int b = l; b * p.QB < q.n; b += sub) {
            PagedItem it;
            item_span<KT>(p, q, b, it);
            s += uint32_t(it.units);
            biggest = max(biggest, uint32_t(it.units));
            ++items;
        }
        if constexpr (ONE) {
            s = __reduce_add_sync(0xffffffffu, s);
        } else {
            for (int o = sub >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(gmask, s, o);
        }
        return s;
    };
    uint32_t sum = 0;
    float claim = 0.0f;  // queries of all requests
    for (int k = 0; k < per; ++k)
        if (r0 + k < p.n_req) {
            const PagedReq q = paged_req(p, r0 + k);
            sum += units_of(q) * uint32_t(p.Hk);
            if (l == 0) claim += float(q.n);
        }
    __syncwarp();
    uint32_t incl = l == 0 || ONE ? sum : 0u;
    if constexpr (!ONE) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += u;
        }
    }
    if constexpr (!ONE)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) claim += __shfl_xor_sync(0xffffffffu, claim, o);
    biggest = __reduce_max_sync(0xffffffffu, biggest);
    items = __reduce_add_sync(0xffffffffu, items);
    uint32_t total = ONE ? sum : __shfl_sync(0xffffffffu, incl, 31), before = 0;
    if constexpr (kBlock) {
        if (lane == 0) {
            warp_sum[warp] = total;
            warp_max[warp] = biggest;
            warp_items[warp] = items;
            warp_claim[warp] = claim;
        }
        __syncthreads();
        total = biggest = items = 0;
        claim = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += warp_sum[w];
            total += warp_sum[w];
            biggest = max(biggest, warp_max[w]);
            items += warp_items[w];
            claim += warp_claim[w];
        }
    }
    // Starts that go back can let requests claim more queries than there are tokens, and then the units may pass 32 bits:
    // there is no telling whose work is whose, so none is done.
    if (!ONE && claim > 1.0001f * float(p.n_tokens)) return PagedStretch{};
    // (lane 0 of a group holds the sum up to and with its group)
    const uint32_t end = ONE ? sum : __shfl_sync(0xffffffffu, incl, lane & ~(sub - 1)) + before, begin = end - sum;
    auto find = [&](uint32_t x) {
        PagedPlace at{};
        bool here = false;
        if (x >= begin && x < end) {
            uint32_t rem = x - begin;
            for (int k = 0; k < per && r0 + k < p.n_req; ++k) {
                const PagedReq q = paged_req(p, r0 + k);
                const uint32_t s = ONE ? sum / uint32_t(p.Hk) : units_of(q);
                if (rem >= s * uint32_t(p.Hk)) {
                    rem -= s * uint32_t(p.Hk);
                    continue;
                }
                const int g = p.Hk > 1 ? int(rem / s) : 0;
                rem -= uint32_t(g) * s;
                for (int base = 0; base * p.QB < q.n; base += sub) {
                    uint32_t u = 0;
                    if ((base + l) * p.QB < q.n) {
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
                        here = rem >= c - u && rem < c;
                        at = PagedPlace{r0 + k, g, base + l, rem - (c - u), c - rem};
                        break;
                    }
                    rem -= all;
                }
                break;
            }
        }
        if constexpr (kBlock) {
            if (here) found = at;
            __syncthreads();
            at = found;
            __syncthreads();
        } else {
            __syncwarp();
            const int src = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
            at.r = __shfl_sync(0xffffffffu, at.r, src);
            at.g = __shfl_sync(0xffffffffu, at.g, src);
            at.b = __shfl_sync(0xffffffffu, at.b, src);
            at.off = __shfl_sync(0xffffffffu, at.off, src);
            at.rest = __shfl_sync(0xffffffffu, at.rest, src);
        }
        return at;
    };
    return cut_stretch(p, total, biggest, items * uint32_t(p.Hk), find);
}
template <int KT, int NT>
__device__ __noinline__ PagedStretch paged_stretch_block(const PagedParams& p) {
    return paged_stretch_by<KT, NT>(p);
}
// Up to 64 requests need no barrier (one decoded token over 867 keys: 4350 cycles by the block, a fifth of the call,
// 1900 by a warp).
// For one request of one block (a decoded token) there is nothing to scan.
template <int KT>
__device__ __forceinline__ PagedStretch paged_stretch_one(const PagedParams& p, const PagedReq& q) {
    PagedItem it;
    item_span<KT>(p, q, 0, it);
    const uint32_t units = uint32_t(it.units), Hk = uint32_t(p.Hk);
    return cut_stretch(p, units * Hk, units, Hk, [&](uint32_t x) {
        const uint32_t g = Hk > 1 ? x / units : 0u, off = x - g * units;
        return PagedPlace{0, int(g), 0, off, units - off};
    });
}
template <int KT, int NT>
__device__ __forceinline__ PagedStretch paged_stretch(const PagedParams& p) {
    PagedReq q{0, 0, 0, 0};
    if (p.n_req == 1) q = paged_req(p, 0);
    PagedStretch st = q.n > 0 && q.n <= p.QB ? paged_stretch_one<KT>(p, q)
                      : p.n_req == 1    ? paged_stretch_by<KT, 32, true>(p)
                      : p.n_req <= 64 ? paged_stretch_by<KT, 32>(p)
                                      : paged_stretch_block<KT, NT>(p);
    // In a form that the compiler knows to be uniform (as an item's numbers are): else its branches are not, and every
    // MMA that depends on them issues slowly (4096 new tokens over 16384 keys: 780 us, so 612).
    st.x0 = ptx::warp_uniform(st.x0);
    st.x1 = ptx::warp_uniform(st.x1);
    st.chunk = ptx::warp_uniform(st.chunk);
    st.r = ptx::warp_uniform(st.r);
    st.g = ptx::warp_uniform(st.g);
    st.b = ptx::warp_uniform(st.b);
    st.off = ptx::warp_uniform(st.off);
    return st;
}

// An item that several CTAs share: CTAs first .. first + count - 1, each with one partial result.
struct PagedJoin {
    int r, g, b, first, count;
};
// The partial result of CTA c for an item that starts in CTA `first`: a CTA has at most one that started
// before it and one that goes on after it.
__device__ __forceinline__ int64_t part_slot(int c, int first) { return 2 * int64_t(c) + (c == first ? 1 : 0); }

// Waits until *flag >= count (acquire); gives up like ptx::mbar_wait.
__device__ __forceinline__ bool join_wait(const uint32_t* flag, uint32_t count, volatile int* abort, int* status, uint64_t limit_ns) {
    if (ptx::ld_acquire_gpu(flag) >= count) return true;
    const uint64_t t0 = ptx::globaltimer();
    for (;;) {
        if (ptx::ld_acquire_gpu(flag) >= count) return true;
        if (*abort) return false;
        if (ptx::globaltimer() - t0 > limit_ns) {
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
// What the kernels are told of a call, but for the tensor maps, the work's split and the grid.
PagedParams paged_params(const PagedAttnArgs& a);
// What a launch of `grid` CTAs (two at least), of which joining an item costs join_units, tells its kernel.
inline void set_grid(PagedParams& p, unsigned grid, unsigned join_units) {
    p.join_units = join_units;
    p.grid_inv = uint32_t(((uint64_t(1) << 32) + grid - 1) / grid);
}
// The tcgen05 kernel (paged_many.cu).
cudaError_t launch_paged_many(PagedParams& p, const PagedAttnArgs& a, cudaStream_t s);

}  // namespace emb
