// Attention of new tokens over a paged key/value cache, many query rows per request: tcgen05
// (definition in include/emb_paged.h, work split in paged_sched.cuh).
//
// An item has two tiles of up to 128 rows (queries times the heads of one key/value head), or one where heads of 256
// leave the tensor memory no room for two. Keys and values come in tiles of 128 (64) through one ring of TMA
// copies, keys and values in turn. One warp issues the MMAs: S = Q K^T from shared memory into tensor memory, and O += P V with
// P read from tensor memory, where it takes the place of its scores. Each row tile has a warpgroup for its
// softmax, a thread a row, so a row's maximum and sum need no exchange. While one tile's softmax runs the tensor
// cores work for the other; with one tile its scores have two places in turn. The running maximum moves only when it
// grows by more than 2^8 (P and its sums stay far within fp32 and bf16's relative precision), so the output in tensor
// memory is seldom rescaled. The weights are rounded once to bf16: hi + lo would double the value product for outputs
// that are rounded to bf16 anyway (error against 64 bits 0.0023 of the outputs' norm, of which 0.0017 is that rounding).
// What bounds it. Heads of 128: 4096 new tokens of 32 heads over 16384 keys take 599 to 639 us, called or replayed (1600 to 1510
// TFLOP/s, 0.84 to 0.79 of the measured matrix rate; the spread, also between boxes, was not traced); by nominal rates the
// softmax's powers of two (16 a cycle and SM) take as long as the MMAs. Heads of 64: half the MMAs for the same powers. Heads of
// 256: not established. Every key and value is fetched for 128 rows instead of 256, and one row tile with one softmax warpgroup
// leaves a tile's chain of steps exposed (2048 over 4096, 16 heads on 2, 135 us; 129 of then 137 with the softmax left out). Small
// calls: latency and the join.
#include <algorithm>
#include <mutex>

#include "paged_math.cuh"

namespace emb {
namespace {

template <int D>
struct ManyTraits {
    static constexpr int NQ = D == 256 ? 1 : 2;        // row tiles of an item
    static constexpr int KT = D == 256 ? 64 : 128;     // keys of a tile
    static constexpr int kSoftWarps = 4 * NQ;
    // then the MMA and the producer warp; with two row tiles their warpgroup is filled up by two idle warps, so that
    // it can hand registers to the softmax, a thread of which holds 128 scores: 384 threads x 168 at launch, then
    // 2 x 128 x 216 + 128 x 72
    static constexpr int kThreads = NQ == 2 ? 384 : 192;
    static constexpr int kQTile = 128 * D * 2;         // bytes of a row tile's queries
    static constexpr int kSlot = KT * D * 2;           // bytes of a tile of keys or values
    static constexpr int kSlots = D == 64 ? 8 : 5;
    static constexpr int kSmem = 1024 + NQ * kQTile + kSlots * kSlot;
    static constexpr int kSub = KT * 128;              // bytes of 64 dims of a tile
    // columns of tensor memory: scores (two places), outputs
    static constexpr int kO = 2 * KT;
};
constexpr uint32_t kTmemAll = 512;
static_assert(ManyTraits<64>::kSmem > 114 * 1024 && ManyTraits<128>::kSmem > 114 * 1024 && ManyTraits<256>::kSmem > 114 * 1024,
              "one CTA per SM: tensor memory is allocated whole (see ptx::tmem_alloc)");

// Largest of three.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float d;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// A place of the ring and the parity of the turn it is in, carried along (a division per wait costs more than the wait).
template <int S>
struct RingPlace {
    int slot = 0;
    uint32_t turn = 0;
    __device__ __forceinline__ void next() {
        if (++slot == S) {
            slot = 0;
            turn ^= 1u;
        }
    }
};

// The part of an item that lies in this CTA's stretch: tiles [j0, j1), of which row tile t has [a[t], b[t]).
template <int D>
struct Segment {
    PagedItem it;
    uint32_t take;
    int j0, j1;
    int a[2], b[2], nq[2];
};
template <int D>
__device__ __forceinline__ Segment<D> segment_of(const PagedParams& p, int r, int g, int b, uint32_t off, uint32_t x, uint32_t x1) {
    using T = ManyTraits<D>;
    Segment<D> s;
    s.it = paged_item<T::KT>(p, r, g, b);
    s.take = min(x1 - x, uint32_t(s.it.units) - off);
    s.j0 = s.it.t0 + int(off);
    s.j1 = s.it.t0 + min(int(off + s.take), s.it.nt);
    const int qt = p.QT;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        s.nq[t] = t < T::NQ ? max(0, min(qt, s.it.nq - t * qt)) : 0;
        s.a[t] = s.b[t] = 0;
        if (s.nq[t] == 0) continue;
        const int i0 = s.it.i0 + t * qt;
        const KeyRange first = query_keys(p, s.it.q, i0), last = query_keys(p, s.it.q, i0 + s.nq[t] - 1);
        if (last.hi <= first.lo) continue;
        s.a[t] = max(s.j0, first.lo / T::KT);
        s.b[t] = min(s.j1, (last.hi + T::KT - 1) / T::KT);
        if (s.b[t] < s.a[t]) s.b[t] = s.a[t];
    }
    return s;
}

template <int D, int CAP>
__global__ void __launch_bounds__(ManyTraits<D>::kThreads, 1) paged_many_kernel(const __grid_constant__ PagedParams p) {
    using T = ManyTraits<D>;
    constexpr int NQ = T::NQ, KT = T::KT, S = T::kSlots;
    constexpr int kRows = 128 * NQ;
    using PL = PartLayout<D, kRows>;
    // what stands for the score of a key that a row does not see (a cap would make -infinity finite)
    constexpr float kHidden = CAP ? -3.402823466e38f : -INFINITY;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t kv_full[S], kv_empty[S], q_full, q_empty, s_full[2], p_ready[2], o_done[2], o_free[2], drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, joined, odd_seen;
    __shared__ PagedJoin cut[2];
    uint8_t* sq = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* ring = sq + NQ * T::kQTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned all = 0xffffffffu;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            ptx::mbar_init(&kv_full[i], 1);
            ptx::mbar_init(&kv_empty[i], 1);
        }
        ptx::mbar_init(&q_full, 1);
        ptx::mbar_init(&q_empty, 1);
        for (int t = 0; t < 2; ++t) {
            ptx::mbar_init(&s_full[t], 1);
            ptx::mbar_init(&p_ready[t], 4);
            ptx::mbar_init(&o_done[t], 1);
            ptx::mbar_init(&o_free[t], 4);
        }
        ptx::mbar_init(&drain, 1);
        abort_flag = 0;
        odd_seen = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tmap(&p.q_map);
        ptx::prefetch_tmap(&p.k_map);
        ptx::prefetch_tmap(&p.v_map);
    }
    if (warp == T::kSoftWarps) {
        ptx::tmem_alloc(&tmem_slot, kTmemAll);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ptx::warp_uniform(tmem_slot);
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();  // lengths, queries and the new tokens' keys and values come from earlier launches
    const PagedStretch st = paged_stretch<KT, T::kThreads>(p);

    int r = st.r, g = st.g, b = st.b;
    uint32_t x = st.x0, off = st.off;
    auto wait = [&](uint64_t* bar, uint32_t phase) {
        return __all_sync(all, ptx::mbar_wait(bar, phase & 1, &abort_flag, p.status, kWaitLimitNs)) != 0;
    };
    // the tiles of the stretch are numbered through; each has its keys in one place of the ring, its values in the next

    if (warp == T::kSoftWarps + 1) {
        // ---------------------------------------------------------------------- producer
        if constexpr (NQ == 2) ptx::regs_down<72>();
        ptx::fence_proxy_async_global();  // (the cache and the queries were written by ordinary stores)
        const int page_size = 1 << p.page_shift, box = min(page_size, KT), n_box = KT / box;
        const int qt = p.QT;
        uint32_t loads = 0, items = 0;  // ring copies and items with queries issued
        RingPlace<S> at;
        bool ok = true;
        while (x < st.x1 && ok) {
            const Segment<D> sg = segment_of<D>(p, r, g, b, off, x, st.x1);
            const PagedItem& it = sg.it;
            if (sg.j1 > sg.j0) {
                if (items > 0) ok = wait(&q_empty, items - 1);
                if (!ok) break;
                const int tiles_q = sg.nq[1] > 0 ? 2 : 1;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(&q_full, uint32_t(tiles_q * (D / 64) * qt * p.G * 128));
                    for (int t = 0; t < tiles_q; ++t)
#pragma unroll
                        for (int c = 0; c < D / 64; ++c)
                            ptx::tma_load_3d(sq + t * T::kQTile + c * 16384, &p.q_map, &q_full, c * 64, g * p.G, it.q.q0 + it.i0 + t * qt);
                }
                __syncwarp();
                ++items;
            }
            const int32_t* row = p.table + int64_t(r) * p.max_pages;
            // lane i looks up the page of the tile's box i; boxes that no query sees, and pages that do not exist,
            // are fetched from behind the cache: zeros
            auto page_of = [&](int j) {
                const int key = j * KT + lane * box;
                int page = p.n_pages;
                if (lane < n_box && j < sg.j1 && key < it.hi && key + box > it.lo) {
                    page = row[key >> p.page_shift];
                    if (page < 0 || page > p.n_pages) page = p.n_pages;
                }
                return page;
            };
            int page = page_of(sg.j0);
            for (int j = sg.j0; j < sg.j1 && ok; ++j) {
                const int next = page_of(j + 1);
                const int place = (j * KT) & (page_size - 1);
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    const int s = at.slot;
                    if (loads >= uint32_t(S)) ok = wait(&kv_empty[s], at.turn ^ 1u);
                    if (!ok) break;
                    if (ptx::elect_one()) ptx::mbar_arrive_expect_tx(&kv_full[s], T::kSlot);
                    __syncwarp();
                    for (int i = 0; i < n_box; ++i) {
                        const int pg = __shfl_sync(all, page, i);
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int c = 0; c < D / 64; ++c)
                                ptx::tma_load_4d(ring + s * T::kSlot + c * T::kSub + i * box * 128, kv ? &p.v_map : &p.k_map,
                                                 &kv_full[s], c * 64, g, place, pg);
                        }
                        __syncwarp();
                    }
                    ++loads;
                    at.next();
                }
                page = next;
            }
            x += sg.take;
            off = 0;
            if (x < st.x1) next_item(p, r, g, b, it.q.n);
        }
        // every copy must land before this CTA's shared memory is released
        for (uint32_t i = loads > uint32_t(S) ? loads - S : 0; i < loads; ++i)
            ptx::mbar_wait(&kv_full[i % S], (i / S) & 1, nullptr, p.status, kWaitLimitNs);
        if (items > 0) ptx::mbar_wait(&q_full, (items - 1) & 1, nullptr, p.status, kWaitLimitNs);
    } else if (warp == T::kSoftWarps) {
        // ------------------------------------------------------------------------- MMAs
        if constexpr (NQ == 2) ptx::regs_down<72>();
        const uint32_t idesc_qk = ptx::idesc_bf16_f32(128, KT) | (p.negate ? ptx::kIdescNegateA : 0u), idesc_pv = ptx::idesc_bf16_f32(128, D) | ptx::kIdescMnMajorB;
        const uint32_t sq_u = ptx::smem_u32(sq), ring_u = ptx::smem_u32(ring);
        uint32_t n = 0, items = 0;
        RingPlace<S> keys, values;  // of tile j, and of the tile before it
        uint32_t scores[2] = {0, 0}, owned[2] = {0, 0};  // score tiles by place, items with outputs by row tile
        bool ok = true;
        // (operands in a form that the compiler knows to be uniform: see ptx::elect_one)
        auto qk = [&](int t, int place, int slot) {  // S[place] = Q[t] K^T
            const uint32_t k = ptx::warp_uniform(ring_u + uint32_t(slot * T::kSlot));
            const uint32_t d = ptx::warp_uniform(tmem + uint32_t(place * KT));
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                ptx::mma_bf16_ss(d, ptx::smem_desc_sw128(sq_u + t * T::kQTile + (ks / 4) * 16384) + 2 * (ks & 3),
                                 ptx::smem_desc_sw128(k + (ks / 4) * T::kSub) + 2 * (ks & 3), idesc_qk, ks != 0);
            ptx::mma_commit(&s_full[place]);
        };
        auto pv = [&](int t, int place, int slot, bool first) {  // O[t] (+)= P[place] V
            const uint64_t desc = ptx::smem_desc_mn_sw128(ptx::warp_uniform(ring_u + uint32_t(slot * T::kSlot)), T::kSub);
            const uint32_t d = ptx::warp_uniform(tmem + uint32_t(T::kO + t * D)), a = ptx::warp_uniform(tmem + uint32_t(place * KT));
            const uint32_t more = ptx::warp_uniform(first ? 0u : 1u);
#pragma unroll
            for (int kk = 0; kk < KT / 16; ++kk)
                ptx::mma_bf16_ta(d, a + uint32_t(8 * kk), desc + uint32_t(kk * 2048 / 16), idesc_pv, kk == 0 ? more : 1u);
            ptx::mma_commit(&o_done[t]);
        };
        while (x < st.x1 && ok) {
            const Segment<D> sg = segment_of<D>(p, r, g, b, off, x, st.x1);
            if (sg.j1 > sg.j0) {
                ok = wait(&q_full, items++);
                for (int j = sg.j0; j <= sg.j1 && ok; ++j) {
                    if (j < sg.j1) ok = wait(&kv_full[keys.slot], keys.turn);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    auto finish = [&](int t, int place) {  // P V of tile j - 1
                        const bool first = j - 1 == sg.a[t];
                        ok = wait(&kv_full[values.slot], values.turn) && wait(&p_ready[place], scores[place] - 1);
                        if (ok && first && owned[t] > 0) ok = wait(&o_free[t], owned[t] - 1);
                        if (!ok) return;
                        ptx::tc_fence_after();
                        pv(t, place, values.slot, first);
                        if (first) ++owned[t];
                    };
                    if constexpr (NQ == 2) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if (j > sg.a[t] && j <= sg.b[t]) finish(t, t);
                            if (!ok) break;
                            if (j >= sg.a[t] && j < sg.b[t]) {
                                qk(t, t, keys.slot);
                                ++scores[t];
                            }
                        }
                    } else {
                        if (j < sg.j1) {
                            qk(0, int(n & 1), keys.slot);
                            ++scores[n & 1];
                        }
                        if (j > sg.j0) finish(0, int((n - 1) & 1));
                    }
                    if (!ok) break;
                    if (j > sg.j0) ptx::mma_commit(&kv_empty[values.slot]);
                    if (j < sg.j1) {
                        ptx::mma_commit(&kv_empty[keys.slot]);
                        ++n;
                        keys.next();
                        values = keys;
                        keys.next();
                        if (j == sg.j1 - 1) ptx::mma_commit(&q_empty);
                    }
                }
            }
            x += sg.take;
            off = 0;
            if (x < st.x1) next_item(p, r, g, b, sg.it.q.n);
        }
        // whatever was issued finishes before tensor memory is freed
        ptx::mma_commit(&drain);
        ptx::mbar_wait(&drain, 0, nullptr, p.status, kWaitLimitNs);
    } else if (warp >= T::kSoftWarps) {
        if constexpr (NQ == 2) ptx::regs_down<72>();  // (idle)
    } else {
        // ---------------------------------------------------------------------- softmax
        if constexpr (NQ == 2) ptx::regs_up<216>();
        zero_padding(p, D, threadIdx.x, 32 * T::kSoftWarps);
        const int t = warp >> 2;  // row tile
        const int row = 32 * (warp & 3) + lane, qt = p.QT, i = row / p.G;
        const uint32_t lanes = uint32_t(32 * (warp & 3)) << 16;
        const uint32_t o_col = tmem + lanes + uint32_t(T::kO + t * D);
        uint32_t n = 0, seen[2] = {0, 0}, outs = 0;
        int joins = 0;
        auto soft_bar = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * T::kSoftWarps) : "memory"); };
        // A wait that gave up sets abort_flag; later waits then return at once, and the loops run to their end (the
        // outputs are undefined then), so that every barrier still meets all its threads.
        while (x < st.x1) {
            const Segment<D> sg = segment_of<D>(p, r, g, b, off, x, st.x1);
            const PagedItem& it = sg.it;
            const bool live = i < (t ? sg.nq[1] : sg.nq[0]);
            const KeyRange keys = live ? query_keys(p, it.q, it.i0 + t * qt + i) : KeyRange{0, 0};
            // (selected, not indexed: t is a run-time value)
            const int a_t = t ? sg.a[1] : sg.a[0], b_t = t ? sg.b[1] : sg.b[0];
            // whether the row has seen a score, its running maximum in base 2 (negated, so that it is added), sums of weights. A
            // cap makes a score of -infinity one of -cap, which counts.
            bool any = false;
            float mc = 0.0f;
            float2 l2[2] = {make_float2(0, 0), make_float2(0, 0)};
            for (int j = sg.j0; j < sg.j1; ++j, ++n) {
                if (j < a_t || j >= b_t) continue;
                const int place = NQ == 2 ? t : int(n & 1);
                wait(&s_full[place], seen[place]++);
                ptx::tc_fence_after();
                const uint32_t s_col = tmem + lanes + uint32_t(place * KT);
                const int key0 = j * KT;
                const bool edge = key0 < it.lo_all || key0 + KT > it.hi_all;
                const int lo = keys.lo - key0, hi = keys.hi - key0;
                // Votes are taken among rows that see a key of the tile. A tile's other rows are not of this request, or not
                // even filled (3 heads: 126 of 128 rows), and what they hold may not decide how a warp computes.
                const bool sees = max(lo, 0) < min(hi, KT);
                float low = INFINITY;  // the lowest score that the row sees (for a cap)
                if (edge) {
                    // scores that the row does not see, in tensor memory: rolled up and away from the path of most tiles
#pragma unroll 1
                    for (int c = 0; c < KT; c += 32) {
                        float v[32];
                        uint32_t w[32];
                        ptx::tmem_ld_32(s_col + c, v);
                        ptx::tmem_ld_wait_32(v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const bool sees = c + e >= lo && c + e < hi;
                            if (CAP && sees) low = fminf(low, v[e]);
                            w[e] = __float_as_uint(sees ? v[e] : kHidden);
                        }
                        ptx::tmem_st_32(s_col + c, w);
                    }
                    ptx::tmem_st_wait();
                }
                float s[KT];
#pragma unroll
                for (int c = 0; c < KT; c += 32) ptx::tmem_ld_32(s_col + c, s + c);
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < KT; c += 32) {
                    ptx::tmem_ld_wait_32(s + c);
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
#pragma unroll
                        for (int k = 0; k < 4; ++k) top[k] = max3(top[k], s[c + e + k], s[c + e + 4 + k]);
                }
                if (CAP && !edge) {
                    float l4[4] = {INFINITY, INFINITY, INFINITY, INFINITY};
#pragma unroll
                    for (int e = 0; e < KT; e += 8)
#pragma unroll
                        for (int k = 0; k < 4; ++k) l4[k] = min3(l4[k], s[e + k], s[e + 4 + k]);
                    low = fminf(min3(l4[0], l4[1], l4[2]), l4[3]);
                }
                // (the maximum is of raw scores: a cap keeps their order)
                const float mt = fmaxf(max3(top[0], top[1], top[2]), top[3]);
                auto base2 = [&](float v) {
                    if constexpr (CAP) return capped2<CAP>(make_float2(v, v), p).x;
                    else return v * p.scale2;
                };
                const float zt = base2(mt);
                const bool grow = sees && (any ? zt + mc > 8.0f : CAP || mt > -INFINITY);
                if (__any_sync(all, grow)) {
                    const float f = !grow ? 1.0f : any ? exp2_fast(-mc - zt) : 0.0f;
                    if (j > a_t) {
                        wait(&o_done[t], outs - 1);  // every product issued so far is in
                        ptx::tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            float o[32];
                            uint32_t w[32];
                            ptx::tmem_ld_32(o_col + c, o);
                            ptx::tmem_ld_wait_32(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(o[e] * f);
                            ptx::tmem_st_32(o_col + c, w);
                        }
                    }
                    if (grow) {
                        const float2 ff = make_float2(f, f), z = make_float2(0, 0);
                        l2[0] = fma2(l2[0], ff, z);
                        l2[1] = fma2(l2[1], ff, z);
                        any = true;
                        mc = -zt;
                    }
                }
                // The weights, 32 at a time, over the scores. `base` gives two scores in base 2 less the row's maximum.
                auto weights = [&](auto base) {
#pragma unroll
                    for (int c = 0; c < KT; c += 32) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float2 u = base(make_float2(s[c + e], s[c + e + 1]));
                            u.x = exp2_fast(u.x);
                            u.y = exp2_fast(u.y);
                            l2[(e >> 1) & 1] = add2(l2[(e >> 1) & 1], u);
                            w[e / 2] = pack_bf16x2(u.x, u.y);
                        }
                        ptx::tmem_st_16(s_col + c / 2, w);
                    }
                };
                const float2 mm = make_float2(mc, mc);
                if constexpr (!CAP) {
                    const float2 sc = make_float2(p.scale2, p.scale2);
                    weights([&](float2 u) { return fma2(u, sc, mm); });
                } else if (__all_sync(all, !sees || fmaxf(fabsf(mt), fabsf(low)) * p.scale2 < kNearCap)) {
                    // far below the cap one power of two per score, where exponential and reciprocal take two more turns of
                    // the same unit. (The series runs away to -infinity at what stands for a hidden score.)
                    weights([&](float2 u) { return capped_near2(u, p, mm); });
                } else {
                    weights([&](float2 u) {
                        const float2 z = capped2<CAP>(u, p);
                        return add2(make_float2(u.x == kHidden ? -INFINITY : z.x, u.y == kHidden ? -INFINITY : z.y), mm);
                    });
                }
                const bool tail = key0 + KT > it.q.L, hidden = key0 < it.lo_all || min(key0 + KT, it.q.L) > it.hi_all;
                if ((tail || hidden) && t == (NQ == 2 && !(j >= sg.a[0] && j < sg.b[0]) ? 1 : 0)) {
                    // values behind the request's last key are anything; those hidden from some rows may not be multiplied
                    // by their weights of 0 if they are not finite: such values leave the tile here and are added
                    // at the item's end for the rows that see them
                    const uint32_t pos = 2 * n + 1;
                    wait(&kv_full[pos % uint32_t(S)], pos / uint32_t(S));
                    uint4* v = reinterpret_cast<uint4*>(ring + (pos % uint32_t(S)) * T::kSlot);
                    uint32_t odd = 0;
                    // 16 bytes of one key at a time, whatever their dims
                    if (hidden) {
#pragma unroll 4
                        for (int e = row; e < KT * (D / 8); e += 128) {
                            const uint4 u = v[e];
                            odd |= not_finite2(u.x) | not_finite2(u.y) | not_finite2(u.z) | not_finite2(u.w);
                        }
                    }
                    if (tail)
                        for (int e = row; e < KT * (D / 8); e += 128)
                            if (key0 + (e / 8) % KT >= it.q.L) v[e] = make_uint4(0, 0, 0, 0);
                    if (odd) {
                        for (int e = row; e < KT * (D / 8); e += 128) {
                            uint4 u = v[e];
                            uint32_t* h = reinterpret_cast<uint32_t*>(&u);
                            bool hit = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t bad = not_finite2(h[k]);
                                if (bad & 0x8000u) h[k] &= 0xFFFF0000u;
                                if (bad & 0x80000000u) h[k] &= 0x0000FFFFu;
                                hit |= bad != 0;
                            }
                            if (hit) {
                                v[e] = u;
                                // (never taken back: the other row tile may be some items behind. Items without such values are
                                // then searched for nothing)
                                *reinterpret_cast<volatile int*>(&odd_seen) = 1;
                            }
                        }
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                }
                // every phase of o_done is waited for, so that a wait cannot take the one before the last for the last:
                // with two score places the last scores do not tell that the product before theirs is in
                if (NQ == 1 && j > a_t) wait(&o_done[t], outs - 1);
                ptx::tmem_st_wait();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&p_ready[place]);
                ++outs;
            }
            // the segment's result: outputs, or this CTA's part of them
            const bool has = b_t > a_t;
            float l = (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
            if (has) {
                wait(&o_done[t], outs - 1);
                ptx::tc_fence_after();
            }
            const bool whole = off == 0 && sg.take == uint32_t(it.units);
            const uint32_t a = x - off;  // the item's first unit
            PagedJoin J{r, g, b, int(a / st.chunk), 0};
            J.count = int((a + uint32_t(it.units) - 1) / st.chunk) - J.first + 1;
            float* part = p.part + part_slot(int(blockIdx.x), J.first) * PL::kFloats;
            const int prow = t * qt * p.G + row;  // rows of both tiles in order
            __nv_bfloat16* out = p.O + (int64_t(it.q.q0 + it.i0 + t * qt + i) * p.H + g * p.G + (row - i * p.G)) * D;
            const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
            const bool odd = has && *reinterpret_cast<volatile int*>(&odd_seen) != 0;
            if (!whole && live) {
                part[prow] = any ? -mc : -INFINITY;
                part[kRows + prow] = l;
            }
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                float o[32];
                __syncwarp();
                if (has) {
                    ptx::tmem_ld_32(o_col + c, o);
                    ptx::tmem_ld_wait_32(o);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0.0f;
                }
                if (odd) {
                    for (int j = sg.j0; j < sg.j1; ++j) {  // the tiles that such values left
                        const int key0 = j * KT;
                        if (!(key0 < it.lo_all || min(key0 + KT, it.q.L) > it.hi_all)) continue;
                        for (int key = max(keys.lo, key0); key < min(keys.hi, key0 + KT); ++key) {
                            const int page = p.table[int64_t(r) * p.max_pages + (key >> p.page_shift)];
                            if (page < 0 || page >= p.n_pages) continue;
                            const int64_t slot = (int64_t(page) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
                            const uint32_t* v = reinterpret_cast<const uint32_t*>(p.V + (slot * p.Hk + g) * D + c);
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const uint32_t w = v[e];
                                const float2 f = unpack_bf16x2(w);
                                if (not_finite(w)) o[2 * e] += f.x;
                                if (not_finite(w >> 16)) o[2 * e + 1] += f.y;
                            }
                        }
                    }
                }
                if (!live) continue;
                if (whole) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint4 u;
                        u.x = pack_bf16x2(__fmul_rn(o[e], inv), __fmul_rn(o[e + 1], inv));
                        u.y = pack_bf16x2(__fmul_rn(o[e + 2], inv), __fmul_rn(o[e + 3], inv));
                        u.z = pack_bf16x2(__fmul_rn(o[e + 4], inv), __fmul_rn(o[e + 5], inv));
                        u.w = pack_bf16x2(__fmul_rn(o[e + 6], inv), __fmul_rn(o[e + 7], inv));
                        *reinterpret_cast<uint4*>(out + c + e) = u;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<float4*>(PL::value(part, prow, c + e)) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                }
            }
            if (has) {
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&o_free[t]);
            }
            if (!whole) {
                soft_bar();
                if (threadIdx.x == 0) part_publish(p.flags + J.first);
                if (threadIdx.x == 0) cut[joins] = J;
                ++joins;
            }
            x += sg.take;
            off = 0;
            if (x < st.x1) next_item(p, r, g, b, it.q.n);
        }
        // Every CTA joins its share of the items that it has a part in, once all their parts are there. The CTAs of
        // the grid all run at once (a cooperative launch), and each publishes its parts before it waits.
        if (joins > 0) soft_bar();
        for (int k = 0; k < joins; ++k) {
            const PagedJoin J = cut[k];
            if (threadIdx.x == 0) joined = part_wait(p.flags + J.first, J.count, &abort_flag, p.status);
            soft_bar();
            const bool in = joined != 0;
            if (in) join_store<D, kRows, 4, 2>(p, J, paged_req(p, J.r), int(blockIdx.x) - J.first, threadIdx.x, 32 * T::kSoftWarps);
            soft_bar();  // before the next item's answer
        }
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == T::kSoftWarps) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, kTmemAll);
    }
}

template <int D, int CAP>
cudaError_t launch_many(PagedParams& p, const PagedAttnArgs& a, cudaStream_t s) {
    using T = ManyTraits<D>;
    // the opt-in shared-memory size is a per-device function attribute
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (dev < 0 || dev >= 64 || !done[dev]) {
            e = cudaFuncSetAttribute(paged_many_kernel<D, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
            if (e != cudaSuccess) return e;
            if (dev >= 0 && dev < 64) done[dev] = true;
        }
    }
    // An item has two full row tiles (one with heads of 256), less while the call would leave SMs without a unit: a small
    // item's partial results are sooner written and joined (50 queries of 8 heads over 866 keys: 256 rows 16.2 us, 32 rows 11.0)
    const int sms = std::max(1, device_sm_count());
    p.QT = 128 / p.G;
    p.QB = T::NQ * p.QT;
    while (p.QB * p.G > 16 && p.QB > 1 && unit_bound(a, p.QB, T::KT) < 0.6 * sms) {
        if (p.QB > p.QT) p.QB = p.QT;
        else p.QB = p.QT = (p.QT + 1) / 2;
    }
    const uint32_t box = uint32_t(std::min<int64_t>(a.page_size, T::KT));
    if (!encode_cache(&p.k_map, a.k_cache, a, box) || !encode_cache(&p.v_map, a.v_cache, a, box) ||
        !encode_queries(&p.q_map, a, uint32_t(p.G), uint32_t(p.QT)))
        return cudaErrorInvalidValue;
    const size_t part = size_t(128 * T::NQ) * (D + 2) * 4;
    const int fit = int((EMB_PAGED_WORKSPACE - kPagedFlagBytes) / (2 * part));
    const int ctas = std::max(1, std::min({sms, fit, int(kPagedFlagBytes / 4)}));
    void* args[] = {&p};
    const unsigned grid = unsigned(std::max(2.0, std::min(double(ctas), unit_bound(a, p.QB, T::KT))));
    set_grid(p, grid, D == 256 ? 8 : 2);

    return launch_serialised(reinterpret_cast<const void*>(paged_many_kernel<D, CAP>), grid, T::kThreads, T::kSmem, s, args, 1, true);
}

template <int D>
cudaError_t launch_many_d(PagedParams& p, const PagedAttnArgs& a, cudaStream_t s) {
    return a.cap > kMostLowCap ? launch_many<D, kAnyCap>(p, a, s) : a.cap > 0.0f ? launch_many<D, kLowCap>(p, a, s) : launch_many<D, kUncapped>(p, a, s);
}

}  // namespace

cudaError_t launch_paged_many(PagedParams& p, const PagedAttnArgs& a, cudaStream_t s) {
    return a.head_dim == 64 ? launch_many_d<64>(p, a, s) : a.head_dim == 128 ? launch_many_d<128>(p, a, s) : launch_many_d<256>(p, a, s);
}

}  // namespace emb
