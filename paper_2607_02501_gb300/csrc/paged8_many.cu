// Attention of new tokens over the 8-bit paged cache, many query rows per request: tcgen05 (definition in
// include/emb_paged.h, work split in paged_sched.cuh).
//
// As the kernel for the bf16 cache (paged_many.cu): an item has two tiles of up to 128 rows (one with heads of 256), S = Q K^T
// into tensor memory, a warpgroup of softmax per row tile with a thread a row, O += P V with P in the place of its
// scores. What differs:
// - Keys stay codes: they are the B operand of kind::f8f6f4 as TMA brings them. A row of queries, times a power of two, is
//   split into two e4m3 numbers per element, the nearest and the rest, by its softmax thread when the tile has arrived: 8 bits
//   of significand together, as bf16 has, so the split is exact but for elements below 2^-9 of the row's largest (within
//   2^-17 of it). Two products at twice the f16 rate cost what one would, the keys need no conversion, and shared
//   memory, whose bandwidth f16 operands of this shape use up, has less to move.
// - Values become f16 tiles in shared memory by two warps of their own. Weights are f16 (as e4m3, also in two parts, tails of
//   many small ones would be lost).
// - The blocks' powers: a row's scores of a block are multiplied by its key power, the running maximum is that of score plus value
//   exponent, and the sum of weights takes the value power out again (see paged8_few.cu). Weights are times 2^6, and
//   the maximum may lag by 2^8: below f16's largest.
// What bounds it. Heads of 128: 4096 new tokens of 32 heads over 16384 keys take 761 us (1260 TFLOP/s, 0.66 of the measured matrix rate; the
// bf16 cache's kernel 600 to 674): a tile's chain of scores, softmax and product, of which the blocks' powers lengthen the softmax, beside some 272 KB
// that two row tiles move through shared memory a key tile, half of its time. Heads of 256: 816 tokens of two requests 33 us, shared memory's
// bandwidth (values are read, written and read).
#include <algorithm>
#include <cfloat>
#include <mutex>

#include "paged8.cuh"

namespace emb {
namespace {

template <int D>
struct Many8Traits {
    static constexpr int NQ = D == 256 ? 1 : 2;        // row tiles of an item
    static constexpr int KT = D == 256 ? 64 : 128;     // keys of a tile
    static constexpr int NB = KT / kBlock8;            // blocks of a tile
    static constexpr int kSoftWarps = 4 * NQ;
    // then the MMA and the producer warp and two that convert values; with two row tiles these hand registers to the
    // softmax, a thread of which holds 128 scores: 384 threads x 168 at launch, then 2 x 128 x 216 + 128 x 72
    static constexpr int kThreads = 32 * (kSoftWarps + 4);
    static constexpr int kQTile = 128 * D * 2;         // bytes of a row tile's queries
    static constexpr int kRaw = KT * D;                // bytes of a tile of codes
    static constexpr int kConv = KT * D * 2;           // bytes of a tile of f16 values
    static constexpr int kKeys = D == 64 ? 6 : 3, kVals = D == 64 ? 6 : 3, kConvs = D == 64 ? 4 : 2;  // ring places
    static constexpr int kSmem = 1024 + NQ * kQTile + (kKeys + kVals) * kRaw + kConvs * kConv;
    static constexpr int W = D < 128 ? D : 128;        // bytes of a row of a code tile's part
    static constexpr int kSub = KT * 128;              // bytes of 64 dims of an f16 tile, and of 128 of a code tile
    // columns of tensor memory: scores (two places), outputs
    static constexpr int kO = 2 * KT;
    // and, where there is room (not with heads of 128), the split queries: as an operand in shared memory they take as much of its
    // bandwidth as the keys and more (816 tokens of two requests, heads of 256: 38.8 us, so 35.2)
    static constexpr bool kQTmem = D != 128;
    static constexpr int kQ = kO + NQ * D, kQCols = D / 2;
    static_assert(!kQTmem || kQ + NQ * kQCols <= 512, "columns");
    // Byte offset of 16-byte chunk c of row r in a code tile as TMA swizzles it.
    static __device__ __forceinline__ uint32_t place(int r, int c) {
        if constexpr (D == 64) return uint32_t(r * 64 + ((c ^ (r >> 1 & 3)) << 4));
        return uint32_t((c >> 3) * kSub + r * 128 + (((c & 7) ^ (r & 7)) << 4));
    }
};
constexpr uint32_t kTmemAll = 512;
static_assert(Many8Traits<64>::kSmem > 114 * 1024 && Many8Traits<128>::kSmem > 114 * 1024 && Many8Traits<256>::kSmem > 114 * 1024,
              "one CTA per SM: tensor memory is allocated whole (see ptx::tmem_alloc)");
// Tiles whose exponents are held. The producer writes them ahead of a tile's keys; the softmax reads them once it has the tile's scores,
// and the producer writes those of tile n + kKeys + 1 only behind products that wait for the weights of tile n. (With a barrier of their
// own, awaited ahead of the scores, warps whose rows do not see a tile need holding back too; 4096 tokens of 32 heads of 128 that see all of
// 16384 keys took 864 us so and 824 this way, with heads of 64 816 and 715.)
constexpr int kScaleTiles = 8;
static_assert(Many8Traits<64>::kKeys < kScaleTiles && Many8Traits<128>::kKeys < kScaleTiles && Many8Traits<256>::kKeys < kScaleTiles,
              "a tile's exponents outlast the wait for its weights");
constexpr float kLift = 6.0f;     // the running maximum is held that much lower: weights are times 2^6,
constexpr float kMostLag = 8.0f;  // and it moves when it is exceeded by as much more

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// A place of a ring and the parity of the turn it is in, carried along.
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
    using T = Many8Traits<D>;
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

// Row `row` of a tile of bf16 queries (rows of 64 dims, 128 bytes, swizzled): 16-byte chunk c of it, the largest magnitude.
__device__ __forceinline__ uint4* query_chunk(uint8_t* tile, int row, int c) {
    return reinterpret_cast<uint4*>(tile + (c >> 3) * 16384 + row * 128 + (((c & 7) ^ (row & 7)) << 4));
}
template <int D>
__device__ __forceinline__ float query_top(uint8_t* tile, int row) {
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
        const uint4 w = *query_chunk(tile, row, c);
        const uint32_t h[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 u = unpack_bf16x2(h[e]);
            top = max3(top, fabsf(u.x), fabsf(u.y));
        }
    }
    return top;
}
// Sixteen elements (chunks c and c + 1) times `by` as nearest codes and rests.
__device__ __forceinline__ void split16(uint8_t* tile, int row, int c, float by, uint32_t* hi, uint32_t* lo) {
    const uint4 w0 = *query_chunk(tile, row, c), w1 = *query_chunk(tile, row, c + 1);
    const uint32_t h[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 x = unpack_bf16x2(h[2 * q]), y = unpack_bf16x2(h[2 * q + 1]);
        const float f[4] = {x.x * by, x.y * by, y.x * by, y.y * by};
        hi[q] = codes_of(f[0], f[1]) | codes_of(f[2], f[3]) << 16;
        uint32_t h0, h1;
        codes_to_f16x4(hi[q], h0, h1);
        const float2 g0 = __half22float2(*reinterpret_cast<__half2*>(&h0)), g1 = __half22float2(*reinterpret_cast<__half2*>(&h1));
        lo[q] = codes_of(f[0] - g0.x, f[1] - g0.y) | codes_of(f[2] - g1.x, f[3] - g1.y) << 16;
    }
}
// Splits a row: into tensor memory from column q_col on (called by whole warps), nearest codes first; or in place, the nearest codes in
// the first parts of 64 dims, the rests in the others. Returns the power that takes the scores back.
template <int D, bool TMEM>
__device__ __forceinline__ float split_row(uint8_t* tile, int row, bool negate, uint32_t q_col) {
    constexpr int C = D / 8;
    const RowPower pr = row_power(query_top<D>(tile, row));
    const float by = pr.to * (negate ? -0.0078125f : 0.0078125f);  // below 2^8
    if constexpr (TMEM) {
#pragma unroll 1
        for (int c = 0; c < C; c += 8) {
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) split16(tile, row, c + 2 * i, by, hi + 4 * i, lo + 4 * i);
            ptx::tmem_st_16(q_col + c * 2, hi);
            ptx::tmem_st_16(q_col + D / 4 + c * 2, lo);
        }
        ptx::tmem_st_wait();
    } else {
        // (the nearest codes take the place of what has been read, the rests wait until all has been)
        uint32_t rest[C / 2][4];
#pragma unroll
        for (int c = 0; c < C; c += 2) {
            uint32_t hi[4];
            split16(tile, row, c, by, hi, rest[c / 2]);
            *query_chunk(tile, row, c / 2) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        }
#pragma unroll
        for (int c = 0; c < C / 2; ++c) *query_chunk(tile, row, C / 2 + c) = make_uint4(rest[c][0], rest[c][1], rest[c][2], rest[c][3]);
    }
    return pr.back * 128.0f;
}

template <int D, int CAP>
__global__ void __launch_bounds__(Many8Traits<D>::kThreads, 1) paged_codes_many_kernel(const __grid_constant__ Paged8Params p) {
    using T = Many8Traits<D>;
    constexpr int NQ = T::NQ, KT = T::KT, NB = T::NB;
    constexpr int kRows = 128 * NQ;
    using PL = PartLayout<D, kRows>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t k_full[T::kKeys], k_empty[T::kKeys], raw_full[T::kVals], raw_empty[T::kVals], v_full[T::kConvs], v_empty[T::kConvs];
    __shared__ uint64_t q_full, q_ready, q_empty, s_full[2], p_ready[2], o_done[2], o_free[2], drain;
    __shared__ float2 scales[kScaleTiles][NB];  // of a block: block_power of its keys, e of its values
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, joined, odd_seen;
    __shared__ PagedJoin cut[2];
    uint8_t* sq = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* kring = sq + NQ * T::kQTile;
    uint8_t* vring = kring + T::kKeys * T::kRaw;
    uint8_t* conv = vring + T::kVals * T::kRaw;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned all = 0xffffffffu;

    if (threadIdx.x == 0) {
        for (int i = 0; i < T::kKeys; ++i) {
            ptx::mbar_init(&k_full[i], 1);
            ptx::mbar_init(&k_empty[i], 1);
        }
        for (int i = 0; i < T::kVals; ++i) {
            ptx::mbar_init(&raw_full[i], 1);
            ptx::mbar_init(&raw_empty[i], 2);
        }
        for (int i = 0; i < T::kConvs; ++i) {
            ptx::mbar_init(&v_full[i], 2);
            ptx::mbar_init(&v_empty[i], 1);
        }
        ptx::mbar_init(&q_full, 1);
        ptx::mbar_init(&q_ready, T::kSoftWarps);
        ptx::mbar_init(&q_empty, T::kQTmem ? T::kSoftWarps : 1);
        for (int t = 0; t < 2; ++t) {
            ptx::mbar_init(&s_full[t], 2);
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
    // (the tiles of the stretch are numbered through, over all its items)

    if (warp == T::kSoftWarps + 1) {
        // ---------------------------------------------------------------------- producer
        if constexpr (NQ == 2) ptx::regs_down<72>();
        ptx::fence_proxy_async_global();  // (the cache and the queries were written by ordinary stores)
        const int page_size = 1 << p.page_shift, box = min(page_size, KT), n_box = KT / box;
        const int qt = p.QT;
        uint32_t keys = 0, values = 0, items = 0;  // tiles of codes and items with queries issued
        RingPlace<T::kKeys> ka;
        RingPlace<T::kVals> va;
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
            // A round of tiles at a time, 2 NB lanes each: first for the tile's blocks of keys, then for those of values. A lane looks up its
            // block's page one round ahead of its exponent, and that a round before it is used. Boxes that no query sees, and pages
            // that do not exist, are fetched from behind the cache: zeros.
            constexpr int kRound = 32 / (2 * NB);
            // (unsigned: a few tiles behind the longest request's end it may wrap, and is not used)
            auto key_of = [&](int j) { return int(uint32_t(j + lane / (2 * NB)) * KT + (lane & (NB - 1)) * kBlock8); };
            auto page_of = [&](int j) {
                const int key = key_of(j), key_box = key & ~(box - 1);
                int page = p.n_pages;
                if (j + lane / (2 * NB) < sg.j1 && key_box < it.hi && key_box + box > it.lo) {
                    page = row[key >> p.page_shift];
                    if (page < 0 || page > p.n_pages) page = p.n_pages;
                }
                return page;
            };
            auto exp_of = [&](int j, int page) {
                const int64_t at = ((int64_t(page) << p.page_shift) + (key_of(j) & (page_size - 1))) / kBlock8 * p.Hk + g;
                uint32_t e = kExpBias;
                if (page < p.n_pages) e = (lane & NB ? p.v_exp : p.k_exp)[at];
                return e;
            };
            int page = page_of(sg.j0), page1 = page_of(sg.j0 + kRound), page2 = 0;
            uint32_t ex = exp_of(sg.j0, page), ex1 = 0;
            for (int j = sg.j0; j < sg.j1 && ok; ++j) {
                const int turn = (j - sg.j0) & (kRound - 1);
                if (turn == 0) {
                    if (j > sg.j0) {
                        page = page1;
                        page1 = page2;
                        ex = ex1;
                    }
                    page2 = page_of(j + 2 * kRound);
                    ex1 = exp_of(j + kRound, page1);
                }
                const int place = (j * KT) & (page_size - 1);
                auto fetch = [&](uint8_t* to, const CUtensorMap* map, uint64_t* bar) {
                    if (ptx::elect_one()) ptx::mbar_arrive_expect_tx(bar, T::kRaw);
                    __syncwarp();
                    for (int i = 0; i < n_box; ++i) {
                        const int pg = __shfl_sync(all, page, turn * 2 * NB + i * (box / kBlock8));
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int c = 0; c < D / T::W; ++c)
                                ptx::tma_load_4d(to + c * T::kSub + i * box * T::W, map, bar, c * T::W, g, place, pg);
                        }
                        __syncwarp();
                    }
                };
                if (keys >= uint32_t(T::kKeys)) ok = wait(&k_empty[ka.slot], ka.turn ^ 1u);
                if (!ok) break;
                const int e = exp_of_byte(ex), s = int(keys % kScaleTiles);
                if (lane / (2 * NB) == turn) {
                    if (lane & NB) scales[s][lane & (NB - 1)].y = float(e);
                    else scales[s][lane & (NB - 1)].x = block_power<CAP>(e);
                }
                __syncwarp();  // (published with the keys' barrier)
                fetch(kring + ka.slot * T::kRaw, &p.k_map, &k_full[ka.slot]);
                ++keys;
                ka.next();
                if (values >= uint32_t(T::kVals)) ok = wait(&raw_empty[va.slot], va.turn ^ 1u);
                if (!ok) break;
                fetch(vring + va.slot * T::kRaw, &p.v_map, &raw_full[va.slot]);
                ++values;
                va.next();
            }
            x += sg.take;
            off = 0;
            if (x < st.x1) next_item(p, r, g, b, it.q.n);
        }
        // every copy must land before this CTA's shared memory is released
        for (uint32_t i = keys > uint32_t(T::kKeys) ? keys - T::kKeys : 0; i < keys; ++i)
            ptx::mbar_wait(&k_full[i % T::kKeys], (i / T::kKeys) & 1, nullptr, p.status, kWaitLimitNs);
        for (uint32_t i = values > uint32_t(T::kVals) ? values - T::kVals : 0; i < values; ++i)
            ptx::mbar_wait(&raw_full[i % T::kVals], (i / T::kVals) & 1, nullptr, p.status, kWaitLimitNs);
        if (items > 0) ptx::mbar_wait(&q_full, (items - 1) & 1, nullptr, p.status, kWaitLimitNs);
    } else if (warp == T::kSoftWarps) {
        // ------------------------------------------------------------------------- MMAs
        if constexpr (NQ == 2) ptx::regs_down<72>();
        constexpr uint32_t idesc_qk = ptx::idesc_e4m3_f32(128, KT), idesc_pv = ptx::idesc_f16_f32(128, D) | ptx::kIdescMnMajorB;
        const uint32_t sq_u = ptx::smem_u32(sq), kring_u = ptx::smem_u32(kring), conv_u = ptx::smem_u32(conv);
        uint32_t n = 0, items = 0;
        RingPlace<T::kKeys> keys;     // of tile j
        RingPlace<T::kConvs> values;  // of the tile before it
        uint32_t scores[2] = {0, 0}, owned[2] = {0, 0};  // score tiles by place, items with outputs by row tile
        bool ok = true, used = false;  // used: a product of the tile's values was issued
        // (operands in a form that the compiler knows to be uniform: see ptx::elect_one)
        auto qk = [&](int t, int place, int slot) {  // S[place] = Q[t] K^T, nearest codes and rests
            const uint32_t k = ptx::warp_uniform(kring_u + uint32_t(slot * T::kRaw));
            const uint32_t q = T::kQTmem ? ptx::warp_uniform(tmem + uint32_t(T::kQ + t * T::kQCols)) : sq_u + uint32_t(t * T::kQTile);
            const uint32_t d = ptx::warp_uniform(tmem + uint32_t(place * KT));
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int ks = 0; ks < D / 32; ++ks) {
                    const uint32_t more = part + ks != 0;
                    if constexpr (T::kQTmem) {
                        const uint64_t db = D == 64 ? ptx::smem_desc_sw64(k) + 2 * ks : ptx::smem_desc_sw128(k + (ks / 4) * T::kSub) + 2 * (ks & 3);
                        ptx::mma_f8_ta(d, q + uint32_t(part * (D / 4) + ks * 8), db, idesc_qk, more);
                    } else {
                        ptx::mma_f8_ss(d, ptx::smem_desc_sw128(q + (part * (D / 128) + ks / 4) * 16384) + 2 * (ks & 3),
                                       ptx::smem_desc_sw128(k + (ks / 4) * T::kSub) + 2 * (ks & 3), idesc_qk, more);
                    }
                }
            ptx::mma_commit(&s_full[place]);
            if (lane == 0) ptx::mbar_arrive(&s_full[place]);  // (and hands on what the keys' barrier published: the block powers)
        };
        auto pv = [&](int t, int place, int slot, bool first) {  // O[t] (+)= P[place] V
            const uint64_t desc = ptx::smem_desc_mn_sw128(ptx::warp_uniform(conv_u + uint32_t(slot * T::kConv)), T::kSub);
            const uint32_t d = ptx::warp_uniform(tmem + uint32_t(T::kO + t * D)), a = ptx::warp_uniform(tmem + uint32_t(place * KT));
            const uint32_t more = ptx::warp_uniform(first ? 0u : 1u);
#pragma unroll
            for (int kk = 0; kk < KT / 16; ++kk)
                ptx::mma_f16_ta(d, a + uint32_t(8 * kk), desc + uint32_t(kk * 2048 / 16), idesc_pv, kk == 0 ? more : 1u);
            ptx::mma_commit(&o_done[t]);
        };
        while (x < st.x1 && ok) {
            const Segment<D> sg = segment_of<D>(p, r, g, b, off, x, st.x1);
            if (sg.j1 > sg.j0) {
                ok = wait(&q_ready, items++);
                ptx::tc_fence_after();
                for (int j = sg.j0; j <= sg.j1 && ok; ++j) {
                    if (j < sg.j1) ok = wait(&k_full[keys.slot], keys.turn);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    auto finish = [&](int t, int place) {  // P V of tile j - 1
                        const bool first = j - 1 == sg.a[t];
                        ok = wait(&v_full[values.slot], values.turn) && wait(&p_ready[place], scores[place] - 1);
                        if (ok && first && owned[t] > 0) ok = wait(&o_free[t], owned[t] - 1);
                        if (!ok) return;
                        ptx::tc_fence_after();
                        pv(t, place, values.slot, first);
                        used = true;
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
                    if (j > sg.j0) {
                        // (a tile that no row tile needed is handed back no sooner than it has arrived)
                        if (!used) ok = wait(&v_full[values.slot], values.turn);
                        if (!ok) break;
                        used = false;
                        ptx::mma_commit(&v_empty[values.slot]);
                        values.next();
                    }
                    if (j < sg.j1) {
                        ptx::mma_commit(&k_empty[keys.slot]);
                        ++n;
                        keys.next();
                        if (!T::kQTmem && j == sg.j1 - 1) ptx::mma_commit(&q_empty);
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
        // ------------------------------------------------------ values to f16, half a tile a warp
        if constexpr (NQ == 2) ptx::regs_down<72>();
        // a thread's first key and chunk, keys to its next one, steps over the keys (heads of 256: twice)
        constexpr int kStep = D == 64 ? 16 : 8, kSteps = KT / kStep, kEach = KT * D / 16 / 64;
        // Chunks in flight: more of them hold up the softmax, whose accesses stand behind these in the load and store unit (when it was
        // chosen, us: 4096 tokens over 16384 keys 1 808, 2 818, 4 843, 8 936; 816 of two requests with heads of 256 1 41, 2 39, 4 41).
        constexpr int kBatch = D == 256 ? 2 : 1;
        const int key_first = (lane & 7) + (D == 64 ? (warp & 1) * 8 : 0), c_first = (D == 64 ? 0 : (warp & 1) * 4) + lane / 8;
        uint32_t n = 0;
        RingPlace<T::kVals> from;
        RingPlace<T::kConvs> to;
        bool ok = true;
        while (x < st.x1 && ok) {
            int j, j1, L, lo_all, hi_all, queries;  // (little of a segment is kept: registers are few here)
            {
                const Segment<D> sg = segment_of<D>(p, r, g, b, off, x, st.x1);
                j = sg.j0;
                j1 = sg.j1;
                L = sg.it.q.L;
                lo_all = sg.it.lo_all;
                hi_all = sg.it.hi_all;
                queries = sg.it.q.n;
                x += sg.take;
                off = 0;
            }
            for (; j < j1 && ok; ++j, ++n) {
                const int key0 = j * KT;
                // Values behind the request's last key are anything: zeros. NaN codes hidden from some rows may not be
                // multiplied by their weights of 0: they leave the tile here and are added at the item's end for the rows that
                // see them.
                const bool tail = key0 + KT > L, hidden = key0 < lo_all || min(key0 + KT, L) > hi_all;
                ok = wait(&raw_full[from.slot], from.turn);
                if (ok && n >= uint32_t(T::kConvs)) ok = wait(&v_empty[to.slot], to.turn ^ 1u);
                if (!ok) break;
                const uint8_t* in = vring + from.slot * T::kRaw;
                uint8_t* out = conv + to.slot * T::kConv;
                uint32_t odd = 0;
                // 16 codes of a key at a time; eight lanes have neighbouring keys, which meet in no bank
                const uint8_t* at = in + T::place(key_first, c_first);
                uint8_t* row = out + (c_first >> 2) * T::kSub + key_first * 128;
                const int s0 = (((c_first & 3) * 2) ^ (key_first & 7)) << 4, s1 = (((c_first & 3) * 2 + 1) ^ (key_first & 7)) << 4;
                auto from_of = [](int i) { return (i % kSteps) * kStep * T::W + (i / kSteps) * T::kSub; };
                auto to_of = [](int i) { return (i % kSteps) * kStep * 128 + (i / kSteps) * 2 * T::kSub; };
                auto fetch = [&](int i, uint4 (&w)[kBatch]) {
#pragma unroll
                    for (int k = 0; k < kBatch; ++k) w[k] = *reinterpret_cast<const uint4*>(at + from_of(i + k));
                };
                auto put = [&](int i, uint4 (&w)[kBatch]) {
#pragma unroll
                    for (int k = 0; k < kBatch; ++k) {
                        if (tail && key0 + key_first + (i + k) % kSteps * kStep >= L) w[k] = make_uint4(0, 0, 0, 0);
                        if (hidden) {
                            const uint32_t bx = nan_codes(w[k].x), by = nan_codes(w[k].y), bz = nan_codes(w[k].z), bw = nan_codes(w[k].w);
                            odd |= bx | by | bz | bw;
                            w[k] = make_uint4(without(w[k].x, bx), without(w[k].y, by), without(w[k].z, bz), without(w[k].w, bw));
                        }
                        uint4 a, d;
                        codes_to_f16x4(w[k].x, a.x, a.y);
                        codes_to_f16x4(w[k].y, a.z, a.w);
                        codes_to_f16x4(w[k].z, d.x, d.y);
                        codes_to_f16x4(w[k].w, d.z, d.w);
                        *reinterpret_cast<uint4*>(row + to_of(i + k) + s0) = a;
                        *reinterpret_cast<uint4*>(row + to_of(i + k) + s1) = d;
                    }
                };
                uint4 w[kBatch];
#pragma unroll 1
                for (int i = 0; i < kEach; i += kBatch) {
                    fetch(i, w);
                    put(i, w);
                }
                // (never taken back: the softmax may be some items behind. Items without such codes are then searched for nothing)
                if (odd) *reinterpret_cast<volatile int*>(&odd_seen) = 1;
                ptx::fence_proxy_async_smem();
                __threadfence_block();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(&v_full[to.slot]);
                    ptx::mbar_arrive(&raw_empty[from.slot]);
                }
                from.next();
                to.next();
            }
            if (x < st.x1) next_item(p, r, g, b, queries);
        }
    } else {
        // ---------------------------------------------------------------------- softmax
        if constexpr (NQ == 2) ptx::regs_up<216>();
        zero_padding(p, D, threadIdx.x, 32 * T::kSoftWarps);
        const int t = warp >> 2;  // row tile
        const int row = 32 * (warp & 3) + lane, qt = p.QT, i = row / p.G;
        const uint32_t lanes = uint32_t(32 * (warp & 3)) << 16;
        const uint32_t o_col = tmem + lanes + uint32_t(T::kO + t * D);
        uint32_t n = 0, seen[2] = {0, 0}, outs = 0, items = 0;
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
            float back = 1.0f;
            if (sg.j1 > sg.j0) {
                wait(&q_full, items++);
                // (this row tile's products of the item before have read its queries: their scores were waited for)
                const float power = split_row<D, T::kQTmem>(sq + t * T::kQTile, row, p.negate, tmem + lanes + uint32_t(T::kQ + t * T::kQCols));
                if (live) back = power;
                if constexpr (T::kQTmem) ptx::tc_fence_before();
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(&q_ready);
                    if (T::kQTmem) ptx::mbar_arrive(&q_empty);
                }
            }
            if constexpr (!CAP) back = row_factor(back, p.scale2);
            // whether the row has seen a score, its running maximum of score plus value exponent in base 2 (negated and lifted, so
            // that it is added), sums of weights without the values' powers
            bool any = false;
            float mc = 0.0f;
            float2 l2 = make_float2(0, 0);
            const uint32_t behind = n + uint32_t(sg.j1 - sg.j0);
            n += uint32_t(max(a_t - sg.j0, 0));
            for (int j = a_t; j < b_t; ++j, ++n) {
                const int place = NQ == 2 ? t : int(n & 1);
                wait(&s_full[place], seen[place]++);
                ptx::tc_fence_after();
                // The factors of the blocks' raw scores, held so that a product neither overflows nor makes NaN of what is hidden,
                // and the values' exponents: read beside the first scores.
                const float2* block = scales[n % kScaleTiles];
                float by[NB], up[NB];
                auto factor = [&](float power) { return fminf(fmaxf(back * power, 1e-37f), 3.0e38f); };
#pragma unroll
                for (int k = 0; k < NB; ++k) {
                    const float2 bl = block[k];
                    by[k] = factor(bl.x);
                    up[k] = bl.y;
                }
                const uint32_t s_col = tmem + lanes + uint32_t(place * KT);
                const int key0 = j * KT;
                const bool edge = key0 < it.lo_all || key0 + KT > it.hi_all;
                const int lo = keys.lo - key0, hi = keys.hi - key0;
                // Votes are taken among rows that see a key of the tile. A tile's other rows are not of this request, or not
                // even filled (3 heads: 126 of 128 rows), and what they hold may not decide how a warp computes.
                const bool sees = max(lo, 0) < min(hi, KT);
                float zt = -INFINITY, far = 0.0f;  // far, for a cap: the largest magnitude of q.k that the row sees
                // What stands for a score that the row does not see: of a tile without any, nothing. (A product q.k of -infinity is a score
                // of -cap and counts.)
                const float gone = edge ? -INFINITY : NAN;
                if (edge) {
                    // Scores that the row does not see, in tensor memory: rolled up and away from the path of most tiles. Under a cap the
                    // others become the products q.k here, held above what stands for those.
#pragma unroll 1
                    for (int c = 0; c < KT; c += 32) {
                        float v[32];
                        uint32_t w[32];
                        ptx::tmem_ld_32(s_col + c, v);
                        ptx::tmem_ld_wait_32(v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const bool in = c + e >= lo && c + e < hi;
                            float u = v[e];
                            if constexpr (CAP) {
                                u *= factor(block[c / 16 + e / 16].x);
                                if (in) far = fmaxf(far, fabsf(u));
                                u = u < -FLT_MAX ? -FLT_MAX : u;  // (NaN stays NaN)
                            }
                            w[e] = __float_as_uint(in ? u : -INFINITY);
                        }
                        ptx::tmem_st_32(s_col + c, w);
                    }
                    ptx::tmem_st_wait();
                    if constexpr (CAP) {
#pragma unroll
                        for (int k = 0; k < NB; ++k) by[k] = 1.0f;
                    }
                }
                float s[KT];
#pragma unroll
                for (int c = 0; c < KT; c += 32) ptx::tmem_ld_32(s_col + c, s + c);
#pragma unroll
                for (int c = 0; c < KT; c += 32) {
                    ptx::tmem_ld_wait_32(s + c);
#pragma unroll
                    for (int h = c; h < c + 32; h += 16) {
                        // score plus value exponent, rounded here, so that what exceeds no maximum exceeds no bound below; or for a
                        // cap q.k yet
                        const float2 f = make_float2(by[h / 16], by[h / 16]), e2 = make_float2(up[h / 16], up[h / 16]);
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            const float2 u = make_float2(s[h + e], s[h + e + 1]), z = CAP ? mul2(u, f) : fma2(u, f, e2);
                            s[h + e] = z.x;
                            s[h + e + 1] = z.y;
                        }
                        float top[5];
#pragma unroll
                        for (int k = 0; k < 5; ++k) top[k] = max3(s[h + 3 * k], s[h + 3 * k + 1], s[h + 3 * k + 2]);
                        const float most = max3(max3(top[0], top[1], top[2]), max3(top[3], top[4], s[h + 15]), -INFINITY);
                        if constexpr (CAP) {
                            // (the maximum is of what the cap is put on: it keeps their order)
                            if (!edge) {
                                float low[5];
#pragma unroll
                                for (int k = 0; k < 5; ++k) low[k] = fminf(fminf(s[h + 3 * k], s[h + 3 * k + 1]), s[h + 3 * k + 2]);
                                const float least = fminf(fminf(fminf(low[0], low[1]), fminf(low[2], low[3])), fminf(low[4], s[h + 15]));
                                far = max3(far, fabsf(most), fabsf(least));
                            }
                            const float z = capped2<CAP>(make_float2(most, most), p).x + up[h / 16];
                            zt = most == gone ? zt : fmaxf(zt, z);
                        } else {
                            zt = fmaxf(zt, most);
                        }
                    }
                }
                const bool grow = sees && (any ? zt + mc > kLift + kMostLag : zt > -INFINITY);
                if (__any_sync(all, grow)) {
                    const float now = kLift - zt;
                    const float f = !grow ? 1.0f : any ? exp2_fast(now - mc) : 0.0f;
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
                        l2.x *= f;
                        l2.y *= f;
                        any = true;
                        mc = now;
                    }
                }
                // The weights, 32 at a time, over the scores. base(u, m) gives two weights' exponents from s, and for q.k that a cap is still to be
                // put on m, their block's value exponent less the row's maximum.
                auto weights = [&](auto base) {
#pragma unroll
                    for (int c = 0; c < KT; c += 32) {
                        uint32_t w[16];
#pragma unroll
                        for (int h = c; h < c + 32; h += 16) {
                            const float m = up[h / 16] + mc;
                            float2 sum = make_float2(0, 0);
#pragma unroll
                            for (int e = 0; e < 16; e += 2) {
                                float2 u = base(make_float2(s[h + e], s[h + e + 1]), make_float2(m, m));
                                u.x = exp2_fast(u.x);
                                u.y = exp2_fast(u.y);
                                sum = add2(sum, u);
                                w[(h - c + e) / 2] = pack_f16x2(u.x, u.y);
                            }
                            const float inv = exp2_fast(-up[h / 16]);
                            l2 = fma2(sum, make_float2(inv, inv), l2);
                        }
                        ptx::tmem_st_16(s_col + c / 2, w);
                    }
                };
                if constexpr (!CAP) {
                    const float2 mm = make_float2(mc, mc);
                    weights([&](float2 u, float2) { return add2(u, mm); });
                } else {
                    auto shown = [gone](float2 u, float2 z) {
                        return make_float2(u.x == gone ? -INFINITY : z.x, u.y == gone ? -INFINITY : z.y);
                    };
                    // (under a large cap a maximum's rounding may be felt in f16's range. NaN stays NaN)
                    auto held = [](float2 z) {
                        if constexpr (CAP == kLowCap) return z;
                        return make_float2(z.x > kLift + kMostLag ? kLift + kMostLag : z.x, z.y > kLift + kMostLag ? kLift + kMostLag : z.y);
                    };
                    // far below the cap one power of two per score, where exponential and reciprocal take two more turns of
                    // the same unit (the series runs away to -infinity at what stands for a hidden score)
                    if (__all_sync(all, !sees || far * p.scale2 < kNearCap))
                        weights([&](float2 u, float2 m) { return held(capped_near2(u, p, m)); });
                    else
                        weights([&](float2 u, float2 m) { return shown(u, held(add2(capped2<CAP>(u, p), m))); });
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
            n = behind;
            // the segment's result: outputs, or this CTA's part of them
            const bool has = b_t > a_t;
            const float l = l2.x + l2.y;
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
                    for (int j = sg.j0; j < sg.j1; ++j) {  // the tiles that such codes left
                        const int key0 = j * KT;
                        if (!(key0 < it.lo_all || min(key0 + KT, it.q.L) > it.hi_all)) continue;
                        for (int key = max(keys.lo, key0); key < min(keys.hi, key0 + KT); ++key) {
                            const int page = p.table[int64_t(r) * p.max_pages + (key >> p.page_shift)];
                            if (page < 0 || page >= p.n_pages) continue;
                            const int64_t slot = (int64_t(page) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
                            const uint32_t* v = reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(p.V) + (slot * p.Hk + g) * D + c);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (nan_codes(v[e / 4]) >> (8 * (e & 3) + 7) & 1u) o[e] = NAN;
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
cudaError_t launch_many8(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s) {
    using T = Many8Traits<D>;
    // the opt-in shared-memory size is a per-device function attribute
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (dev < 0 || dev >= 64 || !done[dev]) {
            e = cudaFuncSetAttribute(paged_codes_many_kernel<D, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
            if (e != cudaSuccess) return e;
            if (dev >= 0 && dev < 64) done[dev] = true;
        }
    }
    // (as for the bf16 cache: full row tiles, less while the call would leave SMs without a unit)
    const int sms = std::max(1, device_sm_count());
    p.QT = 128 / p.G;
    p.QB = T::NQ * p.QT;
    while (p.QB * p.G > 16 && p.QB > 1 && unit_bound(a, p.QB, T::KT) < 0.6 * sms) {
        if (p.QB > p.QT) p.QB = p.QT;
        else p.QB = p.QT = (p.QT + 1) / 2;
    }
    const uint32_t box = uint32_t(std::min<int64_t>(a.page_size, T::KT));
    if (!encode_codes(&p.k_map, a.k_cache, a, box) || !encode_codes(&p.v_map, a.v_cache, a, box) ||
        !encode_queries(&p.q_map, a, uint32_t(p.G), uint32_t(p.QT)))
        return cudaErrorInvalidValue;
    const size_t part = size_t(128 * T::NQ) * (D + 2) * 4;
    const int fit = int((EMB_PAGED_WORKSPACE - kPagedFlagBytes) / (2 * part));
    const int ctas = std::max(1, std::min({sms, fit, int(kPagedFlagBytes / 4)}));
    void* args[] = {&p};
    const unsigned grid = unsigned(std::max(2.0, std::min(double(ctas), unit_bound(a, p.QB, T::KT))));
    set_grid(p, grid, D == 256 ? 8 : 2);
    return launch_serialised(reinterpret_cast<const void*>(paged_codes_many_kernel<D, CAP>), grid, T::kThreads, T::kSmem, s, args, 1, true);
}

template <int D>
cudaError_t launch_many8_d(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s) {
    return a.cap > kMostLowCap ? launch_many8<D, kAnyCap>(p, a, s) : a.cap > 0.0f ? launch_many8<D, kLowCap>(p, a, s) : launch_many8<D, kUncapped>(p, a, s);
}

}  // namespace

cudaError_t launch_paged8_many(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s) {
    return a.head_dim == 64 ? launch_many8_d<64>(p, a, s) : a.head_dim == 128 ? launch_many8_d<128>(p, a, s) : launch_many8_d<256>(p, a, s);
}

}  // namespace emb
