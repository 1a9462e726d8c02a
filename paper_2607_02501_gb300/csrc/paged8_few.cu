// Attention of new tokens over the 8-bit paged cache, few query rows per request: mma.sync (definition in
// include/emb_paged.h, work split in paged_sched.cuh), and the choice between this kernel and that for many rows.
//
// As the kernel for the bf16 cache: a producer warp brings tiles of keys and values by TMA into a ring, an item has 16 rows
// (queries times heads), and each of four warps takes a quarter of a tile's keys; the warps' results are merged at the
// item's end. What differs:
// - Tiles of 128 keys: twice the keys for the same steps of a warp, which are a chain of latencies (64 requests of up to 16384 keys
//   of 8 heads of 128 with tiles of 64 252 us, whatever the stages, 241 with 128).
// - A warp's 32 keys are two blocks of the cache, with a key power and a value power each. The producer looks them up two
//   rounds ahead and lays them beside the tile.
// - Codes become f16 in registers, after ldmatrix, by the hardware's conversion of two at a time. A key's 16 bytes give a lane four
//   neighbouring dims, so the queries' fragments have their dims in that order; transposed by pairs of bytes, a value's 16 bytes
//   give it two dims of two keys, whose even and odd bytes are one fragment of the even dims' outputs and one of the odd dims'.
// - Softmax with the values' powers: with z the score in base 2 and e the exponent of its key's values, the running maximum m is that
//   of z + e, the weight w = 2^(z + e - m) <= 1 multiplies the bare codes, and the sum of weights adds w 2^-e. So w is in f16's
//   range whatever the blocks' powers are: times 2^14, those above 2^-28 of the largest are rounded to 11 bits.
// HBM bounds long histories: those 64 requests' 1.09 GB take 199 to 211 us now, 0.77 to 0.81 of the measured copy rate, and 181 if nothing
// is computed. Latency and the joins bound small calls: one token over 867 keys 6.2 us.
#include <algorithm>
#include <cmath>
#include <mutex>

#include "paged8.cuh"

namespace emb {
namespace {

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm_x4(uint32_t saddr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(saddr));
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t saddr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(saddr));
}

constexpr int kFewWarps = 4;
constexpr int kFewThreads = 32 * (kFewWarps + 1);
constexpr int kFewTile = 128;
constexpr int kFewBlocks = kFewTile / kBlock8;
constexpr int kFewRows = 16;
constexpr int kFewCluster = 8;    // CTAs of a cluster, at most (the portable size)
constexpr float kWeightUnit = 16384.0f;  // the largest weight
static_assert(kFewBlocks == 2 * kFewWarps, "a warp's keys are two blocks");

template <int D>
struct Few8Traits {
    static constexpr int kHalf = kFewTile * D;         // bytes of a tile's keys, and of its values
    static constexpr int kStage = 2 * kHalf;
    static constexpr int kStages = D == 64 ? 6 : 3;
    static constexpr int kCtas = D == 256 ? 1 : 2;     // per SM
    static constexpr int kQPitch = D + 8;              // queries in shared memory (D = 256), f16 per padded row
    static constexpr int kQBytes = D == 256 ? kFewRows * kQPitch * 2 : 0;
    static constexpr int kFinPitch = D + 4;            // a CTA's result for its cluster, fp32 per padded row
    static constexpr int kSmem = 1024 + kStages * kStage + kQBytes;
    static constexpr int kSmemCluster = kSmem + kFewRows * (kFinPitch + 2) * 4;
    static_assert(kFewWarps * kFewRows * D * 4 <= kStage, "the warps' results fit where a tile was");
    // Byte offset of 16-byte chunk c of row r in a tile as TMA swizzles it.
    static __device__ __forceinline__ uint32_t place(int r, int c) {
        if constexpr (D == 64) return uint32_t(r * 64 + ((c ^ (r >> 1 & 3)) << 4));
        return uint32_t((c >> 3) * kFewTile * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
    }
};

template <int D, int CAP, bool CL>
__global__ void __launch_bounds__(kFewThreads, Few8Traits<D>::kCtas) paged_codes_few_kernel(const __grid_constant__ Paged8Params p) {
    using T = Few8Traits<D>;
    constexpr int KS = D / 16, NT = D / 8, ROWS = kFewRows;
    constexpr bool QS = D == 256;  // queries stay in shared memory: their fragments would not fit the registers
    using PL = PartLayout<D, ROWS>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[T::kStages], empty[T::kStages];
    __shared__ float4 powers[T::kStages][kFewBlocks];  // of a block: block_power of its keys; e of its values, 2^-e
    __shared__ int abort_flag, joined;
    __shared__ PagedJoin cut[2];
    __shared__ float warp_m[kFewWarps][16], warp_l[kFewWarps][16], row_back[16];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < T::kStages; ++i) {
            ptx::mbar_init(&full[i], 1);
            ptx::mbar_init(&empty[i], kFewWarps);
        }
        abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tmap(&p.k_map);
        ptx::prefetch_tmap(&p.v_map);
    }
    __syncthreads();
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();  // lengths, queries and the new tokens' keys and values come from earlier launches
    if (p.n_req == 1 && warp == kFewWarps && lane * 32 < p.max_pages) {
        // the only request's row of the table on its way to L1 while the stretch is found
        uint32_t page;
        asm volatile("ld.global.u32 %0, [%1];" : "=r"(page) : "l"(p.table + lane * 32));
    }
    PagedStretch st{};
    int r, g, b = 0, blocks = 0;
    const int S = CL ? p.cluster : 1, rank = CL ? int(blockIdx.x) % S : 0;
    if constexpr (CL) {
        const int id = int(blockIdx.x) / S;
        b = id % p.side;
        g = id / p.side % p.Hk;
        r = id / p.side / p.Hk;
        blocks = (ptx::warp_uniform(paged_req(p, r).n) + p.QB - 1) / p.QB;
    } else {
        st = paged_stretch<kFewTile, kFewThreads>(p);
        r = st.r;
        g = st.g;
        b = st.b;
    }
    uint32_t x = st.x0, off = st.off;
    uint32_t issued = 0;  // tiles so far (ring position and phase)
    if (warp == kFewWarps) {
        // -------------------------------------------------------------------- producer
        ptx::fence_proxy_async_global();  // (the cache was written by ordinary stores)
        const int page_size = 1 << p.page_shift, box = min(page_size, kFewTile), n_box = kFewTile / box;
        uint32_t loads = 0;  // tiles issued: all that were walked through, unless a wait gave up
        while (CL ? b < blocks : x < st.x1) {
            const PagedItem it = paged_item<kFewTile>(p, r, g, b);
            const uint32_t take = min(st.x1 - x, uint32_t(it.units) - off);
            const int j0 = CL ? rank * it.nt / S : int(off), j1 = CL ? (rank + 1) * it.nt / S : min(int(off + take), it.nt);
            const int32_t* row = p.table + int64_t(r) * p.max_pages;
            // Two tiles at a time, sixteen lanes each: eight for the tile's blocks of keys, eight for those of values. A lane looks up its
            // block's page one round ahead of its exponent, and that a round before it is used. Boxes that no query sees, and
            // pages that do not exist, are fetched from behind the cache: zeros.
            constexpr int kRound = 32 / (2 * kFewBlocks);
            // (unsigned: a few tiles behind the longest request's end it may wrap, and is not used)
            auto key_of = [&](int j) { return int(uint32_t(it.t0 + j + lane / (2 * kFewBlocks)) * kFewTile + (lane & (kFewBlocks - 1)) * kBlock8); };
            auto page_of = [&](int j) {
                const int key = key_of(j), key_box = key & ~(box - 1);
                int page = p.n_pages;
                if (j + lane / (2 * kFewBlocks) < j1 && key_box < it.hi && key_box + box > it.lo) {
                    page = row[key >> p.page_shift];
                    if (page < 0 || page > p.n_pages) page = p.n_pages;
                }
                return page;
            };
            auto exp_of = [&](int j, int page) {
                const int64_t at = ((int64_t(page) << p.page_shift) + (key_of(j) & (page_size - 1))) / kBlock8 * p.Hk + g;
                uint32_t e = kExpBias;
                if (page < p.n_pages) e = (lane & kFewBlocks ? p.v_exp : p.k_exp)[at];
                return e;
            };
            int page = page_of(j0), page1 = page_of(j0 + kRound), page2 = 0;
            uint32_t ex = exp_of(j0, page), ex1 = 0;
            for (int j = j0; j < j1; ++j, ++issued) {
                const int in = (j - j0) & (kRound - 1);
                if (in == 0) {
                    if (j > j0) {
                        page = page1;
                        page1 = page2;
                        ex = ex1;
                    }
                    page2 = page_of(j + 2 * kRound);
                    ex1 = exp_of(j + kRound, page1);
                }
                const int s = issued % T::kStages;
                if (issued >= uint32_t(T::kStages))
                    ptx::mbar_wait(&empty[s], (issued / T::kStages - 1) & 1, &abort_flag, p.status, kWaitLimitNs);
                const bool stop = __any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&abort_flag) != 0);
                uint8_t* k = ring + s * T::kStage;
                uint8_t* v = k + T::kHalf;
                if (!stop) {
                    const int e = exp_of_byte(ex);
                    if (lane / (2 * kFewBlocks) == in) {
                        float4& to = powers[s][lane & (kFewBlocks - 1)];
                        if (lane & kFewBlocks) to.y = float(e), to.z = pow2i(-e);
                        else to.x = block_power<CAP>(e);
                    }
                    __syncwarp();
                    if (ptx::elect_one()) ptx::mbar_arrive_expect_tx(&full[s], T::kStage);
                    __syncwarp();
                    const int place = ((it.t0 + j) * kFewTile) & (page_size - 1);
                    for (int i = 0; i < n_box; ++i) {
                        const int pg = __shfl_sync(0xffffffffu, page, in * 2 * kFewBlocks + i * (box / kBlock8));
                        if (ptx::elect_one()) {
                            constexpr int W = D < 128 ? D : 128;
#pragma unroll
                            for (int c = 0; c < D / W; ++c) {
                                ptx::tma_load_4d(k + c * kFewTile * W + i * box * W, &p.k_map, &full[s], c * W, g, place, pg);
                                ptx::tma_load_4d(v + c * kFewTile * W + i * box * W, &p.v_map, &full[s], c * W, g, place, pg);
                            }
                        }
                        __syncwarp();
                    }
                    ++loads;
                }
            }
            if constexpr (CL) {
                ptx::cluster_sync();  // (the compute warps' two)
                ptx::cluster_sync();
                b += p.side;
            } else {
                x += take;
                off = 0;
                if (x < st.x1) next_item(p, r, g, b, it.q.n);
            }
        }
        // every copy must land before this CTA's shared memory is released, also where a wait gave up
        for (uint32_t i = loads > uint32_t(T::kStages) ? loads - T::kStages : 0; i < loads; ++i)
            ptx::mbar_wait(&full[i % T::kStages], (i / T::kStages) & 1, nullptr, p.status, kWaitLimitNs);
        return;
    }

    // ------------------------------------------------------------------------ compute
    // A wait that gave up sets abort_flag; later waits then return at once, and the loops run to their end (the
    // outputs are undefined then), so that every barrier still meets all its threads.
    zero_padding(p, D, threadIdx.x, 32 * kFewWarps);
    auto bar = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
    const int quad = lane >> 2, qc = lane & 3;
    const int wkey = warp * 32;  // the warp's keys of a tile
    const uint32_t ring_u = ptx::smem_u32(ring);
    uint8_t* behind = ring + T::kStages * T::kStage;
    __half* sq = reinterpret_cast<__half*>(behind);
    float* fin = reinterpret_cast<float*>(behind + T::kQBytes);  // [rows][pitch], CL only
    float *fin_m = fin + ROWS * T::kFinPitch, *fin_l = fin_m + ROWS;
    int joins = 0;

    while (CL ? b < blocks : x < st.x1) {
        const PagedItem it = paged_item<kFewTile>(p, r, g, b);
        const uint32_t take = min(st.x1 - x, uint32_t(it.units) - off);
        const int j0 = CL ? rank * it.nt / S : int(off), j1 = CL ? (rank + 1) * it.nt / S : min(int(off + take), it.nt);
        // this thread's two rows: query and head, keys they see
        const int rA = quad, rB = rA + 8, iA = rA / p.G, iB = rB / p.G;
        const bool okA = iA < it.nq, okB = iB < it.nq;
        const KeyRange none{0, 0};
        const KeyRange kA = okA ? query_keys(p, it.q, it.i0 + iA) : none, kB = okB ? query_keys(p, it.q, it.i0 + iB) : none;
        auto row_of = [&](int i, int rr) { return (int64_t(it.q.q0 + it.i0 + i) * p.H + g * p.G + (rr - i * p.G)) * D; };
        const int64_t offA = okA ? row_of(iA, rA) : 0, offB = okB ? row_of(iB, rB) : 0;

        // Queries as f16 fragments: a lane's elements of k-step ks are dims 16 ks + 4 qc .. + 3 (the order of the keys' bytes).
        uint32_t qf[QS ? 1 : KS][4];
        float backA, backB;
        if constexpr (!QS) {
            auto ldq = [&](bool ok, int64_t at) { return ok ? *reinterpret_cast<const uint2*>(p.Q + at) : make_uint2(0, 0); };
            uint2 qa[KS], qb[KS];
            float topA = 0.0f, topB = 0.0f;
            auto most = [](float m, uint2 w) {
                const float2 u = unpack_bf16x2(w.x), v = unpack_bf16x2(w.y);
                return fmaxf(fmaxf(m, fmaxf(fabsf(u.x), fabsf(u.y))), fmaxf(fabsf(v.x), fabsf(v.y)));
            };
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qa[ks] = ldq(okA, offA + ks * 16 + 4 * qc);
                qb[ks] = ldq(okB, offB + ks * 16 + 4 * qc);
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                topA = most(topA, qa[ks]);
                topB = most(topB, qb[ks]);
            }
#pragma unroll
            for (int i = 1; i <= 2; i <<= 1) {
                topA = fmaxf(topA, __shfl_xor_sync(0xffffffffu, topA, i));
                topB = fmaxf(topB, __shfl_xor_sync(0xffffffffu, topB, i));
            }
            const RowPower pa = row_power(topA), pb = row_power(topB);
            backA = pa.back;
            backB = pb.back;
            auto scaled = [](uint32_t w, float by) {
                const float2 u = unpack_bf16x2(w);
                return pack_f16x2(u.x * by, u.y * by);
            };
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qf[ks][0] = scaled(qa[ks].x, pa.to);
                qf[ks][1] = scaled(qb[ks].x, pb.to);
                qf[ks][2] = scaled(qa[ks].y, pa.to);
                qf[ks][3] = scaled(qb[ks].y, pb.to);
            }
        } else {
            bar();  // (the last item's rows are done with)
            for (int rr = warp; rr < ROWS; rr += kFewWarps) {  // a row a warp, eight elements a lane
                const int i = rr / p.G;
                uint4 w = make_uint4(0, 0, 0, 0);
                if (i < it.nq) w = *reinterpret_cast<const uint4*>(p.Q + row_of(i, rr) + lane * 8);
                uint32_t* h = reinterpret_cast<uint32_t*>(&w);
                float top = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 u = unpack_bf16x2(h[e]);
                    top = fmaxf(top, fmaxf(fabsf(u.x), fabsf(u.y)));
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const RowPower pr = row_power(top);
                if (lane == 0) row_back[rr] = pr.back;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 u = unpack_bf16x2(h[e]);
                    h[e] = pack_f16x2(u.x * pr.to, u.y * pr.to);
                }
                *reinterpret_cast<uint4*>(sq + rr * T::kQPitch + lane * 8) = w;
            }
            bar();
            backA = row_back[rA];
            backB = row_back[rB];
        }
        if constexpr (!CAP) {
            backA = row_factor(backA, p.scale2);
            backB = row_factor(backB, p.scale2);
        }

        float o[NT][4];  // of n-tiles 2 c and 2 c + 1: dims 16 c + 4 qc + {0, 2} and + {1, 3}
#pragma unroll
        for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f;
        float mA = -INFINITY, mB = -INFINITY, lA = 0.0f, lB = 0.0f;
        bool odd = false;  // a NaN code was left out of a product

        for (int j = j0; j < j1; ++j, ++issued) {
            const int s = issued % T::kStages;
            ptx::mbar_wait(&full[s], (issued / T::kStages) & 1, &abort_flag, p.status, kWaitLimitNs);
            __syncwarp();
            const uint32_t kb = ring_u + uint32_t(s * T::kStage), vb = kb + T::kHalf;
            const int key0 = (it.t0 + j) * kFewTile;
            const bool edge = key0 < it.lo_all || key0 + kFewTile > it.hi_all;
            // whether it holds places behind the request's last key, and keys that some row does not see
            const bool tail = key0 + kFewTile > it.q.L, hidden = key0 < it.lo_all || min(key0 + kFewTile, it.q.L) > it.hi_all;
            const float4 pw[2] = {powers[s][2 * warp], powers[s][2 * warp + 1]};

            // S = Q K^T, the warp's 32 keys in four n-tiles; one ldmatrix gives the codes of four k-steps
            float sc[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.0f;
#pragma unroll
            for (int k4 = 0; k4 < KS; k4 += 4) {
                uint32_t bk[4][4];
#pragma unroll
                for (int n = 0; n < 4; ++n) ldsm_x4(kb + T::place(wkey + n * 8 + (lane & 7), k4 + (lane >> 3)), bk[n]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t a[4];
                    if constexpr (QS) {
                        const uint2 u = *reinterpret_cast<const uint2*>(sq + rA * T::kQPitch + (k4 + i) * 16 + 4 * qc);
                        const uint2 v = *reinterpret_cast<const uint2*>(sq + rB * T::kQPitch + (k4 + i) * 16 + 4 * qc);
                        a[0] = u.x;
                        a[1] = v.x;
                        a[2] = u.y;
                        a[3] = v.y;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = qf[k4 + i][e];
                    }
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        uint32_t b0, b1;
                        codes_to_f16x4(bk[n][i], b0, b1);
                        mma_f16(sc[n], a, b0, b1);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float fA = score_factor(backA * pw[n / 2].x), fB = score_factor(backB * pw[n / 2].x), ve = pw[n / 2].y;
                float2 zA = mul2(make_float2(sc[n][0], sc[n][1]), make_float2(fA, fA));
                float2 zB = mul2(make_float2(sc[n][2], sc[n][3]), make_float2(fB, fB));
                if constexpr (CAP) {
                    zA = capped2<CAP>(zA, p);
                    zB = capped2<CAP>(zB, p);
                }
                sc[n][0] = zA.x + ve;
                sc[n][1] = zA.y + ve;
                sc[n][2] = zB.x + ve;
                sc[n][3] = zB.y + ve;
            }
            if (edge) {
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = key0 + wkey + n * 8 + 2 * qc + e;
                        if (key < kA.lo || key >= kA.hi) sc[n][e] = -INFINITY;
                        if (key < kB.lo || key >= kB.hi) sc[n][2 + e] = -INFINITY;
                    }
            }
            float tA = -INFINITY, tB = -INFINITY;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                tA = fmaxf(tA, fmaxf(sc[n][0], sc[n][1]));
                tB = fmaxf(tB, fmaxf(sc[n][2], sc[n][3]));
            }
#pragma unroll
            for (int i = 1; i <= 2; i <<= 1) {
                tA = fmaxf(tA, __shfl_xor_sync(0xffffffffu, tA, i));
                tB = fmaxf(tB, __shfl_xor_sync(0xffffffffu, tB, i));
            }
            const float nA = fmaxf(mA, tA), nB = fmaxf(mB, tB);
            // (a row without a finite score so far subtracts 0: its weights are 2^-inf = 0)
            const float sA0 = nA == -INFINITY ? 0.0f : nA, sB0 = nB == -INFINITY ? 0.0f : nB;
            const float cA = exp2_fast(mA - sA0), cB = exp2_fast(mB - sB0);
            lA *= cA;  // lane-partial sums; the four lanes of a row are added at the end
            lB *= cB;
#pragma unroll
            for (int n = 0; n < 4; n += 2) {
                float sA = 0.0f, sB = 0.0f;
#pragma unroll
                for (int m = n; m < n + 2; ++m)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // (the difference first: it is never above 0, however large the scores)
                        sc[m][e] = exp2_fast(sc[m][e] - sA0) * kWeightUnit;
                        sc[m][2 + e] = exp2_fast(sc[m][2 + e] - sB0) * kWeightUnit;
                        sA += sc[m][e];
                        sB += sc[m][2 + e];
                    }
                lA = fmaf(sA, pw[n / 2].z, lA);
                lB = fmaf(sB, pw[n / 2].z, lB);
            }
            if (__any_sync(0xffffffffu, nA != mA || nB != mB)) {  // else every factor is 1
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    o[n][0] *= cA;
                    o[n][1] *= cA;
                    o[n][2] *= cB;
                    o[n][3] *= cB;
                }
            }
            mA = nA;
            mB = nB;
            // O += P V in two k-steps of 16 keys
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const float* s0 = sc[2 * kk];
                const float* s1 = sc[2 * kk + 1];
                const uint32_t pf[4] = {pack_f16x2(s0[0], s0[1]), pack_f16x2(s0[2], s0[3]), pack_f16x2(s1[0], s1[1]), pack_f16x2(s1[2], s1[3])};
                // (of the fragments' keys 2 qc, 2 qc + 1 and the same + 8, those that the request has)
                const int left = it.q.L - (key0 + wkey + kk * 16 + 2 * qc);
                const uint32_t in0 = (left > 0 ? 0x0000FFFFu : 0u) | (left > 1 ? 0xFFFF0000u : 0u);
                const uint32_t in1 = (left > 8 ? 0x0000FFFFu : 0u) | (left > 9 ? 0xFFFF0000u : 0u);
                const int vrow = wkey + kk * 16 + (lane & 15);
#pragma unroll
                for (int c = 0; c < KS; c += 2) {
                    uint32_t bv[4];  // chunk c: keys 0-7, 8-15; chunk c + 1
                    ldsm_x4_trans(vb + T::place(vrow, c + (lane >> 4)), bv);
                    // values behind the request's last key are anything; NaN codes hidden from some rows may not be multiplied
                    // by their weights of 0: they are left out here and added at the end for the rows that see them
                    if (tail) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) bv[e] &= e & 1 ? in1 : in0;
                    }
                    if (hidden) {
                        const uint32_t bad = nan_codes(bv[0]) | nan_codes(bv[1]) | nan_codes(bv[2]) | nan_codes(bv[3]);
                        if (__any_sync(0xffffffffu, bad != 0)) {
                            odd = true;
#pragma unroll
                            for (int e = 0; e < 4; ++e) bv[e] = without(bv[e], nan_codes(bv[e]));
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t e0, o0, e1, o1;  // even and odd dims, keys 0-7 and 8-15
                        codes_to_f16x4(__byte_perm(bv[2 * i], 0, 0x3120), e0, o0);
                        codes_to_f16x4(__byte_perm(bv[2 * i + 1], 0, 0x3120), e1, o1);
                        mma_f16(o[2 * (c + i)], pf, e0, e1);
                        mma_f16(o[2 * (c + i) + 1], pf, o0, o1);
                    }
                }
            }
            __syncwarp();
            // (the last tile makes room for the warps' merge first)
            if (lane == 0 && j + 1 < j1) ptx::mbar_arrive(&empty[s]);
        }
#pragma unroll
        for (int i = 1; i <= 2; i <<= 1) {
            lA += __shfl_xor_sync(0xffffffffu, lA, i);
            lB += __shfl_xor_sync(0xffffffffu, lB, i);
        }
        if (__any_sync(0xffffffffu, odd)) {
            for (int key = (it.t0 + j0) * kFewTile; key < min((it.t0 + j1) * kFewTile, it.hi); ++key) {
                const int in = key & (kFewTile - 1), key0 = key - in;
                if (!(key0 < it.lo_all || min(key0 + kFewTile, it.q.L) > it.hi_all)) continue;
                if (in < wkey || in >= wkey + 32) continue;
                const int page = p.table[int64_t(r) * p.max_pages + (key >> p.page_shift)];
                if (page < 0 || page >= p.n_pages) continue;
                const int64_t slot = (int64_t(page) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
                const uint32_t* v = reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(p.V) + (slot * p.Hk + g) * D) + qc;
                const bool inA = key >= kA.lo && key < kA.hi, inB = key >= kB.lo && key < kB.hi;
#pragma unroll
                for (int c = 0; c < KS; ++c) {
                    const uint32_t bad = nan_codes(v[c * 4]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (bad >> (8 * e + 7) & 1u) {
                            float* to = o[2 * c + (e & 1)];
                            if (inA) to[e >> 1] = NAN;
                            if (inB) to[2 + (e >> 1)] = NAN;
                        }
                }
            }
        }

        // The warps lay their results side by side where the last tile was (a lane's four values of n-tile n at [n][lane]: no two
        // lanes meet in a bank), and each adds up a quarter of the n-tiles.
        constexpr int kMine = NT / kFewWarps;
        const int n0 = warp * kMine;
        if (j1 > j0) {
            const int s = (issued - 1) % T::kStages;
            float4* merge = reinterpret_cast<float4*>(ring + s * T::kStage);  // [warp][n-tile][lane]
            bar();  // every warp is done with the keys and values
#pragma unroll
            for (int n = 0; n < NT; ++n) merge[(warp * NT + n) * 32 + lane] = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
            if (qc == 0) {
                warp_m[warp][quad] = mA;
                warp_l[warp][quad] = lA;
                warp_m[warp][quad + 8] = mB;
                warp_l[warp][quad + 8] = lB;
            }
            bar();
            mA = mB = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                mA = fmaxf(mA, warp_m[w][quad]);
                mB = fmaxf(mB, warp_m[w][quad + 8]);
            }
            const float zA = mA == -INFINITY ? 0.0f : mA, zB = mB == -INFINITY ? 0.0f : mB;
            lA = lB = 0.0f;
#pragma unroll
            for (int n = 0; n < kMine; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                // weight 0 of a warp without a finite score: its sums are 0, or NaN, which has to show
                const float wA = exp2_fast(warp_m[w][quad] - zA), wB = exp2_fast(warp_m[w][quad + 8] - zB);
                lA = fmaf(warp_l[w][quad], wA, lA);
                lB = fmaf(warp_l[w][quad + 8], wB, lB);
#pragma unroll
                for (int n = 0; n < kMine; ++n) {
                    const float4 u = merge[(w * NT + n0 + n) * 32 + lane];
                    o[n][0] = fmaf(u.x, wA, o[n][0]);
                    o[n][1] = fmaf(u.y, wA, o[n][1]);
                    o[n][2] = fmaf(u.z, wB, o[n][2]);
                    o[n][3] = fmaf(u.w, wB, o[n][3]);
                }
            }
            ptx::fence_proxy_async_smem();  // before the next copy into this buffer
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&empty[s]);
        }

        // a lane's four neighbouring dims of its n-tiles 2 c and 2 c + 1, for row A (h = 0) or B (h = 2)
        auto dims = [&](int c, int h) { return make_float4(o[2 * c][h], o[2 * c + 1][h], o[2 * c][h + 1], o[2 * c + 1][h + 1]); };
        auto dim_of = [&](int c) { return (n0 + 2 * c) * 8 + 4 * qc; };
        if constexpr (CL) {
            // every CTA of the cluster lays down its result, and each adds up its share of the outputs, in CTA order
            if (qc == 0 && warp == 0) {
                fin_m[quad] = mA;
                fin_m[quad + 8] = mB;
                fin_l[quad] = lA;
                fin_l[quad + 8] = lB;
            }
#pragma unroll
            for (int c = 0; c < kMine / 2; ++c) {
                *reinterpret_cast<float4*>(fin + quad * T::kFinPitch + dim_of(c)) = dims(c, 0);
                *reinterpret_cast<float4*>(fin + (quad + 8) * T::kFinPitch + dim_of(c)) = dims(c, 2);
            }
            __syncwarp();
            ptx::cluster_sync();
            for (int e = rank * 32 * kFewWarps + int(threadIdx.x); e < it.nq * p.G * (D / 4); e += S * 32 * kFewWarps) {
                const int row = e / (D / 4), c = e % (D / 4) * 4;
                float m[kFewCluster], l[kFewCluster], M = -INFINITY, L = 0.0f;
                float4 v[kFewCluster], a = make_float4(0, 0, 0, 0);
                const uint32_t am = ptx::smem_u32(fin_m + row), al = ptx::smem_u32(fin_l + row);
                const uint32_t av = ptx::smem_u32(fin + row * T::kFinPitch + c);
#pragma unroll
                for (int q = 0; q < kFewCluster; ++q) {
                    m[q] = -INFINITY;
                    l[q] = 0.0f;
                    v[q] = make_float4(0, 0, 0, 0);
                    if (q < S) {
                        m[q] = ptx::ld_dsmem_f32(ptx::map_dsmem(am, q));
                        l[q] = ptx::ld_dsmem_f32(ptx::map_dsmem(al, q));
                        v[q] = ptx::ld_dsmem_f32x4(ptx::map_dsmem(av, q));
                    }
                    M = fmaxf(M, m[q]);
                }
                const float z = M == -INFINITY ? 0.0f : M;
#pragma unroll
                for (int q = 0; q < kFewCluster; ++q) {
                    // weight 0 of a result without a finite score: its sums are 0, or NaN, which has to show
                    const float w = exp2_fast(m[q] - z);
                    L = fmaf(l[q], w, L);
                    a.x = fmaf(v[q].x, w, a.x);
                    a.y = fmaf(v[q].y, w, a.y);
                    a.z = fmaf(v[q].z, w, a.z);
                    a.w = fmaf(v[q].w, w, a.w);
                }
                const float inv = L == 0.0f ? 0.0f : __fdiv_rn(1.0f, L);
                uint2 u;
                u.x = pack_bf16x2(__fmul_rn(a.x, inv), __fmul_rn(a.y, inv));
                u.y = pack_bf16x2(__fmul_rn(a.z, inv), __fmul_rn(a.w, inv));
                *reinterpret_cast<uint2*>(p.O + row_of(row / p.G, row) + c) = u;
            }
            __syncwarp();
            ptx::cluster_sync();  // remote shared memory must outlive its readers
            b += p.side;
            continue;
        }
        const bool whole = off == 0 && take == uint32_t(it.units);
        if (whole) {
            const float iv = lA == 0.0f ? 0.0f : __fdiv_rn(1.0f, lA), iw = lB == 0.0f ? 0.0f : __fdiv_rn(1.0f, lB);
#pragma unroll
            for (int c = 0; c < kMine / 2; ++c) {
                const float4 a = dims(c, 0), w = dims(c, 2);
                if (okA)
                    *reinterpret_cast<uint2*>(p.O + offA + dim_of(c)) =
                        make_uint2(pack_bf16x2(__fmul_rn(a.x, iv), __fmul_rn(a.y, iv)), pack_bf16x2(__fmul_rn(a.z, iv), __fmul_rn(a.w, iv)));
                if (okB)
                    *reinterpret_cast<uint2*>(p.O + offB + dim_of(c)) =
                        make_uint2(pack_bf16x2(__fmul_rn(w.x, iw), __fmul_rn(w.y, iw)), pack_bf16x2(__fmul_rn(w.z, iw), __fmul_rn(w.w, iw)));
            }
        } else {
            const uint32_t a = x - off;  // the item's first unit
            PagedJoin J{r, g, b, int(a / st.chunk), 0};
            J.count = int((a + uint32_t(it.units) - 1) / st.chunk) - J.first + 1;
            float* part = p.part + part_slot(int(blockIdx.x), J.first) * PL::kFloats;
            if (qc == 0 && warp == 0) {
                if (okA) {
                    part[rA] = mA;
                    part[ROWS + rA] = lA;
                }
                if (okB) {
                    part[rB] = mB;
                    part[ROWS + rB] = lB;
                }
            }
#pragma unroll
            for (int c = 0; c < kMine / 2; ++c) {
                if (okA) *reinterpret_cast<float4*>(PL::value(part, rA, dim_of(c))) = dims(c, 0);
                if (okB) *reinterpret_cast<float4*>(PL::value(part, rB, dim_of(c))) = dims(c, 2);
            }
            bar();
            if (threadIdx.x == 0) part_publish(p.flags + J.first);
            if (threadIdx.x == 0) cut[joins] = J;
            ++joins;
        }
        x += take;
        off = 0;
        if (x < st.x1) next_item(p, r, g, b, it.q.n);
    }

    // Every CTA joins its share of the items that it has a part in, once all their parts are there. The CTAs of
    // the grid all run at once (a cooperative launch), and each publishes its parts before it waits.
    if (joins > 0) bar();
    for (int k = 0; k < joins; ++k) {
        const PagedJoin J = cut[k];
        if (threadIdx.x == 0) joined = part_wait(p.flags + J.first, J.count, &abort_flag, p.status);
        bar();
        const bool in = joined != 0;
        if (in) join_store<D, ROWS, 16, 1>(p, J, paged_req(p, J.r), int(blockIdx.x) - J.first, threadIdx.x, 32 * kFewWarps);
        bar();  // before the next item's answer
    }
}

// CTAs that run at once, asked once per device; the opt-in shared memory is a per-device attribute too.
template <int D, int CAP>
cudaError_t few8_resident(int& ctas) {
    static std::mutex mu;
    static int known[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    if (dev >= 0 && dev < 64 && known[dev]) {
        ctas = known[dev];
        return cudaSuccess;
    }
    auto* kernel = paged_codes_few_kernel<D, CAP, false>;
    int per_sm = 0;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Few8Traits<D>::kSmem);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(paged_codes_few_kernel<D, CAP, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Few8Traits<D>::kSmemCluster);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kFewThreads, Few8Traits<D>::kSmem);
    if (e != cudaSuccess) return e;
    // a partial result per item border: two per CTA, within the workspace
    const size_t slot = size_t(kFewRows) * (D + 2) * 4;
    const int fit = int((EMB_PAGED_WORKSPACE - kPagedFlagBytes) / (2 * slot));
    ctas = std::max(1, std::min({std::max(1, per_sm) * std::max(1, device_sm_count()), fit, int(kPagedFlagBytes / 4)}));
    if (dev >= 0 && dev < 64) known[dev] = ctas;
    return cudaSuccess;
}

// Blocks of a request's queries that its clusters take side by side.
int few8_blocks(const PagedAttnArgs& a) {
    const int64_t qb = kFewRows / (a.n_heads / a.n_kv_heads);
    return int((std::min(a.max_q, a.n_tokens) + qb - 1) / qb);
}
// CTAs of the cluster that takes a block, or 0 where equal stretches of all the work are sooner done: the rule of the bf16
// cache's kernel (paged_attention.cu, where its measurements stand), in keys: tiles here have twice as many, so its limits are halved.
// With it, where more than 16 rows have clusters (us, and the tcgen05 kernel): 24 requests of 4 queries of 16 heads on 2 over 1500 keys 11.4 and 19.0
// (heads of 64), 15.6 and 21.5 (128), one of 8 queries over 4000 keys 8.9 and 14.9, 11.5 and 16.9, 14.8 and 23.2 (256).
int few8_cluster(const PagedAttnArgs& a) {
    double keys = double(a.max_pages * a.page_size);
    if (a.window > 0) keys = std::min(keys, double(a.window) + kFewRows + kFewTile);
    const double items = double(a.n_req * a.n_kv_heads) * few8_blocks(a), tiles = std::ceil(keys / kFewTile);
    const double ctas = (a.head_dim == 256 ? 1.0 : 2.0) * std::max(1, device_sm_count());
    constexpr double longest = 12.0;
    int S = kFewCluster;
    while (S > 0 && items * S > ctas) S /= 2;
    return S > 0 && tiles <= longest * S && tiles / S <= items * tiles / ctas + 4.0 ? S : 0;
}

template <int D, int CAP>
cudaError_t launch_few8(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s) {
    int ctas = 0;
    const cudaError_t e = few8_resident<D, CAP>(ctas);
    if (e != cudaSuccess) return e;
    p.QB = kFewRows / p.G;
    const uint32_t box = uint32_t(std::min<int64_t>(a.page_size, kFewTile));
    if (!encode_codes(&p.k_map, a.k_cache, a, box) || !encode_codes(&p.v_map, a.v_cache, a, box)) return cudaErrorInvalidValue;
    void* args[] = {&p};
    p.side = few8_blocks(a);
    p.cluster = few8_cluster(a);
    if (p.cluster > 0)
        return launch_serialised(reinterpret_cast<const void*>(paged_codes_few_kernel<D, CAP, true>), unsigned(a.n_req * a.n_kv_heads * p.side * p.cluster),
                                 kFewThreads, Few8Traits<D>::kSmemCluster, s, args, unsigned(p.cluster));
    const unsigned grid = unsigned(std::max(2.0, std::min(double(ctas), unit_bound(a, p.QB, kFewTile))));
    set_grid(p, grid, 2);
    return launch_serialised(reinterpret_cast<const void*>(paged_codes_few_kernel<D, CAP, false>), grid, kFewThreads, Few8Traits<D>::kSmem, s, args, 1, true);
}

template <int D>
cudaError_t launch_few8_d(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s) {
    return a.cap > kMostLowCap ? launch_few8<D, kAnyCap>(p, a, s) : a.cap > 0.0f ? launch_few8<D, kLowCap>(p, a, s) : launch_few8<D, kUncapped>(p, a, s);
}

}  // namespace

cudaError_t launch_paged8_few(Paged8Params& p, const PagedAttnArgs& a, cudaStream_t s) {
    return a.head_dim == 64    ? launch_few8_d<64>(p, a, s)
           : a.head_dim == 128 ? launch_few8_d<128>(p, a, s)
                               : launch_few8_d<256>(p, a, s);
}

cudaError_t launch_paged8_attention(const Paged8AttnArgs& args, cudaStream_t s) {
    const PagedAttnArgs& a = args.a;
    Paged8Params p;
    static_cast<PagedParams&>(p) = paged_params(a);
    p.k_exp = args.k_exp;
    p.v_exp = args.v_exp;
    // Rows of a request: up to 16 go to the mma.sync kernel, and more where all its blocks of 16 have a cluster at once. Up to 32 do
    // too, though their keys come twice: the second time from L2, and every CTA of two takes a stretch of its own (us, mma.sync and
    // tcgen05: 32 requests of 4 queries of 16 heads on 2 of 128 over 8000 keys 62 and 67, one over 16000 18 and 25, of 64 15 and 23); but
    // heads of 256, and up to 64 rows, only where the call has few blocks to share out (one request of 8 queries of 16 heads
    // on 2 over 16000 keys, heads of 64, 128 and 256: 17 and 23, 22 and 25, 27 and 39; 4 requests 22 and 24, 33 and 27, 75 and 46; 24
    // requests of 4 queries of heads of 256 over 1500 keys 39 and 29). The rest goes to the tcgen05 kernel.
    bool few = false;
    if (p.G <= 16) {
        const int64_t rows = std::min(a.max_q, a.n_tokens) * p.G;
        const bool fine = double(a.n_req * a.n_kv_heads) * few8_blocks(a) <= 16.0;
        few = rows <= 16 || few8_cluster(a) > 0 || (rows <= 32 && a.head_dim < 256) || (rows <= 64 && fine);
    }
    if (!few) {
        p.negate = a.scale < 0.0f;
        p.scale2 = std::max(std::fabs(p.scale2), 1e-37f);  // (hidden scores are the lowest there are times this)
        p.lin2 = std::max(std::fabs(p.lin2), 1e-37f);
        return launch_paged8_many(p, a, s);
    }
    return launch_paged8_few(p, a, s);
}

}  // namespace emb
