// Attention of new tokens over a paged key/value cache (definition in include/emb_paged.h). Both kernels take
// their work from paged_sched.cuh: few query rows per request on mma.sync, many on tcgen05.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <mutex>

#include "paged_math.cuh"

namespace emb {
namespace {

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
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
// ------------------------------------------------------------------ few rows: mma.sync
// A producer warp brings tiles of 64 keys and values by TMA (a box per page, 128-byte swizzled rows) into a ring;
// four warps compute. An item has 16 rows (queries times heads), every warp takes 16 of a tile's keys, and the
// warps' results are merged at the item's end. Scores, softmax in base 2 with a running maximum and the value
// product (weights as bf16 hi + lo) stay in registers. HBM bounds it: the cache is read once for the 16 rows (64
// requests of 32 heads on 8 of 128, 100 to 16384 keys: 2.2 GB in 334 to 348 us, 0.94 to 0.98 of the measured copy rate; 78 % of
// the DRAM's own peak in the counters of a smaller call, 26 % of the tensor pipe). Small calls are latency: one token over 867
// keys 6.0 to 6.2 us.
// CL: for few and short requests a cluster of CTAs takes a request's key/value head and shares out its tiles, and
// the results are joined through distributed shared memory: no search for the work, no workspace.
constexpr int kFewWarps = 4;
constexpr int kFewThreads = 32 * (kFewWarps + 1);
constexpr int kFewTile = 64;
constexpr int kFewRows = 16;
constexpr int kFewCluster = 8;  // CTAs of a cluster, at most (the portable size)

template <int D>
struct FewTraits {
    static constexpr int kStage = kFewTile * D * 4;  // bytes of keys and values
    static constexpr int kStages = D == 64 ? 6 : 3;
    static constexpr int kCtas = D == 256 ? 1 : 2;   // per SM
    static constexpr int kQPitch = D + 8;            // queries in shared memory (D = 256), bf16 per padded row
    static constexpr int kQBytes = D == 256 ? kFewRows * kQPitch * 2 : 0;
    static constexpr int kFinPitch = D + 4;          // a CTA's result for its cluster, fp32 per padded row
    static constexpr int kSmem = 1024 + kStages * kStage + kQBytes;
    static constexpr int kSmemCluster = kSmem + kFewRows * (kFinPitch + 2) * 4;
};

template <int D, int CAP, bool CL>
__global__ void __launch_bounds__(kFewThreads, FewTraits<D>::kCtas) paged_few_kernel(const __grid_constant__ PagedParams p) {
    using T = FewTraits<D>;
    constexpr int KS = D / 16, NT = D / 8, NJ = kFewTile / 8 / kFewWarps, ROWS = kFewRows;
    constexpr bool QS = D == 256;  // queries stay in shared memory: their fragments would not fit the registers
    constexpr int kSub = kFewTile * 128;  // bytes of a 64-dim part of a tile
    using PL = PartLayout<D, ROWS>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[T::kStages], empty[T::kStages];
    __shared__ int abort_flag, joined;
    __shared__ PagedJoin cut[2];
    __shared__ float warp_m[kFewWarps][16], warp_l[kFewWarps][16];
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
            // lane i looks up the page of the tile's box i; boxes that no query sees, and pages that do not
            // exist, are fetched from behind the cache: zeros
            auto page_of = [&](int j) {
                const int key = (it.t0 + j) * kFewTile + lane * box;
                int page = p.n_pages;
                if (lane < n_box && j < j1 && key < it.hi && key + box > it.lo) {
                    page = row[key >> p.page_shift];
                    if (page < 0 || page > p.n_pages) page = p.n_pages;
                }
                return page;
            };
            int page = page_of(j0);
            for (int j = j0; j < j1; ++j, ++issued) {
                const int next = page_of(j + 1);
                const int s = issued % T::kStages;
                if (issued >= uint32_t(T::kStages))
                    ptx::mbar_wait(&empty[s], (issued / T::kStages - 1) & 1, &abort_flag, p.status, kWaitLimitNs);
                const bool stop = __any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&abort_flag) != 0);
                uint8_t* k = ring + s * T::kStage;
                uint8_t* v = k + T::kStage / 2;
                if (!stop) {
                    if (ptx::elect_one()) ptx::mbar_arrive_expect_tx(&full[s], T::kStage);
                    __syncwarp();
                    const int place = ((it.t0 + j) * kFewTile) & (page_size - 1);
                    for (int i = 0; i < n_box; ++i) {
                        const int pg = __shfl_sync(0xffffffffu, page, i);
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int c = 0; c < D / 64; ++c) {
                                ptx::tma_load_4d(k + c * kSub + i * box * 128, &p.k_map, &full[s], c * 64, g, place, pg);
                                ptx::tma_load_4d(v + c * kSub + i * box * 128, &p.v_map, &full[s], c * 64, g, place, pg);
                            }
                        }
                        __syncwarp();
                    }
                    ++loads;
                }
                page = next;
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
    const int wkey = warp * 16;  // the warp's keys of a tile
    const uint32_t ring_u = ptx::smem_u32(ring);
    __nv_bfloat16* sq = reinterpret_cast<__nv_bfloat16*>(ring + T::kStages * T::kStage);
    float* fin = reinterpret_cast<float*>(ring + T::kStages * T::kStage + T::kQBytes);  // [rows][pitch], CL only
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

        uint32_t qf[QS ? 1 : KS][4];
        if constexpr (!QS) {
            auto ldq = [&](bool ok, int64_t at) { return ok ? *reinterpret_cast<const uint32_t*>(p.Q + at) : 0u; };
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int c = ks * 16 + 2 * qc;
                qf[ks][0] = ldq(okA, offA + c);
                qf[ks][1] = ldq(okB, offB + c);
                qf[ks][2] = ldq(okA, offA + c + 8);
                qf[ks][3] = ldq(okB, offB + c + 8);
            }
        } else {
            bar();  // (the last item's rows are done with)
            for (int e = threadIdx.x; e < ROWS * (D / 8); e += 32 * kFewWarps) {
                const int rr = e / (D / 8), c = (e % (D / 8)) * 8, i = rr / p.G;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (i < it.nq) v = *reinterpret_cast<const uint4*>(p.Q + row_of(i, rr) + c);
                *reinterpret_cast<uint4*>(sq + rr * T::kQPitch + c) = v;
            }
            bar();
        }

        float o[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f;
        float mA = -INFINITY, mB = -INFINITY, lA = 0.0f, lB = 0.0f;
        bool odd = false;  // a value that is not finite was left out of a product

        for (int j = j0; j < j1; ++j, ++issued) {
            const int s = issued % T::kStages;
            ptx::mbar_wait(&full[s], (issued / T::kStages) & 1, &abort_flag, p.status, kWaitLimitNs);
            __syncwarp();
            const uint32_t kb = ring_u + uint32_t(s * T::kStage), vb = kb + T::kStage / 2;
            const int key0 = (it.t0 + j) * kFewTile;
            const bool edge = key0 < it.lo_all || key0 + kFewTile > it.hi_all;
            // whether it holds places behind the request's last key, and keys that some row does not see
            const bool tail = key0 + kFewTile > it.q.L, hidden = key0 < it.lo_all || min(key0 + kFewTile, it.q.L) > it.hi_all;

            // S = Q K^T, the warp's keys in n-tiles of 8; one ldmatrix gives the fragments of two k-steps
            float sc[NJ][4];
#pragma unroll
            for (int n = 0; n < NJ; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.0f;
            const uint32_t krow = kb + uint32_t(wkey + (lane & 7)) * 128;
#pragma unroll
            for (int ks = 0; ks < KS; ks += 2) {
                uint32_t a0[4], a1[4];
                if constexpr (QS) {
                    const uint32_t qa = ptx::smem_u32(sq + (lane & 15) * T::kQPitch + ks * 16 + (lane >> 4) * 8);
                    ldsm_x4(qa, a0);
                    ldsm_x4(qa + 32, a1);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        a0[i] = qf[ks][i];
                        a1[i] = qf[ks + 1][i];
                    }
                }
                uint32_t bk[NJ][4];
                const uint32_t at = krow + (ks / 4) * kSub + (((((ks & 3) * 2) + (lane >> 3)) ^ (lane & 7)) << 4);
#pragma unroll
                for (int n = 0; n < NJ; ++n) ldsm_x4(at + n * 1024, bk[n]);
#pragma unroll
                for (int n = 0; n < NJ; ++n) mma_16816(sc[n], a0, bk[n][0], bk[n][1]);
#pragma unroll
                for (int n = 0; n < NJ; ++n) mma_16816(sc[n], a1, bk[n][2], bk[n][3]);
            }
#pragma unroll
            for (int n = 0; n < NJ; ++n)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    float2 z = make_float2(sc[n][e], sc[n][e + 1]);
                    if constexpr (CAP) z = capped2<CAP>(z, p);
                    else z = make_float2(__fmul_rn(z.x, p.scale2), __fmul_rn(z.y, p.scale2));
                    sc[n][e] = z.x;
                    sc[n][e + 1] = z.y;
                }
            if (edge) {
#pragma unroll
                for (int n = 0; n < NJ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = key0 + wkey + n * 8 + 2 * qc + e;
                        if (key < kA.lo || key >= kA.hi) sc[n][e] = -INFINITY;
                        if (key < kB.lo || key >= kB.hi) sc[n][2 + e] = -INFINITY;
                    }
            }
            float tA = -INFINITY, tB = -INFINITY;
#pragma unroll
            for (int n = 0; n < NJ; ++n) {
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
            float sA = 0.0f, sB = 0.0f;
#pragma unroll
            for (int n = 0; n < NJ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    sc[n][e] = exp2_fast(sc[n][e] - sA0);
                    sc[n][2 + e] = exp2_fast(sc[n][2 + e] - sB0);
                    sA += sc[n][e];
                    sB += sc[n][2 + e];
                }
            lA = lA * cA + sA;  // lane-partial sums; the four lanes of a row are added at the end
            lB = lB * cB + sB;
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
            // O += P V in k-steps of 16 keys, P as hi + lo
#pragma unroll
            for (int kk = 0; kk < NJ / 2; ++kk) {
                uint32_t ah[4], al[4];
                const float* s0 = sc[2 * kk];
                const float* s1 = sc[2 * kk + 1];
                const float src[4][2] = {{s0[0], s0[1]}, {s0[2], s0[3]}, {s1[0], s1[1]}, {s1[2], s1[3]}};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ah[i] = pack_bf16x2(src[i][0], src[i][1]);
                    const float2 h = unpack_bf16x2(ah[i]);
                    al[i] = pack_bf16x2(__fsub_rn(src[i][0], h.x), __fsub_rn(src[i][1], h.y));
                }
                // (of the fragments' keys 2 qc, 2 qc + 1 and the same + 8, those that the request has)
                const int left = it.q.L - (key0 + wkey + kk * 16 + 2 * qc);
                const uint32_t in0 = (left > 0 ? 0x0000FFFFu : 0u) | (left > 1 ? 0xFFFF0000u : 0u);
                const uint32_t in1 = (left > 8 ? 0x0000FFFFu : 0u) | (left > 9 ? 0xFFFF0000u : 0u);
                const int kl = wkey + kk * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
                const uint32_t vrow = vb + uint32_t(kl) * 128;
#pragma unroll
                for (int jj = 0; jj < NT; jj += 4) {
                    uint32_t bv[2][4];
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        ldsm_x4_trans(vrow + (jj / 8) * kSub + ((((jj & 7) + 2 * i + (lane >> 4)) ^ (lane & 7)) << 4), bv[i]);
                    // values behind the request's last key are anything; those hidden from some rows may not be
                    // multiplied by their weights of 0 if they are not finite: such values are left out here and
                    // added at the end for the rows that see them
                    if (tail) {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) bv[i][e] &= e & 1 ? in1 : in0;
                    }
                    if (hidden) {
                        uint32_t bad = 0;
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) bad |= not_finite2(bv[i][e]);
                        if (__any_sync(0xffffffffu, bad != 0)) {
                            odd = true;
#pragma unroll
                            for (int i = 0; i < 2; ++i)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint32_t w = not_finite2(bv[i][e]);
                                    if (w & 0x8000u) bv[i][e] &= 0xFFFF0000u;
                                    if (w & 0x80000000u) bv[i][e] &= 0x0000FFFFu;
                                }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) mma_16816(o[jj + i], ah, bv[i >> 1][2 * (i & 1)], bv[i >> 1][2 * (i & 1) + 1]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) mma_16816(o[jj + i], al, bv[i >> 1][2 * (i & 1)], bv[i >> 1][2 * (i & 1) + 1]);
                }
            }
            __syncwarp();
            // (the last tile's keys make room for the warps' merge first)
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
                if (in < wkey || in >= wkey + 16) continue;
                const int page = p.table[int64_t(r) * p.max_pages + (key >> p.page_shift)];
                if (page < 0 || page >= p.n_pages) continue;
                const int64_t slot = (int64_t(page) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
                const uint32_t* v = reinterpret_cast<const uint32_t*>(p.V + (slot * p.Hk + g) * D) + qc;
                const bool inA = key >= kA.lo && key < kA.hi, inB = key >= kB.lo && key < kB.hi;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t w = v[n * 4];
                    const float2 f = unpack_bf16x2(w);
                    if (not_finite(w)) {
                        if (inA) o[n][0] += f.x;
                        if (inB) o[n][2] += f.x;
                    }
                    if (not_finite(w >> 16)) {
                        if (inA) o[n][1] += f.y;
                        if (inB) o[n][3] += f.y;
                    }
                }
            }
        }

        // The warps lay their results side by side where the last tile was (a lane's four values of n-tile n at
        // [n][lane]: no two lanes meet in a bank), and each adds up a quarter of the n-tiles
        constexpr int kMine = NT / kFewWarps;
        const int n0 = warp * kMine;
        if (j1 > j0) {
            const int s = (issued - 1) % T::kStages;
            float4* buf = reinterpret_cast<float4*>(ring + s * T::kStage);  // [warp][n-tile][lane]
            bar();  // every warp is done with the keys and values
#pragma unroll
            for (int n = 0; n < NT; ++n) buf[(warp * NT + n) * 32 + lane] = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
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
                    const float4 u = buf[(w * NT + n0 + n) * 32 + lane];
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

        if constexpr (CL) {
            // every CTA of the cluster lays down its result, and each adds up its share of the outputs, in CTA order
            if (qc == 0 && warp == 0) {
                fin_m[quad] = mA;
                fin_m[quad + 8] = mB;
                fin_l[quad] = lA;
                fin_l[quad + 8] = lB;
            }
#pragma unroll
            for (int n = 0; n < kMine; ++n) {
                const int c = (n0 + n) * 8 + 2 * qc;
                *reinterpret_cast<float2*>(fin + quad * T::kFinPitch + c) = make_float2(o[n][0], o[n][1]);
                *reinterpret_cast<float2*>(fin + (quad + 8) * T::kFinPitch + c) = make_float2(o[n][2], o[n][3]);
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
            for (int n = 0; n < kMine; ++n) {
                const int c = (n0 + n) * 8 + 2 * qc;
                if (okA) *reinterpret_cast<uint32_t*>(p.O + offA + c) = pack_bf16x2(__fmul_rn(o[n][0], iv), __fmul_rn(o[n][1], iv));
                if (okB) *reinterpret_cast<uint32_t*>(p.O + offB + c) = pack_bf16x2(__fmul_rn(o[n][2], iw), __fmul_rn(o[n][3], iw));
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
            for (int n = 0; n < kMine; ++n) {
                const int c = (n0 + n) * 8 + 2 * qc;
                if (okA) *reinterpret_cast<float2*>(PL::value(part, rA, c)) = make_float2(o[n][0], o[n][1]);
                if (okB) *reinterpret_cast<float2*>(PL::value(part, rB, c)) = make_float2(o[n][2], o[n][3]);
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

// A CTA's part of an item whose other part never comes: published and waited for as in the kernels.
__global__ void paged_selftest_kernel(uint32_t* flags, uint64_t limit_ns, int* status) {
    __shared__ int abort_flag;
    abort_flag = 0;
    part_publish(flags);
    part_wait(flags, 2, &abort_flag, status, limit_ns);
}

// ------------------------------------------------------------------ host side

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(f);
    });
    return fn;
}

}  // namespace

bool encode_cache(CUtensorMap* m, const void* base, const PagedAttnArgs& a, uint32_t box) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t D = cuuint64_t(a.head_dim), Hk = cuuint64_t(a.n_kv_heads), P = cuuint64_t(a.page_size);
    const cuuint64_t dims[4] = {D, Hk, P, cuuint64_t(a.n_pages)};
    const cuuint64_t strides[3] = {D * 2, Hk * D * 2, P * Hk * D * 2};
    const cuuint32_t boxes[4] = {64, 1, box, 1}, ones[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, boxes, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool encode_queries(CUtensorMap* m, const PagedAttnArgs& a, uint32_t heads, uint32_t tokens) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t D = cuuint64_t(a.head_dim), H = cuuint64_t(a.n_heads);
    const cuuint64_t dims[3] = {D, H, cuuint64_t(a.n_tokens)};
    const cuuint64_t strides[2] = {D * 2, H * D * 2};
    const cuuint32_t boxes[3] = {64, heads, tokens}, ones[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t*>(a.Q), dims, strides, boxes, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

double unit_bound(const PagedAttnArgs& a, int qb, int kt) {
    const double keys = std::min(double(a.max_pages) * double(a.page_size), 2147483647.0);
    const double blocks = std::floor(double(a.n_tokens) / qb) + double(std::min(a.n_req, a.n_tokens));
    return double(a.n_kv_heads) * blocks * (std::ceil(keys / kt) + 1.0);
}

namespace {

// CTAs that run at once, asked once per device; the opt-in shared memory is a per-device attribute too.
template <int D, int CAP>
cudaError_t few_resident(int& ctas) {
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
    auto* kernel = paged_few_kernel<D, CAP, false>;
    int per_sm = 0;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FewTraits<D>::kSmem);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(paged_few_kernel<D, CAP, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewTraits<D>::kSmemCluster);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kFewThreads, FewTraits<D>::kSmem);
    if (e != cudaSuccess) return e;
    // a partial result per item border: two per CTA, within the workspace
    const size_t slot = size_t(kFewRows) * (D + 2) * 4;
    const int fit = int((EMB_PAGED_WORKSPACE - kPagedFlagBytes) / (2 * slot));
    ctas = std::max(1, std::min({std::max(1, per_sm) * std::max(1, device_sm_count()), fit, int(kPagedFlagBytes / 4)}));
    if (dev >= 0 && dev < 64) known[dev] = ctas;
    return cudaSuccess;
}

// Blocks of a request's queries that its clusters take side by side.
int few_blocks(const PagedAttnArgs& a) {
    const int64_t qb = kFewRows / (a.n_heads / a.n_kv_heads);
    return int((std::min(a.max_q, a.n_tokens) + qb - 1) / qb);
}
// CTAs of the cluster that takes a block, or 0 where equal stretches of all the work are sooner done: a cluster keeps its
// CTAs for the longest request that the table has room for, stretches take their share of the total and a join worth eight
// tiles. Measured (us replayed, stretches and clusters; called, stretches take 2 to 3 more, being cooperative): one token of 8
// heads on one of 128 over 867 keys 7.5 and 6.0, 3000 9.1 and 8.8, 6000 10.0 and 13.1; 32 heads on 8 over 4000 13.0 and 11.0; 8
// requests of them over 900 16.2 and 8.8; 32 requests on one over up to 1500 14.8 and 8.2. The table's room stands for the
// length, which the host does not know: one token over 867 keys with room for 16384 takes 7.7 (10.4 called).
int few_cluster(const PagedAttnArgs& a) {
    double keys = double(a.max_pages * a.page_size);
    if (a.window > 0) keys = std::min(keys, double(a.window) + kFewRows + kFewTile);
    const double items = double(a.n_req * a.n_kv_heads) * few_blocks(a), tiles = std::ceil(keys / kFewTile);
    const double ctas = (a.head_dim == 256 ? 1.0 : 2.0) * std::max(1, device_sm_count());
    // A CTA's tiles, at most. 144 calls drawn where limits of 16 and 24 differ (1 to 64 requests, heads of 64 to 256, capped and
    // not, windows and none): with 24 the time is 0.83 of that with 16 called and 0.90 replayed (geometric means), for calls of
    // up to 16 rows and larger ones, capped and not alike; dearer by more than a tenth for 4 of them called and 9 replayed, by
    // 0.6 at most (few items of long requests, which stretches spread over more SMs).
    constexpr double longest = 24.0;
    int S = kFewCluster;
    while (S > 0 && items * S > ctas) S /= 2;
    return S > 0 && tiles <= longest * S && tiles / S <= items * tiles / ctas + 8.0 ? S : 0;
}

template <int D, int CAP>
cudaError_t launch_few(PagedParams& p, const PagedAttnArgs& a, cudaStream_t s) {
    int ctas = 0;
    const cudaError_t e = few_resident<D, CAP>(ctas);
    if (e != cudaSuccess) return e;
    p.QB = kFewRows / p.G;
    const uint32_t box = uint32_t(std::min<int64_t>(a.page_size, kFewTile));
    if (!encode_cache(&p.k_map, a.k_cache, a, box) || !encode_cache(&p.v_map, a.v_cache, a, box)) return cudaErrorInvalidValue;
    void* args[] = {&p};
    p.side = few_blocks(a);
    p.cluster = few_cluster(a);
    if (p.cluster > 0)
        return launch_serialised(reinterpret_cast<const void*>(paged_few_kernel<D, CAP, true>), unsigned(a.n_req * a.n_kv_heads * p.side * p.cluster),
                                 kFewThreads, FewTraits<D>::kSmemCluster, s, args, unsigned(p.cluster));
    const unsigned grid = unsigned(std::max(2.0, std::min(double(ctas), unit_bound(a, p.QB, kFewTile))));
    set_grid(p, grid, 3);
    return launch_serialised(reinterpret_cast<const void*>(paged_few_kernel<D, CAP, false>), grid, kFewThreads, FewTraits<D>::kSmem, s, args, 1, true);
}

template <int D>
cudaError_t launch_few_d(PagedParams& p, const PagedAttnArgs& a, cudaStream_t s) {
    return a.cap > kMostLowCap ? launch_few<D, kAnyCap>(p, a, s) : a.cap > 0.0f ? launch_few<D, kLowCap>(p, a, s) : launch_few<D, kUncapped>(p, a, s);
}

}  // namespace

double paged_attention_tiles(const PagedAttnArgs& a) { return unit_bound(a, std::max<int>(1, int(16 / (a.n_heads / a.n_kv_heads))), kFewTile); }

cudaError_t launch_paged_selftest(void* workspace, uint64_t limit_ns, int* status, cudaStream_t s) {
    paged_selftest_kernel<<<1, 1, 0, s>>>(static_cast<uint32_t*>(workspace), limit_ns, status);
    return cudaGetLastError();
}

cudaError_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t s) {
    PagedParams p;
    std::memset(&p, 0, sizeof(p));
    p.Q = reinterpret_cast<const __nv_bfloat16*>(a.Q);
    p.K = reinterpret_cast<const __nv_bfloat16*>(a.k_cache);
    p.V = reinterpret_cast<const __nv_bfloat16*>(a.v_cache);
    p.O = reinterpret_cast<__nv_bfloat16*>(a.O);
    p.table = a.table;
    p.q_start = a.q_start;
    p.kv_len = a.kv_len;
    p.prefix = a.prefix;
    p.flags = static_cast<uint32_t*>(a.workspace);
    p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + kPagedFlagBytes);
    p.status = a.status;
    p.max_pages = a.max_pages;
    p.n_tokens = int(a.n_tokens);
    p.n_req = int(a.n_req);
    p.n_pages = int(a.n_pages);
    while ((int64_t(1) << p.page_shift) < a.page_size) ++p.page_shift;
    p.kv_limit = int(a.max_pages * a.page_size);
    p.window = int(std::min<int64_t>(a.window, 2147483647));
    p.H = int(a.n_heads);
    p.Hk = int(a.n_kv_heads);
    p.G = p.H / p.Hk;
    constexpr double kLog2e = 1.4426950408889634;
    p.lin2 = float(kLog2e * double(a.scale));
    p.scale2 = p.lin2;
    if (a.cap > 0.0f) {  // (held within fp32's range for the least and the largest caps)
        p.scale2 = float(std::max(-double(FLT_MAX), std::min(2.0 * kLog2e * double(a.scale) / double(a.cap), double(FLT_MAX))));
        p.cap2 = float(std::min(kLog2e * double(a.cap), double(FLT_MAX)));
    }
    // Up to 16 rows of a request go to the mma.sync kernel, and more where all its blocks of 16 have a cluster at once: such
    // calls are small, and it has them sooner done (us replayed, tcgen05 and mma.sync: 50 queries of 8 heads over 866 keys 11.0
    // and 8.3, 8 over 816 10.1 and 6.5, 24 requests of 3 queries of 14 heads on 2 of 64 over up to 900 15.4 and 9.7, 280 of 8
    // heads of 64 alone 9.6 and 6.5). The rest goes to the tcgen05 kernel.
    const bool few = p.G <= 16 && (a.max_q * p.G <= 16 || few_cluster(a) > 0);
    if (!few) {
        p.negate = a.scale < 0.0f;
        p.scale2 = std::max(std::fabs(p.scale2), 1e-37f);  // (hidden scores are the lowest there are times this)
        p.lin2 = std::max(std::fabs(p.lin2), 1e-37f);
        return launch_paged_many(p, a, s);
    }
    return a.head_dim == 64    ? launch_few_d<64>(p, a, s)
           : a.head_dim == 128 ? launch_few_d<128>(p, a, s)
                               : launch_few_d<256>(p, a, s);
}

}  // namespace emb
