// Declarations shared by the translation units of libembpaged.so (not installed).
#pragma once

#include "../../include/emb_paged.h"
#include "ptx.cuh"

namespace emb {

struct SlotArgs {
    const int32_t* cached;
    const int32_t* added;
    const int32_t* free_pages;
    const int32_t* used;
    int32_t* table;
    int32_t* q_start;
    int32_t* kv_len;
    int64_t* slots;
    int32_t* positions;
    int32_t* used_out;
    int64_t n_free, max_pages, n_tokens;
    int n_req, page_size;
};
cudaError_t launch_paged_slots(const SlotArgs& a, cudaStream_t s);

struct QkArgs {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const float* q_gamma;
    const float* k_gamma;
    const int32_t* positions;
    const uint8_t* axis_of_pair;  // host, or NULL
    const int64_t* slots;
    uint16_t* q_out;
    uint16_t* k_cache;
    uint16_t* v_cache;
    int64_t q_stride, k_stride, v_stride, pos_stride, n_tokens, n_heads, n_kv_heads, head_dim, rot_dim, n_slots, n_axes;
    float eps, base;
    int* status;
};
cudaError_t launch_qk_norm_rope(const QkArgs& a, cudaStream_t s);

struct PagedAttnArgs {
    const uint16_t* Q;
    const uint16_t* k_cache;
    const uint16_t* v_cache;
    const int32_t* table;
    const int32_t* q_start;
    const int32_t* kv_len;
    const int32_t* prefix;
    uint16_t* O;
    void* workspace;
    int* status;
    int64_t n_pages, page_size, max_pages, n_req, n_tokens, max_q, n_heads, n_kv_heads, head_dim, window;
    float scale, cap;
};
// Key tiles of a call, at most (an upper bound from the host's sizes).
double paged_attention_tiles(const PagedAttnArgs& a);
cudaError_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t s);
cudaError_t launch_paged_selftest(void* workspace, uint64_t limit_ns, int* status, cudaStream_t s);

// Two fp32 products, FMAs and sums at once.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "mul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// A launch with programmatic stream serialisation, in clusters if `cluster` is above one. `together`: its CTAs wait for one
// another, so it is launched cooperatively. That all of them run at once is then a promise of the launch (or an error of it),
// whatever runs on other streams; by the occupancy API alone it would hold on an idle device only. It costs a call the
// overlap with the launch before it (one token over 6000 keys 11.1 -> 12.3 us, 816 of two requests, heads of 256, 28.4 -> 30.8),
// a recorded one nothing (10.5 -> 10.0, 28.1 -> 28.3).
inline cudaError_t launch_serialised(const void* fn, unsigned grid, unsigned block, size_t smem, cudaStream_t s,
                                     void** args, unsigned cluster = 1, bool together = false) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    } else if (together) {
        attr[1].id = cudaLaunchAttributeCooperative;
        attr[1].val.cooperative = 1;
        cfg.numAttrs = 2;
    }
    return cudaLaunchKernelExC(&cfg, fn, args);
}

}  // namespace emb
