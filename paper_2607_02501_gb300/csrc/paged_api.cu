// C ABI of libembpaged.so (declarations and contracts in include/emb_paged.h): argument validation, every
// error reported before anything is enqueued, and the status word that bounded device-side waits report into.
#include <algorithm>
#include <cmath>
#include <mutex>

#include "paged8.cuh"

namespace emb {
namespace {

__device__ int g_status_word;  // OR of kStatus* flags; read and cleared by emb_paged_status
__device__ int g_status_read;  // where emb_paged_status's exchange leaves the value it read

// Device addresses of the two words, asked once per device; NULL if they cannot be told.
int* device_words(bool read_slot) {
    static std::mutex mu;
    static int* ptrs[64][2] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!ptrs[dev][0]) {
        void *a = nullptr, *b = nullptr;
        if (cudaGetSymbolAddress(&a, g_status_word) != cudaSuccess || cudaGetSymbolAddress(&b, g_status_read) != cudaSuccess)
            return nullptr;
        ptrs[dev][0] = static_cast<int*>(a);
        ptrs[dev][1] = static_cast<int*>(b);
    }
    return ptrs[dev][read_slot ? 1 : 0];
}

__global__ void paged_status_kernel(int* status, int* out) { *out = atomicExch(status, 0); }

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
constexpr int64_t k31 = int64_t(1) << 31, k46 = int64_t(1) << 46;
bool within(int64_t v, int64_t lo, int64_t end) { return v >= lo && v < end; }

// A buffer of a call: [p, p + bytes). Empty ones overlap nothing.
struct Span {
    const void* p;
    int64_t bytes;
};
bool overlap(const Span& a, const Span& b) {
    const uintptr_t x = uintptr_t(a.p), y = uintptr_t(b.p);
    return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + uintptr_t(b.bytes) && y < x + uintptr_t(a.bytes);
}
// Whether any of the n_out outputs overlaps an input or another output.
bool clash(const Span* outs, int n_out, const Span* ins, int n_in) {
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (overlap(outs[i], ins[j])) return true;
        for (int j = i + 1; j < n_out; ++j)
            if (overlap(outs[i], outs[j])) return true;
    }
    return false;
}
emb_status from_cuda(cudaError_t e) { return e == cudaSuccess ? EMB_OK : EMB_ECUDA; }
cudaStream_t stream_of(emb_stream_t s) { return reinterpret_cast<cudaStream_t>(s); }

// A number as the sum of two fp64 ones, the second below half a unit of the first's last place: about 2^-104 of it (Dekker, 1971;
// Knuth, The Art of Computer Programming, volume 2, 4.2.2). `volatile`: no product is contracted with a sum, on any machine.
struct Twofold {
    double hi, lo;
};
Twofold sum_of(double a, double b) {
    const volatile double s = a + b, t = s - a;
    const volatile double u = s - t;
    return {s, (a - u) + (b - t)};
}
Twofold operator+(Twofold a, Twofold b) {
    const Twofold s = sum_of(a.hi, b.hi);
    return sum_of(s.hi, s.lo + (a.lo + b.lo));
}
Twofold operator*(Twofold a, Twofold b) {
    const volatile double p = a.hi * b.hi;
    const double e = std::fma(a.hi, b.hi, -p);
    return sum_of(p, std::fma(a.hi, b.lo, std::fma(a.lo, b.hi, e)));
}
Twofold operator/(Twofold a, Twofold b) {  // two steps of long division, and the rest's rest
    const double q0 = a.hi / b.hi;
    const Twofold r = a + Twofold{-q0, 0.0} * b;
    const double q1 = r.hi / b.hi;
    const Twofold s = r + Twofold{-q1, 0.0} * b;
    return sum_of(q0, q1) + Twofold{s.hi / b.hi, 0.0};
}
Twofold power(Twofold x, int64_t n) {
    Twofold y{1.0, 0.0};
    for (; n > 0; n >>= 1) {
        if (n & 1) y = y * x;
        if (n > 1) x = x * x;
    }
    return y;
}
// x^(-1 / n), x in [1/2, 2]: Newton's step on x y^n = 1, which doubles the digits of the first guess.
Twofold inverse_root(double x, int64_t n) {
    Twofold y{std::pow(x, -1.0 / double(n)), 0.0};
    for (int k = 0; k < 2; ++k) {
        const Twofold off = Twofold{1.0, 0.0} + Twofold{-x, 0.0} * power(y, n);
        y = y + y * (off / Twofold{double(n), 0.0});
    }
    return y;
}

bool cache8_supported(int64_t head_dim, int64_t page_size) {
    return (head_dim == 64 || head_dim == 128 || head_dim == 256) &&
           (page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128 || page_size == 256);
}

// The checks of an attention call over a cache whose elements have `size` bytes, and its arguments for a launch. `exps`: what else
// the cache consists of, or nothing.
emb_status attention_args(PagedAttnArgs& a, int64_t size, const Span (&exps)[2], const uint16_t* Q, const void* k_cache,
                          const void* v_cache, int64_t n_pages, int64_t page_size, const int32_t* table, int64_t max_pages,
                          const int32_t* q_start, const int32_t* kv_len, const int32_t* prefix, int64_t n_req, int64_t n_tokens,
                          int64_t max_q, uint16_t* O, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim, float scale,
                          float cap, int64_t window, void* workspace, size_t ws_bytes) {
    if (!within(n_req, 1, 65537) || !within(n_tokens, 1, k31) || !within(n_pages, 1, k31) || max_q < 1 ||
        !within(max_pages, 1, k31) || !within(n_heads, 1, 4097) || n_kv_heads < 1 || n_heads % n_kv_heads != 0 ||
        !std::isfinite(scale) || !std::isfinite(cap) || cap < 0.0f || window < 0 || head_dim < 1 || page_size < 1 ||
        n_req * max_pages >= k46)
        return EMB_EINVAL;
    if (!Q || !k_cache || !v_cache || !table || !q_start || !kv_len || !O || !workspace) return EMB_EINVAL;
    if ((head_dim != 64 && head_dim != 128 && head_dim != 256) || n_heads / n_kv_heads > 64 ||
        (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128 && page_size != 256))
        return EMB_EUNSUPPORTED;
    // (a key's number plus two tiles stays within 31 bits)
    if (max_pages * page_size > k31 - 512 || n_tokens >= k46 / (n_heads * head_dim) ||
        n_pages * page_size >= k46 / (n_kv_heads * head_dim))
        return EMB_EINVAL;
    const void* rows[] = {Q, k_cache, v_cache, O};
    for (const void* w : rows)
        if (!aligned(w, 16)) return EMB_EALIGN;
    const void* ints[] = {table, q_start, kv_len, prefix};
    for (const void* w : ints)
        if (!aligned(w, 4)) return EMB_EALIGN;
    if (!aligned(workspace, 256)) return EMB_EALIGN;
    if (ws_bytes < EMB_PAGED_WORKSPACE) return EMB_ENOSPC;
    const int64_t rows_bytes = n_tokens * n_heads * head_dim * 2, cache = n_pages * page_size * n_kv_heads * head_dim * size;
    const Span ins[] = {{Q, rows_bytes}, {k_cache, cache}, {v_cache, cache}, {table, n_req * max_pages * 4},
                        {q_start, (n_req + 1) * 4}, {kv_len, n_req * 4}, {prefix, n_req * 4}, exps[0], exps[1]};
    const Span outs[] = {{O, rows_bytes}, {workspace, int64_t(EMB_PAGED_WORKSPACE)}};
    if (clash(outs, 2, ins, 9)) return EMB_EINVAL;
    a = PagedAttnArgs{};
    a.Q = Q;
    a.k_cache = static_cast<const uint16_t*>(k_cache);
    a.v_cache = static_cast<const uint16_t*>(v_cache);
    a.table = table;
    a.q_start = q_start;
    a.kv_len = kv_len;
    a.prefix = prefix;
    a.O = O;
    a.workspace = workspace;
    a.n_pages = n_pages;
    a.page_size = page_size;
    a.max_pages = max_pages;
    a.n_req = n_req;
    a.n_tokens = n_tokens;
    a.max_q = max_q;
    a.n_heads = n_heads;
    a.n_kv_heads = n_kv_heads;
    a.head_dim = head_dim;
    a.window = window;
    a.scale = scale;
    a.cap = cap;
    if (paged_attention_tiles(a) >= double(k31)) return EMB_EUNSUPPORTED;
    a.status = device_words(false);
    return a.status ? EMB_OK : EMB_ECUDA;
}

}  // namespace

int device_sm_count() {
    static std::mutex mu;
    static int counts[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    std::lock_guard<std::mutex> lock(mu);
    if (!counts[dev] && cudaDeviceGetAttribute(&counts[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        counts[dev] = 0;
    return counts[dev];
}

}  // namespace emb

using namespace emb;

extern "C" {

emb_status emb_paged_slots(const int32_t* cached, const int32_t* added, int64_t n_req, const int32_t* free_pages,
                           int64_t n_free, const int32_t* used, int64_t page_size, int32_t* table, int64_t max_pages,
                           int32_t* q_start, int32_t* kv_len, int64_t* slots, int32_t* positions, int64_t n_tokens,
                           int32_t* used_out, emb_stream_t stream) {
    if (!within(n_req, 1, 65537) || !within(n_tokens, 0, k31) || !within(n_free, 0, k31) ||
        !within(page_size, 1, 65537) || !within(max_pages, 1, k31) || n_req * max_pages >= k46)
        return EMB_EINVAL;
    if (!cached || !added || !used || !table || !q_start || !kv_len || !used_out || (n_free > 0 && !free_pages) ||
        (n_tokens > 0 && (!slots || !positions)))
        return EMB_EINVAL;
    const void* words[] = {cached, added, free_pages, used, table, q_start, kv_len, positions, used_out};
    for (const void* w : words)
        if (!aligned(w, 4)) return EMB_EALIGN;
    if (!aligned(slots, 8)) return EMB_EALIGN;
    const Span ins[] = {{cached, n_req * 4}, {added, n_req * 4}, {free_pages, n_free * 4}, {used, 4}};
    const Span outs[] = {{table, n_req * max_pages * 4}, {q_start, (n_req + 1) * 4}, {kv_len, n_req * 4},
                         {slots, n_tokens * 8}, {positions, n_tokens * 4}, {used_out, 4}};
    if (clash(outs, 6, ins, 4)) return EMB_EINVAL;
    SlotArgs a = {};
    a.cached = cached;
    a.added = added;
    a.free_pages = free_pages;
    a.used = used;
    a.table = table;
    a.q_start = q_start;
    a.kv_len = kv_len;
    a.slots = slots;
    a.positions = positions;
    a.used_out = used_out;
    a.n_free = n_free;
    a.max_pages = max_pages;
    a.n_tokens = n_tokens;
    a.n_req = int(n_req);
    a.page_size = int(page_size);
    return from_cuda(launch_paged_slots(a, stream_of(stream)));
}

emb_status emb_qk_norm_rope(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                            const uint16_t* v, int64_t v_stride, int64_t n_tokens, int64_t n_heads,
                            int64_t n_kv_heads, int64_t head_dim, const float* q_gamma, const float* k_gamma,
                            float eps, const int32_t* positions, int64_t pos_stride, int64_t n_axes,
                            const uint8_t* axis_of_pair, int64_t rot_dim, float base, const int64_t* slots,
                            uint16_t* q_out, uint16_t* k_cache, uint16_t* v_cache, int64_t n_pages,
                            int64_t page_size, emb_stream_t stream) {
    if (!within(n_tokens, 1, k31) || !within(n_heads, 1, 4097) || !within(n_kv_heads, 1, 4097) ||
        !within(head_dim, 8, 257) || head_dim % 8 != 0 || !within(rot_dim, 0, head_dim + 1) || rot_dim % 8 != 0 ||
        !within(n_axes, 1, 5) || !within(pos_stride, n_tokens, k46) || !within(n_pages, 1, k31) ||
        !within(page_size, 1, 65537) || !(base > 0.0f) || !std::isfinite(base) || !(eps >= 0.0f) || !std::isfinite(eps))
        return EMB_EINVAL;
    const int64_t qw = n_heads * head_dim, kw = n_kv_heads * head_dim;
    const int64_t strides[] = {q_stride - qw, k_stride - kw, v_stride - kw};
    for (int64_t over : strides)
        if (over < 0 || over % 8 != 0) return EMB_EINVAL;
    if (q_stride >= k46 / n_tokens || k_stride >= k46 / n_tokens || v_stride >= k46 / n_tokens ||
        n_pages * page_size >= k46 / kw)
        return EMB_EINVAL;
    if (!q || !k || !v || !positions || !slots || !q_out || !k_cache || !v_cache) return EMB_EINVAL;
    if (axis_of_pair)
        for (int64_t i = 0; i < rot_dim / 2; ++i)
            if (axis_of_pair[i] >= n_axes) return EMB_EINVAL;
    const void* rows[] = {q, k, v, q_gamma, k_gamma, q_out, k_cache, v_cache};
    for (const void* w : rows)
        if (!aligned(w, 16)) return EMB_EALIGN;
    if (!aligned(positions, 4) || !aligned(slots, 8)) return EMB_EALIGN;
    auto rows_bytes = [&](int64_t stride, int64_t width) { return ((n_tokens - 1) * stride + width) * 2; };
    const Span ins[] = {{q, rows_bytes(q_stride, qw)}, {k, rows_bytes(k_stride, kw)}, {v, rows_bytes(v_stride, kw)},
                        {q_gamma, head_dim * 4}, {k_gamma, head_dim * 4},
                        {positions, ((n_axes - 1) * pos_stride + n_tokens) * 4}, {slots, n_tokens * 8}};
    const int64_t cache = n_pages * page_size * kw * 2;
    const Span outs[] = {{q_out, n_tokens * qw * 2}, {k_cache, cache}, {v_cache, cache}};
    if (clash(outs, 3, ins, 7)) return EMB_EINVAL;
    QkArgs a = {};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_gamma = q_gamma;
    a.k_gamma = k_gamma;
    a.positions = positions;
    a.axis_of_pair = axis_of_pair;
    a.slots = slots;
    a.q_out = q_out;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pos_stride = pos_stride;
    a.n_tokens = n_tokens;
    a.n_heads = n_heads;
    a.n_kv_heads = n_kv_heads;
    a.head_dim = head_dim;
    a.rot_dim = rot_dim;
    a.n_slots = n_pages * page_size;
    a.eps = eps;
    a.base = base;
    a.n_axes = n_axes;
    a.status = device_words(false);
    if (!a.status) return EMB_ECUDA;
    return from_cuda(launch_qk_norm_rope(a, stream_of(stream)));
}

emb_status emb_paged_attention(const uint16_t* Q, const uint16_t* k_cache, const uint16_t* v_cache,
                               int64_t n_pages, int64_t page_size, const int32_t* table, int64_t max_pages,
                               const int32_t* q_start, const int32_t* kv_len, const int32_t* prefix, int64_t n_req,
                               int64_t n_tokens, int64_t max_q, uint16_t* O, int64_t n_heads, int64_t n_kv_heads,
                               int64_t head_dim, float scale, float cap, int64_t window, void* workspace,
                               size_t ws_bytes, emb_stream_t stream) {
    PagedAttnArgs a;
    const emb_status e = attention_args(a, 2, {{nullptr, 0}, {nullptr, 0}}, Q, k_cache, v_cache, n_pages, page_size, table, max_pages,
                                        q_start, kv_len, prefix, n_req, n_tokens, max_q, O, n_heads, n_kv_heads, head_dim, scale,
                                        cap, window, workspace, ws_bytes);
    return e != EMB_OK ? e : from_cuda(launch_paged_attention(a, stream_of(stream)));
}

emb_status emb_paged_status(emb_stream_t stream) {
    const cudaStream_t s = stream_of(stream);
    int *st = device_words(false), *slot = device_words(true);
    if (!st || !slot) return EMB_ECUDA;
    // one read slot per device: concurrent callers take turns
    static std::mutex mu;
    std::lock_guard<std::mutex> lock(mu);
    paged_status_kernel<<<1, 1, 0, s>>>(st, slot);
    if (cudaGetLastError() != cudaSuccess) return EMB_ECUDA;
    int host = 0;
    if (cudaMemcpyAsync(&host, slot, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess) return EMB_ECUDA;
    if (cudaStreamSynchronize(s) != cudaSuccess) return EMB_ECUDA;
    return (host & kStatusTimeout) ? EMB_ETIMEOUT : EMB_OK;
}

emb_status emb_paged_selftest_wait_timeout(void* workspace, size_t ws_bytes, int64_t timeout_ns, emb_stream_t stream) {
    if (!workspace || timeout_ns < 1000 || timeout_ns > 1000000000) return EMB_EINVAL;
    if (!aligned(workspace, 256)) return EMB_EALIGN;
    if (ws_bytes < EMB_PAGED_WORKSPACE) return EMB_ENOSPC;
    int* st = device_words(false);
    if (!st) return EMB_ECUDA;
    return from_cuda(launch_paged_selftest(workspace, uint64_t(timeout_ns), st, stream_of(stream)));
}

// ------------------------------------------------------------------ the 8-bit cache (include/emb_paged.h)

emb_status emb_rotary_turns(int64_t rot_dim, double base, double stretch, double original, double low, double high, uint64_t* turns) {
    if (!within(rot_dim, 2, 257) || rot_dim % 2 != 0 || !(base > 0.0) || !std::isfinite(base) || !(stretch >= 1.0) ||
        !std::isfinite(stretch) || !(original >= 0.0) || !std::isfinite(original) || !(low >= 0.0) || !(high > low) ||
        !std::isfinite(high) || !turns)
        return EMB_EINVAL;
    // base^(-i / n) for base = m 2^e, i e = q n + j: m^(-i / n) 2^(-j / n) 2^-q, the first two of which are near one
    const int64_t n = rot_dim / 2;
    int e = 0;
    const double m = std::frexp(base, &e);
    const Twofold root = inverse_root(m, n), half = inverse_root(2.0, n), one{1.0, 0.0};
    const Twofold per_radian{0x1.45f306dc9c883p-3, -0x1.6b01ec5417056p-57};  // 1 / (2 pi)
    for (int64_t i = 0; i < n; ++i) {
        const int64_t q = i * e >= 0 ? i * e / n : -((-i * e + n - 1) / n), j = i * e - q * n;
        Twofold t = power(root, i) * power(half, j) * per_radian;  // turns a position
        t = {std::ldexp(t.hi, int(-q)), std::ldexp(t.lo, int(-q))};
        if (stretch > 1.0) {
            const double turned = original * t.hi;
            Twofold keep{turned >= 2.0 * high ? 1.0 : 0.0, 0.0};
            if (turned < 2.0 * high && turned > 0.5 * low) keep = (Twofold{original, 0.0} * t + Twofold{-low, 0.0}) / sum_of(high, -low);
            if (!(keep.hi > 0.0)) keep = {0.0, 0.0};
            if (!(keep.hi < 1.0)) keep = one;
            t = t * (keep + (one + Twofold{-keep.hi, -keep.lo}) / Twofold{stretch, 0.0});
        }
        // whole turns are none; whole units and the rest of both parts
        const double a = std::ldexp(std::fmod(t.hi, 1.0), 64), b = std::ldexp(std::fmod(t.lo, 1.0), 64);
        const double down = std::floor(b), rest = (a - std::floor(a)) + (b - down);
        turns[i] = uint64_t(std::floor(a)) + (down < 0.0 ? 0 - uint64_t(-down) : uint64_t(down)) + uint64_t(std::floor(rest + 0.5));
    }
    return EMB_OK;
}

emb_status emb_paged8_store(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                            int64_t v_stride, int64_t n_tokens, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                            const float* q_gamma, const float* k_gamma, float eps, const int32_t* positions, int64_t pos_stride,
                            int64_t n_axes, const uint8_t* axis_of_pair, const uint64_t* turns, int64_t rot_dim,
                            int32_t neighbours, float factor, const int64_t* slots, uint16_t* q_out, uint8_t* k_codes,
                            uint8_t* v_codes, uint8_t* k_exp, uint8_t* v_exp, int64_t n_pages, int64_t page_size,
                            emb_stream_t stream) {
    if (head_dim < 1 || page_size < 1) return EMB_EINVAL;
    if (!cache8_supported(head_dim, page_size)) return EMB_EUNSUPPORTED;
    if (!within(n_tokens, 1, k31) || !within(n_heads, 1, 4097) || !within(n_kv_heads, 1, 4097) ||
        !within(rot_dim, 0, head_dim + 1) || rot_dim % 8 != 0 || !within(n_axes, 1, 5) ||
        !within(pos_stride, n_tokens, k46) || !within(n_pages, 1, k31) || !(eps >= 0.0f) || !std::isfinite(eps) ||
        !std::isfinite(factor) || (neighbours != 0 && neighbours != 1))
        return EMB_EINVAL;
    const int64_t qw = n_heads * head_dim, kw = n_kv_heads * head_dim;
    const int64_t strides[] = {q_stride - qw, k_stride - kw, v_stride - kw};
    for (int64_t over : strides)
        if (over < 0 || over % 8 != 0) return EMB_EINVAL;
    if (q_stride >= k46 / n_tokens || k_stride >= k46 / n_tokens || v_stride >= k46 / n_tokens || n_pages * page_size >= k46 / kw)
        return EMB_EINVAL;
    // (its CTAs stay within a launch's grid)
    if (n_tokens * (n_heads + n_kv_heads) >= (int64_t(1) << 33)) return EMB_EUNSUPPORTED;
    if (!q || !k || !v || !positions || (rot_dim > 0 && !turns) || !slots || !q_out || !k_codes || !v_codes || !k_exp || !v_exp)
        return EMB_EINVAL;
    const void* rows[] = {q, k, v, q_gamma, k_gamma, q_out, k_codes, v_codes};
    for (const void* w : rows)
        if (!aligned(w, 16)) return EMB_EALIGN;
    if (!aligned(positions, 4) || !aligned(slots, 8) || !aligned(turns, 8)) return EMB_EALIGN;
    auto rows_bytes = [&](int64_t stride, int64_t width) { return ((n_tokens - 1) * stride + width) * 2; };
    const Span ins[] = {{q, rows_bytes(q_stride, qw)}, {k, rows_bytes(k_stride, kw)}, {v, rows_bytes(v_stride, kw)},
                        {q_gamma, head_dim * 4}, {k_gamma, head_dim * 4},
                        {positions, ((n_axes - 1) * pos_stride + n_tokens) * 4}, {slots, n_tokens * 8},
                        {turns, rot_dim / 2 * 8}, {axis_of_pair, rot_dim / 2}};
    const int64_t codes = n_pages * page_size * kw, exps = n_pages * (page_size / kBlock8) * n_kv_heads;
    const Span outs[] = {{q_out, n_tokens * qw * 2}, {k_codes, codes}, {v_codes, codes}, {k_exp, exps}, {v_exp, exps}};
    if (clash(outs, 5, ins, 9)) return EMB_EINVAL;
    Store8Args a = {};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_gamma = q_gamma;
    a.k_gamma = k_gamma;
    a.positions = positions;
    a.axis_of_pair = axis_of_pair;
    a.turns = turns;
    a.slots = slots;
    a.q_out = q_out;
    a.k_codes = k_codes;
    a.v_codes = v_codes;
    a.k_exp = k_exp;
    a.v_exp = v_exp;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pos_stride = pos_stride;
    a.n_tokens = n_tokens;
    a.n_slots = n_pages * page_size;
    a.n_heads = int(n_heads);
    a.n_kv_heads = int(n_kv_heads);
    a.head_dim = int(head_dim);
    a.rot_dim = int(rot_dim);
    a.n_axes = int(n_axes);
    a.eps = eps;
    a.factor = factor;
    a.neighbours = neighbours != 0;
    return from_cuda(launch_paged8_store(a, stream_of(stream)));
}

emb_status emb_paged8_read(const uint8_t* k_codes, const uint8_t* v_codes, const uint8_t* k_exp, const uint8_t* v_exp,
                           int64_t n_pages, int64_t page_size, int64_t n_kv_heads, int64_t head_dim, const int64_t* slots,
                           int64_t n_rows, uint16_t* k_out, uint16_t* v_out, emb_stream_t stream) {
    if (!within(n_rows, 0, k31) || !within(n_kv_heads, 1, 4097) || !within(n_pages, 1, k31) || head_dim < 1 || page_size < 1)
        return EMB_EINVAL;
    if (!cache8_supported(head_dim, page_size)) return EMB_EUNSUPPORTED;
    const int64_t kw = n_kv_heads * head_dim;
    if (n_pages * page_size >= k46 / kw || n_rows >= k46 / kw) return EMB_EINVAL;
    if (n_rows * kw >= int64_t(1) << 42) return EMB_EUNSUPPORTED;  // (its CTAs stay within a launch's grid)
    if (!k_codes || !v_codes || !k_exp || !v_exp || (n_rows > 0 && (!slots || !k_out || !v_out))) return EMB_EINVAL;
    const void* rows[] = {k_codes, v_codes, k_out, v_out};
    for (const void* w : rows)
        if (!aligned(w, 16)) return EMB_EALIGN;
    if (!aligned(slots, 8)) return EMB_EALIGN;
    const int64_t codes = n_pages * page_size * kw, exps = n_pages * (page_size / kBlock8) * n_kv_heads;
    const Span ins[] = {{k_codes, codes}, {v_codes, codes}, {k_exp, exps}, {v_exp, exps}, {slots, n_rows * 8}};
    const Span outs[] = {{k_out, n_rows * kw * 2}, {v_out, n_rows * kw * 2}};
    if (clash(outs, 2, ins, 5)) return EMB_EINVAL;
    if (n_rows == 0) return EMB_OK;
    Read8Args a = {k_codes, v_codes, k_exp, v_exp, slots, k_out, v_out, n_rows, n_pages * page_size, int(n_kv_heads), int(head_dim)};
    return from_cuda(launch_paged8_read(a, stream_of(stream)));
}

emb_status emb_paged8_attention(const uint16_t* Q, const uint8_t* k_codes, const uint8_t* v_codes, const uint8_t* k_exp,
                                const uint8_t* v_exp, int64_t n_pages, int64_t page_size, const int32_t* table,
                                int64_t max_pages, const int32_t* q_start, const int32_t* kv_len, const int32_t* prefix,
                                int64_t n_req, int64_t n_tokens, int64_t max_q, uint16_t* O, int64_t n_heads,
                                int64_t n_kv_heads, int64_t head_dim, float scale, float cap, int64_t window, void* workspace,
                                size_t ws_bytes, emb_stream_t stream) {
    Paged8AttnArgs a;
    if (!k_exp || !v_exp) return EMB_EINVAL;
    // (sizes that make no sense are refused below; here they only must not overflow)
    const bool sane = within(n_pages, 1, k31) && within(page_size, 1, 65537) && within(n_kv_heads, 1, 4097);
    const int64_t exps = sane ? n_pages * (page_size / kBlock8) * n_kv_heads : 0;
    const emb_status e = attention_args(a.a, 1, {{k_exp, exps}, {v_exp, exps}}, Q, k_codes, v_codes, n_pages, page_size, table,
                                        max_pages, q_start, kv_len, prefix, n_req, n_tokens, max_q, O, n_heads, n_kv_heads,
                                        head_dim, scale, cap, window, workspace, ws_bytes);
    if (e != EMB_OK) return e;
    a.k_exp = k_exp;
    a.v_exp = v_exp;
    return from_cuda(launch_paged8_attention(a, stream_of(stream)));
}

}  // extern "C"
