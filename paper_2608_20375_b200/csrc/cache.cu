// The paged key/value cache of the verifier: entries written (and quantised), read back, and moved up after the walk.
#include "cache.cuh"

namespace graft {

namespace {

constexpr int kThreads = 256;

struct CacheRowsParams {
    CacheView c;
    const int32_t* prefix_len;
    const int32_t* count;
    int rows;
    long long stride;  // of the rows of key and value, in numbers
    const uint8_t* key;   // (cache_read: written)
    const uint8_t* value;
    int32_t* status;
};

// Rows in use and the first slot of sequence b, or no row at all when something about them is wrong.  A block finds it once; the first
// block of a sequence reports it.
__device__ __forceinline__ int rows_of(const CacheRowsParams& p, int b, int& base) {
    __shared__ int use;
    const int n = p.count[b];
    base = p.prefix_len[b] - 1;
    if (threadIdx.x < 32) {
        const bool ok = n >= 0 && n <= p.rows && base >= 0 && cache_slots_ok(p.c, p.c.table + (size_t)b * p.c.width, base, (long long)base + n);
        if (threadIdx.x == 0) {
            use = ok ? n : 0;
            if (p.status && blockIdx.x == 0) p.status[b] = ok ? 0 : GRAFT_ST_BAD_CACHE;
        }
    }
    __syncthreads();
    return use;
}

// What a thread does of one (row, K or V, head): sixteen numbers, head_dim / 16 threads a head.
struct Item {
    bool there, is_v;
    long long at;      // of the thread's numbers in key or value
    size_t entry;      // of the cache
};
__device__ __forceinline__ Item item_of(const CacheRowsParams& p, int b, int n, int base, unsigned item, int part) {
    const CacheView& c = p.c;
    Item t;
    const unsigned row = item / (2u * c.kv_heads), hk = item - row * 2u * c.kv_heads;
    t.there = (int)row < n;
    t.is_v = hk >= (unsigned)c.kv_heads;
    const int head = (int)hk - (t.is_v ? c.kv_heads : 0), slot = base + (int)row;
    t.at = ((long long)b * p.rows + row) * p.stride + head * c.head_dim + part * 16;
    const int page = t.there ? __ldg(c.table + (size_t)b * c.width + (slot >> c.page_shift)) : 0;
    t.entry = cache_row(c, page, head, slot & ((1 << c.page_shift) - 1));
    return t;
}

constexpr int kItems = 4;  // that a thread has under way: 128 bytes of its input

// Two 16-byte loads a thread and item, the largest of the row by shuffles, one 16-byte store (two into a bf16 cache).  A row's exponent
// follows from the bits of its largest magnitude alone.  Prompts of 1000 to 8192 tokens, 8 sequences, 8 heads of 128, written and
// read back: 453 MB in 107 us, 4.2 TB/s (165 us with one item a thread).
template <bool Q8>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const CacheRowsParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const CacheView& c = p.c;
    const int b = blockIdx.y, tpr = c.head_dim >> 4, per = kThreads / tpr;
    int base;
    const int n = rows_of(p, b, base);
    const unsigned first = blockIdx.x * (unsigned)(per * kItems);
    if (first / (2u * c.kv_heads) >= (unsigned)n) return;
    const int part = threadIdx.x & (tpr - 1);
    Item t[kItems];
    uint4 in[kItems][2];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        t[i] = item_of(p, b, n, base, first + i * per + threadIdx.x / tpr, part);
        const uint4* src = (const uint4*)((t[i].is_v ? p.value : p.key) + (t[i].there ? 2 * t[i].at : 0));
        in[i][0] = __ldg(src), in[i][1] = __ldg(src + 1);
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        uint8_t* dst = (t[i].is_v ? c.v : c.k) + t[i].entry * c.row_bytes;
        if (!Q8) {
            if (t[i].there) ((uint4*)dst)[2 * part] = in[i][0], ((uint4*)dst)[2 * part + 1] = in[i][1];
            continue;
        }
        const uint32_t w[8] = {in[i][0].x, in[i][0].y, in[i][0].z, in[i][0].w, in[i][1].x, in[i][1].y, in[i][1].z, in[i][1].w};
        uint32_t amax = 0;  // as the bits of a bf16: magnitudes are ordered like their bits, NaN above infinity
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = max(amax, max(w[j] & 0x7FFFu, (w[j] >> 16) & 0x7FFFu));
        for (int o = tpr >> 1; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
        if (!t[i].there) continue;
        const bool bad = amax >= 0x7F80u;
        // amax = f 2^x with f in [1, 2): amax <= 448 2^e = 1.75 2^(e + 8) iff e >= x - 8, or x - 7 where f > 1.75.  Subnormal numbers are
        // below 2^-126, where e is at its least.
        int e = (int)(amax >> 7) - 127 - 8 + ((amax & 0x7Fu) > 0x60u);
        e = e < -120 ? -120 : e;
        const float up = __int_as_float((uint32_t)(127 - (e > 0 ? e : e / 2)) << 23);       // 2^-e in two factors: -e goes up to 120,
        const float more = __int_as_float((uint32_t)(127 - (e > 0 ? 0 : e - e / 2)) << 23); // and both are normal numbers
        uint32_t y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t four = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t u = w[2 * j + k];
                const float2 x = make_float2(__uint_as_float(u << 16) * up * more, __uint_as_float(u & 0xFFFF0000u) * up * more);
                four |= (uint32_t)__nv_cvt_float2_to_fp8x2(x, __NV_SATFINITE, __NV_E4M3) << (16 * k);
            }
            y[j] = bad ? 0u : four;
        }
        ((uint4*)dst)[part] = make_uint4(y[0], y[1], y[2], y[3]);
        if (part == 0) (t[i].is_v ? c.v_exp : c.k_exp)[t[i].entry] = bad ? 255 : (uint8_t)(e + 127);
    }
}

template <bool Q8>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheRowsParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const CacheView& c = p.c;
    const int b = blockIdx.y, tpr = c.head_dim >> 4, per = kThreads / tpr;
    int base;
    const int n = rows_of(p, b, base);
    const unsigned first = blockIdx.x * (unsigned)(per * kItems);
    if (first / (2u * c.kv_heads) >= (unsigned)n) return;
    const int part = threadIdx.x & (tpr - 1);
    Item t[kItems];
    uint4 in[kItems][2];
    uint32_t exps[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        t[i] = item_of(p, b, n, base, first + i * per + threadIdx.x / tpr, part);
        const size_t entry = t[i].there ? t[i].entry : 0;
        const uint4* src = (const uint4*)((t[i].is_v ? c.v : c.k) + entry * c.row_bytes);
        in[i][0] = src[Q8 ? part : 2 * part];
        if (Q8)
            exps[i] = (t[i].is_v ? c.v_exp : c.k_exp)[entry];
        else
            in[i][1] = src[2 * part + 1];
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        if (!t[i].there) continue;
        uint4* dst = (uint4*)((t[i].is_v ? p.value : p.key) + 2 * t[i].at);
        if (Q8) {
            uint32_t f, more;
            e4m3_factors(exps[i], f, more);
            const uint4 y = in[i][0];
            const uint2 a = e4m3x4_to_bf16(y.x, f, more), d = e4m3x4_to_bf16(y.y, f, more);
            const uint2 g = e4m3x4_to_bf16(y.z, f, more), h = e4m3x4_to_bf16(y.w, f, more);
            dst[0] = make_uint4(a.x, a.y, d.x, d.y);
            dst[1] = make_uint4(g.x, g.y, h.x, h.y);
        } else {
            dst[0] = in[i][0];
            dst[1] = in[i][1];
        }
    }
}

struct CacheKeepParams {
    CacheView c;
    const int32_t* prefix_len;
    const int32_t* accept_len;
    const int32_t* accept_path;
    int32_t* next_prefix;
    int32_t* status;
    int L, layers;
    size_t layer_bytes, layer_rows;
};

constexpr int kKeepChunks = 4;  // 16-byte pieces a thread holds: 32 entries of 256 bytes over 128 threads
constexpr int kKeepThreads = 128;
constexpr int kKeepLayers = 4;  // a block's: where entries stand is found once, and the layers' loads are under way together
// (on the device, in a graph: 24 layers of 64 sequences, 101 MB, 20 us, 28 with a layer a block; 36 layers of one sequence 2.4 us; called one by
// one they take 26 and 9.7, the second the host's time)

// A block a (sequence, some layers, head, K or V): all entries of the path are in registers before the first is written, so that their
// order and overlaps do not matter.
__global__ void __launch_bounds__(kKeepThreads) cache_keep_kernel(const CacheKeepParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const CacheView& c = p.c;
    const int b = blockIdx.y;
    int x = blockIdx.x;
    const bool is_v = x & 1;
    x >>= 1;
    const int head = x % c.kv_heads, layer0 = x / c.kv_heads * kKeepLayers, layers = min(kKeepLayers, p.layers - layer0);
    const int a = p.accept_len[b], base = p.prefix_len[b] - 1;
    __shared__ int src_row[kMaxL], dst_row[kMaxL];
    __shared__ int fine;
    const int32_t* table = c.table + (size_t)b * c.width;
    if (threadIdx.x < 32) {
        const int k = threadIdx.x;
        bool ok = base >= 0 && a >= 0 && a <= p.L;
        if (ok && k < a) {
            const int node = p.accept_path[(size_t)b * p.L + k];
            const long long s = (long long)base + node, d = (long long)base + 1 + k, most = (long long)c.width << c.page_shift;
            ok = node >= 0 && s < most && d < most;
            if (ok) {
                const int ps = table[s >> c.page_shift], pd = table[d >> c.page_shift], low = (1 << c.page_shift) - 1;
                ok = (unsigned)ps < (unsigned)c.n_pages && (unsigned)pd < (unsigned)c.n_pages;
                if (ok) {
                    src_row[k] = (int)cache_row(c, ps, head, (int)(s & low));
                    dst_row[k] = (int)cache_row(c, pd, head, (int)(d & low));
                }
            }
        }
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (k == 0) {
            fine = ok;
            if (blockIdx.x == 0) {
                if (p.status) p.status[b] = ok ? 0 : GRAFT_ST_BAD_CACHE;
                if (p.next_prefix) p.next_prefix[b] = ok ? base + 1 + a + 1 : base + 1;
            }
        }
    }
    __syncthreads();
    if (!fine) return;
    uint8_t* rows = (is_v ? c.v : c.k) + (size_t)layer0 * p.layer_bytes;
    const int per = c.row_bytes >> 4, pieces = a * per;
    uint4 held[kKeepLayers][kKeepChunks];
#pragma unroll
    for (int i = 0; i < kKeepChunks; ++i) {
        const int q = threadIdx.x + i * kKeepThreads;
        if (q < pieces) {
            const uint8_t* from = rows + (size_t)src_row[q / per] * c.row_bytes + q % per * 16;
#pragma unroll
            for (int y = 0; y < kKeepLayers; ++y)
                if (y < layers) held[y][i] = *(const uint4*)(from + y * p.layer_bytes);
        }
    }
    uint8_t* exps = is_v ? c.v_exp : c.k_exp;
    uint8_t e[kKeepLayers] = {};
    if (exps) {
        exps += (size_t)layer0 * p.layer_rows;
#pragma unroll
        for (int y = 0; y < kKeepLayers; ++y)
            if (y < layers && threadIdx.x < a) e[y] = exps[y * p.layer_rows + src_row[threadIdx.x]];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kKeepChunks; ++i) {
        const int q = threadIdx.x + i * kKeepThreads;
        if (q < pieces) {
            uint8_t* to = rows + (size_t)dst_row[q / per] * c.row_bytes + q % per * 16;
#pragma unroll
            for (int y = 0; y < kKeepLayers; ++y)
                if (y < layers) *(uint4*)(to + y * p.layer_bytes) = held[y][i];
        }
    }
    if (exps && threadIdx.x < a)
#pragma unroll
        for (int y = 0; y < kKeepLayers; ++y)
            if (y < layers) exps[y * p.layer_rows + dst_row[threadIdx.x]] = e[y];
}

// For next lengths that take the place of the old ones, which every block of the moves reads: a launch of its own behind them.
struct NextPrefixParams {
    const int32_t* prefix_len;
    const int32_t* accept_len;
    const int32_t* accept_path;
    int32_t* next_prefix;
    CacheView c;
    int batch, L;
};
__global__ void __launch_bounds__(kThreads) next_prefix_kernel(const NextPrefixParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, k = lane_id();
    if (b >= p.batch) return;
    const int a = p.accept_len[b], base = p.prefix_len[b] - 1;
    bool ok = base >= 0 && a >= 0 && a <= p.L;
    if (ok && k < a) {
        const int node = p.accept_path[(size_t)b * p.L + k];
        const long long s = (long long)base + node, d = (long long)base + 1 + k, most = (long long)p.c.width << p.c.page_shift;
        ok = node >= 0 && s < most && d < most;
        if (ok) {
            const int32_t* table = p.c.table + (size_t)b * p.c.width;
            ok = (unsigned)table[s >> p.c.page_shift] < (unsigned)p.c.n_pages && (unsigned)table[d >> p.c.page_shift] < (unsigned)p.c.n_pages;
        }
    }
    ok = __all_sync(0xFFFFFFFFu, ok);
    if (k == 0) p.next_prefix[b] = ok ? base + 1 + a + 1 : base + 1;
}

}  // namespace

CacheView cache_view(const graft_cache* c, int layer) {
    CacheView v = {};
    const size_t rows = (size_t)c->n_pages * c->kv_heads * c->page_size;
    v.row_bytes = c->head_dim * (c->dtype == GRAFT_E4M3 ? 1 : 2);
    v.k = (uint8_t*)c->d_k + rows * v.row_bytes * layer;
    v.v = (uint8_t*)c->d_v + rows * v.row_bytes * layer;
    if (c->dtype == GRAFT_E4M3) {
        v.k_exp = c->d_k_exp + rows * layer;
        v.v_exp = c->d_v_exp + rows * layer;
    }
    v.table = c->d_table;
    v.width = c->table_width;
    v.n_pages = c->n_pages;
    v.kv_heads = c->kv_heads;
    v.head_dim = c->head_dim;
    while ((1 << v.page_shift) < c->page_size) v.page_shift += 1;
    return v;
}

cudaError_t cache_rows_launch(graft_ctx* ctx, bool write, int batch, const graft_cache* cache, int layer, const int32_t* d_prefix_len,
                              const int32_t* d_count, int rows, long long stride, const void* d_key, const void* d_value,
                              int32_t* d_status, cudaStream_t st) {
    CacheRowsParams p;
    p.c = cache_view(cache, layer);
    p.prefix_len = d_prefix_len;
    p.count = d_count;
    p.rows = rows;
    p.stride = stride;
    p.key = (const uint8_t*)d_key;
    p.value = (const uint8_t*)d_value;
    p.status = d_status;
    const int per = kItems * (kThreads / (cache->head_dim / 16));
    const long long items = (long long)rows * 2 * cache->kv_heads;
    const dim3 grid((unsigned)((items + per - 1) / per), batch);
    const bool q8 = cache->dtype == GRAFT_E4M3;
    const cudaError_t e = write ? launch_pdl(q8 ? cache_write_kernel<true> : cache_write_kernel<false>, grid, dim3(kThreads), 0, st, p)
                                : launch_pdl(q8 ? cache_read_kernel<true> : cache_read_kernel<false>, grid, dim3(kThreads), 0, st, p);
    ctx->launches += 1;
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t cache_keep_launch(graft_ctx* ctx, int batch, const graft_cache* cache, const int32_t* d_prefix_len,
                              const int32_t* d_accept_len, const int32_t* d_accept_path, int32_t* d_next_prefix, int32_t* d_status,
                              cudaStream_t st) {
    CacheKeepParams p;
    p.c = cache_view(cache, 0);
    p.prefix_len = d_prefix_len;
    p.accept_len = d_accept_len;
    p.accept_path = d_accept_path;
    p.next_prefix = d_next_prefix;
    p.status = d_status;
    p.L = ctx->cfg.L;
    p.layers = cache->layers;
    p.layer_rows = (size_t)cache->n_pages * cache->kv_heads * cache->page_size;
    p.layer_bytes = p.layer_rows * p.c.row_bytes;
    // the new lengths come with the moves, but for an array that overlaps the old ones, which every block reads
    const bool apart = (uintptr_t)d_next_prefix >= (uintptr_t)(d_prefix_len + batch) || (uintptr_t)(d_next_prefix + batch) <= (uintptr_t)d_prefix_len;
    if (!apart) p.next_prefix = nullptr;
    cudaError_t e = launch_pdl(cache_keep_kernel, dim3(2 * cache->kv_heads * ((cache->layers + kKeepLayers - 1) / kKeepLayers), batch), dim3(kKeepThreads), 0, st, p);
    ctx->launches += 1;
    if (e == cudaSuccess && d_next_prefix && !apart) {
        const NextPrefixParams np = {d_prefix_len, d_accept_len, d_accept_path, d_next_prefix, p.c, batch, ctx->cfg.L};
        e = launch_pdl(next_prefix_kernel, dim3((batch + kThreads / 32 - 1) / (kThreads / 32)), dim3(kThreads), 0, st, np);
        ctx->launches += 1;
    }
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace graft
