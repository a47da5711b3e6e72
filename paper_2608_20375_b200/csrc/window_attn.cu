// Attention over a paged cache of rows that see the last `window` positions and the first `sinks` (graft_window_attention).
#include "cache.cuh"

namespace graft {

namespace {

constexpr int kThreads = 128;

struct WindowParams {
    CacheView c;
    const uint8_t* q;
    long long q_stride;
    const int32_t* prefix_len;
    const int32_t* count;
    const uint32_t* mask;
    const int32_t* position;
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
    float scale;
    int rows, q_heads, group, nmax, words, window, sinks;
};

__device__ __forceinline__ float entry_of(const CacheView& c, const uint8_t* x, const uint8_t* exps, size_t row, int d) {
    if (!exps) return __uint_as_float((uint32_t)((const uint16_t*)x)[row * c.head_dim + d] << 16);
    uint32_t f, more;
    e4m3_factors(exps[row], f, more);
    return __uint_as_float(e4m3x4_to_bf16(x[row * c.head_dim + d], f, more).x << 16);
}

// A block a row and head, four warps that take 32 slots in turn: a lane a slot for the scores, some numbers of the head for the sums.
template <int D>
__global__ void __launch_bounds__(kThreads) window_attn_kernel(const __grid_constant__ WindowParams p) {
    constexpr int kWarps = kThreads / 32, kPer = D / 32;
    __shared__ float q[D], sum[kWarps][D], sm[kWarps], sl[kWarps];
    __shared__ int fine;
    pdl_launch_dependents();
    pdl_wait();
    const CacheView& c = p.c;
    const int i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = p.count[b], base = p.prefix_len[b] - 1, end = base + n, lo = max(0, base - p.window + 1), low = (1 << c.page_shift) - 1;
    const int32_t* table = c.table + (size_t)b * c.width;
    if (warp == 0) {
        bool ok = n >= 0 && n <= p.rows && base >= 0 && (long long)base + n <= (long long)c.width << c.page_shift;
        if (ok && n > 0) {
            ok = cache_slots_ok(c, table, 0, min(p.sinks, end)) && cache_slots_ok(c, table, lo, end);
        }
        if (lane == 0) {
            fine = ok;
            if (p.status && i == 0 && h == 0) p.status[b] = ok ? 0 : GRAFT_ST_BAD_CACHE;
        }
    }
    __syncthreads();
    if (!fine || i >= n) return;
    const int kh = h / p.group;
    for (int d = tid; d < D; d += kThreads)
        q[d] = p.scale * __bfloat162float(((const __nv_bfloat16*)p.q)[((long long)b * p.rows + i) * p.q_stride + (long long)h * D + d]);
    __syncthreads();
    const int32_t* pos = p.mask ? p.position + (size_t)b * p.nmax : nullptr;
    const uint32_t* bits = p.mask ? p.mask + ((size_t)b * p.nmax + i) * p.words : nullptr;
    const auto position_of = [&](int j) { return pos ? min(max(pos[j], base), base + j) : base + j; };
    const int mine = position_of(i);
    const auto sees = [&](int s) {
        const int j = s - base;
        if (j >= 0 && !(bits ? j < 32 * p.words && (bits[j >> 5] >> (j & 31) & 1) : j <= i)) return false;
        const int at = j < 0 ? s : position_of(j);
        return mine - at < p.window || at < p.sinks;
    };
    float m = -INFINITY, l = 0.0f, o[kPer] = {};
    const int first = min(p.sinks, lo), total = first + end - lo;
    for (int x0 = warp * 32; x0 < total; x0 += kThreads) {
        const int x = x0 + lane, s = x < first ? x : lo + x - first;
        const bool see = x < total && sees(s);
        float sc = -INFINITY;
        if (see) {
            const size_t row = cache_row(c, table[s >> c.page_shift], kh, s & low);
            sc = 0.0f;
            for (int d = 0; d < D; ++d) sc = fmaf(q[d], entry_of(c, c.k, c.k_exp, row, d), sc);
            if (!(sc < INFINITY)) sc = __int_as_float(0x7FFFFFFF);
        }
        const bool nan = __any_sync(0xFFFFFFFFu, sc != sc);
        float mx = sc;
        for (int y = 16; y > 0; y >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, y));
        const float now = fmaxf(m, mx), f = m > -INFINITY ? expf(m - now) : 0.0f;
        const float w = sc > -INFINITY ? expf(sc - now) : 0.0f;
        float ws = w;
        for (int y = 16; y > 0; y >>= 1) ws += __shfl_xor_sync(0xFFFFFFFFu, ws, y);
        l = nan ? __int_as_float(0x7FFFFFFF) : l * f + ws;
        m = now;
        for (int y = 0; y < kPer; ++y) o[y] *= f;
        const unsigned who = __ballot_sync(0xFFFFFFFFu, see);
        for (int y = 0; y < 32; ++y) {
            if (!(who >> y & 1)) continue;
            const float wy = __shfl_sync(0xFFFFFFFFu, w, y);
            const int sy = __shfl_sync(0xFFFFFFFFu, s, y);
            const size_t row = cache_row(c, table[sy >> c.page_shift], kh, sy & low);
            for (int z = 0; z < kPer; ++z) o[z] += wy * entry_of(c, c.v, c.v_exp, row, z * 32 + lane);
        }
    }
    if (lane == 0) sm[warp] = m, sl[warp] = l;
    for (int z = 0; z < kPer; ++z) sum[warp][z * 32 + lane] = o[z];
    __syncthreads();
    float mm = -INFINITY, ll = 0.0f;
    for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, sm[w]);
    const auto weight = [&](int w) { return sm[w] > -INFINITY ? expf(sm[w] - mm) : 0.0f; };
    for (int w = 0; w < kWarps; ++w) ll += sl[w] != sl[w] ? sl[w] : weight(w) * sl[w];
    const size_t row = ((size_t)b * p.rows + i) * p.q_heads + h;
    for (int d = tid; d < D; d += kThreads) {
        float x = 0.0f;
        for (int w = 0; w < kWarps; ++w) x += weight(w) * sum[w][d];
        p.out[row * D + d] = __float2bfloat16(ll != 0.0f ? x / ll : x);
    }
    if (p.lse && tid == 0) p.lse[row] = ll == 0.0f ? -INFINITY : (mm > -INFINITY ? mm : 0.0f) + logf(ll);
}

}  // namespace

cudaError_t window_attn_launch(graft_ctx* ctx, int batch, const graft_cache* cache, int layer, int q_heads, int rows, long long q_stride,
                               const void* d_q, float scale, const int32_t* d_prefix_len, const int32_t* d_count, const uint32_t* d_mask,
                               const int32_t* d_position, int window, int sinks, void* d_out, float* d_lse, int32_t* d_status, cudaStream_t st) {
    WindowParams p;
    p.c = cache_view(cache, layer);
    p.q = (const uint8_t*)d_q;
    p.q_stride = q_stride;
    p.prefix_len = d_prefix_len;
    p.count = d_count;
    p.mask = d_mask;
    p.position = d_position;
    p.out = (__nv_bfloat16*)d_out;
    p.lse = d_lse;
    p.status = d_status;
    p.scale = scale;
    p.rows = rows;
    p.q_heads = q_heads;
    p.group = q_heads / cache->kv_heads;
    p.nmax = ctx->nmax;
    p.words = ctx->mask_words;
    p.window = window;
    p.sinks = sinks;
    const cudaError_t e = launch_pdl(cache->head_dim == 128 ? window_attn_kernel<128> : window_attn_kernel<64>, dim3(rows, q_heads, batch),
                                     dim3(kThreads), 0, st, p);
    ctx->launches += 1;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace graft
