// Attention of the trees' nodes over a paged cache (graft_tree_attention).
#include <float.h>

#include "cache.cuh"

namespace graft {

namespace {

struct AttnParams {
    CacheView c;
    const uint8_t* q;
    long long q_stride;
    const int32_t* prefix_len;
    const int32_t* count;
    const uint32_t* mask;
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
    float scale;
    int rows, q_heads, shared, nmax, words;
};

// A warp a (row, query head): 32 slots at a time, a lane a slot for the scores, a lane head_dim / 32 numbers for the sums.
template <int D, bool Q8>
__global__ void __launch_bounds__(128) tree_attn_kernel(const AttnParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const CacheView& c = p.c;
    __shared__ float qs[4][D];
    const int lane = lane_id(), w = threadIdx.x >> 5, b = blockIdx.y;
    const long long item = (long long)blockIdx.x * 4 + w;
    const int row = (int)(item / p.q_heads), h = (int)(item % p.q_heads), hk = h / (p.q_heads / c.kv_heads);
    const int n = p.count[b], base = p.prefix_len[b] - 1;
    const int32_t* table = c.table + (size_t)b * c.width;
    const bool ok = n >= 0 && n <= p.rows && base >= 0 && base >= p.shared && cache_slots_ok(c, table, 0, (long long)base + n);
    if (item == 0 && lane == 0 && p.status) p.status[b] = ok ? 0 : GRAFT_ST_BAD_CACHE;
    if (!ok || row >= n) return;
    const uint16_t* q = (const uint16_t*)p.q + ((long long)b * p.rows + row) * p.q_stride + h * D;
    for (int i = lane; i < D; i += 32) qs[w][i] = __uint_as_float((uint32_t)q[i] << 16) * p.scale;
    __syncwarp();
    float m = -INFINITY, l = 0.0f, o[D / 32] = {};
    for (int s0 = 0; s0 < base + n; s0 += 32) {
        const int s = s0 + lane, j = s - base;
        bool seen = s < base + n;
        if (seen && j >= 0) seen = p.mask ? (p.mask[((size_t)b * p.nmax + row) * p.words + (j >> 5)] >> (j & 31)) & 1 : j <= row;
        float x = -INFINITY;
        if (seen) {
            const size_t at = cache_row(c, table[s >> c.page_shift], hk, s & ((1 << c.page_shift) - 1));
            const uint8_t* k = c.k + at * c.row_bytes;
            uint32_t f = 0, more = 0;
            if (Q8) e4m3_factors(c.k_exp[at], f, more);
            x = 0.0f;
            for (int i = 0; i < D; i += 4) {
                uint2 y;
                if (Q8)
                    y = e4m3x4_to_bf16(*(const uint32_t*)(k + i), f, more);
                else
                    y = *(const uint2*)(k + 2 * i);
                x += qs[w][i] * __uint_as_float(y.x << 16) + qs[w][i + 1] * __uint_as_float(y.x & 0xFFFF0000u) +
                     qs[w][i + 2] * __uint_as_float(y.y << 16) + qs[w][i + 3] * __uint_as_float(y.y & 0xFFFF0000u);
            }
        }
        float mm = x;
        for (int d = 16; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xFFFFFFFFu, mm, d));
        mm = fmaxf(mm, m);
        const float keep = m > -INFINITY ? expf(m - mm) : 0.0f, e = seen && mm > -INFINITY ? expf(x - mm) : 0.0f;
        float sum = e;
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        l = l * keep + sum;
        m = mm;
        for (int i = 0; i < D / 32; ++i) o[i] *= keep;
        for (int t = 0; t < 32 && s0 + t < base + n; ++t) {
            const float pe = __shfl_sync(0xFFFFFFFFu, e, t);
            if (pe == 0.0f) continue;
            const size_t at = cache_row(c, table[(s0 + t) >> c.page_shift], hk, (s0 + t) & ((1 << c.page_shift) - 1));
            const uint8_t* v = c.v + at * c.row_bytes;
            for (int i = 0; i < D / 32; ++i) {
                const int d = lane + 32 * i;
                float y;
                if (Q8) {
                    uint32_t f, more;
                    e4m3_factors(c.v_exp[at], f, more);
                    y = __uint_as_float(e4m3x4_to_bf16(v[d], f, more).x << 16);
                } else
                    y = __uint_as_float((uint32_t)((const uint16_t*)v)[d] << 16);
                o[i] += pe * y;
            }
        }
    }
    const size_t oat = ((size_t)b * p.rows + row) * p.q_heads + h;
    for (int i = 0; i < D / 32; ++i) p.out[oat * D + lane + 32 * i] = __float2bfloat16(l > 0.0f ? o[i] / l : o[i]);
    if (p.lse && lane == 0) p.lse[oat] = m > -INFINITY ? m + logf(l) : -INFINITY;
}

}  // namespace

cudaError_t tree_attn_launch(graft_ctx* ctx, int batch, const graft_cache* cache, int layer, int q_heads, int rows, long long q_stride,
                             const void* d_q, float scale, const int32_t* d_prefix_len, const int32_t* d_count, const uint32_t* d_mask,
                             int shared, void* d_out, float* d_lse, int32_t* d_status, cudaStream_t st) {
    AttnParams p;
    p.c = cache_view(cache, layer);
    p.q = (const uint8_t*)d_q;
    p.q_stride = q_stride;
    p.prefix_len = d_prefix_len;
    p.count = d_count;
    p.mask = d_mask;
    p.out = (__nv_bfloat16*)d_out;
    p.lse = d_lse;
    p.status = d_status;
    p.scale = scale;
    p.rows = rows;
    p.q_heads = q_heads;
    p.shared = shared;
    p.nmax = ctx->nmax;
    p.words = ctx->mask_words;
    const dim3 grid((unsigned)(((long long)rows * q_heads + 3) / 4), batch);
    const bool q8 = cache->dtype == GRAFT_E4M3;
    const auto kernel = cache->head_dim == 128 ? (q8 ? tree_attn_kernel<128, true> : tree_attn_kernel<128, false>)
                                               : (q8 ? tree_attn_kernel<64, true> : tree_attn_kernel<64, false>);
    const cudaError_t e = launch_pdl(kernel, grid, dim3(128), 0, st, p);
    ctx->launches += 1;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace graft
