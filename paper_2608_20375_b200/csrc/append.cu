// New rows of a target layer on their way to attention (graft_cache_append): queries and keys are turned by their positions' angles, keys
// and values go into the paged cache.
//
// Pair i of a head, (x, y), becomes gain (x cos a - y sin a, x sin a + y cos a) with a = sum over axes of (position + shift) freq[axis, i].
// A position may be far out and a frequency is up to a turn a step, so angles, their cosines and sines are worked out in fp64, modulo a turn: a
// position of 2^24 costs no more precision than position 1.  (Turns in fp32 into sincospif: twice as many results rounded to the other side as
// with cosines and sines that are right to half a step of fp32; the fp64 pair costs 0.5 % of a prompt's time.)  A block works out the cosines and sines of its
// tokens' pairs once, into shared memory, for all of their heads.  Rotated numbers are fp32 and are rounded once: to bf16, or, into an e4m3
// cache, to e4m3 with the row's exponent taken from the fp32 numbers.
//
// What bounds it.  Every number is read and written once: 8 prompts of up to 8192 rows, 32 query heads on 8 of 128, 904 MB, 162 us: 5.6 TB/s, 0.85 of a plain copy's rate (into an e4m3 cache 829 MB, 159 us),
// with two rows a thread under way (one row a thread that was asked for behind the table and the angles: 209 us).  Clips of three axes 47 us (68 before).  64 trees'
// rows into an e4m3 cache 15.4 us (bytes: 9.0), one tree 3.4: blocks of four tokens, two and a half to a place on an SM, each behind its chain of count, table and angles.
#include <cuda_bf16.h>

#include "cache.cuh"

namespace graft {

namespace {

constexpr int kThreads = 256;
constexpr int kItems = 2;        // rows (token, head) that a thread loads ahead of those that it works on
constexpr int kMostTokens = 16;  // of a block
constexpr int kMostPairs = 64;

struct AppendParams {
    CacheView c;
    const int32_t* prefix_len;
    const int32_t* count;
    int rows, q_heads;
    const uint8_t* q;
    const uint8_t* key;
    const uint8_t* value;
    uint8_t* q_out;
    long long q_stride, kv_stride, out_stride;  // in numbers
    const float* freq;
    const int32_t* position;
    const int32_t* shift;
    int axes, pairs, interleaved, pos_rows, pos_axes;
    float gain;
    int tokens;  // a block's
    int32_t* status;
};

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint4 load16(const uint8_t* p) {
    uint4 r;
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}

// A thread has sixteen numbers of a row, two pieces of eight that hold both numbers of each of their pairs: pieces `part` of both halves of
// what is rotated, or side by side (neighbours paired, and what is not rotated).  Its rows are `per` apart among the block's tokens' heads (queries, keys,
// values); the first are asked for ahead of all that the block looks up.
template <bool Q8>
__global__ void __launch_bounds__(kThreads, 3) cache_append_kernel(const __grid_constant__ AppendParams p) {
    __shared__ int use;
    __shared__ float4 turn[kMostTokens][4][kMostPairs / 8];  // [token][j][part]: cosine and sine of pairs 8 part + 2 j and the next
    __shared__ int entry0[kMostTokens];                      // the token's row of the layer's cache, head 0
    pdl_launch_dependents();
    pdl_wait();
    const CacheView& c = p.c;
    const int b = blockIdx.y, tid = threadIdx.x, first = blockIdx.x * p.tokens;
    const int D = c.head_dim, tpr = D >> 4, part = tid & (tpr - 1), per = kThreads / tpr;
    const int heads = p.q_heads + 2 * c.kv_heads, rot_parts = p.pairs >> 3;
    const bool turned = part < rot_parts;
    const int at0 = p.interleaved || !turned ? 16 * part : 8 * part, at1 = p.interleaved || !turned ? at0 + 8 : at0 + p.pairs;
    const int step_tok = per / heads, step_hd = per - step_tok * heads;
    const auto next = [&](int& tok, int& hd) {
        tok += step_tok, hd += step_hd;
        if (hd >= heads) hd -= heads, tok += 1;
    };
    const long long row0 = (long long)b * p.rows + first;
    const auto bring = [&](uint4 (&in)[2], int tok, int h, int tokens) {
        if (tok >= tokens) return;
        const uint8_t* src = h < p.q_heads ? p.q + 2 * ((row0 + tok) * p.q_stride + (long long)h * D)
                             : h < p.q_heads + c.kv_heads ? p.key + 2 * ((row0 + tok) * p.kv_stride + (long long)(h - p.q_heads) * D)
                                                          : p.value + 2 * ((row0 + tok) * p.kv_stride + (long long)(h - p.q_heads - c.kv_heads) * D);
        in[0] = load16(src + 2 * at0), in[1] = load16(src + 2 * at1);
    };
    uint4 in[kItems][2];
    int tok = tid / tpr / heads, hd = tid / tpr - tok * heads;     // the next row to work on
    int tok_in = tok, hd_in = hd;                                  // the next one to ask for
#pragma unroll
    for (int y = 0; y < kItems; ++y) {  // (rows that are not in use are there all the same)
        bring(in[y], tok_in, hd_in, min(p.tokens, p.rows - first));
        next(tok_in, hd_in);
    }
    const int n0 = p.count[b], base = p.prefix_len[b] - 1;
    const int32_t* table = c.table + (size_t)b * c.width;
    if (tid < 32) {
        const bool ok = n0 >= 0 && n0 <= p.rows && base >= 0 && cache_slots_ok(c, table, base, (long long)base + n0);
        if (tid == 0) {
            use = ok ? n0 : 0;
            if (p.status && blockIdx.x == 0) p.status[b] = ok ? 0 : GRAFT_ST_BAD_CACHE;
        }
    }
    __syncthreads();
    const int tokens = min(p.tokens, use - first);
    if (tokens <= 0) return;
    const long long shift = p.shift ? p.shift[b] : 0;
    for (int x = tid; x < tokens * p.pairs; x += kThreads) {
        const int t = x / p.pairs, i = x - t * p.pairs;
        const int32_t* pos = p.position ? p.position + ((long long)b * p.pos_rows + first + t) * p.pos_axes : nullptr;
        double angle = 0.0;
        for (int a = 0; a < p.axes; ++a) {
            const long long at = (pos ? (long long)pos[p.pos_axes == 1 ? 0 : a] : (long long)base + first + t) + shift;
            angle += (double)at * (double)p.freq[a * p.pairs + i];
        }
        const double turns = angle * 0.15915494309189535;  // 1 / (2 pi)
        double s, co;
        sincospi(2.0 * (turns - rint(turns)), &s, &co);
        ((float2*)&turn[t][(i >> 1) & 3][i >> 3])[i & 1] = make_float2((float)co * p.gain, (float)s * p.gain);
    }
    if (tid < tokens) {
        const int slot = base + first + tid;
        entry0[tid] = (int)cache_row(c, table[slot >> c.page_shift], 0, slot & ((1 << c.page_shift) - 1));
    }
    __syncthreads();
    // (a row's threads are neighbours in a warp and go through the loop together)
    while (__any_sync(0xFFFFFFFFu, tok < tokens)) {
#pragma unroll
        for (int y = 0; y < kItems; ++y) {
            const int h = hd;
            const bool there = tok < tokens, is_q = h < p.q_heads, is_v = h >= p.q_heads + c.kv_heads;
            float x[16];
            const uint32_t w[8] = {in[y][0].x, in[y][0].y, in[y][0].z, in[y][0].w, in[y][1].x, in[y][1].y, in[y][1].z, in[y][1].w};
#pragma unroll
            for (int j = 0; j < 8; ++j) x[2 * j] = __uint_as_float(w[j] << 16), x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            bring(in[y], tok_in, hd_in, tokens);
            next(tok_in, hd_in);
            if (there && turned && !is_v) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 cs = turn[tok][j][part];
                    if (p.interleaved) {
                        const float u0 = x[4 * j], v0 = x[4 * j + 1], u1 = x[4 * j + 2], v1 = x[4 * j + 3];
                        x[4 * j] = u0 * cs.x - v0 * cs.y, x[4 * j + 1] = u0 * cs.y + v0 * cs.x;
                        x[4 * j + 2] = u1 * cs.z - v1 * cs.w, x[4 * j + 3] = u1 * cs.w + v1 * cs.z;
                    } else {
                        const float u0 = x[2 * j], v0 = x[2 * j + 8], u1 = x[2 * j + 1], v1 = x[2 * j + 9];
                        x[2 * j] = u0 * cs.x - v0 * cs.y, x[2 * j + 8] = u0 * cs.y + v0 * cs.x;
                        x[2 * j + 1] = u1 * cs.z - v1 * cs.w, x[2 * j + 9] = u1 * cs.w + v1 * cs.z;
                    }
                }
            }
            uint8_t* dst = nullptr;
            size_t entry = 0;
            if (there) {
                if (is_q)
                    dst = p.q_out + 2 * ((row0 + tok) * p.out_stride + (long long)h * D);
                else {
                    entry = (size_t)entry0[tok] + ((size_t)(h - p.q_heads - (is_v ? c.kv_heads : 0)) << c.page_shift);
                    dst = (is_v ? c.v : c.k) + entry * c.row_bytes;
                }
            }
            if (Q8 && __any_sync(0xFFFFFFFFu, there && !is_q)) {
                uint32_t amax = 0;  // magnitudes are ordered like their bits, NaN above infinity
#pragma unroll
                for (int j = 0; j < 16; ++j) amax = max(amax, __float_as_uint(x[j]) & 0x7FFFFFFFu);
                for (int o = tpr >> 1; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
                if (there && !is_q) {
                    const bool bad = amax >= 0x7F800000u;
                    // amax = f 2^z with f in [1, 2): amax <= 448 2^e = 1.75 2^(e + 8) iff e >= z - 8, or z - 7 where f > 1.75
                    int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u);
                    e = e < -120 ? -120 : e;
                    const float up = bad ? 0.0f : __int_as_float((uint32_t)(127 - e) << 23);  // 2^-e: exact but for what is far below e4m3's smallest
                    uint32_t z[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t four = 0;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float2 v = make_float2(x[4 * j + 2 * k] * up, x[4 * j + 2 * k + 1] * up);
                            four |= (uint32_t)__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3) << (16 * k);
                        }
                        z[j] = bad ? 0u : four;
                    }
                    *(uint2*)(dst + at0) = make_uint2(z[0], z[1]);
                    *(uint2*)(dst + at1) = make_uint2(z[2], z[3]);
                    if (part == 0) (is_v ? c.v_exp : c.k_exp)[entry] = bad ? 255 : (uint8_t)(e + 127);
                }
            }
            if (there && (!Q8 || is_q)) {
                *(uint4*)(dst + 2 * at0) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
                *(uint4*)(dst + 2 * at1) = make_uint4(pack2(x[8], x[9]), pack2(x[10], x[11]), pack2(x[12], x[13]), pack2(x[14], x[15]));
            }
            next(tok, hd);
        }
    }
}

}  // namespace

cudaError_t cache_append_launch(graft_ctx* ctx, int batch, const graft_cache* cache, int layer, const graft_rope* rope, int q_heads,
                                const int32_t* d_prefix_len, const int32_t* d_count, int rows, long long q_stride, const void* d_q,
                                long long kv_stride, const void* d_key, const void* d_value, long long out_stride, void* d_q_out,
                                int32_t* d_status, cudaStream_t st) {
    AppendParams p;
    p.c = cache_view(cache, layer);
    p.prefix_len = d_prefix_len;
    p.count = d_count;
    p.rows = rows;
    p.q_heads = q_heads;
    p.q = (const uint8_t*)d_q;
    p.key = (const uint8_t*)d_key;
    p.value = (const uint8_t*)d_value;
    p.q_out = (uint8_t*)d_q_out;
    p.q_stride = q_stride;
    p.kv_stride = kv_stride;
    p.out_stride = out_stride;
    p.freq = rope->d_freq;
    p.position = rope->d_position;
    p.shift = rope->d_shift;
    p.axes = rope->axes;
    p.pairs = rope->rot_dim / 2;
    p.interleaved = rope->interleaved;
    p.pos_rows = rope->pos_rows;
    p.pos_axes = rope->pos_axes;
    p.gain = rope->gain;
    p.status = d_status;
    // tokens a block: as many as share the work of a block's beginning, as long as there are two rounds of blocks an SM
    const long long share = (long long)batch * rows / (6 * ctx->num_sms);
    p.tokens = share < 1 ? 1 : share > kMostTokens ? kMostTokens : (int)share;
    const dim3 grid((unsigned)((rows + p.tokens - 1) / p.tokens), batch);
    const cudaError_t e = launch_pdl(cache->dtype == GRAFT_E4M3 ? cache_append_kernel<true> : cache_append_kernel<false>, grid, dim3(kThreads), 0, st, p);
    ctx->launches += 1;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace graft
