// What the kernels that read and write a paged key/value cache share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "common.cuh"
#include "internal.h"

namespace graft {

// A graft_cache as the kernels see it: one layer of it (cache_keep: all), addresses in entries.
struct CacheView {
    uint8_t* k;
    uint8_t* v;
    uint8_t* k_exp;  // NULL: bf16
    uint8_t* v_exp;
    const int32_t* table;  // [batch, width]
    int width, n_pages, kv_heads, page_shift, head_dim;
    int row_bytes;  // of an entry (one token, one head)
};

CacheView cache_view(const graft_cache* c, int layer);  // csrc/cache.cu

// row (token, head) of a layer that slot `at` of a page holds
__device__ __forceinline__ size_t cache_row(const CacheView& c, int page, int head, int at) {
    return ((((size_t)page * c.kv_heads + head) << c.page_shift) + at);
}

// Whether slots [first, end) of the sequence lie within its table and in pages of the cache; a whole warp calls it.
__device__ __forceinline__ bool cache_slots_ok(const CacheView& c, const int32_t* table, long long first, long long end) {
    if (first < 0 || end > ((long long)c.width << c.page_shift)) return false;
    bool ok = true;
    if (end > first)
        for (int p = (int)(first >> c.page_shift) + lane_id(); p <= (int)((end - 1) >> c.page_shift); p += 32)
            ok = ok && (unsigned)table[p] < (unsigned)c.n_pages;
    return __all_sync(0xFFFFFFFFu, ok);
}

// Bytes ia and ib (0 .. 3 of a, 4 .. 7 of b), e4m3 numbers -> bf16 times 2^-120; exact.  A byte with its sign eight times above it, moved up
// four places, has sign, exponent and mantissa where bf16 has them, and signs in the exponent's upper bits, which go.  (prmt replicates signs,
// __byte_perm does not.)
__device__ __forceinline__ uint32_t e4m3_pair_small(uint32_t a, uint32_t b, int ia, int ib) {
    uint32_t x;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(x) : "r"(a), "r"(b), "r"(ia | (ia | 8) << 4 | ib << 8 | (ib | 8) << 12));
    return (x << 4) & 0x87F087F0u;
}
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Factors that take what e4m3_pair_small gives to the numbers that it stands for, as pairs of bf16: 2^(e + 120) with
// e = byte - 127.  Up to 2^127 one factor holds it and the second is 1; byte 255 is NaN.
__device__ __forceinline__ void e4m3_factors(uint32_t byte, uint32_t& f, uint32_t& more) {
    int x = (int)byte - 7;  // e + 120
    const int y = x > 127 ? x - 127 : 0;
    x = x > 127 ? 127 : (x < -126 ? -126 : x);
    const uint32_t a = byte == 255 ? 0x7FC0u : (uint32_t)(x + 127) << 7;
    f = a | (a << 16);
    const uint32_t b = (uint32_t)(y + 127) << 7;
    more = b | (b << 16);
}
// four e4m3 numbers -> two pairs of bf16
__device__ __forceinline__ uint2 e4m3x4_to_bf16(uint32_t w, uint32_t f, uint32_t more) {
    uint2 r;
    r.x = bf16x2_mul(e4m3_pair_small(w, 0, 0, 1), f);
    r.y = bf16x2_mul(e4m3_pair_small(w, 0, 2, 3), f);
    if (more != 0x3F803F80u) {
        r.x = bf16x2_mul(r.x, more);
        r.y = bf16x2_mul(r.y, more);
    }
    return r;
}

constexpr uint32_t kOneBf16x2 = 0x3F803F80u;

}  // namespace graft
