// Attention of the trees' nodes over a paged cache (graft_tree_attention), on the tcgen05 tensor cores.  (What other attention shares with it: attn.cuh.)
//
// For a node i and a query head h:  o = sum_j p_j v_j,  p = softmax(scale q . k_j)  over the slots j that i sees.  All query heads of a
// key head and all nodes of a sequence are rows of one matrix product against the same keys, so the prefix is gone through once for a
// whole tree; with a shared prefix, once for the nodes of all sequences.
//
// Units and pieces.  A unit is a sequence (or, for the shared prefix, all of them), a key head and up to 256 rows (two row tiles
// of 128), against all key tiles of 128 slots.  The units' key tiles stand in one line, weighted by what they cost, and every
// CTA takes an equal stretch of it: lengths and trees may be as unlike as they want, and one sequence's prefix spreads over all SMs.  A
// unit that is cut leaves unnormalised sums with their maximum and denominator behind, which a second kernel joins.
//
// Inside a CTA two groups of four warps (`streams`) hold a row tile each and take turns on the tensor cores: while one stream's
// exponentials are worked out, the other's products run.  A unit of one row tile gives the streams the even and the odd key tiles
// instead, joined at the end.  Scores and sums stay in TMEM: S of 128 columns a stream, overwritten in place by the weights p in bf16
// (which are the second product's first operand from there), and O of head_dim columns.  One thread has one row, so maxima and sums need no
// exchange.  O is rescaled only when a row's maximum has grown by more than 2^8 since it was last taken: weights are then up to 256,
// which fp32 sums and bf16 hold as well as those up to 1.
//
// Sequences of up to eight rows a key head (single tokens) have a kernel of their own, on the same plan: see "few rows".
//
// What bounds it.  Large trees (16 of up to 513 nodes behind 6000 to 8192 slots, bf16, 717 GFLOP): 805 to 850 us, the tensor cores busy for 52 % of
// the time, the exponentials' unit for 39 %: a stream's next product waits for all of a tile's weights, and two streams (TMEM holds
// no more) do not fill the gaps; the clock falls to 1.3 GHz under that load in a long run (960 to 1040 us).  A tile of e4m3 slots is converted
// once a unit, 0.5 to 0.6 us: 32 trees of up to 65 nodes behind 500 to 4096 slots 127 us.  17 nodes (68 rows)
// behind 4000 slots, bf16: 213 us, 0.78 of the copy's rate.  Small calls are latencies: one tree of 65 nodes behind 1500 slots 29.5 us, of
// which the plan takes 4, the kernel 10 to 15 and the join 8.
//
// Code counts.  Four roles of warps run in four places of this kernel, and what they go through in a tile has to stay in the SM's instruction cache: with
// every wait unrolled and a copy of the softmax for each half of e4m3 scores it was 185 KB, and the e4m3 case above 177 us (now 111 KB); so
// waits, rescaling and walks along lists are rolled loops and rare paths are functions.
#include "attn.cuh"

namespace graft {

namespace {

// ---- the attention kernel ------------------------------------------------------------------------------------------
constexpr int kPieces = 4;  // that are told ahead
// Pieces that the flags of rows of V that were taken out are held for.  A warp of the first stream may set the next piece's flag while others
// have yet to test this one's (it clears V ahead of its first scores); none is two pieces ahead, as a piece's first scores wait for all eight
// warps' arrivals on q_full, which follow their test.
constexpr int kSpoiltPieces = 2;

// Tiles of V in a row that the first stream may have cleared before the second one asks whether: as many as the ring holds, and they come
// by turns, so that a barrier's phase tells uses apart.
constexpr int kCleared = 8;

// kOne: no unit has more than one row tile, and there is room for more key tiles.
template <int D, bool Q8, bool kOne>
struct Shape {
    static constexpr int kHalf = kTile * 128;                 // 128 rows of 128 bytes: 64 numbers of a row, in the 128-byte swizzle
    static constexpr int kTileBytes = kTile * D * 2;          // a tile of Q, K or V in bf16
    static constexpr int kRawBytes = kTile * D + kTile;       // a tile of e4m3 numbers and its rows' exponents
    static constexpr int kQTiles = kOne ? 1 : 2;
    // Tiles in bf16 (and e4m3 tiles on their way).  Two streams on key tiles of their own have four in use.
    static constexpr int kStages = (Q8 ? kOne ? 5 : 4 : kOne ? 6 : 5) * (128 / D);
    static constexpr int kRaw = Q8 ? 2 * (128 / D) : 0;
    static constexpr int kConvWarps = Q8 ? 8 : 0;
    static constexpr int kThreads = 384 + 32 * kConvWarps;
    // registers a thread: the softmax's eight warps take over what the others leave (of what the launch has)
    static constexpr int kRegsLaunch = Q8 ? 96 : 168;
    static constexpr int kRegsSoftmax = Q8 ? 168 : 224, kRegsOthers = Q8 ? 48 : 56;
    static constexpr int kCols = Q8 ? 64 : 128;  // scores that a softmax thread holds at a time
    static_assert(256 * kRegsSoftmax + (kThreads - 256) * kRegsOthers <= kThreads * kRegsLaunch, "registers of a launch");
    static constexpr size_t kSmem = 1024 + kQTiles * kTileBytes + (size_t)kStages * kTileBytes + (size_t)kRaw * kRawBytes + 1024;
};

// One thread of the warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// D (+)= A B with both operands in shared memory, a CTA by itself; one thread issues it.  Descriptors as their low words; the high one is the
// same for all.
template <bool kAccumulate>
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\tsetp.ne.u32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}" ::"r"(d_tmem),
        "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "n"(kAccumulate ? 1 : 0)
        : "memory");
}
// The same with A in TMEM.
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t hi, uint32_t b_lo, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tmov.b64 b, {%3, %2};\n\tsetp.ne.u32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "r"(hi), "r"(b_lo), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
}
// When every matrix instruction that this thread issued so far has completed: one arrival on the barrier.
__device__ __forceinline__ void umma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// a number that is the same in all lanes, known to be
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
// 32 columns of the lane's row
__device__ __forceinline__ void tmem_ld_32x32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
        "%26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
// the same registers, known to have arrived: nothing that reads them is moved ahead of the wait
template <int N>
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[N]) {
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
// two fp32 numbers in a 64-bit register
__device__ __forceinline__ uint64_t two(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 apart(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm volatile("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm volatile("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// the largest; NaN if one of them is
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max2(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// kCols of the row's scores at tS, from x0 on, all asked for together (while the tensor cores work on the other stream, an answer takes
// several hundred cycles), -inf in the place of those that `sees` leaves out, and their largest (NaN if one of them is).
template <int kCols, int kWords>
__device__ __forceinline__ float scores(uint32_t tS, int x0, uint32_t (&u)[kCols], bool masked, const uint32_t (&sees)[kWords]) {
#pragma unroll
    for (int x = 0; x < kCols; x += 32) tmem_ld_32x32(tS + x0 + x, *(uint32_t(*)[32]) & u[x]);
    tmem_arrived(u);
    if (masked)
#pragma unroll
        for (int w = 0; w < kCols / 32; ++w)
            if (__any_sync(0xFFFFFFFFu, sees[x0 / 32 + w] != 0xFFFFFFFFu))  // (borders cross few of a tile's columns)
#pragma unroll
                for (int x = 0; x < 32; ++x) u[32 * w + x] = (sees[x0 / 32 + w] >> x) & 1 ? u[32 * w + x] : 0xFF800000u;
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int x = 0; x < kCols; x += 2) mx[x / 2 % 4] = max3(mx[x / 2 % 4], __uint_as_float(u[x]), __uint_as_float(u[x + 1]));
    return max2(max3(mx[0], mx[1], mx[2]), mx[3]);
}
// 2^t of two numbers on the FMA pipe: t = n + f, n whole and |f| <= 1/2; 2^f by a polynomial of degree 5 (fitted for the least largest
// relative error, 1e-7, with 1 at f = 0), n added to its exponent.  t is held to -127 .. 127: at -127, where slots that are not seen
// come out, the exponent's field is 0 and the result is 0.  (So it is for NaN, which the kernel knows of from the tile's maximum.)
__device__ __forceinline__ float2 exp2_poly(uint64_t t) {
    float2 x = apart(t);
    t = two(fminf(fmaxf(x.x, -127.0f), 127.0f), fminf(fmaxf(x.y, -127.0f), 127.0f));
    const auto both = [](float c) { return two(c, c); };
    const uint64_t r = add2(t, both(12582912.0f));  // 1.5 2^23: the sum's last bits are n
    const uint64_t f = fma2(add2(r, both(-12582912.0f)), both(-1.0f), t);
    uint64_t q = fma2(both(0.0013264727f), f, both(0.0096715127f));
    q = fma2(q, f, both(0.055507337f));
    q = fma2(q, f, both(0.24022242f));
    q = fma2(q, f, both(0.69314698f));
    q = fma2(q, f, both(1.0f));
    const float2 a = apart(q), n = apart(r);
    return make_float2(__int_as_float(__float_as_int(a.x) + (__float_as_int(n.x) << 23)),
                       __int_as_float(__float_as_int(a.y) + (__float_as_int(n.y) << 23)));
}
// Weights 2^(c2 s + off) of 64 scores as pairs of bf16, and their sum (unrounded).  128 rows' exponentials take the 16-a-clock unit as long
// as both products take the tensor cores, so one pair of four is worked out on the FMA pipe; sums and conversions follow eight pairs
// behind.  Cycles for 128 x 128 scores, one and two warps a scheduler: 1150 and 1910 for two; without polynomials 1350 and 2350, with one in
// three 1180 and 1960.
__device__ __forceinline__ float weigh(uint32_t* v, float c2, float off, uint32_t (&w)[32]) {
    constexpr int kBehind = 8, kPairs = 32;
    uint64_t part[2] = {0, 0};
    const uint64_t cc = two(c2, c2), oo = two(off, off);
#pragma unroll
    for (int y = 0; y < kPairs + kBehind; ++y) {
        if (y < kPairs) {
            const uint64_t t = fma2(two(__uint_as_float(v[2 * y]), __uint_as_float(v[2 * y + 1])), cc, oo);
            const float2 e = y % 4 == 3 ? exp2_poly(t) : make_float2(ex2_in_order(apart(t).x), ex2_in_order(apart(t).y));
            v[2 * y] = __float_as_uint(e.x), v[2 * y + 1] = __float_as_uint(e.y);
        }
        if (y >= kBehind) {
            const int z = y - kBehind;
            const float e0 = __uint_as_float(v[2 * z]), e1 = __uint_as_float(v[2 * z + 1]);
            part[z & 1] = add2(part[z & 1], two(e0, e1));
            w[z] = pack_bf16(e0, e1);
        }
    }
    const float2 a = apart(add2(part[0], part[1]));
    return a.x + a.y;
}
// O of the row times f
template <int D>
__device__ __forceinline__ void rescale(uint32_t tO, float f) {
    uint32_t u[32];
#pragma unroll 1
    for (int x = 0; x < D / 32; ++x) {
        tmem_ld_32x32(tO + 32 * x, u);
        tmem_arrived(u);
#pragma unroll
        for (int y = 0; y < 32; ++y) u[y] = __float_as_uint(__uint_as_float(u[y]) * f);
        tmem_st_32x32(tO + 32 * x, u);
    }
}

// Entries of the ring are used in the order K0 V0 K1 V1 ... (two row tiles against every key tile), or K0 K1 V0 K2 V1 K3 ... (one row tile:
// a stream's product with K(t + 2) follows its product with V(t)); T key tiles are 2 T entries either way.
__device__ __forceinline__ int v_entry(bool two, int T, int t) { return two ? 1 + 2 * t : t <= T - 2 ? 2 + 2 * t : 2 * T - 1; }

// A row of V in its tile: cleared if it is to be, or holds what is not a number; whether it was.
template <int D>
__device__ __noinline__ bool clear_row(uint32_t at, int row, bool clear) {
    constexpr uint32_t kHalf = kTile * 128;
    if (!clear) {
        uint32_t most = 0;  // magnitudes; NaN if one is
#pragma unroll
        for (int x0 = 0; x0 < D / 8; x0 += 4) {
            uint32_t a[4][4];
#pragma unroll
            for (int x = x0; x < x0 + 4; ++x)  // (a row's pieces in an order of its own: eight rows then use all banks)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(a[x - x0][0]), "=r"(a[x - x0][1]), "=r"(a[x - x0][2]), "=r"(a[x - x0][3])
                             : "r"(at + (x >> 3) * kHalf + ((x + row) & 7) * 16)
                             : "memory");
#pragma unroll
            for (int x = 0; x < 16; ++x) most = max_magnitude2(most, a[x >> 2][x & 3]);
        }
        clear = not_finite2(most);
    }
    if (clear) {
#pragma unroll
        for (int x = 0; x < D / 8; ++x)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + (x >> 3) * kHalf + ((x + row) & 7) * 16), "r"(0) : "memory");
    }
    return clear;
}

// What a row sees of new slots whose V is not a number, which was taken out of the products: added to its O in TMEM, with scores of
// its own.  Key tiles t0, t0 + dt, .. of the piece; a whole warp calls it, `sums` are the rows that see anything, m their maxima.
template <int D, bool Q8, bool kWin>
__device__ __noinline__ void add_spoilt(const AttnParams& p, const Piece& pc, uint32_t tO, bool sums, int b, int node, int head, int t0,
                                        int dt, float m) {
    const CacheView& c = p.c;
    const uint32_t* mask_row = p.mask ? p.mask + ((size_t)b * p.nmax + node) * p.words : nullptr;
    const uint16_t* q = (const uint16_t*)p.q + ((long long)b * p.rows + node) * p.q_stride + (long long)head * D;
    for (int t = t0; t < pc.T; t += dt) {
        const int first = pc.first + t * kTile;
        uint32_t sees[4];
        if (kWin)
            window_words(p, pc.gap, pc.lo, pc.base, pc.end, b, node, node - pc.node0,
                         window_step(p.mask ? p.position + (size_t)b * p.nmax : nullptr, node - pc.node0, pc.base + pc.gap), first, sees);
        for (int place = kWin ? first : max(first, pc.base); place < min(pc.end, first + kTile); ++place) {
            if (kWin && place < pc.base && !window_border(place, p.sinks, pc.lo, pc.reach)) continue;
            const int slot = kWin ? slot_at(p, pc.gap, place) : place;
            const size_t at = cache_row(c, __ldg(c.table + (size_t)(kWin ? pc.b : pc.s - 1) * c.width + (slot >> c.page_shift)), pc.h,
                                        slot & ((1 << c.page_shift) - 1));
            const auto entry = [&](const uint8_t* x, const uint8_t* exps, int d) {  // four numbers from d on
                if (!Q8) return *(const uint2*)(x + at * c.row_bytes + 2 * d);
                uint32_t f, more;
                e4m3_factors(exps[at], f, more);
                return e4m3x4_to_bf16(*(const uint32_t*)(x + at * c.row_bytes + d), f, more);
            };
            bool bad = false;  // the same in all lanes: a piece's rows have one sequence where there are new slots
#pragma unroll 1
            for (int d = 0; d < D; d += 4) {
                const uint2 v = entry(c.v, c.v_exp, d);
                bad = bad || not_finite2(v.x) || not_finite2(v.y);
            }
            if (!bad) continue;
            const int j = slot - pc.base;
            bool mine = sums;
            if (kWin) {  // (no index that is not known: the words stay in registers)
                const int x = place - first;
                const uint32_t word = x < 32 ? sees[0] : x < 64 ? sees[1] : x < 96 ? sees[2] : sees[3];
                mine = mine && ((word >> (x & 31)) & 1);
            } else
                mine = mine && (mask_row == nullptr ? j <= node : j < 32 * p.words && ((mask_row[j >> 5] >> (j & 31)) & 1));
            float s = 0.0f;
            if (mine)
#pragma unroll 1
                for (int d = 0; d < D; d += 4) {
                    const uint2 k = entry(c.k, c.k_exp, d);
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t qw = (((uint32_t)q[d + y] << 16) ^ (p.q_flip & 0xFFFF0000u)) & p.q_keep, kw = y < 2 ? k.x : k.y;
                        s += __uint_as_float(qw) * __uint_as_float(y & 1 ? kw & 0xFFFF0000u : kw << 16);
                    }
                }
            const float e = mine ? ex2_approx((s - m) * p.c2) : 0.0f;
#pragma unroll 1
            for (int d = 0; d < D; d += 4) {
                const uint2 v = entry(c.v, c.v_exp, d);
                const uint32_t v0 = v.x << 16, v1 = v.x & 0xFFFF0000u, v2 = v.y << 16, v3 = v.y & 0xFFFF0000u;
                const uint32_t vw[4] = {v0, v1, v2, v3};
                uint32_t o[4];
                asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
                             : "r"(tO + d));
                tmem_wait_ld();
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    asm volatile("" : "+r"(o[y]));
                    if (mine) o[y] = __float_as_uint(__uint_as_float(o[y]) + e * __uint_as_float(vw[y]));
                }
                asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(tO + d), "r"(o[0]), "r"(o[1]), "r"(o[2]),
                             "r"(o[3])
                             : "memory");
                tmem_wait_st();
            }
        }
    }
}

template <int D, bool Q8, bool kOne, bool kWin>
__global__ void __launch_bounds__(Shape<D, Q8, kOne>::kThreads, 1) tree_attn_kernel(const __grid_constant__ AttnParams p) {
    using S = Shape<D, Q8, kOne>;
    constexpr int NS = S::kStages, NR = S::kRaw > 0 ? S::kRaw : 1;
    // Slots whose scores a stream takes at a time.  Whole tiles' scores leave no room for the next ones, and a stream's softmax and products are one
    // chain, two streams by turns: 3450 to 4100 cycles for a key tile and two row tiles, of which the tensor cores work for 1050 (head_dim 64) to 2050.
    // Halves of a key tile have halves of the stream's 128 columns: while one half's exponentials are worked out, the products of the other
    // (its weights' with V, then K of the next tile) run.  That is faster where tiles are converted and arrive late: e4m3 slots behind a window 580
    // us against 600 for 16 trees of up to 513 nodes, 840 against 914 for a prompt of 12000.  It is slower over bf16, where turns do as well and products
    // of 64 slots cost 48 cycles in place of 32: 521 against 490, 780 against 728.  Without a window scores of e4m3 slots are whole tiles' too, which keeps sums in
    // the order that they have had.
    constexpr int kSub = kWin && Q8 ? 64 : kTile, kSubs = kTile / kSub;
    constexpr int kRegsSoftmax = kSubs > 1 ? 144 : S::kRegsSoftmax, kRegsOthers = kSubs > 1 ? 64 : S::kRegsOthers;
    static_assert(256 * kRegsSoftmax + (S::kThreads - 256) * kRegsOthers <= S::kThreads * S::kRegsLaunch, "registers of a launch");
    static_assert(NS / 2 < kCleared, "tiles that the streams may be apart");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base_addr = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base_addr - smem_u32(smem_raw));
    const uint32_t q_addr = base_addr, kv_addr = q_addr + S::kQTiles * S::kTileBytes, raw_addr = kv_addr + NS * S::kTileBytes;
    uint8_t* const raw_ptr = smem + (raw_addr - base_addr);
    uint64_t* bars = (uint64_t*)(raw_ptr + S::kRaw * S::kRawBytes);
    const uint32_t bar0 = smem_u32(bars);
    const auto kv_full = [&](int i) { return bar0 + 8 * i; };
    const auto kv_empty = [&](int i) { return bar0 + 8 * (NS + i); };
    const auto raw_full = [&](int i) { return bar0 + 8 * (2 * NS + i); };
    const auto raw_empty = [&](int i) { return bar0 + 8 * (2 * NS + NR + i); };
    const uint32_t q_full = bar0 + 8 * (2 * NS + 2 * NR), pair = q_full + 8, turn0 = q_full + 16, cleared0 = q_full + 32;
    const uint32_t s_full0 = cleared0 + 8 * kCleared, p_full0 = s_full0 + 32, o_done0 = p_full0 + 32, piece_full0 = o_done0 + 32, piece_empty0 = piece_full0 + 8 * kPieces;
    const auto s_full = [&](int stream, int c) { return s_full0 + 8 * (2 * stream + c); };
    const auto p_full = [&](int stream, int c) { return p_full0 + 8 * (2 * stream + c); };
    const auto o_done = [&](int stream, int c) { return o_done0 + 8 * (2 * stream + c); };
    constexpr int kBars = 2 * NS + 2 * NR + 16 + kCleared + 2 * kPieces;
    volatile int* const gave_up = (volatile int*)(bars + kBars);
    volatile int* const spoilt = gave_up + 1;  // [kSpoiltPieces][2 streams] the last piece (counted from 1) with a row of V that was taken out
    uint32_t* const tmem_at = (uint32_t*)(gave_up + 1 + 2 * kSpoiltPieces);
    Piece* const pieces = (Piece*)(gave_up + 2 + 2 * kSpoiltPieces);  // [kPieces]
    static_assert(kBars * 8 + (2 + 2 * kSpoiltPieces) * 4 + kPieces * sizeof(Piece) <= 1024, "barriers and pieces");
    static_assert((2 + 2 * kSpoiltPieces) * 4 % 8 == 0, "pieces begin where they may be copied eight bytes at a time");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(kv_full(i), Q8 ? S::kConvWarps : 1);
            mbar_init(kv_empty(i), 2);
        }
        for (int i = 0; i < NR; ++i) {
            mbar_init(raw_full(i), 1);
            mbar_init(raw_empty(i), S::kConvWarps > 0 ? S::kConvWarps : 1);
        }
        for (int i = 0; i < kPieces; ++i) {
            mbar_init(piece_full0 + 8 * i, 1);
            mbar_init(piece_empty0 + 8 * i, 11 + S::kConvWarps);
        }
        mbar_init(q_full, 10);
        mbar_init(pair, 8);
        for (int i = 0; i < 2; ++i) {
            for (int c = 0; c < kSubs; ++c) {
                mbar_init(s_full(i, c), 1);
                mbar_init(p_full(i, c), 4);
                mbar_init(o_done(i, c), 1);
            }
            mbar_init(turn0 + 8 * i, 1);
        }
        for (int i = 0; i < kCleared; ++i) mbar_init(cleared0 + 8 * i, 4);
        *gave_up = 0;
        for (int i = 0; i < 2 * kSpoiltPieces; ++i) spoilt[i] = 0;
        mbar_fence_init();
    }
    if (warp == 8) tmem_alloc<false>(smem_u32(tmem_at), 512);
    if (warp == 9 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &p.map_k : &p.map_v) : "memory");
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_at;
    pdl_wait();

    const CacheView& c = p.c;
    // Warp 11 walks along the CTA's stretch and tells the others, a few pieces ahead.
    const auto next_piece = [&](uint32_t n) { return wait_for(piece_full0 + 8 * (n % kPieces), (n / kPieces) & 1, gave_up); };
    const auto piece_done = [&](uint32_t n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(piece_empty0 + 8 * (n % kPieces));
    };

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        // ---- softmax: a thread a row
        const int i = warp >> 2, row_in_tile = tid & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's quarter of the lanes
        const uint32_t tS = tmem + lanes + i * 128, tO = tmem + lanes + 256 + i * 128;
        uint32_t it = 0, n_s = 0, n_piece = 0, n_pair = 0, n_cleared = 0;
        bool ok = true;
        const float c2 = p.c2;
        const auto both = [&]() {  // the two streams meet
            __syncwarp();
            if (lane == 0) mbar_arrive(pair);
            const bool r = wait_for(pair, n_pair & 1, gave_up);
            n_pair += 1;
            return r;
        };
        const auto wait_s = [&](int c) {
            const bool r = wait_for(s_full(i, c), n_s & 1, gave_up);
            tc_fence_after();
            return r;
        };
        // The stream's last product with V that it handed weights over for, ahead of part c of its tile n_s.  (The one before it with the same part is done:
        // scores that have been waited for come from a product behind that.)
        const auto wait_o = [&](int c) {
            const bool r = wait_for(o_done(i, c == 0 ? kSubs - 1 : 0), c == 0 ? (n_s & 1) ^ 1 : n_s & 1, gave_up);
            tc_fence_after();
            return r;
        };
        for (; (ok = next_piece(n_piece)); ++n_piece) {
            const volatile Piece& pc = pieces[n_piece % kPieces];
            const int T = pc.T;
            if (T == 0) break;
            const bool two = !kOne && pc.rows > kTile;
            const int r = (two ? i * kTile : 0) + row_in_tile;  // row of the unit
            const bool live = r < pc.rows;
            int row_b = 0, row_node = 0, row_step = 0;  // kWin: the row's sequence, its number there, and how far its position is behind the first row's
            if (two || i == 0) {
                // a row's pieces side by side in a warp's load; where a row stands is worked out by the lane that has it
                int b = 0, node = 0, g = 0;
                if (live) row_of<kWin>(p, pc, pc.r0 + r, b, node, g);
                if (kWin) row_b = live ? b : pc.b, row_node = live ? node : pc.node0;
                const long long mine = live ? ((long long)b * p.rows + node) * p.q_stride + (long long)(pc.h * p.group + g) * D : -1;
                constexpr int kPer = D / 8, kRows = 32 / kPer;  // lanes a row, rows a load
                const int x = lane % kPer;
                uint4 u[32 / kRows];
#pragma unroll
                for (int y = 0; y < 32 / kRows; ++y) {
                    const long long at = __shfl_sync(0xFFFFFFFFu, mine, y * kRows + lane / kPer);
                    u[y] = __ldg((const uint4*)(p.q + 2 * max(at, 0LL)) + x);  // (no branches between the loads: rows that are not there read row 0)
                }
#pragma unroll
                for (int y = 0; y < 32 / kRows; ++y) {
                    uint4 v = u[y];
                    const uint32_t keep = __shfl_sync(0xFFFFFFFFu, live, y * kRows + lane / kPer) ? p.q_keep : 0u;
                    v.x = (v.x ^ p.q_flip) & keep, v.y = (v.y ^ p.q_flip) & keep;
                    v.z = (v.z ^ p.q_flip) & keep, v.w = (v.w ^ p.q_flip) & keep;
                    const int row = (warp & 3) * 32 + y * kRows + lane / kPer;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_addr + i * S::kTileBytes + row * 128 + (x >> 3) * S::kHalf +
                                                                                  ((((uint32_t)x & 7) ^ (row & 7)) << 4)),
                                 "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                                 : "memory");
                }
                fence_proxy_async();
            } else if (kWin) {
                int g = 0;
                row_b = pc.b, row_node = pc.node0;
                if (live) row_of<kWin>(p, pc, pc.r0 + r, row_b, row_node, g);
            }
            if (kWin) row_step = window_step(p.mask ? p.position + (size_t)row_b * p.nmax : nullptr, row_node - pc.node0, pc.base + pc.gap);
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
            const bool warp_live = __any_sync(0xFFFFFFFFu, live);
            float m = -INFINITY, l = 0.0f;  // maximum of the raw scores, sum of 2^(c2 (s - m))
            bool any = false;               // this stream has had a tile
            // from this tile on there are new slots, or slots that are not there (the shared prefix: base is its end)
            const int first0 = pc.first, to_base = pc.base - kTile - first0, t_masked = to_base < 0 ? 0 : to_base / kTile + 1;
            // (kWin: and tiles at the window's border, with places that some rows do not see)
            const int border0 = kWin ? p.sinks : 0, border1 = kWin ? pc.lo + pc.reach : 0;
            // Slots that are not there hold anything, and new slots may hold what is not a number and is not for every row: weights of zero do
            // not keep it out of the sums.  Their rows of V are cleared (a thread a slot); rows that see such a slot get it in the end.
            const auto clear_v = [&](int t, int first) {
                const uint32_t entry = it + v_entry(two, T, t);
                if (!wait_for(kv_full(entry % NS), (entry / NS) & 1, gave_up)) return false;
                const int slot = first + row_in_tile, end = pc.end;
                if (slot >= pc.base || (kWin && slot >= border0 && slot < border1)) {
                    const bool unseen = kWin && slot >= border0 && slot < min(pc.lo, pc.base);  // by all rows
                    if (clear_row<D>(kv_addr + (entry % NS) * S::kTileBytes + row_in_tile * 128, row_in_tile, slot >= end || unseen) && slot < end && !unseen)
                        spoilt[2 * (n_piece % kSpoiltPieces) + i] = (int)n_piece + 1;
                }
                fence_proxy_async();
                return true;
            };
            for (int t = two ? 0 : i; t < T; t += two ? 1 : 2) {
                const int first = first0 + t * kTile;
                const bool masked = t >= t_masked || (kWin && first < border1 && first + kTile > border0 && border0 < border1);
                uint32_t sees[4];
                if (masked) {
                    if (kWin) {
                        window_words(p, pc.gap, pc.lo, pc.base, live ? pc.end : 0, row_b, row_node, row_node - pc.node0, row_step, first, sees);
                    } else {
                        int b = 0, node = 0, g = 0;
                        if (live) row_of<kWin>(p, pc, pc.r0 + r, b, node, g);
                        const uint32_t* mask_row = p.mask ? p.mask + ((size_t)b * p.nmax + node) * p.words : nullptr;
                        seen_words(mask_row, p.words, node, pc.base, live ? pc.end : 0, first, sees);
                    }
                    // (with two row tiles every entry ahead of V's in the ring has been used by this stream, so its phase is certain: see `pass`)
                    if (two && i == 0) {
                        if (!(ok = clear_v(t, first))) break;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(cleared0 + 8 * (n_cleared % kCleared));
                    }
                }
#pragma unroll 1
                for (int c = 0; c < kSubs; ++c) {
                    if (!(ok = wait_s(c))) break;
                    if (warp_live) {
                        // (with fewer registers: the maximum first, then the scores again, 64 at a time; one piece of code for both halves, which has to stay
                        // in the instruction cache beside that of the other warps: 32 trees behind 500 to 4096 e4m3 slots 160 -> 129 us)
                        constexpr int kCols = S::kCols < kSub ? S::kCols : kSub;
                        uint32_t u[kCols], w[32], part[kCols / 32];
                        const uint32_t tSc = tS + c * kSub;
                        const auto words = [&](int second) {
#pragma unroll
                            for (int x = 0; x < kCols / 32; ++x) part[x] = second ? sees[(x + 2) & 3] : sees[x];
                        };
                        float mx = -INFINITY;
#pragma unroll 1
                        for (int h = 0; h < kSub / kCols; ++h) {
                            words(kCols < kTile && c + h > 0);
                            mx = max2(mx, scores(tSc + 64 * h, 0, u, masked, part));
                        }
                        // (m = -inf: nothing seen so far, and what O holds is zero)
                        const bool grown = mx > m && !((mx - m) * c2 <= kMostGrowth);
                        if (__any_sync(0xFFFFFFFFu, grown)) {
                            const float now = fmaxf(m, mx), f = m > -INFINITY ? ex2_approx((m - now) * c2) : 1.0f;
                            if (any) {
                                if (kSubs > 1 && !(ok = wait_o(c))) break;
                                rescale<D>(tO, f);
                            }
                            l *= f;
                            m = now;
                        }
                        // (a score of NaN or +inf, which some of the exponentials below would lose: the row's sum is NaN from here on, and so is all that
                        // is divided by it)
                        if (!(mx < INFINITY)) l = __int_as_float(0x7FFFFFFF);
                        const float off = m > -INFINITY ? -m * c2 : 0.0f;
#pragma unroll 1
                        for (int h = 0; h < kSub / kCols; ++h) {
                            if (kCols < kSub) {
                                words(h);
                                scores(tSc + 64 * h, 0, u, masked, part);
                            }
                            l += weigh(u, c2, off, w);
                            tmem_st_32x32(tSc + 32 * h, w);
                            if (kCols == kTile) {
                                l += weigh(u + kCols - 64, c2, off, w);
                                tmem_st_32x32(tSc + 32, w);
                            }
                        }
                        tmem_wait_st();
                    }
                    if (masked && c == 0) {
                        if (!two && !(ok = clear_v(t, first))) break;
                        // (the first stream clears for both)
                        if (two && i == 1 && !(ok = wait_for(cleared0 + 8 * (n_cleared % kCleared), (n_cleared / kCleared) & 1, gave_up))) break;
                        n_cleared += two ? 1 : 0;
                    }
                    any = true;
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full(i, c));
                }
                if (!ok) break;
                n_s += 1;
            }
            if (!ok) break;
            it += 2 * T;
            if (any)
                ok = wait_o(0);
            else
                ok = wait_for(q_full, n_piece & 1, gave_up);  // (nor does a stream without a tile run ahead)
            if (!ok) break;

            // ---- the end of a piece: O as far as it goes
            int b = 0, node = 0, g = 0;
            if (live) row_of<kWin>(p, pc, pc.r0 + r, b, node, g);
            const int head = pc.h * p.group + g;
            if (spoilt[2 * (n_piece % kSpoiltPieces) + (two ? 0 : i)] == (int)n_piece + 1)
                add_spoilt<D, Q8, kWin>(p, pieces[n_piece % kPieces], tO, live && m > -INFINITY, b, node, head, two ? 0 : i, two ? 1 : 2, m);
            const bool whole = pc.whole;
            const size_t slot = p.shared > 0 ? (size_t)pc.unit + blockIdx.x : 2 * (size_t)blockIdx.x + pc.head;
            const size_t out_row = ((size_t)b * p.rows + node) * p.q_heads + head;
            const auto put = [&](int d0, uint32_t (&u)[32], float inv) {
                if (!live) return;
                if (whole) {
                    uint4* to = (uint4*)(p.out + out_row * D + d0);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        uint32_t w[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            w[y] = pack_bf16(__uint_as_float(u[8 * x + 2 * y]) * inv, __uint_as_float(u[8 * x + 2 * y + 1]) * inv);
                        to[x] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else {
                    // (four columns of all rows side by side: a warp's stores are whole lines)
                    float4* to = (float4*)p.part_o + (slot * (D / 4) + d0 / 4) * p.part_rows + r;
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        to[x * p.part_rows] = make_float4(__uint_as_float(u[4 * x]), __uint_as_float(u[4 * x + 1]), __uint_as_float(u[4 * x + 2]),
                                            __uint_as_float(u[4 * x + 3]));
                }
            };
            const auto put_sums = [&](float mm, float ll) {
                if (!live) return;
                if (!whole)
                    p.part_ml[slot * p.part_rows + r] = make_float2(mm > -INFINITY ? mm * c2 : -INFINITY, ll);
                else if (p.lse)
                    p.lse[out_row] = log_sum(mm > -INFINITY ? mm * c2 : -INFINITY, ll);
            };
            uint32_t u[32];
            if (two || T == 1) {
                if (two || i == 0) {
                    const float inv = l != 0.0f ? 1.0f / l : 1.0f;  // (a row that sees nothing: O is zero)
                    if (!whole) {
#pragma unroll 1
                        for (int x = 0; x < D / 32; ++x) {
                            tmem_ld_32x32(tO + 32 * x, u);
                            tmem_arrived(u);
                            put(32 * x, u, inv);
                        }
                    } else {
                        // rows go through their own places in Q's tile, which nobody reads any more, so that a warp's stores are whole rows
                        constexpr int kPer = D / 8, kRows = 32 / kPer;  // lanes a row, rows a store
                        const uint32_t tile = q_addr + i * S::kTileBytes;
                        const auto piece_at = [&](int row, int x) { return tile + row * 128 + (x >> 3) * S::kHalf + (((x & 7) ^ (row & 7)) << 4); };
#pragma unroll 1
                        for (int x = 0; x < D / 32; ++x) {
                            tmem_ld_32x32(tO + 32 * x, u);
                            tmem_arrived(u);
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                uint32_t w[4];
#pragma unroll
                                for (int z = 0; z < 4; ++z)
                                    w[z] = pack_bf16(__uint_as_float(u[8 * y + 2 * z]) * inv, __uint_as_float(u[8 * y + 2 * z + 1]) * inv);
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece_at(row_in_tile, 4 * x + y)), "r"(w[0]),
                                             "r"(w[1]), "r"(w[2]), "r"(w[3])
                                             : "memory");
                            }
                        }
                        __syncwarp();
                        const long long mine = live ? (long long)(out_row * D) : -1;
#pragma unroll
                        for (int y = 0; y < 32 / kRows; ++y) {
                            const int from = y * kRows + lane / kPer;
                            const long long at = __shfl_sync(0xFFFFFFFFu, mine, from);
                            uint4 v;
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                                         : "r"(piece_at((warp & 3) * 32 + from, lane % kPer))
                                         : "memory");
                            if (at >= 0) ((uint4*)(p.out + at))[lane % kPer] = v;
                        }
                    }
                    put_sums(m, l);
                }
            } else {
                // the streams' halves are joined: the second one's goes through the shared memory of Q, which nobody reads any more
                float* const tmp = (float*)smem;  // [D / 2 columns][128 rows]
                float m1 = 0.0f, l1 = 0.0f, f0 = 1.0f, f1 = 0.0f, ms = 0.0f, ls = 0.0f, inv = 1.0f;
#pragma unroll 1
                for (int half = 0; half < 2 && ok; ++half) {
                    // maximum and sum of the second stream go ahead of its sums
                    if (half == 0) {
                        if (!(ok = both())) break;  // (both are through with Q)
                        if (i == 1) {
                            tmp[row_in_tile] = m;
                            tmp[128 + row_in_tile] = l;
                        }
                        if (!(ok = both())) break;
                        if (i == 0) {
                            m1 = tmp[row_in_tile];
                            l1 = tmp[128 + row_in_tile];
                            ms = fmaxf(m, m1);
                            f0 = m > -INFINITY ? ex2_approx((m - ms) * c2) : 0.0f;
                            f1 = m1 > -INFINITY ? ex2_approx((m1 - ms) * c2) : 0.0f;
                            ls = l * f0 + l1 * f1;
                            inv = ls != 0.0f ? 1.0f / ls : 1.0f;
                        }
                        if (!(ok = both())) break;
                    }
                    if (i == 1) {
#pragma unroll 1
                        for (int x = 0; x < D / 64; ++x) {
                            const int d0 = half * (D / 2) + 32 * x;
                            tmem_ld_32x32(tO + d0, u);
                            tmem_arrived(u);
#pragma unroll
                            for (int y = 0; y < 32; ++y) tmp[(32 * x + y) * 128 + row_in_tile] = __uint_as_float(u[y]);
                        }
                    }
                    if (!(ok = both())) break;
                    if (i == 0) {
#pragma unroll 1
                        for (int x = 0; x < D / 64; ++x) {
                            const int d0 = half * (D / 2) + 32 * x;
                            tmem_ld_32x32(tO + d0, u);
                            tmem_arrived(u);
#pragma unroll
                            for (int y = 0; y < 32; ++y)
                                u[y] = __float_as_uint(__uint_as_float(u[y]) * f0 + tmp[(32 * x + y) * 128 + row_in_tile] * f1);
                            put(d0, u, inv);
                        }
                    }
                    ok = both();
                }
                if (i == 0 && ok) put_sums(ms, ls);
            }
            tc_fence_before();  // what follows in TMEM follows these reads
            if (!ok) break;
            piece_done(n_piece);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOthers));
        uint32_t n_piece = 0;
        bool ok = true;
        if (warp == 11) {
            Walk<kWin> walk;
            Piece pc;
            walk.begin(p, blockIdx.x);
            for (bool more = true; ok && more; ++n_piece) {
                more = walk.next(pc);
                if (!more) pc.T = 0;
                ok = wait_for(piece_empty0 + 8 * (n_piece % kPieces), ((n_piece / kPieces) & 1) ^ 1, gave_up);
                if (ok && lane == 0) {
                    pieces[n_piece % kPieces] = pc;
                    mbar_arrive(piece_full0 + 8 * (n_piece % kPieces));
                }
                if (more && pc.s > 0)  // its rows of Q come to L2 while the pieces ahead are worked on
                    for (int r = lane; r < pc.rows; r += 32) {
                        int b, node, g;
                        row_of<kWin>(p, pc, pc.r0 + r, b, node, g);
                        const uint8_t* at = p.q + 2 * (((long long)b * p.rows + node) * p.q_stride + (long long)(pc.h * p.group + g) * D);
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
                        if (D > 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + 128));
                    }
            }
        } else if (warp == 9) {
            // ---- copies: K and V tiles page by page, into the ring (bf16) or to where the conversion takes them from (e4m3)
            constexpr int N = Q8 ? NR : NS;
            constexpr int kParts = Q8 ? 2 : D / 64;  // copies a page and tile: halves of its rows, or numbers and exponents
            uint32_t it = 0;
            const int box = p.box_rows, shift = c.page_shift, low = (1 << shift) - 1;
            for (; (ok = next_piece(n_piece)); ++n_piece) {
                const volatile Piece& pc = pieces[n_piece % kPieces];
                const int T = pc.T, h = pc.h, end = pc.end, first0 = pc.first;
                if (T == 0) break;
                const bool two = !kOne && pc.rows > kTile;
                const int32_t* table = c.table + (kWin ? (size_t)pc.b * c.width : pc.s == 0 ? 0 : (size_t)(pc.s - 1) * c.width);
                const int gap = kWin ? pc.gap : 0;
                const auto bring = [&](int t, bool is_v) {
                    const int first = first0 + t * kTile, upto = min(end, first + kTile);
                    const int copies = (upto - first + box - 1) / box;  // boxes with a slot in use
                    const int i = lane / kParts, part = lane % kParts;
                    int page = 0, at = 0;
                    if (i < copies) {
                        const int slot = kWin ? slot_at(p, gap, first + i * box) : first + i * box;
                        page = __ldg(table + (slot >> shift));
                        at = slot & low;
                    }
                    const uint32_t st = it % N, full = Q8 ? raw_full(st) : kv_full(st), empty = Q8 ? raw_empty(st) : kv_empty(st);
                    if (!wait_for(empty, ((it / N) & 1) ^ 1, gave_up)) return false;
                    const uint32_t to = Q8 ? raw_addr + st * S::kRawBytes : kv_addr + st * S::kTileBytes;
                    if (lane == 0) mbar_arrive_expect_tx(full, copies * box * (Q8 ? D + 1 : 2 * D));
                    __syncwarp();
                    if (i < copies) {
                        const size_t row = cache_row(c, page, h, at);
                        if (!Q8 || part == 0)
                            tma_load_2d(to + (Q8 ? i * box * D : part * S::kHalf + i * box * 128), is_v ? &p.map_v : &p.map_k,
                                        Q8 ? 0 : part * 64, (int)row, full);
                        else
                            tma_load_1d(to + kTile * D + i * box, (is_v ? c.v_exp : c.k_exp) + row, box, full);
                    }
                    it += 1;
                    return true;
                };
                // (in the order of the ring, see v_entry)
#pragma unroll 1
                for (int e = 0; ok && e < 2 * T; ++e) {
                    const bool is_v = two ? e & 1 : e == 2 * T - 1 || (e > 0 && !(e & 1));
                    ok = bring(two ? e >> 1 : e == 2 * T - 1 ? T - 1 : is_v ? (e - 2) >> 1 : (e + 1) >> 1, is_v);
                }
                if (!ok) break;
                piece_done(n_piece);
            }
            // (after a wait that ran out: what is on its way arrives before the CTA ends)
            if (!ok && lane == 0)
                for (uint32_t i = it > (uint32_t)N ? it - N : 0; i < it; ++i)
                    for (int w = 0; w < (1 << 16) && !mbar_try_wait(Q8 ? raw_full(i % N) : kv_full(i % N), (i / N) & 1); ++w) {
                    }
            __syncwarp();
        } else if (warp == 8 || warp == 10) {
            // ---- products, a warp a stream: while one waits for weights or signals, the other's instructions keep the tensor cores busy
            constexpr uint32_t id_s = umma_idesc(128, kSub, true), id_o = umma_idesc(128, D, true) | (1u << 16);  // (V: head_dim is contiguous)
            const uint32_t i = warp == 8 ? 0 : 1;
            uint32_t it = 0, n_p = 0, n_turn = 0;
            // (descriptors differ in their low words alone; the numbers that choose them are loaded, so the compiler is told that they are uniform)
            constexpr uint32_t kDescHi = (uint32_t)(umma_desc_sw128(0) >> 32);
            const uint32_t tS = uniform(tmem + i * 128), tO = uniform(tmem + 256 + i * 128);
            const uint32_t q_lo = uniform((uint32_t)umma_desc_sw128(q_addr)), kv_lo = uniform((uint32_t)umma_desc_sw128(kv_addr));
            const auto qk = [&](int c, uint32_t a, uint32_t b) {  // (rows of K: slots)
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t at = ((ks >> 2) * S::kHalf + (ks & 3) * 32) / 16, row = c * (kSub * 128 / 16);
                    if (ks == 0)
                        umma_ss<false>(tS + c * kSub, a + at, b + at + row, kDescHi, id_s);
                    else
                        umma_ss<true>(tS + c * kSub, a + at, b + at + row, kDescHi, id_s);
                }
            };
            // V as the second operand of P V: rows (slots) of 64 numbers of head_dim side by side, so head_dim is the contiguous direction.  In
            // the 128-byte swizzle: blocks of 64 numbers kHalf apart (a field that the other operands leave at 1), groups of eight slots 1024 bytes.
            constexpr uint32_t kHalfField = (uint32_t)(S::kHalf / 16) << 16, kOneField = 1u << 16;
            const auto pv = [&](int c, bool first, uint32_t b) {
#pragma unroll
                for (int ks = 0; ks < kSub / 16; ++ks)
                    umma_ts(tO, tS + c * kSub + ks * 8, kDescHi, b + (c * (kSub / 16) + ks) * (2048 / 16), id_o, c > 0 || ks > 0 || !first);
            };
            const auto at_entry = [&](uint32_t entry) { return uniform(kv_lo + (entry % NS) * (S::kTileBytes / 16)); };
            const auto wait_kv = [&](uint32_t entry) { return wait_for(kv_full(entry % NS), (entry / NS) & 1, gave_up); };
            // Both streams go through all entries in order and an entry is free when both have: one that the other stream alone reads is seen
            // to be full and let go.  So neither is ever more than one use of a stage away from what it waits for, which is as far as a
            // barrier's phase tells uses apart (copies may arrive out of order).
            const auto pass = [&](uint32_t upto) {
                for (; it != upto; ++it) {
                    if (!wait_kv(it)) return false;
                    if (lane == 0) mbar_arrive(kv_empty(it % NS));
                }
                return true;
            };
            // Two row tiles, whole tiles' scores: the streams issue by turns.  Side by side, their instructions would share the tensor cores and both streams'
            // softmax would then share the rest of the time; by turns, one stream's softmax runs under the other's products.
            const auto my_turn = [&](bool two) {
                if (!two || kSubs > 1) return true;
                const bool r = wait_for(turn0 + 8 * i, (n_turn & 1) ^ (1 - i), gave_up);
                n_turn += 1;
                return r;
            };
            for (; (ok = next_piece(n_piece)); ++n_piece) {
                const volatile Piece& pc = pieces[n_piece % kPieces];
                const int T = pc.T;
                if (T == 0) break;
                const bool two = !kOne && pc.rows > kTile;
                if (lane == 0) mbar_arrive(q_full);  // (with the rows' own arrivals: a piece begins when this warp is there too)
                if (!(ok = wait_for(q_full, n_piece & 1, gave_up))) break;
                const uint32_t a = uniform(q_lo + (two ? i : 0) * (S::kTileBytes / 16)), it0 = it;
                const int t0 = two ? 0 : (int)i, dt = two ? 1 : 2;
                if (t0 < T) {
                    if (!(ok = pass(it0 + t0) && wait_kv(it) && my_turn(two))) break;
                    tc_fence_after();
                    const uint32_t bk = at_entry(it);
                    if (elect_one()) {
#pragma unroll
                        for (int c = 0; c < kSubs; ++c) {
                            qk(c, a, bk);
                            if (c == kSubs - 1) {
                                if (two && kSubs == 1) mbar_arrive(turn0 + 8 * (1 - i));
                                umma_commit(kv_empty(it % NS));
                            }
                            umma_commit(s_full(i, c));
                        }
                    }
                    __syncwarp();
                    it += 1;
                }
                // P V of a tile, then Q K of the next, which takes the weights' place
                for (int t = t0; t < T; t += dt) {
                    const bool more = t + dt < T;
                    if (!(ok = pass(it0 + v_entry(two, T, t)) && wait_kv(it))) break;
                    const uint32_t bv = uniform(at_entry(it) - kOneField + kHalfField), bk = at_entry(it + 1);
#pragma unroll 1
                    for (int c = 0; c < kSubs; ++c) {
                        if (!(ok = wait_for(p_full(i, c), n_p & 1, gave_up) && my_turn(two))) break;
                        tc_fence_after();
                        if (elect_one()) {
                            pv(c, t == t0, bv);
                            umma_commit(o_done(i, c));
                            if (c == kSubs - 1) umma_commit(kv_empty(it % NS));
                        }
                        __syncwarp();
                        if (more && c == 0) {
                            if (!(ok = wait_kv(it + 1))) break;
                            tc_fence_after();
                        }
                        if (elect_one()) {
                            if (more) qk(c, a, bk);
                            if (two && kSubs == 1) mbar_arrive(turn0 + 8 * (1 - i));
                            if (more) umma_commit(s_full(i, c));
                            if (more && c == kSubs - 1) umma_commit(kv_empty((it + 1) % NS));
                        }
                        __syncwarp();
                    }
                    n_p += 1;
                    if (!ok) break;
                    it += more ? 2 : 1;
                }
                ok = ok && pass(it0 + 2 * T);
                if (!ok) break;
                piece_done(n_piece);
            }
        } else if (Q8 && warp >= 12) {
            // ---- e4m3 tiles to bf16 tiles in the 128-byte swizzle: sixteen numbers a thread and step
            const int ct = tid - 384;
            constexpr int kPer = D / 16, kRowsStep = (Q8 ? 32 * S::kConvWarps : 256) / kPer, kSteps = kTile / kRowsStep;
            const int col = ct % kPer, row0 = ct / kPer;
            constexpr int kBatch = kSteps < 4 ? kSteps : 4;
            uint32_t it = 0;
            for (; (ok = next_piece(n_piece)); ++n_piece) {
                const int T = ((const volatile Piece&)pieces[n_piece % kPieces]).T;
                if (T == 0) break;
                const auto convert = [&]() {
                    const uint32_t rs = it % NR, ks = it % NS;
                    if (!wait_for(raw_full(rs), (it / NR) & 1, gave_up)) return false;
                    if (!wait_for(kv_empty(ks), ((it / NS) & 1) ^ 1, gave_up)) return false;
                    const uint8_t* raw = raw_ptr + rs * S::kRawBytes;
                    const uint32_t to = kv_addr + ks * S::kTileBytes + (col >> 2) * S::kHalf;
#pragma unroll
                    for (int x0 = 0; x0 < kSteps; x0 += kBatch) {
                        uint4 y[kBatch];
                        uint32_t e[kBatch];
#pragma unroll
                        for (int x = 0; x < kBatch; ++x) {
                            const int row = (x0 + x) * kRowsStep + row0;
                            y[x] = *(const uint4*)(raw + row * D + col * 16);
                            e[x] = raw[kTile * D + row];
                        }
                        // (scales above 2^7 take a second factor: rows of their kind are looked for once a batch)
                        bool large = false;
#pragma unroll
                        for (int x = 0; x < kBatch; ++x) large = large || (e[x] > 134 && e[x] != 255);
                        const auto put_rows = [&](auto two_factors) {
#pragma unroll
                            for (int x = 0; x < kBatch; ++x) {
                                const int row = (x0 + x) * kRowsStep + row0;
                                uint32_t f, more;
                                if (decltype(two_factors)::value)
                                    e4m3_factors(e[x], f, more);
                                else
                                    f = e[x] == 255 ? 0x7FC07FC0u : (e[x] + 120) * 0x00800080u, more = kOneBf16x2;
                                uint32_t r[8];
#pragma unroll
                                for (int y4 = 0; y4 < 4; ++y4) {
                                    const uint32_t v4 = y4 == 0 ? y[x].x : y4 == 1 ? y[x].y : y4 == 2 ? y[x].z : y[x].w;
                                    const uint2 a = make_uint2(bf16x2_mul(e4m3_pair_small(v4, 0, 0, 1), f), bf16x2_mul(e4m3_pair_small(v4, 0, 2, 3), f));
                                    r[2 * y4] = decltype(two_factors)::value ? bf16x2_mul(a.x, more) : a.x;
                                    r[2 * y4 + 1] = decltype(two_factors)::value ? bf16x2_mul(a.y, more) : a.y;
                                }
                                // (the second half of a row's threads store their second piece first: eight threads then use all banks)
                                const uint32_t chunk = (col & 3) * 2, at = to + row * 128, swap = D == 128 ? (uint32_t)col >> 2 : 0u;
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (((chunk + swap) ^ (row & 7)) << 4)),
                                             "r"(swap ? r[4] : r[0]), "r"(swap ? r[5] : r[1]), "r"(swap ? r[6] : r[2]), "r"(swap ? r[7] : r[3])
                                             : "memory");
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (((chunk + 1 - swap) ^ (row & 7)) << 4)),
                                             "r"(swap ? r[0] : r[4]), "r"(swap ? r[1] : r[5]), "r"(swap ? r[2] : r[6]), "r"(swap ? r[3] : r[7])
                                             : "memory");
                            }
                        };
                        if (__any_sync(0xFFFFFFFFu, large))
                            put_rows(Yes());
                        else
                            put_rows(No());
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(raw_empty(rs));
                        mbar_arrive(kv_full(ks));
                    }
                    it += 1;
                    return true;
                };
                for (int e = 0; ok && e < 2 * T; ++e) ok = convert();
                if (!ok) break;
                piece_done(n_piece);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*gave_up && p.status)
        for (int i = tid; i < p.batch; i += blockDim.x) atomicOr(p.status + i, GRAFT_ST_INTERNAL);
    if (warp == 8) tmem_free<false>(tmem, 512);
}

// ---- its plan and its launch ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kPlanThreads) attn_plan_kernel(const __grid_constant__ AttnParams p) {
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kWarps = kPlanThreads / 32;
    const CacheView& c = p.c;
    __shared__ int fine[kWarps], last;
    __shared__ int scratch[3][kWarps];
    __shared__ PlanSeq entries[kPlanSeqs + 1];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int n0 = p.count[b], base0 = p.prefix_len[b] - 1;
    {
        const int32_t* table = c.table + (size_t)b * c.width;
        const long long end = (long long)base0 + n0;
        bool ok = n0 >= 0 && n0 <= p.rows && base0 >= 0 && base0 >= p.shared && end <= ((long long)c.width << c.page_shift);
        if (ok && n0 > 0)
            for (int i = tid; i <= (int)((end - 1) >> c.page_shift); i += kPlanThreads) {
                ok = ok && (unsigned)table[i] < (unsigned)c.n_pages;
                // (the shared pages are read from the first sequence's table)
                if (i < p.shared >> c.page_shift) ok = ok && (unsigned)c.table[i] < (unsigned)c.n_pages;
            }
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (lane == 0) fine[warp] = ok;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) ok = ok && fine[w];
        n0 = ok ? n0 : 0;
        if (tid == 0) {
            if (p.status) p.status[b] = ok ? 0 : GRAFT_ST_BAD_CACHE;
            *(int2*)&p.seq[b + 1] = make_int2(n0, base0);
            last = gridDim.x == 1 || atom_add_acq_rel(p.arrivals, 1) == (int)gridDim.x - 1;
        }
        __syncthreads();
        if (!last) return;
    }
    // the last block: what sequence i has
    const int Hk = c.kv_heads;
    const bool held = p.batch <= kPlanSeqs, small = p.batch <= 32;  // (few sequences: every warp goes through them by itself)
    const int me = small ? lane : tid;
    const auto of = [&](int i, int& n, int& base, int& kt, int& R) {
        n = base = 0;
        if (gridDim.x == 1) {
            if (i == 0) n = n0, base = base0;
        } else if (i < p.batch) {
            const int2 v = __ldcg((const int2*)&p.seq[i + 1]);
            n = v.x, base = v.y;
        }
        kt = n > 0 ? (base + n - p.shared + kTile - 1) / kTile : 0;
        R = n * p.group;
    };
    int nodes = 0, total = 0, chunk = 1;
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
        int n, base, kt, R;
        of(b0 + me, n, base, kt, R);
        const Sums s = block_sums(scratch, small, n, Hk * head_cost(R, kt, 1), 0);
        nodes += s.all[0], total += s.all[1];
    }
    const int Rs = p.shared > 0 ? nodes * p.group : 0, kts = (p.shared + kTile - 1) / kTile;
    total += Hk * head_cost(Rs, kts, 1);
    // A CTA's share of the line may begin and end inside of units; every piece of one costs some microseconds beside its tiles.  Where shares
    // are short, units are given lengths of whole shares instead, so that a CTA has one piece, if shares a few tiles longer than equal ones
    // are enough for it.
    const int share = (total + p.ctas - 1) / p.ctas;
    if (share > 1 && share <= p.most_share && p.batch <= kPlanThreads) {
        int n, base, kt, R;
        of(me, n, base, kt, R);
        for (int c2 = (share + 5) / 6 * 6; c2 <= share + 11; c2 += 6) {  // (whole tiles of either weight)
            const Sums s = block_sums(scratch, small, Hk * (head_cost(R, kt, c2) / c2), 0, 0);
            if (s.all[0] + Hk * (head_cost(Rs, kts, c2) / c2) <= p.ctas) {
                chunk = c2;
                break;
            }
        }
    }
    // (the shared prefix goes first)
    int units = Hk * row_tiles2(Rs), cost = Hk * head_cost(Rs, kts, chunk), seen = 0;
    if (tid == 0) {
        PlanSeq s = {Rs > 0 ? nodes : 0, p.shared, 0, 0, 0, kts, 0, 0};
        p.seq[0] = s;
        entries[0] = s;
    }
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
        const int i = b0 + me;
        int n, base, kt, R;
        of(i, n, base, kt, R);
        const Sums s = block_sums(scratch, small, n, Hk * row_tiles2(R), Hk * head_cost(R, kt, chunk));
        if (i < p.batch && (!small || warp == 0)) {
            PlanSeq q = {n, base, seen + s.before[0], units + s.before[1], cost + s.before[2], kt, 0, 0};
            p.seq[i + 1] = q;
            if (held) entries[i + 1] = q;
        }
        seen += s.all[0], units += s.all[1], cost += s.all[2];
    }
    total = cost;
    const int parts = chunk > 1 ? total / chunk : min(p.ctas, total);
    if (tid == 0) {
        p.head->total = total;
        p.head->parts = parts;
        p.head->chunk = chunk;
        *p.arrivals = 0;
    }
    __syncthreads();
    plan_starts<false>(p, entries, held, p.batch, total, parts, chunk);
}

// Behind a shared prefix every row has pieces of two units; 32 rows of a sequence may lie in two units of the prefix.
template <int D>
__global__ void __launch_bounds__(kJoinThreads, 4) attn_join_shared_kernel(const __grid_constant__ AttnParams p) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ JoinList j;
    const int b = blockIdx.z, h = blockIdx.y, r0 = blockIdx.x * kJoinRows;
    PlanSeq all, q;
    load_seq(all, p.seq);
    load_seq(q, p.seq + b + 1);
    const int total = __ldcg(&p.head->total), parts = __ldcg(&p.head->parts), chunk = __ldcg(&p.head->chunk), R = q.n * p.group;
    if (r0 >= R) return;
    if (threadIdx.x < 32) {
        if (threadIdx.x == 0) j.n = 0;
        __syncwarp();
        const int Ra = all.n * p.group, ra = q.node0 * p.group + r0, mt = ra / kUnitRows, upto = (mt + 1) * kUnitRows - ra;
        const int ua = all.unit0 + h * row_tiles2(Ra);
        UnitAt u = unit_at(all, p.group, h, mt, chunk);
        const auto cta = [&](int k) { return cta_of(u.x0 + k * u.w, total, parts); };
        list_unit(j, u, cta(0), cta(u.kt - 1), total, parts, ua + mt, ra - mt * kUnitRows, 0, min(upto, kJoinRows));
        if (upto < kJoinRows && (mt + 1) * kUnitRows < Ra) {
            u = unit_at(all, p.group, h, mt + 1, chunk);
            list_unit(j, u, cta(0), cta(u.kt - 1), total, parts, ua + mt + 1, -upto, upto, kJoinRows);
        }
        const int mo = r0 / kUnitRows;
        u = unit_at(q, p.group, h, mo, chunk);
        list_unit(j, u, cta(0), cta(u.kt - 1), total, parts, q.unit0 + h * row_tiles2(R) + mo, r0 - mo * kUnitRows, 0, kJoinRows);
    }
    __syncthreads();
    const int r = r0 + lane_id(), node = r / p.group;
    join_rows<D, 2>(p, j, r < R, ((size_t)b * p.rows + node) * p.q_heads + h * p.group + (r - node * p.group));
}

template <int D, typename Kernel>
cudaError_t launch_tree(graft_ctx* ctx, const AttnParams& p, Kernel kernel, int threads, size_t smem, uint32_t ready, bool join, cudaStream_t st) {
    return launch_kernels(ctx, p, attn_plan_kernel, kernel, threads, smem, &ctx->attn_ready, ready, [&] {
        if (!join) return cudaSuccess;
        if (p.shared == 0) return launch_join<D>(ctx, p, st);
        ctx->launches += 1;
        const long long most = (long long)p.rows * p.group;  // rows of a sequence and key head
        return launch_pdl(attn_join_shared_kernel<D>, dim3((unsigned)((most + kJoinRows - 1) / kJoinRows), p.c.kv_heads, p.batch),
                          dim3(kJoinThreads), 0, st, p);
    }, st);
}
template <int D, bool Q8, bool kOne>
cudaError_t launch_attn(graft_ctx* ctx, const AttnParams& p, cudaStream_t st) {
    using S = Shape<D, Q8, kOne>;
    return launch_tree<D>(ctx, p, tree_attn_kernel<D, Q8, kOne, false>, S::kThreads, S::kSmem, 1u << ((D == 128) + 2 * Q8 + 4 * kOne), true, st);
}
template <int D, bool Q8>
cudaError_t launch_any(graft_ctx* ctx, const AttnParams& p, cudaStream_t st) {
    const long long rows = (long long)p.rows * p.group;
    if (few_rows(p.group, p.rows, p.shared))
        return launch_tree<D>(ctx, p, few_attn_kernel<D, Q8, false>, FewShape<D, Q8, false>::kThreads, FewShape<D, Q8, false>::kSmem,
                                 256u << ((D == 128) + 2 * Q8), false, st);
    return p.shared == 0 && rows <= kTile ? launch_attn<D, Q8, true>(ctx, p, st) : launch_attn<D, Q8, false>(ctx, p, st);
}

template <int D, bool Q8, bool kOne>
TilesKernel window_tiles() {
    using S = Shape<D, Q8, kOne>;
    return {tree_attn_kernel<D, Q8, kOne, true>, S::kThreads, S::kSmem};
}

}  // namespace

TilesKernel window_tiles_kernel(int head_dim, bool q8, bool one) {
    if (head_dim == 128)
        return q8 ? (one ? window_tiles<128, true, true>() : window_tiles<128, true, false>())
                  : (one ? window_tiles<128, false, true>() : window_tiles<128, false, false>());
    return q8 ? (one ? window_tiles<64, true, true>() : window_tiles<64, true, false>())
              : (one ? window_tiles<64, false, true>() : window_tiles<64, false, false>());
}

size_t tree_attn_scratch_bytes(const graft_ctx* ctx, int batch, const graft_cache* cache, int q_heads, int rows, int shared) {
    const int group = q_heads / cache->kv_heads, ctas = attn_ctas<false>(ctx, cache->dtype == GRAFT_E4M3, cache->head_dim, group, rows, shared);
    return attn_sizes(ctas, batch, batch, 0, cache->kv_heads, cache->head_dim, group, rows, shared).total;
}

cudaError_t tree_attn_launch(graft_ctx* ctx, int batch, const graft_cache* cache, int layer, int q_heads, int rows, long long q_stride,
                             const void* d_q, float scale, const int32_t* d_prefix_len, const int32_t* d_count, const uint32_t* d_mask,
                             int shared, void* d_out, float* d_lse, int32_t* d_status, void* scratch, cudaStream_t st) {
    const bool q8 = cache->dtype == GRAFT_E4M3, few = few_rows(q_heads / cache->kv_heads, rows, shared);
    AttnParams p;
    const cudaError_t e = attn_params(p, ctx, batch, cache, layer, q_heads, rows, q_stride, d_q, scale, d_prefix_len, d_count, d_mask, d_out, d_lse,
                                      d_status, !few, cache->page_size < kTile ? cache->page_size : kTile);
    if (e != cudaSuccess) return e;
    p.shared = shared;
    p.ctas = attn_ctas<false>(ctx, q8, cache->head_dim, p.group, rows, shared);
    attn_places(p, attn_sizes(p.ctas, batch, batch, 0, cache->kv_heads, cache->head_dim, p.group, rows, shared), scratch);
    p.most_share = few ? 0 : 128;
    const auto launch = cache->head_dim == 128 ? (q8 ? launch_any<128, true> : launch_any<128, false>)
                                               : (q8 ? launch_any<64, true> : launch_any<64, false>);
    return launch(ctx, p, st);
}

}  // namespace graft

