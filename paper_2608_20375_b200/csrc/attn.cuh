// Attention over a paged cache: what graft_tree_attention (tree_attn.cu) and graft_window_attention (window_attn.cu, kWin) have in common.  The
// kernels and the line of key tiles that they share out are described in tree_attn.cu.
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include <float.h>
#include <string.h>

#include "cache.cuh"
#include "umma.cuh"

namespace graft {

constexpr int kTile = 128;      // slots of a key tile, rows of a row tile
constexpr int kUnitRows = 256;
constexpr uint32_t kWaitNs = 500;  // that a poll may sleep
constexpr float kMostGrowth = 8.0f;  // (powers of two) of a row's maximum, before O is rescaled

struct Yes {
    static constexpr bool value = true;
};
struct No {
    static constexpr bool value = false;
};

// What the plan says of a sequence (entry 0: the shared prefix with the rows of all of them; entry b + 1: sequence b).  Behind a window (kWin)
// entries are blocks of a sequence's rows, entry 0 is empty, and slots are counted along what the block's rows see: see "windows".
struct __align__(16) PlanSeq {
    int n;       // rows in use (nodes); 0: none, or left out
    int base;    // slots before the first row's (shared prefix: its length)
    int node0;   // nodes of the sequences before (kWin: of the sequence, before the block)
    int unit0;   // units before (kWin: how far behind the first row's position another row's is at most)
    int cost0;   // position in the line: lengths of the units before
    int kt;      // key tiles
    int b, gap;  // kWin: the sequence; slots that are left out
};
struct __align__(16) PlanStart {
    int s, h, mt, k;         // where a CTA begins: entry, key head, unit of the head, key tile (may be one behind the unit's last)
    int x, x1, chunk, pad;   // that tile's position in the line, and where the CTA's stretch ends
    PlanSeq q;               // the entry
};
// A unit that is cut at the beginning of CTA c's stretch for the first time: what joining it takes.
struct __align__(16) PlanJoin {
    int rows;          // of the unit; 0: nothing to join here
    int f, l;          // first and last CTA that may have tiles of it
    int total, parts;  // as in PlanHead
    int x0, w, kt;     // the unit in the line
    int s, h, r0;      // entry (kWin: sequence + 1), key head, first row of the unit among the entry's
    int node0;         // kWin: nodes of the sequence before the entry's
};
struct PlanHead {
    int total;  // length of the line
    int parts;  // CTAs that it is cut for
    int chunk;  // units begin at multiples of it
    int entries;  // kWin: how many there are behind entry 0
};

struct __align__(64) AttnParams {
    CUtensorMap map_k, map_v;
    CacheView c;
    const uint8_t* q;
    long long q_stride;
    const int32_t* prefix_len;
    const int32_t* count;
    const uint32_t* mask;
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
    float c2;            // |scale| log2(e)
    uint32_t q_flip;     // a negative scale: the sign of q
    uint32_t q_keep;     // 0: a scale of zero
    int rows, q_heads, group, shared, nmax, words, batch;
    int box_rows;        // slots of a page that one copy brings
    PlanHead* head;
    PlanSeq* seq;        // [batch + 1]
    PlanStart* start;    // [gridDim of the attention kernel]
    PlanJoin* join;      // the same
    int ctas;
    int most_share;      // shares up to this length may be made whole
    int part_rows;       // rows that a piece has room for
    int* arrivals;       // zero between calls
    int* ready;          // [ctas] few rows: pieces that are there of the unit that is cut behind its beginning in a CTA
    float* part_o;       // [slots][D / 4][part_rows][4]
    float2* part_ml;     // [slots][part_rows]: maximum (log2 domain), sum
    // kWin
    const int32_t* position;  // with a mask: [batch, nmax]
    int window, sinks;
    int grain;           // slots are left out in whole multiples of it, from `sink_pad` on
    int sink_pad;
    int block_rows;      // nodes of an entry at most
    int4* use;           // [batch] rows in use, the slots before them, and unit0 of a tree
    int* entry0;         // [batch] entries before the sequence's
    int self_plan;       // few rows: every CTA works out the plan by itself (`ready` is zero between calls then)
};

// A kernel of tiles (tree_attn.cu) for rows behind a window: units of one row tile at most, or of two.
struct TilesKernel {
    void (*kernel)(AttnParams);
    int threads;
    size_t smem;
};
TilesKernel window_tiles_kernel(int head_dim, bool q8, bool one);

namespace {

// ---- windows -------------------------------------------------------------------------------------------------------
// Rows of a block whose first one stands in slot `base` see the slots below `sinks` and those from lo = base - window + 1 on.  What lies between
// is left out, in whole grains: places 0, 1, .. of the block's line of slots are slots 0 .. sink_pad - 1 and, behind them, the slots from
// sink_pad + gap on.  All that is said of a piece (its first place, its end, the place of its first new row) is said in places.
__device__ __forceinline__ int gap_of(const AttnParams& p, int base) {
    const int lo = base - p.window + 1;
    return max(0, (max(lo, 0) & ~(p.grain - 1)) - p.sink_pad);
}
__device__ __forceinline__ int slot_at(const AttnParams& p, int gap, int place) { return place + (place >= p.sink_pad ? gap : 0); }
// Slots ahead of the new rows that some row of the block does not see: those behind the sinks and ahead of the window of the row that is `reach`
// positions behind the first.
__device__ __forceinline__ bool window_border(int place, int sinks, int lo, int reach) { return place >= sinks && place < lo + reach; }
__device__ __forceinline__ uint32_t low_bits(int n) {  // (a shift by 32 or more leaves nothing)
    uint32_t r;
    asm("shl.b32 %0, %1, %2;" : "=r"(r) : "r"(1), "r"(max(n, 0)));
    return r - 1;
}
// how far behind the first row's slot row i's position is; base: that slot
__device__ __forceinline__ int window_step(const int32_t* position, int i, int base) {
    if (position == nullptr) return i;
    const int at = __ldg(position + i);
    return at <= base ? 0 : min(at - base, i);
}

__device__ __forceinline__ void load_seq(PlanSeq& q, const PlanSeq* from) {
    ((int4*)&q)[0] = __ldcg((const int4*)from);
    ((int4*)&q)[1] = __ldcg((const int4*)from + 1);
}


// ---- the plan ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int row_tiles2(int R) { return (R + kUnitRows - 1) / kUnitRows; }  // units of R rows
// What a key tile weighs: one row tile keeps the streams half as busy as two, but copies and conversions are the same (256 rows take 1.5 times as
// long as 68, in bf16 and e4m3).
constexpr int kOneTile = 2, kTwoTiles = 3;
__device__ __forceinline__ int unit_weight(int R, int mt) { return R - mt * kUnitRows > kTile ? kTwoTiles : kOneTile; }
// A unit's length in the line: its tiles' and kPieceCost for what a piece costs beside them (Q's rows, the first products, O), or what fills
// the last share.  64 x 17 nodes behind 8192 shared slots, where 256 short pieces follow the long ones: 317 us with 0, 243 with 4, 214 with 7,
// 215 with 10, 218 with 14; 32 sequences of up to 65 nodes over e4m3: 234, 196, 186, 175, 176.
constexpr int kPieceCost = 8;
__device__ __forceinline__ int padded(int cost, int chunk) { return chunk == 1 ? cost + kPieceCost : (cost + chunk - 1) / chunk * chunk; }
__device__ __forceinline__ int head_cost(int R, int kt, int chunk) {
    const int u = row_tiles2(R);
    return u == 0 ? 0 : (u - 1) * padded(kTwoTiles * kt, chunk) + padded(kt * unit_weight(R, u - 1), chunk);
}

// first position of CTA c's stretch: ceil(c total / parts)
__device__ __forceinline__ int part_first(int total, int parts, int c) {
    const int q = total / parts;
    return c * q + (c * (total - q * parts) + parts - 1) / parts;
}

// A unit in the line: where its first tile stands, what a tile weighs, how many there are.
struct UnitAt {
    int x0, w, kt;
};
__device__ __forceinline__ UnitAt unit_at(const PlanSeq& q, int group, int h, int mt, int chunk) {
    const int R = q.n * group;
    UnitAt u;
    u.x0 = q.cost0 + h * head_cost(R, q.kt, chunk) + padded(kTwoTiles * q.kt, chunk) * mt;
    u.w = unit_weight(R, mt);
    u.kt = q.kt;
    return u;
}
// first tile of the unit that is not ahead of CTA c's stretch
__device__ __forceinline__ int first_tile(const UnitAt& u, int total, int parts, int c) {
    const int d = part_first(total, parts, c) - u.x0;
    return d <= 0 ? 0 : min((d + u.w - 1) / u.w, u.kt);
}
__device__ __forceinline__ int cta_of(int x, int total, int parts) { return (int)((long long)x * parts / total); }

constexpr int kPlanThreads = 256;
constexpr int kPlanSeqs = 512;  // sequences whose entries are held in shared memory; more are read from global memory

// Sums of three numbers over the block, and over the threads before this one; by_warp: every warp by itself.
struct Sums {
    int before[3], all[3];
};
__device__ __forceinline__ Sums block_sums(int (*scratch)[kPlanThreads / 32], bool by_warp, int a, int b, int c) {
    constexpr int kWarps = kPlanThreads / 32;
    const int lane = lane_id(), warp = threadIdx.x >> 5, mine[3] = {a, b, c};
    Sums s;
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        int x = mine[q];
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
            if (lane >= o) x += y;
        }
        s.before[q] = x - mine[q];
        s.all[q] = __shfl_sync(0xFFFFFFFFu, x, 31);
        if (!by_warp && lane == 31) scratch[q][warp] = x;
    }
    if (by_warp) return s;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        s.all[q] = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) s.before[q] += s.all[q];
            s.all[q] += scratch[q][w];
        }
    }
    __syncthreads();
    return s;
}
// Where every CTA begins, and the units that are joined at the beginnings; by the block that wrote the entries.  held: they are in `entries`.
template <bool kWin>
__device__ __forceinline__ void plan_starts(const AttnParams& p, const PlanSeq* entries, bool held, int last_s, int total, int parts, int chunk) {
    const int tid = threadIdx.x;
    for (int i = tid; i < p.ctas; i += kPlanThreads) {
        PlanStart st = {};
        PlanJoin j = {};
        if (i < parts) {
            st.x = part_first(total, parts, i);
            st.x1 = part_first(total, parts, i + 1);
            st.chunk = chunk;
            int lo = kWin ? 1 : 0, hi = last_s;  // the last entry whose position is not above x: one that has any, as the ones behind it begin above x
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if ((held ? entries[mid].cost0 : __ldcg(&p.seq[mid].cost0)) <= st.x)
                    lo = mid;
                else
                    hi = mid - 1;
            }
            PlanSeq q;
            if (held)
                q = entries[lo];
            else
                load_seq(q, p.seq + lo);
            const int R = q.n * p.group, hc = head_cost(R, q.kt, chunk), local = st.x - q.cost0, full = padded(kTwoTiles * q.kt, chunk);
            st.s = lo;
            st.h = local / hc;
            int rem = local - st.h * hc;
            st.mt = min(rem / full, row_tiles2(R) - 1);
            rem -= full * st.mt;
            const int w = unit_weight(R, st.mt);
            st.k = min((rem + w - 1) / w, q.kt);  // (behind the tiles: kt, as if at their end)
            st.x += st.k * w - rem;
            st.q = q;
            if ((kWin || p.shared == 0) && st.k > 0 && st.k < q.kt) {  // (else the stretch begins with a unit)
                const UnitAt un = unit_at(q, p.group, st.h, st.mt, chunk);
                j.f = cta_of(un.x0, total, parts);
                // the tiles ahead of this CTA's are those of the unit's first CTA, and this one has some
                if (first_tile(un, total, parts, j.f + 1) == st.k && first_tile(un, total, parts, i + 1) > st.k)
                    j.rows = min(kUnitRows, R - st.mt * kUnitRows);
                j.l = cta_of(un.x0 + (un.kt - 1) * un.w, total, parts);
                j.total = total, j.parts = parts;
                j.x0 = un.x0, j.w = un.w, j.kt = un.kt;
                j.s = kWin ? q.b + 1 : lo, j.h = st.h, j.r0 = st.mt * kUnitRows;
                if (kWin) j.node0 = q.node0;
            }
        }
        p.start[i] = st;
        p.join[i] = j;
        p.ready[i] = 0;
    }
}

// ---- walking along a CTA's stretch -----------------------------------------------------------------------------------
// A bounded wait whose polls sleep: the polls of warps that wait would otherwise take the shared-memory pipe from those that work.  (mbar_wait_bounded_hint
// with its loop kept small: unrolled, a wait is 2 KB of code, thirty of them are more than the instruction cache next to the cores, and the softmax
// waited a quarter of its time for instructions.)
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*gave_up) return false;
#pragma unroll 1
    for (uint32_t it = 0; it < GRAFT_SPIN_LIMIT; ++it) {
        if (mbar_try_wait_hint(bar, parity, kWaitNs)) return true;
        if ((it & 15u) == 15u && *gave_up) return false;
    }
    *gave_up = 1;
    return false;
}

// What the warps of a CTA are told of a piece.
struct Piece {
    int T;          // key tiles; 0: there are no more pieces
    int s, h;       // entry of the plan, key head
    int first, end; // first slot, and how many slots there are
    int n, base;    // new rows, slots before the first of them
    int r0, rows;   // first row of the unit among the entry's, rows of the unit
    int unit;       // number of the unit
    int head, whole;  // the piece begins with the unit's first tile; is all of it
    int b, node0, gap, lo, reach;  // kWin: the sequence, its nodes before the entry's, slots left out, the place that the first row's window begins at, and
                                   // how far behind it the last one begins
};
template <bool kWin>
struct Walk {
    const PlanSeq* seq;
    int last_s, Hk, group, shared, window;
    int x, x1, chunk;
    int s, h, mt, k;
    bool own;  // entries are in this CTA's shared memory
    PlanSeq q;
    __device__ __forceinline__ void of(const AttnParams& p) {
        Hk = p.c.kv_heads;
        group = p.group;
        shared = kWin ? 0 : p.shared;
        window = p.window;
    }
    __device__ __forceinline__ void begin(const AttnParams& p, int cta) {
        seq = p.seq;
        last_s = kWin ? __ldcg(&p.head->entries) : p.batch;
        own = false;
        of(p);
        const PlanStart* from = p.start + cta;
        const int4 st = __ldcg((const int4*)from), en = __ldcg((const int4*)from + 1);
        load_seq(q, &from->q);
        s = st.x, h = st.y, mt = st.z, k = st.w, x = en.x, x1 = en.y, chunk = en.z;
    }
    // the same from entries of its own and where its stretch begins
    __device__ __forceinline__ void begin(const AttnParams& p, const PlanSeq* entries, const PlanStart& from) {
        seq = entries;
        last_s = p.batch;
        own = true;
        of(p);
        q = entries[from.s];
        s = from.s, h = from.h, mt = 0, k = from.k, x = from.x, x1 = from.x1, chunk = 1;
    }
    __device__ __forceinline__ bool next(Piece& pc) {
        if (x >= x1) return false;
        int R = q.n * group;
        if (k >= q.kt) {
            x = padded(x, chunk);
            if (x >= x1) return false;
        }
        while (q.n == 0 || k >= q.kt) {  // the next unit
            k = 0;
            mt += 1;
            if (q.n == 0 || mt >= row_tiles2(R)) {
                mt = 0;
                h += 1;
                if (q.n == 0 || h >= Hk) {
                    h = 0;
                    s += 1;
                    if (s > last_s) return false;
                    if (kWin && own)
                        q = seq[s];
                    else
                        load_seq(q, seq + s);
                    R = q.n * group;
                }
            }
        }
        const int w = unit_weight(R, mt), left = (x1 - x + w - 1) / w, kv0 = s == 0 ? 0 : shared;
        pc.T = min(left, q.kt - k);
        pc.s = s, pc.h = h;
        pc.first = kv0 + k * kTile;
        pc.end = s == 0 ? shared : q.base + q.n;
        pc.n = q.n, pc.base = q.base;
        pc.r0 = mt * kUnitRows;
        pc.rows = min(kUnitRows, R - pc.r0);
        pc.unit = q.unit0 + h * row_tiles2(R) + mt;
        pc.head = k == 0;
        pc.whole = k == 0 && pc.T == q.kt && shared == 0;
        if (kWin) {
            pc.b = q.b, pc.node0 = q.node0, pc.gap = q.gap, pc.reach = q.unit0;
            pc.lo = q.base - window + 1 - q.gap;
            pc.end -= q.gap, pc.base -= q.gap;
        }
        x += pc.T * w;
        k += pc.T;
        return true;
    }
};

// the sequence, node and query head of row r of an entry's rows
__device__ __forceinline__ void row_of(const AttnParams& p, int s, int r, int& b, int& node, int& g) {
    const int f = r / p.group;
    g = r - f * p.group;
    b = s - 1;
    node = f;
    if (s == 0) {  // all sequences' nodes in a row: the last sequence whose first node is not behind f
        int lo = 1, hi = p.batch;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (__ldcg(&p.seq[mid].node0) <= f)
                lo = mid;
            else
                hi = mid - 1;
        }
        b = lo - 1;
        node = f - __ldcg(&p.seq[lo].node0);
    }
}

// the same of a row of a piece
template <bool kWin>
__device__ __forceinline__ void row_of(const AttnParams& p, const volatile Piece& pc, int r, int& b, int& node, int& g) {
    if (kWin) {
        const int f = r / p.group;
        g = r - f * p.group;
        b = pc.b;
        node = pc.node0 + f;
    } else
        row_of(p, pc.s, r, b, node, g);
}

// which of the 128 slots from `first` on row `node` sees; end: slots there are.  (Words of the mask are loaded without branches, all together.)
__device__ __noinline__ void seen_words(const uint32_t* mask_row, int words, int node, int base, int end, int first, uint32_t (&sees)[4]) {
    const int j0 = first - base, w0 = j0 >> 5;  // new row of the first slot (below 0: slots of the prefix) and its word
    uint32_t m[5] = {0, 0, 0, 0, 0};
    if (mask_row != nullptr)
#pragma unroll
        for (int x = 0; x < 5; ++x) {
            const uint32_t v = __ldg(mask_row + min(max(w0 + x, 0), words - 1));
            m[x] = w0 + x >= 0 && w0 + x < words ? v : 0;
        }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const auto low = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1; };  // the n lowest bits
        const int j = j0 + 32 * x;
        const uint32_t tree = mask_row != nullptr ? __funnelshift_r(m[x], m[x + 1], j0 & 31) : low(node - j + 1);
        sees[x] = (tree | low(-j)) & low(end - first - 32 * x);
    }
}

// Of the new rows from j on that `tree` has, those that a row further than the window behind the first one sees, by their own positions.
__device__ __noinline__ uint32_t near_rows(const AttnParams& p, const int32_t* position, uint32_t tree, int j, int at_base, int step) {
    for (uint32_t left = tree; left != 0; left &= left - 1) {
        const int y = __ffs(left) - 1, at = window_step(position, j + y, at_base);
        if (step - at >= p.window && at + at_base >= p.sinks) tree &= ~(1u << y);
    }
    return tree;
}
// The same behind a window: of the 128 places from `first` on, for row i of a block (the sequence's row `node`) whose first row stands in place
// `base`; step: how far behind that one's position its own is.
__device__ __noinline__ void window_words(const AttnParams& p, int gap, int lo, int base, int end, int b, int node, int i, int step, int first,
                                          uint32_t (&sees)[4]) {
    const int j0 = first - base, w0 = j0 >> 5;
    uint32_t m[5] = {0, 0, 0, 0, 0};
    if (p.mask != nullptr && first + kTile > base) {
        const uint32_t* mask_row = p.mask + ((size_t)b * p.nmax + node) * p.words;
#pragma unroll
        for (int x = 0; x < 5; ++x) {
            const uint32_t v = __ldg(mask_row + min(max(w0 + x, 0), p.words - 1));
            m[x] = w0 + x >= 0 && w0 + x < p.words ? v : 0;
        }
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int j = j0 + 32 * x, place = first + 32 * x;
        const uint32_t near = low_bits(p.sinks - place) | ~low_bits(lo + step - place);
        const uint32_t there = low_bits(end - place);
        uint32_t tree = __funnelshift_r(m[x], m[x + 1], j0 & 31) & there;
        // (with a mask a block is a whole tree: i is its node; a path may be longer than the window)
        if (p.mask != nullptr && step >= p.window) tree = near_rows(p, p.position + (size_t)b * p.nmax, tree, j, base + gap, step);
        sees[x] = (p.mask != nullptr ? (low_bits(-j) & near) | tree : low_bits(i - j + 1) & near) & there;
    }
}
// ---- small parts ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm volatile("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ bool not_finite2(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// the larger magnitudes of two pairs of bf16 (signs mean nothing), NaN where one is
__device__ __forceinline__ uint32_t max_magnitude2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// log(2^m sum); m = -inf: nothing seen, or nothing but what is not a number
__device__ __forceinline__ float log_sum(float m, float sum) {
    return sum == 0.0f ? -INFINITY : (m > -INFINITY ? m * 0.69314718f : 0.0f) + logf(sum);
}

// (the asm statements of a pass over scores are volatile: they stay in the order that hides their latencies)
__device__ __forceinline__ float ex2_in_order(float x) {
    float y;
    asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- joining the pieces ----------------------------------------------------------------------------------------------
constexpr int kJoinThreads = 256;
constexpr int kJoinRows = 32;
constexpr int kJoinMost = 320;  // pieces of a block's rows: no more than CTAs and units (three at most)

struct JoinPiece {
    int slot, shift, lo, hi;  // rows lo .. hi - 1 of the block are rows lo + shift .. of the piece
};
struct JoinList {
    JoinPiece piece[kJoinMost];
    int n;
};

// The pieces of a unit, to the list; a warp calls it, a lane a CTA (of f .. l) that may have tiles of it.  Behind a shared prefix (unit >= 0) a piece's
// slot is the unit's number and the CTA's added up; else the unit's first CTA has it in the odd one of its two slots.
__device__ __forceinline__ void list_unit(JoinList& j, const UnitAt& u, int f, int l, int total, int parts, int unit, int shift, int lo, int hi) {
    const int lane = lane_id();
    for (int d0 = f; d0 <= l; d0 += 32) {
        const int d = d0 + lane;
        const bool has = d <= l && first_tile(u, total, parts, d + 1) > first_tile(u, total, parts, d);
        const unsigned all = __ballot_sync(0xFFFFFFFFu, has);
        const int n = j.n, at = n + __popc(all & ((1u << lane) - 1));
        __syncwarp();
        if (has && at < kJoinMost) j.piece[at] = {unit >= 0 ? unit + d : d == f ? 2 * d + 1 : 2 * d, shift, lo, hi};
        if (lane == 0) j.n = min(n + __popc(all), kJoinMost);
        __syncwarp();
    }
}

// 32 rows of a unit from the pieces on the list: a lane a row, a warp some of the columns.  Pieces are added in their order along the line, results
// repeat; kAhead are on their way at a time (kernels that join have two, as most units were cut once, and four blocks an SM: trees behind a window 75.5 -> 73.1 us).
template <int D, int kAhead>
__device__ __forceinline__ void join_rows(const AttnParams& p, const JoinList& j, bool live, size_t out_row) {
    constexpr int kWarps = kJoinThreads / 32, kQuads = D / 4 / kWarps;  // groups of four columns a warp
    const int lane = lane_id(), warp = threadIdx.x >> 5, n = j.n;
    float m = -INFINITY, l = 0.0f;
    float o[4 * kQuads] = {};
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        float2 ml[kAhead];
        float4 v[kAhead][kQuads];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {  // (rows that a piece does not have, and pieces behind the last, weigh nothing)
            const JoinPiece a = j.piece[min(i0 + i, n - 1)];
            const bool mine = i0 + i < n && lane >= a.lo && lane < a.hi;
            const int r = mine ? lane + a.shift : 0;
            const float2 x = __ldcg(p.part_ml + (size_t)a.slot * p.part_rows + r);
            ml[i] = mine ? x : make_float2(-INFINITY, 0.0f);
            const float4* from = (const float4*)p.part_o + ((size_t)a.slot * (D / 4) + warp * kQuads) * p.part_rows + r;
#pragma unroll
            for (int y = 0; y < kQuads; ++y) {
                const float4 z = __ldcg(from + y * p.part_rows);
                v[i][y] = mine ? z : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const float now = fmaxf(m, ml[i].x), f0 = m > -INFINITY ? ex2_approx(m - now) : 0.0f;
            const float f1 = ml[i].x > -INFINITY ? ex2_approx(ml[i].x - now) : 0.0f;
            m = now;
            l = l * f0 + ml[i].y * f1;
#pragma unroll
            for (int y = 0; y < kQuads; ++y) {
                o[4 * y] = o[4 * y] * f0 + f1 * v[i][y].x, o[4 * y + 1] = o[4 * y + 1] * f0 + f1 * v[i][y].y;
                o[4 * y + 2] = o[4 * y + 2] * f0 + f1 * v[i][y].z, o[4 * y + 3] = o[4 * y + 3] * f0 + f1 * v[i][y].w;
            }
        }
    }
    if (!live) return;
    const float inv = l != 0.0f ? 1.0f / l : 1.0f;
    uint2* to = (uint2*)(p.out + out_row * D + warp * kQuads * 4);
#pragma unroll
    for (int x = 0; x < kQuads; ++x)
        to[x] = make_uint2(pack_bf16(o[4 * x] * inv, o[4 * x + 1] * inv), pack_bf16(o[4 * x + 2] * inv, o[4 * x + 3] * inv));
    if (p.lse && warp == 0) p.lse[out_row] = log_sum(m, l);
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
// Single tokens (up to eight rows a sequence and key head) are bound by the bytes of K and V, and a tile of 128 rows would be nearly empty.
// Here a warp takes 16 slots at a time into the fragments of m16n8k16 products, S^T = K Q^T and O^T = V^T P^T, with slots and head_dim in
// the long directions and the rows in the short one; e4m3 entries become f16 (K) and bf16 (V) in registers, their slots' powers of two go to scores
// and weights.  The order of head_dim inside a product is free, so a lane loads pieces of 16 bytes straight into what it multiplies: of K, a quarter of those of two slots; of V, an eighth of four.  The next
// step's K is asked for when this one's scores are done, and V when its products are: the warps of an SM then have 50 to 60 KB under way.
// 64 sequences of 2000 to 16000 slots, 8 key heads of 128: bf16 354 us (6.6 TB/s; through the tiles of 128 rows 417), e4m3 226 us (5.3
// TB/s; 553), which instructions bound, three warps a scheduler to hide their latencies.  With K and V turned into bf16 and multiplied by their slots'
// powers: 500 instructions for 16 slots, 275 us.  Before pieces' own cost was counted (371 and 288): through a ring of cp.async in shared memory 543 and 295;
// with 8 warps of two steps 297, with 16 warps 294 (registers spill).  Behind a window of 4096, 64 sequences: e4m3 114 us.
constexpr int kFewRows = 8;

template <int D, bool Q8, bool kWin>
struct FewShape {
    static constexpr int kBytes = Q8 ? 1 : 2;
    static constexpr int kK = D / 4 * kBytes / 16;                                     // pieces of a slot's K that a lane has
    static constexpr int kPiece = D / 8 * kBytes < 16 ? D / 8 * kBytes : 16;           // bytes of a piece of V (D = 64, e4m3: 8)
    static constexpr int kV = D / 8 * kBytes / kPiece;                                 // pieces of a slot's V
    // As many warps an SM as have room in registers for a step's K and V (16 to 64 of them) beside Q and O.  In two CTAs one begins a piece while the
    // other is under way: e4m3 slots behind a window, 12 warps an SM, 64 tokens 121 -> 114 us, 12 tokens 33.0 -> 29.9.  Over bf16 slots there are 8, whose
    // loads fill the SM's share of the memory either way (64 tokens 168.0 and 168.8, 4 tokens 19.8 and 20.3).
    static constexpr bool kPair = D == 64 || (Q8 && kWin);
    static constexpr int kWarps = Q8 && D == 128 ? (kPair ? 6 : 12) : 8, kThreads = 32 * kWarps;
    static constexpr int kCtas = kPair ? 2 : 1;
    static constexpr size_t kSmem = (size_t)kWarps * kFewRows * (D + 2) * sizeof(float);
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// four e4m3 numbers as f16, which holds them all
__device__ __forceinline__ uint2 e4m3x4_to_f16(uint32_t w) {
    uint2 r;
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n cvt.rn.f16x2.e4m3x2 %1, hi;\n}" : "=r"(r.x), "=r"(r.y) : "r"(w));
    return r;
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }  // -126 .. 127
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint4 load_once(const uint8_t* p) {
    uint4 r;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
// The plan of few rows behind a window, worked out by every CTA for itself: a launch ahead takes longer than two loads and a sum over the sequences (one
// token behind a window of 4096 18.4 -> 16.2 us, 64 of them, e4m3, 152 -> 130, before the steps below).  More sequences than this have a launch ahead, as their plan takes a block its time.
// Numbers that are wrong by themselves leave a sequence without rows; its pages are looked at with its pieces.
constexpr int kSelfSeqs = 192;
struct SelfPlan {
    PlanSeq entry[kSelfSeqs + 1];
    PlanStart start;
    int sums[kSelfSeqs / 32];
    int total;
};
__device__ __forceinline__ void self_plan(const AttnParams& p, SelfPlan& sm) {
    const int b = threadIdx.x, lane = b & 31, warp = b >> 5;
    PlanSeq q = {};
    int cost = 0, before = 0;
    if (b < kSelfSeqs) {
        if (b < p.batch) {
            const int n = p.count[b], base = p.prefix_len[b] - 1;
            const bool fine = n >= 0 && n <= p.rows && base >= 0 && (long long)base + n <= (long long)p.c.width << p.c.page_shift;
            if (p.status && blockIdx.x == 0 && (!fine || n == 0)) p.status[b] = fine ? 0 : GRAFT_ST_BAD_CACHE;
            if (fine && n > 0) {
                q.n = n, q.base = base, q.b = b;
                q.unit0 = n - 1;  // (at most eight rows)
                q.gap = gap_of(p, base);
                q.kt = (base + n - q.gap + kTile - 1) / kTile;
                cost = p.c.kv_heads * padded(kOneTile * q.kt, 1);
            }
        }
        before = cost;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, before, o);
            if (lane >= o) before += y;
        }
        if (lane == 31) sm.sums[warp] = before;
        before -= cost;
    }
    if (b == 0) sm.start = PlanStart{};
    __syncthreads();
    int total = 0;
    for (int w = 0; w < kSelfSeqs / 32; ++w) {
        if (w == warp) before += total;
        total += sm.sums[w];
    }
    const int parts = min(p.ctas, total), i = blockIdx.x;
    if (b < p.batch && b < kSelfSeqs) {
        q.cost0 = before;
        sm.entry[b + 1] = q;
        if (i < parts) {
            const int x = part_first(total, parts, i);
            if (cost > 0 && before <= x && x < before + cost) {  // the stretch begins here
                const int unit = padded(kOneTile * q.kt, 1), h = (x - before) / unit, rem = x - before - h * unit;
                PlanStart st = {};
                st.s = b + 1, st.h = h;
                st.k = min((rem + kOneTile - 1) / kOneTile, q.kt);
                st.x = x + st.k * kOneTile - rem;
                st.x1 = part_first(total, parts, i + 1);
                sm.start = st;
            }
        }
    }
    if (b == 0) sm.total = total, sm.entry[0] = PlanSeq{};
    __syncthreads();
}

// Up to eight rows of a unit from the pieces on the list, behind a window: a lane a row and every fourth piece, a warp some of the columns; the four
// lanes of a row are added in the end, so results repeat.  Eight pieces are on their way at a time: one token behind a window of 4096, whose units
// have 18 pieces, 16.2 -> 12.4 us beside a lane a row and four pieces at a time (sixteen at a time 12.6, registers spill).
template <int D, int kWarps>
__device__ __forceinline__ void join_few(const AttnParams& p, const JoinList& j, int R, size_t out_row0) {
    constexpr int kQuads = (D / 4 + kWarps - 1) / kWarps, kEach = 2;
    const int lane = lane_id(), warp = threadIdx.x >> 5, n = j.n, row = lane & 7, at = lane >> 3;
    const int r = row < R ? row : 0;
    float m = -INFINITY, l = 0.0f;
    float o[4 * kQuads] = {};
    for (int i0 = 0; i0 < n; i0 += 4 * kEach) {
        float2 ml[kEach];
        float4 v[kEach][kQuads];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = i0 + 4 * i + at;
            const size_t slot = j.piece[min(e, n - 1)].slot;
            ml[i] = make_float2(-INFINITY, 0.0f);
            if (e < n) ml[i] = __ldcg(p.part_ml + slot * p.part_rows + r);
#pragma unroll
            for (int y = 0; y < kQuads; ++y) {
                v[i][y] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (e < n && warp + y * kWarps < D / 4)
                    v[i][y] = __ldcg((const float4*)p.part_o + (slot * (D / 4) + warp + y * kWarps) * p.part_rows + r);
            }
        }
        float now = m;
#pragma unroll
        for (int i = 0; i < kEach; ++i) now = fmaxf(now, ml[i].x);
        const float f0 = m > -INFINITY ? ex2_approx(m - now) : 0.0f;
        m = now;
        l *= f0;
#pragma unroll
        for (int x = 0; x < 4 * kQuads; ++x) o[x] *= f0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const float f = ml[i].x > -INFINITY ? ex2_approx(ml[i].x - m) : 0.0f;
            l += f * ml[i].y;
#pragma unroll
            for (int y = 0; y < kQuads; ++y)
                o[4 * y] += f * v[i][y].x, o[4 * y + 1] += f * v[i][y].y, o[4 * y + 2] += f * v[i][y].z, o[4 * y + 3] += f * v[i][y].w;
        }
    }
    float all = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
    all = fmaxf(all, __shfl_xor_sync(0xFFFFFFFFu, all, 16));
    const float f = m > -INFINITY ? ex2_approx(m - all) : 0.0f;
    const auto sum4 = [&](float x) {
        x *= f;
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
        return x + __shfl_xor_sync(0xFFFFFFFFu, x, 16);
    };
    l = sum4(l);
    const float inv = l != 0.0f ? 1.0f / l : 1.0f;
#pragma unroll
    for (int y = 0; y < kQuads; ++y) {
        const float a = sum4(o[4 * y]), b = sum4(o[4 * y + 1]), c = sum4(o[4 * y + 2]), d = sum4(o[4 * y + 3]);
        const int quad = warp + y * kWarps;
        if (at == 0 && row < R && quad < D / 4)
            ((uint2*)(p.out + (out_row0 + (row / p.group) * (size_t)p.q_heads + row % p.group) * D))[quad] =
                make_uint2(pack_bf16(a * inv, b * inv), pack_bf16(c * inv, d * inv));
    }
    if (p.lse && warp == 0 && at == 0 && row < R) p.lse[out_row0 + (row / p.group) * (size_t)p.q_heads + row % p.group] = log_sum(all, l);
}

template <int D, bool Q8, bool kWin>
__global__ void __launch_bounds__(FewShape<D, Q8, kWin>::kThreads, FewShape<D, Q8, kWin>::kCtas) few_attn_kernel(const __grid_constant__ AttnParams p) {
    using S = FewShape<D, Q8, kWin>;
    constexpr int kBytes = S::kBytes, kK = S::kK, kV = S::kV, kPiece = S::kPiece, kWarps = S::kWarps;
    constexpr int kCk = 16 / kBytes, kCv = kPiece / kBytes;  // numbers of a piece
    extern __shared__ __align__(16) float few_sm[];  // [warps][rows][D], then [warps][rows][2]
    float* const sm_ml = few_sm + kWarps * kFewRows * D;
    __shared__ Piece pc;
    __shared__ JoinList list;
    __shared__ int cut_f, cut_x0, cut_kt, last;  // of the unit that the piece is of
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q4 = lane & 3;
    const CacheView& c = p.c;
    const int shift = c.page_shift, low = (1 << shift) - 1;
    const float c2 = p.c2, most = kMostGrowth / c2;
    pdl_launch_dependents();
    pdl_wait();
    Walk<kWin> walk;
    __shared__ uint4 self_sm[kWin ? (sizeof(SelfPlan) + 15) / 16 : 1];
    SelfPlan* const self = (SelfPlan*)self_sm;
    const bool selfish = kWin && p.self_plan;
    static_assert(S::kThreads >= kSelfSeqs, "a thread a sequence");
    if (selfish) self_plan(p, self[0]);
    const int total = selfish ? self[0].total : __ldcg(&p.head->total), parts = selfish ? min(p.ctas, total) : __ldcg(&p.head->parts);
    if (tid == 0) {
        if (selfish)
            walk.begin(p, self[0].entry, self[0].start);
        else
            walk.begin(p, blockIdx.x);
    }
    for (;;) {
        if (tid == 0) {
            Piece x;
            if (!walk.next(x)) x.T = 0;
            pc = x;
            if (x.T > 0 && !x.whole) {
                cut_x0 = unit_at(walk.q, p.group, walk.h, 0, 1).x0;
                cut_kt = walk.q.kt;
                cut_f = cta_of(cut_x0, total, parts);
                list.n = 0;
            }
        }
        __syncthreads();
        const int T = pc.T;
        if (T == 0) break;
        const int h = pc.h, b = kWin ? pc.b : pc.s - 1, base = pc.base, end = pc.end, R = pc.rows, first0 = pc.first;
        const int gap = kWin ? pc.gap : 0, lo = kWin ? pc.lo : 0, border1 = kWin ? lo + pc.n - 1 : 0;
        const int32_t* table = c.table + (size_t)b * c.width;
        // A step's 16 slots lie in one page; the warps take steps by turns.
        const int all = min(8 * T, (end - first0 + 15) / 16), steps = warp < all ? (all - warp + kWarps - 1) / kWarps : 0;
        const auto slot_of = [&](int step) { return first0 + (warp + step * kWarps) * 16; };  // (kWin: the place)
        const auto stored_at = [&](int step) { return kWin ? slot_at(p, gap, slot_of(step)) : slot_of(step); };
        const auto page_of = [&](int step) {
            const int page = __ldg(table + (stored_at(min(step, steps - 1)) >> shift));
            return kWin && (unsigned)page >= (unsigned)c.n_pages ? 0 : page;  // (what is read there is not used, see `fine`)
        };
        const auto row_at = [&](int step, int page) { return cache_row(c, page, h, stored_at(step) & low); };
        uint4 kr[2][kK], k_exps = {}, v_exps = {};  // (exponents of all 16 slots)
        uint32_t vr[4][4 * kV];
        const auto bring_k = [&](size_t row0) {
            const uint8_t* const k = c.k + (row0 + g) * (D * kBytes) + q4 * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int y = 0; y < kK; ++y) kr[i][y] = load_once(k + i * 8 * (D * kBytes) + y * 64);
            }
            if (Q8) k_exps = __ldg((const uint4*)(c.k_exp + row0));
        };
        const auto bring_v = [&](size_t row0) {
            const uint8_t* const v = c.v + (row0 + 2 * q4) * (D * kBytes) + g * kPiece;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int y = 0; y < kV; ++y) {
                    const uint8_t* const from = v + ((i & 1) + 8 * (i >> 1)) * (D * kBytes) + y * 8 * kPiece;
                    if (kPiece == 16) {
                        const uint4 u = load_once(from);
                        vr[i][4 * y] = u.x, vr[i][4 * y + 1] = u.y, vr[i][4 * y + 2] = u.z, vr[i][4 * y + 3] = u.w;
                    } else {
                        const uint2 u = __ldg((const uint2*)from);
                        vr[i][0] = u.x, vr[i][1] = u.y, vr[i][2] = vr[i][3] = 0;
                    }
                }
            if (Q8) v_exps = __ldg((const uint4*)(c.v_exp + row0));
        };
        // Whether the sequence's pages are all there: this thread's share of them.
        bool fine = true;
        if (selfish) {
            const int last_page = (end + gap - 1) >> shift, sinks = p.sinks > 0 ? min((p.sinks - 1) >> shift, last_page) : -1;
            for (int i = tid; i <= sinks; i += S::kThreads) fine = fine && (unsigned)__ldg(table + i) < (unsigned)c.n_pages;
            for (int i = max(max(lo + gap, 0) >> shift, sinks + 1) + tid; i <= last_page; i += S::kThreads)
                fine = fine && (unsigned)__ldg(table + i) < (unsigned)c.n_pages;
        }
        size_t row0 = 0;
        int page = 0;
        if (steps > 0) {
            row0 = row_at(0, page_of(0));
            page = page_of(1);
            bring_k(row0);
            bring_v(row0);
        }
        // rows of Q: lane (g, q4) has row g of the second operand, in the order of K's pieces
        uint32_t qf[D / 8];
        {
            const bool live = g < R;
            const int node = live ? g / p.group : 0, hg = live ? g - node * p.group : 0;
            const uint8_t* from = p.q + 2 * (((long long)b * p.rows + node) * p.q_stride + (long long)(h * p.group + hg) * D);
            const uint32_t keep = live ? p.q_keep : 0u;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const int d = 8 * i / kCk * (4 * kCk) + q4 * kCk + 8 * i % kCk;
                uint4 u = __ldg((const uint4*)(from + 2 * d));
                u.x = (u.x ^ p.q_flip) & keep, u.y = (u.y ^ p.q_flip) & keep, u.z = (u.z ^ p.q_flip) & keep, u.w = (u.w ^ p.q_flip) & keep;
                qf[4 * i] = u.x, qf[4 * i + 1] = u.y, qf[4 * i + 2] = u.z, qf[4 * i + 3] = u.w;
            }
        }
        // Over e4m3 slots: f16 holds e4m3 numbers, and a row of Q when its largest number is brought to 2^14 by a power of two, unless others are
        // 2^31 times smaller; scores take the powers of both back.  With a row that f16 does not hold bit for bit, Q stays as it is and K becomes bf16
        // (rare; 64 tokens behind a window of 4096 114 us, with such rows 122).
        float q_down[2] = {1.0f, 1.0f};  // of rows 2 q4, 2 q4 + 1
        bool q_far = false, q_wide = false;
        if (Q8) {
            uint32_t most2 = 0;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) most2 = max_magnitude2(most2, qf[i]);
            uint32_t top = max(most2 & 0x7FFFu, most2 >> 16 & 0x7FFFu);
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const int up = top == 0 ? 0 : min(127 + 14 - (int)(top >> 7), 126);  // (from -114 on)
            const float f = power_of_two(up), down = power_of_two(-up);
            uint32_t qh[D / 8];
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const float lo = __uint_as_float(qf[i] << 16), hi = __uint_as_float(qf[i] & 0xFFFF0000u);
                asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(qh[i]) : "f"(hi * f), "f"(lo * f));
                const float2 back = __half22float2(*(const __half2*)&qh[i]);
                const float2 again = make_float2(back.x * down, back.y * down);
                q_wide = q_wide || again.x < lo || again.x > lo || again.y < hi || again.y > hi;  // (what is not a number is none in f16 either)
            }
            q_wide = __any_sync(0xFFFFFFFFu, q_wide);
            if (!q_wide) {
#pragma unroll
                for (int i = 0; i < D / 8; ++i) qf[i] = qh[i];
                q_far = __any_sync(0xFFFFFFFFu, up > 60 || up < -60);
#pragma unroll
                for (int i = 0; i < 2; ++i) q_down[i] = power_of_two(-__shfl_sync(0xFFFFFFFFu, up, (2 * q4 + i) * 4));
            }
        }
        float o[D / 16][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, upto[2] = {-INFINITY, -INFINITY}, off[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        // (its steps with K as bf16 are code of their own: a branch inside of them costs 2 %)
        const auto steps_of_piece = [&](auto wide) {
            constexpr bool kF16 = Q8 && !decltype(wide)::value;
            for (int step = 0; step < steps; ++step) {
                const int s0 = slot_of(step);
                const bool more_steps = step + 1 < steps;
                const size_t row1 = row_at(step + 1, page);
                page = page_of(step + 2);
                // powers of two of K's slots g, g + 8
                uint32_t ke[2] = {0, 0};
                if (Q8)
#pragma unroll
                    for (int i = 0; i < 2; ++i) ke[i] = __byte_perm(i ? k_exps.z : k_exps.x, i ? k_exps.w : k_exps.y, g) & 255;
                // ---- scores: rows 2 q4, 2 q4 + 1 at slots g, g + 8
                float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, s2[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                uint32_t f[2] = {0, 0}, more[2] = {kOneBf16x2, kOneBf16x2};
                if (Q8 && !kF16)
#pragma unroll
                    for (int i = 0; i < 2; ++i) e4m3_factors(ke[i], f[i], more[i]);
#pragma unroll
                for (int y = 0; y < kK; ++y) {
                    uint2 a[4 / kBytes][2];
#pragma unroll
                    for (int x = 0; x < 4 / kBytes; ++x)  // four numbers of the lane's a product
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t w[4] = {kr[i][y].x, kr[i][y].y, kr[i][y].z, kr[i][y].w};
                            a[x][i] = kF16 ? e4m3x4_to_f16(w[x]) : Q8 ? e4m3x4_to_bf16(w[x], f[i], kOneBf16x2) : make_uint2(w[2 * x & 3], w[(2 * x + 1) & 3]);
                        }
#pragma unroll
                    for (int x = 0; x < 4 / kBytes; ++x) {
                        const int ks = y * (4 / kBytes) + x;
                        const auto mma = kF16 ? mma_16816_f16 : mma_16816;
                        mma(x & 1 ? s2 : s, a[x][0].x, a[x][1].x, a[x][0].y, a[x][1].y, qf[2 * ks], qf[2 * ks + 1]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i] += s2[i];
                    if (Q8 && !kF16) s[i] *= __uint_as_float(more[i >> 1] << 16);  // (what is above bf16's largest power)
                }
                if (kF16) {
                    if (q_far || __any_sync(0xFFFFFFFFu, max(ke[0] - 67, ke[1] - 67) > 120)) {  // (rare: in two steps, and what is not a number)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int e = (int)ke[i >> 1] - 127, d = (__float_as_int(q_down[i & 1]) >> 23) - 127, e1 = e >> 1, d1 = d >> 1;
                            s[i] = ke[i >> 1] == 255 ? __int_as_float(0x7FFFFFFF) : s[i] * power_of_two(e1 + d1) * power_of_two(e - e1 + d - d1);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[i] *= q_down[i & 1] * __uint_as_float(ke[i >> 1] << 23);
                    }
                }
                if (more_steps) bring_k(row1);
                // What e4m3_pair_small makes of V lacks a power of two a slot, 2^(e + 120).  It goes to the slot's weights, where it changes no rounding, as long
                // as those stay below 2^128; else (rare, and not numbers) to V, with what is above bf16's largest power going to the weights.
                uint32_t f2[2] = {0, 0}, x[2] = {0, 0};  // (x: the exponents of two slots)
                float big[2] = {1.0f, 1.0f};
                bool large_v = false;
                if (Q8) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        x[i] = __byte_perm(i ? v_exps.z : v_exps.x, i ? v_exps.w : v_exps.y, 2 * q4 | (2 * q4 + 1) << 8) & 0x00FF00FFu;
                        big[i] = __uint_as_float(((__byte_perm(i ? v_exps.z : v_exps.x, i ? v_exps.w : v_exps.y, g) & 255) + 120) << 23);
                    }
                    large_v = __any_sync(0xFFFFFFFFu, ((x[0] + 0x00810081u) | (x[1] + 0x00810081u)) & 0x01000100u);  // (one above 126: weights are up to 2^8)
                    if (large_v)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t fa, fb, y;
                            e4m3_factors(x[i] & 255, fa, y), e4m3_factors(x[i] >> 16, fb, y);
                            f2[i] = __byte_perm(fa, fb, 0x5410);
                            const uint32_t pair = __shfl_sync(0xFFFFFFFFu, x[i], g >> 1);
                            e4m3_factors(g & 1 ? pair >> 16 : pair & 255, fa, y);
                            big[i] = __uint_as_float(y << 16);
                        }
                }
                const bool masked = s0 + 16 > base || (kWin && s0 < border1 && s0 + 16 > p.sinks);
                bool spoilt[4] = {false, false, false, false};
                uint32_t sees = 0;  // bit i: score i is of a slot that its row sees
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int slot = s0 + g + 8 * (i >> 1), r = 2 * q4 + (i & 1), j = slot - base, node = r / p.group;
                        bool seen = slot < end && r < R;
                        if (kWin) {
                            if (seen) {
                                const int32_t* position = p.mask != nullptr ? p.position + (size_t)b * p.nmax : nullptr;
                                const int step = window_step(position, node, base + gap);
                                if (j < 0 || p.mask == nullptr)
                                    seen = j <= node && (slot < p.sinks || slot >= lo + step);
                                else {
                                    seen = j < 32 * p.words && ((p.mask[((size_t)b * p.nmax + node) * p.words + (j >> 5)] >> (j & 31)) & 1);
                                    if (seen && step >= p.window) {
                                        const int at = window_step(position, j, base + gap);
                                        seen = step - at < p.window || at + base + gap < p.sinks;
                                    }
                                }
                            }
                        } else if (seen && j >= 0)
                            seen = p.mask == nullptr ? j <= node
                                                     : j < 32 * p.words && ((p.mask[((size_t)b * p.nmax + node) * p.words + (j >> 5)] >> (j & 31)) & 1);
                        s[i] = seen ? s[i] : -INFINITY;
                        sees |= (seen ? 1u : 0u) << i;
                    }
                    // V of slots that are not there is taken out, and of new slots that are not numbers: what of those is seen is added in the end
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int slot = s0 + 2 * q4 + (i & 1) + 8 * (i >> 1);
                        bool bad = Q8 && (x[i >> 1] >> (16 * (i & 1)) & 255) > 246;  // (up to 480 2^119 is below 2^128)
                        if (!Q8)
#pragma unroll
                            for (int x = 0; x < 4 * kV; ++x) bad = bad || not_finite2(vr[i][x]);
                        // (a slot's lanes differ in g: any of them)
                        const bool unseen = kWin && slot >= p.sinks && slot < min(lo, base);  // (by all rows)
                        const unsigned who = __ballot_sync(0xFFFFFFFFu, bad && slot < end && (slot >= base || (kWin && !unseen && window_border(slot, p.sinks, lo, pc.n - 1))));
                        spoilt[i] = (who & (0x11111111u << q4)) != 0;
                        if (slot >= end || spoilt[i] || unseen) {
#pragma unroll
                            for (int x = 0; x < 4 * kV; ++x) vr[i][x] = 0;
                            f2[i >> 1] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                        }
                    }
                }
                // ---- weights, against the maximum known before as long as it has not grown by more than 2^8
                if (__any_sync(0xFFFFFFFFu, fmaxf(s[0], s[2]) > upto[0] || fmaxf(s[1], s[3]) > upto[1])) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float x = fmaxf(s[i], s[i + 2]);
                        for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, d));
                        const float now = fmaxf(m[i], x), k = m[i] > -INFINITY ? ex2_approx((m[i] - now) * c2) : 1.0f;
                        m[i] = now;
                        upto[i] = now + most;
                        off[i] = now > -INFINITY ? -now * c2 : 0.0f;
                        l[i] *= k;
#pragma unroll
                        for (int y = 0; y < D / 16; ++y) o[y][i] *= k, o[y][i + 2] *= k;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i] = ex2_approx(fmaf(s[i], c2, off[i & 1]));
                    l[i & 1] += s[i];
                }
                // P^T as the second operand: rows where the slots were
                float e[4] = {s[0], s[1], s[2], s[3]};
                if (Q8)
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[i] *= big[i >> 1];
                const uint32_t pb0 = transpose_8x8(pack_bf16(e[0], e[1])), pb1 = transpose_8x8(pack_bf16(e[2], e[3]));
                // ---- O^T += V^T P^T: rows of the first operand are head_dim, two numbers of the lane's D / 8 a product
#pragma unroll
                for (int y0 = 0; y0 < D / 16; y0 += 4) {
                    uint32_t a[4][2][2];  // [product][slot pair][number]
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int z = 0; z < 2; ++z) {
                                const int y = y0 + x, byte = (2 * y + z) & 3;
                                if (Q8) {
                                    a[x][i][z] = e4m3_pair_small(vr[2 * i][y / 2], vr[2 * i + 1][y / 2], byte, 4 + byte);
                                } else
                                    a[x][i][z] = __byte_perm(vr[2 * i][y], vr[2 * i + 1][y], z ? 0x7632 : 0x5410);
                            }
                    if (Q8 && large_v)
#pragma unroll
                        for (int x = 0; x < 16; ++x) a[x >> 2][x >> 1 & 1][x & 1] = bf16x2_mul(a[x >> 2][x >> 1 & 1][x & 1], f2[x >> 1 & 1]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) mma_16816(o[y0 + x], a[x][0][0], a[x][0][1], a[x][1][0], a[x][1][1], pb0, pb1);
                }
                if (more_steps) bring_v(row1);
                // number y of the lane's of V: o[y / 2][..], [rows + 2 (y & 1)]
                const auto dim = [&](int y) { return y / kCv * (8 * kCv) + g * kCv + y % kCv; };
                // ---- new slots whose V is not a number: to the rows that see them
                if (masked && __any_sync(0xFFFFFFFFu, spoilt[0] || spoilt[1] || spoilt[2] || spoilt[3])) {
#pragma unroll 1
                    for (int i = 0; i < 16; ++i) {
                        const int owner = (i & 7) >> 1, which = (i & 1) + 2 * (i >> 3);
                        const bool bad = __shfl_sync(0xFFFFFFFFu, which == 0 ? spoilt[0] : which == 1 ? spoilt[1] : which == 2 ? spoilt[2] : spoilt[3], owner);
                        if (!bad) continue;
                        const size_t r = row0 + i;
                        uint32_t fv = 0, mv = kOneBf16x2;
                        if (Q8) e4m3_factors(__ldg(c.v_exp + r), fv, mv);
                        const float w0 = __shfl_sync(0xFFFFFFFFu, i < 8 ? s[0] : s[2], (i & 7) * 4 + q4);
                        const float w1 = __shfl_sync(0xFFFFFFFFu, i < 8 ? s[1] : s[3], (i & 7) * 4 + q4);
                        // (a weight of a slot that is seen may be too small for fp32 and 0: what it stands before is not a number all the same)
                        const uint32_t see = __shfl_sync(0xFFFFFFFFu, sees >> (i < 8 ? 0 : 2), (i & 7) * 4 + q4);
#pragma unroll
                        for (int y = 0; y < D / 8; ++y) {
                            const uint8_t* from = c.v + (r * D + dim(y)) * kBytes;
                            float v;
                            if (Q8)
                                v = __uint_as_float(e4m3x4_to_bf16(*from, fv, mv).x << 16);
                            else
                                v = __uint_as_float((uint32_t) * (const uint16_t*)from << 16);
                            if (see & 1) o[y / 2][2 * (y & 1)] += w0 * v;
                            if (see & 2) o[y / 2][2 * (y & 1) + 1] += w1 * v;
                        }
                    }
                }
                row0 = row1;
            }
        };
        if (Q8 && q_wide)
            steps_of_piece(Yes());
        else
            steps_of_piece(No());
        // ---- the warps' sums are joined
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x = l[i];
            for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
            const int r = 2 * q4 + i;
            if (g == 0) {
                sm_ml[(warp * kFewRows + r) * 2] = m[i] > -INFINITY ? m[i] * c2 : -INFINITY;
                sm_ml[(warp * kFewRows + r) * 2 + 1] = x;
            }
#pragma unroll
            for (int y = 0; y < D / 16; ++y)
                *(float2*)&few_sm[(warp * kFewRows + r) * D + 2 * y / kCv * (8 * kCv) + g * kCv + 2 * y % kCv] = make_float2(o[y][i], o[y][i + 2]);
        }
        if (selfish) {
            fine = __syncthreads_and(fine);
            if (tid == 0 && h == 0 && pc.head && p.status) p.status[b] = fine ? 0 : GRAFT_ST_BAD_CACHE;
            if (!fine) {  // (so it is for all CTAs that have pieces of the sequence: it is left out)
                __syncthreads();
                continue;
            }
        } else
            __syncthreads();
        const bool whole = pc.whole;
        const size_t slot = 2 * (size_t)blockIdx.x + pc.head;
        for (int x = tid; x < R * (D / 4); x += S::kThreads) {
            const int r = x / (D / 4), d = x % (D / 4) * 4;
            float mm = -INFINITY, ll = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, sm_ml[(w * kFewRows + r) * 2]);
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float mw = sm_ml[(w * kFewRows + r) * 2], lw = sm_ml[(w * kFewRows + r) * 2 + 1];
                const float k = mw > -INFINITY ? ex2_approx(mw - mm) : 0.0f;
                ll += k * lw;
                const float4 v = *(const float4*)&few_sm[(w * kFewRows + r) * D + d];
                sum.x += k * v.x, sum.y += k * v.y, sum.z += k * v.z, sum.w += k * v.w;
            }
            const int node = r / p.group;
            const size_t out_row = ((size_t)b * p.rows + node) * p.q_heads + h * p.group + (r - node * p.group);
            if (whole) {
                const float inv = ll != 0.0f ? 1.0f / ll : 1.0f;
                *(uint2*)(p.out + out_row * D + d) = make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
                if (p.lse && d == 0) p.lse[out_row] = log_sum(mm, ll);
            } else {
                ((float4*)p.part_o)[(slot * (D / 4) + d / 4) * p.part_rows + r] = sum;
                if (d == 0) p.part_ml[slot * p.part_rows + r] = make_float2(mm, ll);
            }
        }
        if (!whole) __threadfence();
        __syncthreads();  // (the sums and the piece are read)
        if (!whole) {
            // The last of a unit's pieces to be there joins them, in the pieces' order: eight rows are little work, and a kernel behind this one
            // takes longer to begin.  One token behind 1000 and 32000 slots: 17.0 -> 14.2 and 34.3 -> 28.3 us (e4m3), 64 tokens 269 -> 274.
            if (warp == 0) {
                list_unit(list, {cut_x0, kOneTile, cut_kt}, cut_f, cta_of(cut_x0 + (cut_kt - 1) * kOneTile, total, parts), total, parts, -1, 0, 0,
                          kJoinRows);
                if (lane == 0) {
                    last = atomicAdd(p.ready + cut_f, 1) == list.n - 1;
                    if (selfish && last) p.ready[cut_f] = 0;  // (nobody else comes)
                }
            }
            __syncthreads();
            if (last) {
                __threadfence();
                const int node = lane / p.group;
                if (kWin)
                    join_few<D, kWarps>(p, list, R, (size_t)b * p.rows * p.q_heads + h * p.group);
                else if (tid < kJoinThreads)
                    join_rows<D, 4>(p, list, lane < R, ((size_t)b * p.rows + node) * p.q_heads + h * p.group + (lane - node * p.group));
            }
            __syncthreads();
        }
    }
}

// Units that were cut, without a shared prefix: blocks for every boundary between CTAs; the first boundary inside a unit joins it.
template <int D>
__global__ void __launch_bounds__(kJoinThreads, 4) attn_join_kernel(const __grid_constant__ AttnParams p) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ JoinList j;
    const int4* from = (const int4*)(p.join + blockIdx.y + 1);
    PlanJoin q;
#pragma unroll
    for (int i = 0; i < 3; ++i) ((int4*)&q)[i] = __ldcg(from + i);
    const int r0 = blockIdx.x * kJoinRows;
    if (r0 >= q.rows) return;
    if (threadIdx.x < 32) {
        if (threadIdx.x == 0) j.n = 0;
        __syncwarp();
        list_unit(j, {q.x0, q.w, q.kt}, q.f, q.l, q.total, q.parts, -1, r0, 0, kJoinRows);
    }
    __syncthreads();
    const int r = q.r0 + r0 + lane_id(), node = r / p.group;
    const bool live = r0 + lane_id() < q.rows;
    join_rows<D, 2>(p, j, live, ((size_t)(q.s - 1) * p.rows + q.node0 + node) * p.q_heads + q.h * p.group + (r - node * p.group));
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled() {
    static const EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return (EncodeTiledFn) nullptr;
        }
        return (EncodeTiledFn)f;
    }();
    return fn;
}
// Entries of one layer as rows: boxes of 64 bf16 numbers in the 128-byte swizzle, or of whole rows of e4m3 numbers as they are.
bool encode_map(CUtensorMap* map, const void* base, bool q8, int D, uint64_t rows, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)D, rows}, strides[1] = {(cuuint64_t)D * (q8 ? 1 : 2)};
    const cuuint32_t box[2] = {(cuuint32_t)(q8 ? D : 64), (cuuint32_t)box_rows}, step[2] = {1, 1};
    return encode_tiled()(map, q8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
                          strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, q8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool few_rows(int group, int rows, int shared) { return shared == 0 && (long long)rows * group <= kFewRows; }
template <bool kWin>
int attn_ctas(const graft_ctx* ctx, bool q8, int head_dim, int group, int rows, int shared) {
    const int ctas = head_dim == 128 ? (q8 ? FewShape<128, true, kWin>::kCtas : FewShape<128, false, kWin>::kCtas)
                                     : (q8 ? FewShape<64, true, kWin>::kCtas : FewShape<64, false, kWin>::kCtas);
    return ctx->num_sms * (few_rows(group, rows, shared) ? ctas : 1);
}

struct AttnSizes {
    int part_rows;
    size_t o_seq, o_start, o_join, o_ready, o_use, o_entry0, o_ml, o_o, total;
};
// entries: of the plan, behind entry 0; use: sequences that a plan of blocks keeps numbers of (else 0)
AttnSizes attn_sizes(int ctas, int batch, int entries, int use, int kv_heads, int head_dim, int group, int rows, int shared) {
    const auto units = [&](long long nodes) { return (size_t)kv_heads * (size_t)((nodes * group + kUnitRows - 1) / kUnitRows); };
    const size_t slots = shared > 0 ? units((long long)batch * rows) + (size_t)batch * units(rows) + ctas : 2 * (size_t)ctas;
    AttnSizes z;
    z.part_rows = shared > 0 ? kUnitRows : (int)min((long long)kUnitRows, ((long long)rows * group + 31) / 32 * 32);
    size_t off = 256;
    const auto take = [&](size_t bytes) {
        const size_t o = off;
        off = (off + bytes + 255) / 256 * 256;
        return o;
    };
    z.o_seq = take((size_t)(entries + 1) * sizeof(PlanSeq));
    z.o_start = take((size_t)ctas * sizeof(PlanStart));
    z.o_join = take((size_t)(ctas + 1) * sizeof(PlanJoin));
    z.o_ready = take((size_t)ctas * sizeof(int));
    z.o_use = take((size_t)use * sizeof(int4));
    z.o_entry0 = take((size_t)use * sizeof(int));
    z.o_ml = take(slots * z.part_rows * sizeof(float2));
    z.o_o = take(slots * z.part_rows * head_dim * sizeof(float));
    z.total = off;
    return z;
}

// The plan, the attention kernel, the joining of what it cut (unless the kernel joins it itself).
template <typename Plan, typename Kernel, typename Join>
cudaError_t launch_kernels(graft_ctx* ctx, const AttnParams& p, Plan plan, Kernel kernel, int threads, size_t smem, uint32_t* done, uint32_t ready,
                           Join join, cudaStream_t st) {
    cudaError_t e;
    if (!(*done & ready)) {
        e = allow_smem((const void*)kernel, smem);
        if (e != cudaSuccess) return e;
        *done |= ready;
    }
    e = launch_pdl(plan, dim3(p.batch), dim3(kPlanThreads), 0, st, p);
    if (e != cudaSuccess) return e;
    ctx->launches += 1;
    e = launch_pdl(kernel, dim3(p.ctas), dim3(threads), smem, st, p);
    if (e != cudaSuccess) return e;
    ctx->launches += 1;
    return join();
}
template <int D>
cudaError_t launch_join(graft_ctx* ctx, const AttnParams& p, cudaStream_t st) {
    const long long most = (long long)p.rows * p.group;  // rows of a sequence and key head
    ctx->launches += 1;
    return launch_pdl(attn_join_kernel<D>, dim3((unsigned)((min(most, (long long)kUnitRows) + kJoinRows - 1) / kJoinRows), max(p.ctas - 1, 1)),
                      dim3(kJoinThreads), 0, st, p);
}
// What a call's parameters are whatever its rows see; maps: the kernel copies by TMA, box_rows slots at a time.
cudaError_t attn_params(AttnParams& p, const graft_ctx* ctx, int batch, const graft_cache* cache, int layer, int q_heads, int rows, long long q_stride,
                        const void* d_q, float scale, const int32_t* d_prefix_len, const int32_t* d_count, const uint32_t* d_mask, void* d_out,
                        float* d_lse, int32_t* d_status, bool maps, int box_rows) {
    memset(&p, 0, sizeof p);
    p.c = cache_view(cache, layer);
    p.box_rows = box_rows;
    if (maps) {
        const bool q8 = cache->dtype == GRAFT_E4M3;
        const uint64_t cache_rows = (uint64_t)cache->n_pages * cache->kv_heads * cache->page_size;
        if (encode_tiled() == nullptr) return cudaErrorNotSupported;
        if (!encode_map(&p.map_k, p.c.k, q8, cache->head_dim, cache_rows, box_rows) ||
            !encode_map(&p.map_v, p.c.v, q8, cache->head_dim, cache_rows, box_rows))
            return cudaErrorInvalidValue;
    }
    p.q = (const uint8_t*)d_q;
    p.q_stride = q_stride;
    p.prefix_len = d_prefix_len;
    p.count = d_count;
    p.mask = d_mask;
    p.out = (__nv_bfloat16*)d_out;
    p.lse = d_lse;
    p.status = d_status;
    p.c2 = scale == 0.0f ? kLog2e : fabsf(scale) * kLog2e;
    p.q_flip = scale < 0.0f ? 0x80008000u : 0u;
    p.q_keep = scale == 0.0f ? 0u : 0xFFFFFFFFu;
    p.rows = rows;
    p.q_heads = q_heads;
    p.group = q_heads / cache->kv_heads;
    p.nmax = ctx->nmax;
    p.words = ctx->mask_words;
    p.batch = batch;
    p.arrivals = ctx->w_attn_n;
    return cudaSuccess;
}
// and where its scratch is
void attn_places(AttnParams& p, const AttnSizes& z, void* scratch) {
    uint8_t* base = (uint8_t*)scratch;
    p.head = (PlanHead*)base;
    p.seq = (PlanSeq*)(base + z.o_seq);
    p.start = (PlanStart*)(base + z.o_start);
    p.join = (PlanJoin*)(base + z.o_join);
    p.ready = (int*)(base + z.o_ready);
    p.use = (int4*)(base + z.o_use);
    p.entry0 = (int*)(base + z.o_entry0);
    p.part_ml = (float2*)(base + z.o_ml);
    p.part_o = (float*)(base + z.o_o);
    p.part_rows = z.part_rows;
}

}  // namespace

}  // namespace graft
