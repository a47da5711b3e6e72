// Attention of the trees' nodes over a paged cache (graft_tree_attention), on the tcgen05 tensor cores.
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
// What bounds it.  Large trees (16 of up to 513 nodes behind 6000 to 8192 slots, bf16, 717 GFLOP): 840 to 875 us, the tensor cores busy for 47 % of
// the time, the exponentials' unit for 36 %: a stream's next product waits for all of a tile's weights, and two streams (TMEM holds
// no more) do not fill the gaps; the clock falls to 1.3 GHz under that load in a long run (980 to 1060 us).  A tile of e4m3 slots is converted
// once a unit, 0.5 to 0.6 us, and is as long on its way as the products: 823 us against 621 for 8 sequences of 512 nodes.  17 nodes (68 rows)
// behind 4000 slots, bf16: 213 us, 0.78 of the copy's rate.  Small calls are latencies: one tree of 65 nodes behind 1500 slots 31 us, of
// which plan 4, attention 10 to 15, joining 8, and the hand-overs of three kernels.
#include <cuda.h>
#include <float.h>
#include <string.h>

#include "cache.cuh"
#include "umma.cuh"

namespace graft {

namespace {

constexpr int kTile = 128;      // slots of a key tile, rows of a row tile
constexpr int kUnitRows = 256;
constexpr uint32_t kWaitNs = 500;  // that a poll may sleep
constexpr float kMostGrowth = 8.0f;  // (powers of two) of a row's maximum, before O is rescaled

// What the plan says of a sequence (entry 0: the shared prefix with the rows of all of them; entry b + 1: sequence b).
struct __align__(16) PlanSeq {
    int n;       // rows in use (nodes); 0: none, or left out
    int base;    // slots before the first row's (shared prefix: its length)
    int node0;   // nodes of the sequences before
    int unit0;   // units before
    int cost0;   // position in the line: lengths of the units before
    int kt;      // key tiles
    int pad[2];
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
    int s, h, r0;      // entry, key head, first row of the unit among the entry's
    int pad;
};
struct PlanHead {
    int total;  // length of the line
    int parts;  // CTAs that it is cut for
    int chunk;  // units begin at multiples of it
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
};

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
        PlanSeq s = {Rs > 0 ? nodes : 0, p.shared, 0, 0, 0, kts, {0, 0}};
        p.seq[0] = s;
        entries[0] = s;
    }
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
        const int i = b0 + me;
        int n, base, kt, R;
        of(i, n, base, kt, R);
        const Sums s = block_sums(scratch, small, n, Hk * row_tiles2(R), Hk * head_cost(R, kt, chunk));
        if (i < p.batch && (!small || warp == 0)) {
            PlanSeq q = {n, base, seen + s.before[0], units + s.before[1], cost + s.before[2], kt, {0, 0}};
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
    // where every CTA begins
    for (int i = tid; i < p.ctas; i += kPlanThreads) {
        PlanStart st = {};
        PlanJoin j = {};
        if (i < parts) {
            st.x = part_first(total, parts, i);
            st.x1 = part_first(total, parts, i + 1);
            st.chunk = chunk;
            int lo = 0, hi = p.batch;  // the last entry whose position is not above x: one that has any, as the ones behind it begin above x
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
            if (p.shared == 0 && st.k > 0 && st.k < q.kt) {  // (else the stretch begins with a unit)
                const UnitAt un = unit_at(q, p.group, st.h, st.mt, chunk);
                j.f = cta_of(un.x0, total, parts);
                // the tiles ahead of this CTA's are those of the unit's first CTA, and this one has some
                if (first_tile(un, total, parts, j.f + 1) == st.k && first_tile(un, total, parts, i + 1) > st.k)
                    j.rows = min(kUnitRows, R - st.mt * kUnitRows);
                j.l = cta_of(un.x0 + (un.kt - 1) * un.w, total, parts);
                j.total = total, j.parts = parts;
                j.x0 = un.x0, j.w = un.w, j.kt = un.kt;
                j.s = lo, j.h = st.h, j.r0 = st.mt * kUnitRows;
            }
        }
        p.start[i] = st;
        p.join[i] = j;
        p.ready[i] = 0;
    }
}

// ---- walking along a CTA's stretch -----------------------------------------------------------------------------------
// A bounded wait whose polls sleep: the polls of warps that wait would otherwise take the shared-memory pipe from those that work.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    return mbar_wait_bounded_hint(bar, parity, gave_up, kWaitNs);
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
};
struct Walk {
    const PlanSeq* seq;
    int last_s, Hk, group, shared;
    int x, x1, chunk;
    int s, h, mt, k;
    PlanSeq q;
    __device__ __forceinline__ void begin(const AttnParams& p, int cta) {
        seq = p.seq;
        last_s = p.batch;
        Hk = p.c.kv_heads;
        group = p.group;
        shared = p.shared;
        const PlanStart* from = p.start + cta;
        const int4 st = __ldcg((const int4*)from), en = __ldcg((const int4*)from + 1);
        load_seq(q, &from->q);
        s = st.x, h = st.y, mt = st.z, k = st.w, x = en.x, x1 = en.y, chunk = en.z;
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

// which of the 128 slots from `first` on row `node` sees; end: slots there are.  (Words of the mask are loaded without branches, all together.)
__device__ __forceinline__ void seen_words(const uint32_t* mask_row, int words, int node, int base, int end, int first, uint32_t (&sees)[4]) {
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

// ---- the attention kernel ------------------------------------------------------------------------------------------
constexpr int kPieces = 4;  // that are told ahead
// Pieces that the flags of rows of V that were taken out are held for.  A warp of the first stream may set the next piece's flag while others
// have yet to test this one's (it clears V ahead of its first scores); none is two pieces ahead, as a piece's first scores wait for all eight
// warps' arrivals on q_full, which follow their test.
constexpr int kSpoiltPieces = 2;

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
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm volatile("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ bool not_finite2(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

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
struct Yes {
    static constexpr bool value = true;
};
struct No {
    static constexpr bool value = false;
};
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
template <int kCols>
__device__ __forceinline__ float scores(uint32_t tS, int x0, uint32_t (&u)[kCols], bool masked, const uint32_t (&sees)[4]) {
#pragma unroll
    for (int x = 0; x < kCols; x += 32) tmem_ld_32x32(tS + x0 + x, *(uint32_t(*)[32]) & u[x]);
    tmem_arrived(u);
    if (masked)
#pragma unroll
        for (int x = 0; x < kCols; ++x) u[x] = (sees[(x0 + x) / 32] >> (x % 32)) & 1 ? u[x] : 0xFF800000u;
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
#pragma unroll
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

// What a row sees of new slots whose V is not a number, which was taken out of the products: added to its O in TMEM, with scores of
// its own.  Key tiles t0, t0 + dt, .. of the piece; a whole warp calls it, `sums` are the rows that see anything, m their maxima.
template <int D, bool Q8>
__device__ __noinline__ void add_spoilt(const AttnParams& p, const Piece& pc, uint32_t tO, bool sums, int b, int node, int head, int t0,
                                        int dt, float m) {
    const CacheView& c = p.c;
    const uint32_t* mask_row = p.mask ? p.mask + ((size_t)b * p.nmax + node) * p.words : nullptr;
    const uint16_t* q = (const uint16_t*)p.q + ((long long)b * p.rows + node) * p.q_stride + (long long)head * D;
    for (int t = t0; t < pc.T; t += dt) {
        const int first = pc.first + t * kTile;
        for (int slot = max(first, pc.base); slot < min(pc.end, first + kTile); ++slot) {
            const size_t at = cache_row(c, __ldg(c.table + (size_t)(pc.s - 1) * c.width + (slot >> c.page_shift)), pc.h,
                                        slot & ((1 << c.page_shift) - 1));
            const auto entry = [&](const uint8_t* x, const uint8_t* exps, int d) {  // four numbers from d on
                if (!Q8) return *(const uint2*)(x + at * c.row_bytes + 2 * d);
                uint32_t f, more;
                e4m3_factors(exps[at], f, more);
                return e4m3x4_to_bf16(*(const uint32_t*)(x + at * c.row_bytes + d), f, more);
            };
            bool bad = false;  // the same in all lanes: a piece's rows have one sequence where there are new slots
            for (int d = 0; d < D; d += 4) {
                const uint2 v = entry(c.v, c.v_exp, d);
                bad = bad || not_finite2(v.x) || not_finite2(v.y);
            }
            if (!bad) continue;
            const int j = slot - pc.base;
            const bool mine = sums && (mask_row == nullptr ? j <= node : j < 32 * p.words && ((mask_row[j >> 5] >> (j & 31)) & 1));
            float s = 0.0f;
            if (mine)
                for (int d = 0; d < D; d += 4) {
                    const uint2 k = entry(c.k, c.k_exp, d);
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t qw = (((uint32_t)q[d + y] << 16) ^ (p.q_flip & 0xFFFF0000u)) & p.q_keep, kw = y < 2 ? k.x : k.y;
                        s += __uint_as_float(qw) * __uint_as_float(y & 1 ? kw & 0xFFFF0000u : kw << 16);
                    }
                }
            const float e = mine ? ex2_approx((s - m) * p.c2) : 0.0f;
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

template <int D, bool Q8, bool kOne>
__global__ void __launch_bounds__(Shape<D, Q8, kOne>::kThreads, 1) tree_attn_kernel(const __grid_constant__ AttnParams p) {
    using S = Shape<D, Q8, kOne>;
    constexpr int NS = S::kStages, NR = S::kRaw > 0 ? S::kRaw : 1;
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
    const uint32_t q_full = bar0 + 8 * (2 * NS + 2 * NR), s_full0 = q_full + 8, p_full0 = q_full + 24, pair = q_full + 40, turn0 = q_full + 48;
    const uint32_t piece_full0 = q_full + 64, piece_empty0 = piece_full0 + 8 * kPieces;
    volatile int* const gave_up = (volatile int*)(bars + 2 * NS + 2 * NR + 8 + 2 * kPieces);
    volatile int* const spoilt = gave_up + 1;  // [kSpoiltPieces][2 streams] the last piece (counted from 1) with a row of V that was taken out
    uint32_t* const tmem_at = (uint32_t*)(gave_up + 1 + 2 * kSpoiltPieces);
    Piece* const pieces = (Piece*)(gave_up + 2 + 2 * kSpoiltPieces);  // [kPieces]
    static_assert((2 * NS + 2 * NR + 8 + 2 * kPieces) * 8 + (2 + 2 * kSpoiltPieces) * 4 + kPieces * sizeof(Piece) <= 1024, "barriers and pieces");
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
            mbar_init(s_full0 + 8 * i, 1);
            mbar_init(p_full0 + 8 * i, 4);
            mbar_init(turn0 + 8 * i, 1);
        }
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
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kRegsSoftmax));
        // ---- softmax: a thread a row
        const int i = warp >> 2, row_in_tile = tid & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's quarter of the lanes
        const uint32_t tS = tmem + lanes + i * 128, tO = tmem + lanes + 256 + i * 128;
        uint32_t it = 0, n_s = 0, n_piece = 0, n_pair = 0;
        bool ok = true;
        const float c2 = p.c2;
        const auto both = [&]() {  // the two streams meet
            __syncwarp();
            if (lane == 0) mbar_arrive(pair);
            const bool r = wait_for(pair, n_pair & 1, gave_up);
            n_pair += 1;
            return r;
        };
        const auto wait_s = [&]() {
            const bool r = wait_for(s_full0 + 8 * i, n_s & 1, gave_up);
            n_s += 1;
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
            if (two || i == 0) {
                // a row's pieces side by side in a warp's load; where a row stands is worked out by the lane that has it
                int b = 0, node = 0, g = 0;
                if (live) row_of(p, pc.s, pc.r0 + r, b, node, g);
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
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
            const bool warp_live = __any_sync(0xFFFFFFFFu, live);
            float m = -INFINITY, l = 0.0f;  // maximum of the raw scores, sum of 2^(c2 (s - m))
            bool any = false;               // this stream has had a tile
            // from this tile on there are new slots, or slots that are not there (the shared prefix: base is its end)
            const int first0 = pc.first, to_base = pc.base - kTile - first0, t_masked = to_base < 0 ? 0 : to_base / kTile + 1;
            // Slots that are not there hold anything, and new slots may hold what is not a number and is not for every row: weights of zero do
            // not keep it out of the sums.  Their rows of V are cleared (a thread a slot); rows that see such a slot get it in the end.
            const auto clear_v = [&](int t, int first) {
                const uint32_t entry = it + v_entry(two, T, t);
                if (!wait_for(kv_full(entry % NS), (entry / NS) & 1, gave_up)) return false;
                const int slot = first + row_in_tile, end = pc.end;
                if (slot >= pc.base) {
                    const uint32_t at = kv_addr + (entry % NS) * S::kTileBytes + row_in_tile * 128;
                    bool clear = slot >= end;
                    if (!clear)
#pragma unroll
                        for (int x = 0; x < D / 8; ++x) {  // (a row's pieces in an order of its own: eight rows then use all banks)
                            uint32_t a0, a1, a2, a3;
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(a0), "=r"(a1), "=r"(a2), "=r"(a3)
                                         : "r"(at + (x >> 3) * S::kHalf + ((x + row_in_tile) & 7) * 16)
                                         : "memory");
                            clear = clear || not_finite2(a0) || not_finite2(a1) || not_finite2(a2) || not_finite2(a3);
                        }
                    if (clear) {
#pragma unroll
                        for (int x = 0; x < D / 8; ++x)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + (x >> 3) * S::kHalf + ((x + row_in_tile) & 7) * 16),
                                         "r"(0)
                                         : "memory");
                        if (slot < end) spoilt[2 * (n_piece % kSpoiltPieces) + i] = (int)n_piece + 1;
                    }
                }
                fence_proxy_async();
                return true;
            };
            for (int t = two ? 0 : i; t < T; t += two ? 1 : 2) {
                const int first = first0 + t * kTile;
                const bool masked = t >= t_masked;
                uint32_t sees[4];
                if (masked) {
                    int b = 0, node = 0, g = 0;
                    if (live) row_of(p, pc.s, pc.r0 + r, b, node, g);
                    const uint32_t* mask_row = p.mask ? p.mask + ((size_t)b * p.nmax + node) * p.words : nullptr;
                    seen_words(mask_row, p.words, node, pc.base, live ? pc.end : 0, first, sees);
                    // (with two row tiles every entry ahead of V's in the ring has been used by this stream, so its phase is certain: see `pass`)
                    if (two && i == 0 && !(ok = clear_v(t, first))) break;
                }
                if (!(ok = wait_s())) break;
                if (warp_live) {
                    // (with fewer registers: the maximum first, then each half again)
                    constexpr bool kAgain = S::kCols < kTile;
                    uint32_t u[S::kCols], w[32];
                    float mx = scores(tS, 0, u, masked, sees);
                    if (kAgain) mx = max2(mx, scores(tS, 64, u, masked, sees));
                    // (m = -inf: nothing seen so far, and what O holds is zero)
                    const bool grown = mx > m && !((mx - m) * c2 <= kMostGrowth);
                    if (__any_sync(0xFFFFFFFFu, grown)) {
                        const float now = fmaxf(m, mx), f = m > -INFINITY ? ex2_approx((m - now) * c2) : 1.0f;
                        if (any) rescale<D>(tO, f);
                        l *= f;
                        m = now;
                    }
                    // (a score of NaN or +inf, which some of the exponentials below would lose: the row's sum is NaN from here on, and so is all that
                    // is divided by it)
                    if (!(mx < INFINITY)) l = __int_as_float(0x7FFFFFFF);
                    const float off = m > -INFINITY ? -m * c2 : 0.0f;
                    if (kAgain) scores(tS, 0, u, masked, sees);
                    l += weigh(u, c2, off, w);
                    tmem_st_32x32(tS, w);
                    if (kAgain) scores(tS, 64, u, masked, sees);
                    l += weigh(u + S::kCols - 64, c2, off, w);
                    tmem_st_32x32(tS + 32, w);
                    tmem_wait_st();
                }
                if (masked && !two && !(ok = clear_v(t, first))) break;
                if (masked && two && !(ok = both())) break;  // (the first stream clears for both)
                any = true;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full0 + 8 * i);
            }
            if (!ok) break;
            it += 2 * T;
            if (any)
                ok = wait_s();  // the last product is done
            else
                ok = wait_for(q_full, n_piece & 1, gave_up);  // (nor does a stream without a tile run ahead)
            if (!ok) break;

            // ---- the end of a piece: O as far as it goes
            int b = 0, node = 0, g = 0;
            if (live) row_of(p, pc.s, pc.r0 + r, b, node, g);
            const int head = pc.h * p.group + g;
            if (spoilt[2 * (n_piece % kSpoiltPieces) + (two ? 0 : i)] == (int)n_piece + 1)
                add_spoilt<D, Q8>(p, pieces[n_piece % kPieces], tO, live && m > -INFINITY, b, node, head, two ? 0 : i, two ? 1 : 2, m);
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
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) {
                        tmem_ld_32x32(tO + 32 * x, u);
                        tmem_arrived(u);
                        put(32 * x, u, inv);
                    }
                    put_sums(m, l);
                }
            } else {
                // the streams' halves are joined: the second one's goes through the shared memory of Q, which nobody reads any more
                float* const tmp = (float*)smem;  // [D / 2 columns][128 rows]
                float m1 = 0.0f, l1 = 0.0f, f0 = 1.0f, f1 = 0.0f, ms = 0.0f, ls = 0.0f, inv = 1.0f;
#pragma unroll
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
#pragma unroll
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
#pragma unroll
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
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kRegsOthers));
        uint32_t n_piece = 0;
        bool ok = true;
        if (warp == 11) {
            Walk walk;
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
                const int32_t* table = c.table + (pc.s == 0 ? 0 : (size_t)(pc.s - 1) * c.width);
                const auto bring = [&](int t, bool is_v) {
                    const int first = first0 + t * kTile, upto = min(end, first + kTile);
                    const int copies = (upto - first + box - 1) / box;  // boxes with a slot in use
                    const int i = lane / kParts, part = lane % kParts;
                    int page = 0, at = 0;
                    if (i < copies) {
                        const int slot = first + i * box;
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
                if (two) {
                    for (int t = 0; ok && t < T; ++t) ok = bring(t, false) && bring(t, true);
                } else {
                    ok = bring(0, false);
                    if (T > 1) ok = ok && bring(1, false);
                    for (int t = 0; ok && t < T; ++t) {
                        ok = bring(t, true);
                        if (t + 2 < T) ok = ok && bring(t + 2, false);
                    }
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
            constexpr uint32_t id_s = umma_idesc(128, 128, true), id_o = umma_idesc(128, D, true) | (1u << 16);  // (V: head_dim is contiguous)
            const uint32_t i = warp == 8 ? 0 : 1;
            uint32_t it = 0, n_p = 0, n_turn = 0;
            // (descriptors differ in their low words alone; the numbers that choose them are loaded, so the compiler is told that they are uniform)
            constexpr uint32_t kDescHi = (uint32_t)(umma_desc_sw128(0) >> 32);
            const uint32_t tS = uniform(tmem + i * 128), tO = uniform(tmem + 256 + i * 128);
            const uint32_t q_lo = uniform((uint32_t)umma_desc_sw128(q_addr)), kv_lo = uniform((uint32_t)umma_desc_sw128(kv_addr));
            const auto qk = [&](uint32_t a, uint32_t b) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t at = ((ks >> 2) * S::kHalf + (ks & 3) * 32) / 16;
                    if (ks == 0)
                        umma_ss<false>(tS, a + at, b + at, kDescHi, id_s);
                    else
                        umma_ss<true>(tS, a + at, b + at, kDescHi, id_s);
                }
            };
            // V as the second operand of P V: rows (slots) of 64 numbers of head_dim side by side, so head_dim is the contiguous direction.  In
            // the 128-byte swizzle: blocks of 64 numbers kHalf apart (a field that the other operands leave at 1), groups of eight slots 1024 bytes.
            constexpr uint32_t kHalfField = (uint32_t)(S::kHalf / 16) << 16, kOneField = 1u << 16;
            const auto pv = [&](bool first, uint32_t b) {
#pragma unroll
                for (int ks = 0; ks < kTile / 16; ++ks) umma_ts(tO, tS + ks * 8, kDescHi, b + ks * (2048 / 16), id_o, ks > 0 || !first);
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
            // Two row tiles: the streams issue by turns.  Side by side, their instructions would share the tensor cores and both streams'
            // softmax would then share the rest of the time; by turns, one stream's softmax runs under the other's products.
            const auto my_turn = [&](bool two) {
                if (!two) return true;
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
                        qk(a, bk);
                        if (two) mbar_arrive(turn0 + 8 * (1 - i));
                        umma_commit(kv_empty(it % NS));
                        umma_commit(s_full0 + 8 * i);
                    }
                    __syncwarp();
                    it += 1;
                }
                // P V of a tile, then Q K of the next, which takes the weights' place
                for (int t = t0; t < T; t += dt) {
                    const bool more = t + dt < T;
                    ok = pass(it0 + v_entry(two, T, t)) && wait_kv(it) && wait_for(p_full0 + 8 * i, n_p & 1, gave_up) && my_turn(two);
                    n_p += 1;
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t bv = uniform(at_entry(it) - kOneField + kHalfField), bk = at_entry(it + 1);
                    if (elect_one()) {
                        pv(t == t0, bv);
                        umma_commit(kv_empty(it % NS));
                    }
                    __syncwarp();
                    if (more) {
                        if (!(ok = wait_kv(it + 1))) break;
                        tc_fence_after();
                    }
                    if (elect_one()) {
                        if (more) qk(a, bk);
                        if (two) mbar_arrive(turn0 + 8 * (1 - i));
                        umma_commit(s_full0 + 8 * i);
                        if (more) umma_commit(kv_empty((it + 1) % NS));
                    }
                    __syncwarp();
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

// 32 rows of a unit from the pieces on the list: a lane a row, a warp some of the columns.  Pieces are added in their order along the line, results repeat; four are on their way at a time.
template <int D>
__device__ __forceinline__ void join_rows(const AttnParams& p, const JoinList& j, bool live, size_t out_row) {
    constexpr int kWarps = kJoinThreads / 32, kQuads = D / 4 / kWarps;  // groups of four columns a warp
    const int lane = lane_id(), warp = threadIdx.x >> 5, n = j.n;
    float m = -INFINITY, l = 0.0f;
    float o[4 * kQuads] = {};
    constexpr int kAhead = 4;
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
// the long directions and the rows in the short one; e4m3 entries become bf16 in registers.  The order of head_dim inside a product is free,
// so a lane loads pieces of 16 bytes straight into what it multiplies: of K, a quarter of those of two slots; of V, an eighth of four.  The next
// step's K is asked for when this one's scores are done, and V when its products are: the warps of an SM then have 50 to 60 KB under way.
// 64 sequences of 2000 to 16000 slots, 8 key heads of 128: bf16 354 us (6.6 TB/s; through the tiles of 128 rows 417), e4m3 274 us (4.3
// TB/s; 553), which conversions bound: 500 instructions for 16 slots, three warps a scheduler to hide their latencies.  Before pieces' own cost
// was counted (371 and 288): through a ring of cp.async in shared memory 543 and 295; with 8 warps of two steps 297, with 16 warps 294 (registers spill).
constexpr int kFewRows = 8;

template <int D, bool Q8>
struct FewShape {
    static constexpr int kBytes = Q8 ? 1 : 2;
    static constexpr int kK = D / 4 * kBytes / 16;                                     // pieces of a slot's K that a lane has
    static constexpr int kPiece = D / 8 * kBytes < 16 ? D / 8 * kBytes : 16;           // bytes of a piece of V (D = 64, e4m3: 8)
    static constexpr int kV = D / 8 * kBytes / kPiece;                                 // pieces of a slot's V
    // as many warps an SM as have room in registers for a step's K and V (16 to 64 of them) beside Q and O
    static constexpr int kWarps = Q8 && D == 128 ? 12 : 8, kThreads = 32 * kWarps;
    static constexpr int kCtas = D == 128 ? 1 : 2;
    static constexpr size_t kSmem = (size_t)kWarps * kFewRows * (D + 2) * sizeof(float);
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
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
template <int D, bool Q8>
__global__ void __launch_bounds__(FewShape<D, Q8>::kThreads, FewShape<D, Q8>::kCtas) few_attn_kernel(const __grid_constant__ AttnParams p) {
    using S = FewShape<D, Q8>;
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
    Walk walk;
    const int total = __ldcg(&p.head->total), parts = __ldcg(&p.head->parts);
    if (tid == 0) walk.begin(p, blockIdx.x);
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
        const int h = pc.h, b = pc.s - 1, base = pc.base, end = pc.end, R = pc.rows, first0 = pc.first;
        const int32_t* table = c.table + (size_t)b * c.width;
        // A step's 16 slots lie in one page; the warps take steps by turns.
        const int all = min(8 * T, (end - first0 + 15) / 16), steps = warp < all ? (all - warp + kWarps - 1) / kWarps : 0;
        const auto slot_of = [&](int step) { return first0 + (warp + step * kWarps) * 16; };
        const auto page_of = [&](int step) { return __ldg(table + (slot_of(min(step, steps - 1)) >> shift)); };
        const auto row_at = [&](int step, int page) { return cache_row(c, page, h, slot_of(step) & low); };
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
        float o[D / 16][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, upto[2] = {-INFINITY, -INFINITY}, off[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        for (int step = 0; step < steps; ++step) {
            const int s0 = slot_of(step);
            const bool more_steps = step + 1 < steps;
            const size_t row1 = row_at(step + 1, page);
            page = page_of(step + 2);
            // factors of K's slots g, g + 8: 2^(e + 120), a second one where that is above bf16's largest (rare, and not numbers)
            uint32_t f[2] = {0, 0}, ke[2] = {0, 0};
            float more[2] = {1.0f, 1.0f};
            bool large = false;
            if (Q8) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    ke[i] = __byte_perm(i ? k_exps.z : k_exps.x, i ? k_exps.w : k_exps.y, g) & 255;
                    f[i] = (ke[i] + 120) * 0x00800080u;
                }
                large = __any_sync(0xFFFFFFFFu, max(ke[0], ke[1]) > 134);
                if (large)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t x;
                        e4m3_factors(ke[i], f[i], x);
                        more[i] = __uint_as_float(x << 16);
                    }
            }
            // ---- scores: rows 2 q4, 2 q4 + 1 at slots g, g + 8
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, s2[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int y = 0; y < kK; ++y) {
                uint2 a[4 / kBytes][2];
#pragma unroll
                for (int x = 0; x < 4 / kBytes; ++x)  // four numbers of the lane's a product
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t w[4] = {kr[i][y].x, kr[i][y].y, kr[i][y].z, kr[i][y].w};
                        a[x][i] = Q8 ? make_uint2(bf16x2_mul(e4m3_pair_small(w[x], 0, 0, 1), f[i]), bf16x2_mul(e4m3_pair_small(w[x], 0, 2, 3), f[i]))
                                     : make_uint2(w[2 * x & 3], w[(2 * x + 1) & 3]);
                    }
#pragma unroll
                for (int x = 0; x < 4 / kBytes; ++x) {
                    const int ks = y * (4 / kBytes) + x;
                    mma_16816(x & 1 ? s2 : s, a[x][0].x, a[x][1].x, a[x][0].y, a[x][1].y, qf[2 * ks], qf[2 * ks + 1]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += s2[i];
            if (Q8 && large)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] *= more[i >> 1];
            if (more_steps) bring_k(row1);
            // the same for V's pairs of slots; second factors go to the weights (slots g, g + 8)
            uint32_t f2[2] = {0, 0}, x[2] = {0, 0};  // (x: the exponents of two slots)
            float big[2] = {1.0f, 1.0f};
            bool large_v = false;
            if (Q8) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[i] = __byte_perm(i ? v_exps.z : v_exps.x, i ? v_exps.w : v_exps.y, 2 * q4 | (2 * q4 + 1) << 8) & 0x00FF00FFu;
                    f2[i] = (x[i] + 0x00780078u) << 7;
                }
                large_v = __any_sync(0xFFFFFFFFu, ((x[0] + 0x00790079u) | (x[1] + 0x00790079u)) & 0x01000100u);  // (one above 134)
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
            const bool masked = s0 + 16 > base;
            bool spoilt[4] = {false, false, false, false};
            uint32_t sees = 0;  // bit i: score i is of a slot that its row sees
            if (masked) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int slot = s0 + g + 8 * (i >> 1), r = 2 * q4 + (i & 1), j = slot - base, node = r / p.group;
                    bool seen = slot < end && r < R;
                    if (seen && j >= 0)
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
                    const unsigned who = __ballot_sync(0xFFFFFFFFu, bad && slot >= base && slot < end);
                    spoilt[i] = (who & (0x11111111u << q4)) != 0;
                    if (slot >= end || spoilt[i]) {
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
            if (Q8 && large_v)
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
                                a[x][i][z] = bf16x2_mul(e4m3_pair_small(vr[2 * i][y / 2], vr[2 * i + 1][y / 2], byte, 4 + byte), f2[i]);
                            } else
                                a[x][i][z] = __byte_perm(vr[2 * i][y], vr[2 * i + 1][y], z ? 0x7632 : 0x5410);
                        }
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
                if (lane == 0) last = atomicAdd(p.ready + cut_f, 1) == list.n - 1;
            }
            __syncthreads();
            if (last) {
                __threadfence();
                const int node = lane / p.group;
                if (tid < kJoinThreads)
                    join_rows<D>(p, list, lane < R, ((size_t)b * p.rows + node) * p.q_heads + h * p.group + (lane - node * p.group));
            }
            __syncthreads();
        }
    }
}

// Units that were cut, without a shared prefix: blocks for every boundary between CTAs; the first boundary inside a unit joins it.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const __grid_constant__ AttnParams p) {
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
    join_rows<D>(p, j, live, ((size_t)(q.s - 1) * p.rows + node) * p.q_heads + q.h * p.group + (r - node * p.group));
}

// Behind a shared prefix every row has pieces of two units; 32 rows of a sequence may lie in two units of the prefix.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attn_join_shared_kernel(const __grid_constant__ AttnParams p) {
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
    join_rows<D>(p, j, r < R, ((size_t)b * p.rows + node) * p.q_heads + h * p.group + (r - node * p.group));
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
int attn_ctas(const graft_ctx* ctx, bool q8, int head_dim, int group, int rows, int shared) {
    const int ctas = head_dim == 128 ? (q8 ? FewShape<128, true>::kCtas : FewShape<128, false>::kCtas)
                                     : (q8 ? FewShape<64, true>::kCtas : FewShape<64, false>::kCtas);
    return ctx->num_sms * (few_rows(group, rows, shared) ? ctas : 1);
}

struct AttnSizes {
    int part_rows;
    size_t o_seq, o_start, o_join, o_ready, o_ml, o_o, total;
};
AttnSizes attn_sizes(const graft_ctx* ctx, int ctas, int batch, int kv_heads, int head_dim, int group, int rows, int shared) {
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
    z.o_seq = take((size_t)(batch + 1) * sizeof(PlanSeq));
    z.o_start = take((size_t)ctas * sizeof(PlanStart));
    z.o_join = take((size_t)(ctas + 1) * sizeof(PlanJoin));
    z.o_ready = take((size_t)ctas * sizeof(int));
    z.o_ml = take(slots * z.part_rows * sizeof(float2));
    z.o_o = take(slots * z.part_rows * head_dim * sizeof(float));
    z.total = off;
    return z;
}

// The plan, the attention kernel, the joining of what it cut (unless the kernel joins it itself).
template <int D, typename Kernel>
cudaError_t launch_kernels(graft_ctx* ctx, const AttnParams& p, Kernel kernel, int threads, size_t smem, uint32_t ready, bool join, cudaStream_t st) {
    cudaError_t e;
    if (!(ctx->attn_ready & ready)) {
        e = allow_smem((const void*)kernel, smem);
        if (e != cudaSuccess) return e;
        ctx->attn_ready |= ready;
    }
    e = launch_pdl(attn_plan_kernel, dim3(p.batch), dim3(kPlanThreads), 0, st, p);
    if (e != cudaSuccess) return e;
    ctx->launches += 1;
    e = launch_pdl(kernel, dim3(p.ctas), dim3(threads), smem, st, p);
    if (e != cudaSuccess) return e;
    ctx->launches += 1;
    if (!join) return e;
    const long long most = (long long)p.rows * p.group;  // rows of a sequence and key head
    if (p.shared > 0)
        e = launch_pdl(attn_join_shared_kernel<D>, dim3((unsigned)((most + kJoinRows - 1) / kJoinRows), p.c.kv_heads, p.batch),
                       dim3(kJoinThreads), 0, st, p);
    else
        e = launch_pdl(attn_join_kernel<D>, dim3((unsigned)((min(most, (long long)kUnitRows) + kJoinRows - 1) / kJoinRows), max(p.ctas - 1, 1)),
                       dim3(kJoinThreads), 0, st, p);
    ctx->launches += 1;
    return e;
}
template <int D, bool Q8, bool kOne>
cudaError_t launch_attn(graft_ctx* ctx, const AttnParams& p, cudaStream_t st) {
    using S = Shape<D, Q8, kOne>;
    return launch_kernels<D>(ctx, p, tree_attn_kernel<D, Q8, kOne>, S::kThreads, S::kSmem, 1u << ((D == 128) + 2 * Q8 + 4 * kOne), true, st);
}
template <int D, bool Q8>
cudaError_t launch_any(graft_ctx* ctx, const AttnParams& p, cudaStream_t st) {
    const long long rows = (long long)p.rows * p.group;
    if (few_rows(p.group, p.rows, p.shared))
        return launch_kernels<D>(ctx, p, few_attn_kernel<D, Q8>, FewShape<D, Q8>::kThreads, FewShape<D, Q8>::kSmem,
                                 256u << ((D == 128) + 2 * Q8), false, st);
    return p.shared == 0 && rows <= kTile ? launch_attn<D, Q8, true>(ctx, p, st) : launch_attn<D, Q8, false>(ctx, p, st);
}

}  // namespace

size_t tree_attn_scratch_bytes(const graft_ctx* ctx, int batch, const graft_cache* cache, int q_heads, int rows, int shared) {
    const int group = q_heads / cache->kv_heads, ctas = attn_ctas(ctx, cache->dtype == GRAFT_E4M3, cache->head_dim, group, rows, shared);
    return attn_sizes(ctx, ctas, batch, cache->kv_heads, cache->head_dim, group, rows, shared).total;
}

cudaError_t tree_attn_launch(graft_ctx* ctx, int batch, const graft_cache* cache, int layer, int q_heads, int rows, long long q_stride,
                             const void* d_q, float scale, const int32_t* d_prefix_len, const int32_t* d_count, const uint32_t* d_mask,
                             int shared, void* d_out, float* d_lse, int32_t* d_status, void* scratch, cudaStream_t st) {
    AttnParams p;
    p.c = cache_view(cache, layer);
    const bool q8 = cache->dtype == GRAFT_E4M3;
    p.box_rows = cache->page_size < kTile ? cache->page_size : kTile;
    const uint64_t cache_rows = (uint64_t)cache->n_pages * cache->kv_heads * cache->page_size;
    const bool few = few_rows(q_heads / cache->kv_heads, rows, shared);
    if (!few && encode_tiled() == nullptr) return cudaErrorNotSupported;
    if (few)  // (no copies by TMA)
        memset(&p.map_k, 0, sizeof p.map_k), memset(&p.map_v, 0, sizeof p.map_v);
    else if (!encode_map(&p.map_k, p.c.k, q8, cache->head_dim, cache_rows, p.box_rows) ||
             !encode_map(&p.map_v, p.c.v, q8, cache->head_dim, cache_rows, p.box_rows))
        return cudaErrorInvalidValue;
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
    p.shared = shared;
    p.nmax = ctx->nmax;
    p.words = ctx->mask_words;
    p.batch = batch;
    p.ctas = attn_ctas(ctx, q8, cache->head_dim, p.group, rows, shared);
    const AttnSizes z = attn_sizes(ctx, p.ctas, batch, cache->kv_heads, cache->head_dim, p.group, rows, shared);
    uint8_t* base = (uint8_t*)scratch;
    p.head = (PlanHead*)base;
    p.seq = (PlanSeq*)(base + z.o_seq);
    p.start = (PlanStart*)(base + z.o_start);
    p.join = (PlanJoin*)(base + z.o_join);
    p.ready = (int*)(base + z.o_ready);
    p.part_ml = (float2*)(base + z.o_ml);
    p.part_o = (float*)(base + z.o_o);
    p.arrivals = ctx->w_attn_n;
    p.part_rows = z.part_rows;
    p.most_share = few ? 0 : 128;
    const auto launch = cache->head_dim == 128 ? (q8 ? launch_any<128, true> : launch_any<128, false>)
                                               : (q8 ? launch_any<64, true> : launch_any<64, false>);
    return launch(ctx, p, st);
}

}  // namespace graft
