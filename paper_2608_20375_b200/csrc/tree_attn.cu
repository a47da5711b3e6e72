// Attention of the trees' nodes over a paged cache (graft_tree_attention), on the tcgen05 tensor cores.  (The kernels are in attn.cuh.)
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
#include "attn.cuh"

namespace graft {

namespace {

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
        return launch_tree<D>(ctx, p, few_attn_kernel<D, Q8, false>, FewShape<D, Q8>::kThreads, FewShape<D, Q8>::kSmem,
                                 256u << ((D == 128) + 2 * Q8), false, st);
    return p.shared == 0 && rows <= kTile ? launch_attn<D, Q8, true>(ctx, p, st) : launch_attn<D, Q8, false>(ctx, p, st);
}

}  // namespace

size_t tree_attn_scratch_bytes(const graft_ctx* ctx, int batch, const graft_cache* cache, int q_heads, int rows, int shared) {
    const int group = q_heads / cache->kv_heads, ctas = attn_ctas(ctx, cache->dtype == GRAFT_E4M3, cache->head_dim, group, rows, shared);
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
    p.ctas = attn_ctas(ctx, q8, cache->head_dim, p.group, rows, shared);
    attn_places(p, attn_sizes(p.ctas, batch, batch, 0, cache->kv_heads, cache->head_dim, p.group, rows, shared), scratch);
    p.most_share = few ? 0 : 128;
    const auto launch = cache->head_dim == 128 ? (q8 ? launch_any<128, true> : launch_any<128, false>)
                                               : (q8 ? launch_any<64, true> : launch_any<64, false>);
    return launch(ctx, p, st);
}

}  // namespace graft

