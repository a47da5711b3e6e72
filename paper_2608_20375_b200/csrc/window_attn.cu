// Attention over a paged cache of rows that see the last `window` positions and the first `sinks` (graft_window_attention).
//
// The kernels are those of graft_tree_attention (attn.cuh, kWin); what differs is what they go through.  A tree, or up to 256 / group rows of a
// chain, is an entry of the plan with a line of slots of its own: the sinks, then the slots from the first row's window on up to the last row's
// own, rounded to whole grains (16 slots for few rows, what a copy brings for others).  Rows see less than that at the line's borders alone: tiles
// there are masked row by row, and V of places that only some rows see is looked at for what is not a number, as V of new rows is.
//
// What bounds it.  One token behind a window of 4096: 12.4 us, latencies (the floor is 2.6); 64 of them over e4m3 slots 114 us, 0.73 of the copy's rate (83).
// 32 trees of up to 65 nodes, window 1024: 73 us (10 of them this plan's launch, 9 the join); 16 of up to 513, window 4096, e4m3, head_dim 64: 538; 4 prompts of up to 8192, window 1024: 505 to 550, tensor cores
// busy for 36 %, over e4m3 slots 630; a prompt of 12000, window 4001: 670 to 740 by the clock that power leaves, over e4m3 slots 885 (tiles are converted for every unit of 36 rows).  Beside the chain of scores, exponentials and products that tree_attn.cu
// describes it is the borders: masked tiles cost 9 to 17 % (two of nine tiles behind a window of 1024, four to six of 35 to 37 of a tree of 257 to 513), and a unit's beginning and end as long as three tiles.
// Chains go in blocks of as many rows as make a unit of 256: smaller blocks would mask less and bring K and V more often, at half-empty row tiles.
#include "attn.cuh"

namespace graft {

namespace {

// Rows of a sequence that are an entry: a mask's all (they see one another by the mask), else as many as a unit holds.
__device__ __forceinline__ int entries_of(const AttnParams& p, int n) { return n > 0 ? (n + p.block_rows - 1) / p.block_rows : 0; }

__global__ void __launch_bounds__(kPlanThreads) window_plan_kernel(const __grid_constant__ AttnParams p) {
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kWarps = kPlanThreads / 32;
    const CacheView& c = p.c;
    __shared__ int fine[kWarps], last;
    __shared__ int scratch[3][kWarps];
    __shared__ PlanSeq entries[kPlanSeqs + 1];
    __shared__ int first_entry[kPlanSeqs];
    __shared__ int4 uses[kPlanSeqs];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    {
        const int b = blockIdx.x;
        int n = p.count[b], base = p.prefix_len[b] - 1;
        const int32_t* table = c.table + (size_t)b * c.width;
        bool ok = n >= 0 && n <= p.rows && base >= 0 && (long long)base + n <= ((long long)c.width << c.page_shift);
        if (ok && n > 0) {
            // pages of the sinks, and from the first row's window on
            const int end = base + n, lo = max(0, base - p.window + 1), pages = (end - 1) >> c.page_shift;
            const int sinks = p.sinks > 0 ? min((min(p.sinks, end) - 1) >> c.page_shift, pages) : -1;
            for (int i = tid; i <= sinks; i += kPlanThreads) ok = ok && (unsigned)table[i] < (unsigned)c.n_pages;
            for (int i = max(lo >> c.page_shift, sinks + 1) + tid; i <= pages; i += kPlanThreads) ok = ok && (unsigned)table[i] < (unsigned)c.n_pages;
        }
        int reach = 0;  // of a tree: the deepest node's, as the window's border is as wide as that
        if (p.mask != nullptr && ok)
            for (int i = tid; i < n; i += kPlanThreads) reach = max(reach, window_step(p.position + (size_t)b * p.nmax, i, base));
        ok = __all_sync(0xFFFFFFFFu, ok);
        reach = __reduce_max_sync(0xFFFFFFFFu, reach);
        if (lane == 0) fine[warp] = ok ? reach : -1;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) ok = ok && fine[w] >= 0, reach = max(reach, fine[w]);
        if (tid == 0) {
            if (p.status) p.status[b] = ok ? 0 : GRAFT_ST_BAD_CACHE;
            p.use[b] = make_int4(ok ? n : 0, base, reach, 0);
            last = gridDim.x == 1 || atom_add_acq_rel(p.arrivals, 1) == (int)gridDim.x - 1;
        }
        __syncthreads();
        if (!last) return;
    }
    // the last block: where the sequences' entries begin, what every entry has, where it stands in the line
    const int Hk = c.kv_heads;
    const bool few_seqs = p.batch <= kPlanSeqs;
    int n_entries = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const int4 u = b < p.batch ? __ldcg(p.use + b) : make_int4(0, 0, 0, 0);
        const int mine = entries_of(p, u.x);
        const Sums s = block_sums(scratch, false, mine, 0, 0);
        if (b < p.batch) {
            if (few_seqs)
                first_entry[b] = n_entries + s.before[0], uses[b] = u;
            else
                p.entry0[b] = n_entries + s.before[0];
        }
        n_entries += s.all[0];
    }
    __syncthreads();
    const auto of = [&](int e, PlanSeq& q) {
        q = {};
        if (e >= n_entries) return;
        int lo = 0, hi = p.batch - 1;  // the last sequence whose first entry is not behind e: it has some, as sequences without begin where the next does
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((few_seqs ? first_entry[mid] : p.entry0[mid]) <= e)
                lo = mid;
            else
                hi = mid - 1;
        }
        const int4 u = few_seqs ? uses[lo] : __ldcg(p.use + lo);
        q.b = lo;
        q.node0 = (e - (few_seqs ? first_entry[lo] : p.entry0[lo])) * p.block_rows;
        q.n = min(p.block_rows, u.x - q.node0);
        q.base = u.y + q.node0;
        q.unit0 = p.mask != nullptr ? u.z : q.n - 1;
        q.gap = gap_of(p, q.base);
        q.kt = (q.base + q.n - q.gap + kTile - 1) / kTile;
    };
    const auto cost_of = [&](const PlanSeq& q, int chunk) { return Hk * head_cost(q.n * p.group, q.kt, chunk); };
    const bool small = n_entries <= 32, held = n_entries <= kPlanSeqs;  // (few entries: every warp goes through them by itself)
    const int me = small ? lane : tid;
    PlanSeq q;
    int total = 0, chunk = 1;
    for (int e0 = 0; e0 < n_entries; e0 += kPlanThreads) {
        of(e0 + me, q);
        total += block_sums(scratch, small, cost_of(q, 1), 0, 0).all[0];
    }
    // (short shares: as in attn_plan_kernel)
    const int share = (total + p.ctas - 1) / p.ctas;
    if (share > 1 && share <= p.most_share && n_entries <= kPlanThreads)
        for (int c2 = (share + 5) / 6 * 6; c2 <= share + 11; c2 += 6)
            if (block_sums(scratch, small, cost_of(q, c2) / c2, 0, 0).all[0] <= p.ctas) {
                chunk = c2;
                break;
            }
    int cost = 0;
    if (tid == 0) {
        const PlanSeq none = {};
        p.seq[0] = none;
        entries[0] = none;
    }
    for (int e0 = 0; e0 < n_entries; e0 += kPlanThreads) {
        const int e = e0 + me;
        if (n_entries > kPlanThreads) of(e, q);
        const Sums s = block_sums(scratch, small, cost_of(q, chunk), 0, 0);
        if (e < n_entries && (!small || warp == 0)) {
            q.cost0 = cost + s.before[0];
            p.seq[e + 1] = q;
            if (held) entries[e + 1] = q;
        }
        cost += s.all[0];
    }
    total = cost;
    const int parts = chunk > 1 ? total / chunk : min(p.ctas, total);
    if (tid == 0) {
        p.head->total = total;
        p.head->parts = parts;
        p.head->chunk = chunk;
        p.head->entries = n_entries;
        *p.arrivals = 0;
    }
    __syncthreads();
    plan_starts<true>(p, entries, held, n_entries, total, parts, chunk);
}

template <int D, bool Q8>
cudaError_t launch_any(graft_ctx* ctx, const AttnParams& p, bool few, cudaStream_t st) {
    const uint32_t bit = 1u << ((D == 128) + 2 * Q8);
    if (few && p.self_plan) {
        if (!(ctx->window_ready & bit)) {
            const cudaError_t e = allow_smem((const void*)few_attn_kernel<D, Q8, true>, FewShape<D, Q8, true>::kSmem);
            if (e != cudaSuccess) return e;
            ctx->window_ready |= bit;
        }
        ctx->launches += 1;
        return launch_pdl(few_attn_kernel<D, Q8, true>, dim3(p.ctas), dim3(FewShape<D, Q8, true>::kThreads), FewShape<D, Q8, true>::kSmem, st, p);
    }
    if (few)
        return launch_kernels(ctx, p, window_plan_kernel, few_attn_kernel<D, Q8, true>, FewShape<D, Q8, true>::kThreads, FewShape<D, Q8, true>::kSmem,
                              &ctx->window_ready, bit, [] { return cudaSuccess; }, st);
    const bool one = (long long)p.block_rows * p.group <= kTile;
    const TilesKernel k = window_tiles_kernel(D, Q8, one);
    return launch_kernels(ctx, p, window_plan_kernel, k.kernel, k.threads, k.smem, &ctx->window_ready, bit << (one ? 4 : 8),
                          [&] { return launch_join<D>(ctx, p, st); }, st);
}

struct WindowShape {
    int ctas, block_rows;
    long long entries;
    AttnSizes z;
};
// block_rows: what a unit holds of a chain's rows; all of a tree's
WindowShape window_shape(const graft_ctx* ctx, int batch, const graft_cache* cache, int q_heads, int rows, bool mask) {
    const int group = q_heads / cache->kv_heads;
    WindowShape w;
    w.ctas = attn_ctas<true>(ctx, cache->dtype == GRAFT_E4M3, cache->head_dim, group, rows, 0);
    w.block_rows = mask || (long long)rows * group <= kUnitRows ? rows : group < kUnitRows ? kUnitRows / group : 1;
    w.entries = (long long)batch * ((rows + w.block_rows - 1) / w.block_rows);
    w.z = attn_sizes(w.ctas, batch, (int)w.entries, batch, cache->kv_heads, cache->head_dim, group, w.block_rows, 0);
    return w;
}

}  // namespace

// Bytes of scratch; 0: positions in the line of key tiles would not fit in 32 bits.
size_t window_attn_scratch_bytes(const graft_ctx* ctx, int batch, const graft_cache* cache, int q_heads, int rows, bool mask, int window, int sinks) {
    const WindowShape w = window_shape(ctx, batch, cache, q_heads, rows, mask);
    const double all = (double)cache->table_width * cache->page_size, seen = (double)window + sinks + w.block_rows + 2 * kTile;
    const double row_tiles = (double)w.entries * ((double)w.block_rows * (q_heads / cache->kv_heads) / 128 + 2);
    if ((double)w.entries >= 2147483648.0 || 2 * row_tiles * cache->kv_heads * ((all < seen ? all : seen) / 128 + 2) >= 2147483648.0) return 0;
    return w.z.total;
}

cudaError_t window_attn_launch(graft_ctx* ctx, int batch, const graft_cache* cache, int layer, int q_heads, int rows, long long q_stride,
                               const void* d_q, float scale, const int32_t* d_prefix_len, const int32_t* d_count, const uint32_t* d_mask,
                               const int32_t* d_position, int window, int sinks, void* d_out, float* d_lse, int32_t* d_status, void* scratch,
                               cudaStream_t st) {
    const bool q8 = cache->dtype == GRAFT_E4M3, few = few_rows(q_heads / cache->kv_heads, rows, 0);
    // (a copy brings no more than 32 slots, so that the line's borders are not rounded by more)
    const int box_rows = cache->page_size < 32 ? cache->page_size : 32;
    AttnParams p;
    const cudaError_t e = attn_params(p, ctx, batch, cache, layer, q_heads, rows, q_stride, d_q, scale, d_prefix_len, d_count, d_mask, d_out, d_lse,
                                      d_status, !few, box_rows);
    if (e != cudaSuccess) return e;
    const WindowShape w = window_shape(ctx, batch, cache, q_heads, rows, d_mask != nullptr);
    p.ctas = w.ctas;
    p.block_rows = w.block_rows;
    attn_places(p, w.z, scratch);
    p.most_share = few ? 0 : 128;
    p.self_plan = few && batch <= kSelfSeqs;
    if (p.self_plan) p.ready = ctx->w_window_n;
    const int most = cache->table_width * cache->page_size;  // (below 2^31 - 65536)
    p.position = d_position;
    p.window = window < most ? window : most;  // (neither changes what is seen)
    p.sinks = sinks < most ? sinks : most;
    p.grain = few ? 16 : box_rows;
    p.sink_pad = (p.sinks + p.grain - 1) / p.grain * p.grain;
    const auto launch = cache->head_dim == 128 ? (q8 ? launch_any<128, true> : launch_any<128, false>)
                                               : (q8 ? launch_any<64, true> : launch_any<64, false>);
    return launch(ctx, p, few, st);
}

}  // namespace graft
