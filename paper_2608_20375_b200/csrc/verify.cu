// The acceptance walk for a target that samples (graft_verify): the tree's tokens are kept with the target's own probability, and
// what is left of its distribution is sampled at the node where none is kept.
//
// One cluster of CTAs a sequence; each CTA goes through its share of the visited node's row.  Visited rows only are read, one after
// another: which row comes next is known when the one before is summed up.
#include <float.h>

#include "common.cuh"
#include "internal.h"
#include "umma.cuh"

namespace graft {

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kVec = 8;              // tokens a step and thread
constexpr float kNear = 1e-5f;       // sums of fp32 exponentials are nearer than that (of the whole) to the exact ones
constexpr uint32_t kAll = 0xFFFFFFFFu;

struct VerifyParams {
    const int32_t* n_nodes;
    const int32_t* token;
    const int32_t* parent;
    const uint8_t* logits;  // [batch, rows, V]
    const float* temperature;
    const float* uniform;
    int32_t* accept_len;
    int32_t* accept_path;
    int32_t* bonus;
    int32_t* status;
    int rows, V, nmax, L;
    int hist_w;
    int32_t* hist_window;
    int32_t* hist_count;
    float* hist_out;
};

// what one CTA tells the others about its share of a row
struct Share {
    float m, s;        // largest logit, sum of exp((z - m) / T)
    double sum;        // fp64 sum of exp((z - row's largest) / T)
    uint64_t key;      // T = 0: (order of the largest logit << 32) | ~its id
    int bad;
};

template <bool BF16>
__device__ __forceinline__ float logit(const uint8_t* row, int v) {
    return BF16 ? __uint_as_float((uint32_t)((const uint16_t*)row)[v] << 16) : ((const float*)row)[v];
}

// eight tokens from v on (those at `end` and behind it: -inf); `al`: rows start on 16-byte boundaries
template <bool BF16>
__device__ __forceinline__ void load8(const uint8_t* row, int v, int end, bool al, float (&x)[kVec]) {
    if (al && v + kVec <= end) {
        if (BF16) {
            const uint4 u = __ldg((const uint4*)((const uint16_t*)row + v));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            const float4 a = __ldg((const float4*)((const float*)row + v)), d = __ldg((const float4*)((const float*)row + v) + 1);
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = d.x, x[5] = d.y, x[6] = d.z, x[7] = d.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = v + i < end ? logit<BF16>(row, v + i) : -INFINITY;
    }
}

__device__ __forceinline__ float warp_max(float x) {
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kAll, x, o));
    return x;
}
template <typename T>
__device__ __forceinline__ T warp_sum(T x) {
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}
__device__ __forceinline__ uint64_t warp_max_key(uint64_t k) {
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t y = __shfl_xor_sync(kAll, k, o);
        k = y > k ? y : k;
    }
    return k;
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyParams p) {
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(16) int32_t vsm[];
    int32_t* first_child = vsm;          // [nmax], 0: none (the root is nobody's child)
    int32_t* par = vsm + p.nmax;         // [nmax]
    int32_t* tok = par + p.nmax;         // [nmax]
    __shared__ Share mine, heard[2][kMaxCluster];
    __shared__ float w_m[kWarps], w_s[kWarps];
    __shared__ double w_d[kWarps];
    __shared__ uint64_t w_k[kWarps];
    __shared__ uint32_t filter[32];      // of the children's tokens
    __shared__ int step_next, step_again, step_first, step_n, found;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t n_cta;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_cta));
    const int rank = (int)cluster_ctarank(), ctas = (int)n_cta;
    const int b = blockIdx.y;
    const size_t ob = (size_t)b * p.nmax;
    const int esz = BF16 ? 2 : 4, V = p.V;

    const int n = p.n_nodes[b];
    const float T = p.temperature ? p.temperature[b] : 1.0f;
    const bool greedy = T == 0.0f;
    const bool tree_ok = n >= 1 && n <= p.rows, t_ok = T >= 0.0f && T <= FLT_MAX;
    for (int i = tid; i < p.nmax; i += kThreads) {
        first_child[i] = 0;
        par[i] = p.parent[ob + i];
        tok[i] = p.token[ob + i];
    }
    __syncthreads();
    if (tree_ok)
        for (int i = 1 + tid; i < n; i += kThreads) {  // siblings stand side by side
            const int q = par[i];
            if (q >= 0 && q < i && (i == 1 || par[i - 1] != q)) first_child[q] = i;
        }
    __syncthreads();
    // every CTA's share of a row: whole steps of kVec tokens
    const int steps = (V + kVec - 1) / kVec;
    const int s0 = (int)((long long)steps * rank / ctas), s1 = (int)((long long)steps * (rank + 1) / ctas);
    const double inv_T = greedy ? 1.0 : 1.0 / (double)T;
    const float cf = (float)((double)kLog2e * inv_T);

    int cur = 0, a = 0, status = !tree_ok ? GRAFT_ST_BAD_TREE : !t_ok ? GRAFT_ST_BAD_LOGITS : 0, bonus = -1;
    int path = -1;  // lane l of warp 0 keeps step l
    // Tell the others, hear the others: `heard` by turns, so that one barrier an exchange is enough (who writes to a half again has
    // passed the barrier that all arrive at after they read it).
    int turn = 0;
    const Share* all = nullptr;
    auto exchange = [&]() {
        __syncthreads();  // `mine` is written
        if (tid < ctas) {
            const uint32_t to = mapa_u32(smem_u32(&heard[turn][rank]), tid);
            const uint32_t* w = (const uint32_t*)&mine;
#pragma unroll
            for (int i = 0; i < (int)(sizeof(Share) / 4); ++i)
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 4 * i), "r"(w[i]) : "memory");
        }
        cluster_sync();
        all = heard[turn];
        turn ^= 1;
    };
    while (status == 0) {
        const uint8_t* row = p.logits + ((size_t)b * p.rows + cur) * V * esz;
        const bool al = ((uintptr_t)row & 15) == 0;
        // ---- largest logit and the sum of exponentials of this CTA's share
        float m = -FLT_MAX, s = 0.0f;
        bool bad = false;
        uint64_t key = 0;
        for (int st = s0 + tid; st < s1; st += kThreads) {
            float x[kVec];
            load8<BF16>(row, st * kVec, V, al, x);
            float vm = x[0];
#pragma unroll
            for (int i = 1; i < kVec; ++i) vm = fmaxf(vm, x[i]);
#pragma unroll
            for (int i = 0; i < kVec; ++i) bad = bad || !(x[i] <= FLT_MAX);
            if (greedy) {
                if (key == 0 || vm > m) {
                    m = vm;
                    int at = 0;
#pragma unroll
                    for (int i = kVec - 1; i >= 0; --i)
                        if (x[i] == vm) at = i;
                    key = make_key(__float_as_uint(vm), (uint32_t)(st * kVec + at));
                }
            } else {
                if (vm > m) {
                    s *= ex2_approx((m - vm) * cf);
                    m = vm;
                }
                float t[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) t[i] = ex2_approx((x[i] - m) * cf);
                s += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
            }
        }
        const float wm = warp_max(m);
        const float ws = warp_sum(s * ex2_approx((m - wm) * cf));
        const uint64_t wk = warp_max_key(key);
        const bool wb = __any_sync(kAll, bad);
        if (lane == 0) {
            w_m[warp] = wm;
            w_s[warp] = ws;
            w_k[warp] = wk;
            w_d[warp] = wb ? 1.0 : 0.0;
        }
        __syncthreads();
        if (warp == 0) {
            const float xm = lane < kWarps ? w_m[lane] : -FLT_MAX, xs = lane < kWarps ? w_s[lane] : 0.0f;
            const float am = warp_max(xm), as = warp_sum(xs * ex2_approx((xm - am) * cf));
            const uint64_t ak = warp_max_key(lane < kWarps ? w_k[lane] : 0);
            const bool ab = __any_sync(kAll, lane < kWarps && w_d[lane] != 0.0);
            if (lane == 0) {
                mine.m = am;
                mine.s = as;
                mine.key = ak;
                mine.bad = ab;
            }
        }
        exchange();
        float top = -FLT_MAX, Zf = 0.0f;
        uint64_t best = 0;
        bool row_bad = false;
        for (int r = 0; r < ctas; ++r) {
            top = fmaxf(top, all[r].m);
            best = all[r].key > best ? all[r].key : best;
            row_bad = row_bad || all[r].bad;
        }
        for (int r = 0; r < ctas; ++r) Zf += all[r].s * ex2_approx((all[r].m - top) * cf);
        // (a row without a finite entry: no exponential above zero, or as key the one of -inf)
        row_bad = row_bad || (greedy ? (uint32_t)(best >> 32) <= ord_from_float(-INFINITY) : !(Zf > 0.0f));
        if (row_bad) {
            status = GRAFT_ST_BAD_LOGITS;
            break;
        }
        const double dtop = (double)top;
        // ---- the children, in turn: every CTA finds the same
        double Z = (double)Zf;
        bool exact = greedy;
        int next = 0, n_child = 0;
        const int fc = a < p.L ? first_child[cur] : 0;
        for (;;) {
            if (warp == 0) {
                double ahead = 0.0;
                int nx = 0, again = 0, c0 = fc;
                if (fc > 0)
                    for (;; c0 += 32) {
                        const int c = c0 + lane;
                        const bool is = c < n && par[c] == cur;
                        const unsigned kids = __ballot_sync(kAll, is);
                        if (kids == 0) break;
                        const int v = is ? tok[c] : -1;
                        double w = 0.0;
                        if (is && v >= 0 && v < V) {
                            if (greedy)
                                w = (uint32_t)v == key_id(best) ? 1.0 : 0.0;
                            else
                                w = exp(((double)logit<BF16>(row, v) - dtop) * inv_T);
                            for (int e = fc; e < c; ++e)
                                if (tok[e] == v) w = 0.0;  // an earlier sibling's token is taken already
                        }
                        double sum = w;
                        for (int o = 1; o < 32; o <<= 1) {
                            const double y = __shfl_up_sync(kAll, sum, o);
                            if (lane >= o) sum += y;
                        }
                        const double left = (greedy ? 1.0 : Z) - (ahead + (sum - w));
                        const double u = is ? (double)p.uniform[ob + c] : 2.0;
                        const bool ok = is && u * left < w;
                        const bool near = is && !exact && w > 0.0 && fabs(u * left - w) <= (double)kNear * Z;
                        const unsigned oks = __ballot_sync(kAll, ok), nears = __ballot_sync(kAll, near);
                        const int f = oks ? __ffs(oks) - 1 : 32;
                        if (nears & (f >= 31 ? kAll : ((2u << f) - 1))) {
                            again = 1;
                            break;
                        }
                        if (oks) {
                            nx = c0 + f;
                            break;
                        }
                        ahead += __shfl_sync(kAll, sum, 31);
                        n_child = c0 + __popc(kids) - fc;
                        if (kids != kAll) break;
                    }
                if (lane == 0) {
                    step_next = nx;
                    step_again = again;
                    step_n = n_child;
                }
            }
            __syncthreads();
            next = step_next;
            n_child = step_n;
            const int again = step_again;
            __syncthreads();
            if (!again) break;
            // too close for sums of fp32 exponentials: the row's sum again in fp64
            double d = 0.0;
            for (int st = s0 + tid; st < s1; st += kThreads) {
                float x[kVec];
                load8<BF16>(row, st * kVec, V, al, x);
#pragma unroll
                for (int i = 0; i < kVec; ++i) d += exp(((double)x[i] - dtop) * inv_T);
            }
            d = warp_sum(d);
            if (lane == 0) w_d[warp] = d;
            __syncthreads();
            if (tid == 0) {
                double t = 0.0;
                for (int i = 0; i < kWarps; ++i) t += w_d[i];
                mine.sum = t;
            }
            exchange();
            Z = 0.0;
            for (int r = 0; r < ctas; ++r) Z += all[r].sum;
            exact = true;
        }
        if (next > 0) {
            if (warp == 0 && lane == a) path = next;
            a += 1;
            cur = next;
            continue;
        }
        // ---- nobody: the bonus token
        if (greedy) {
            bonus = (int)key_id(best);
            break;
        }
        // (a step's tokens share a bit of the filter; a step whose bit is set looks through the children)
        if (tid < 32) filter[tid] = 0;
        __syncthreads();
        for (int e = tid; e < n_child; e += kThreads) {
            const int v = tok[fc + e];
            if (v >= 0 && v < V) atomicOr(&filter[(v >> 8) & 31], 1u << ((v >> 3) & 31));
        }
        __syncthreads();
        auto weights = [&](int st, double (&w)[kVec]) {
            float x[kVec];
            load8<BF16>(row, st * kVec, V, al, x);
#pragma unroll
            for (int i = 0; i < kVec; ++i) w[i] = exp(((double)x[i] - dtop) * inv_T);
            if ((filter[(st >> 5) & 31] >> (st & 31)) & 1)
                for (int e = 0; e < n_child; ++e) {
                    const int v = tok[fc + e];
                    if (v >> 3 == st) {
#pragma unroll
                        for (int i = 0; i < kVec; ++i)
                            if (i == (v & 7)) w[i] = 0.0;
                    }
                }
        };
        // a warp's steps follow one another, so that its sum is one stretch of the distribution
        const int own = s1 - s0, v0 = s0 + (int)((long long)own * warp / kWarps), v1 = s0 + (int)((long long)own * (warp + 1) / kWarps);
        double d = 0.0;
        for (int st = v0 + lane; st < v1; st += 32) {
            double w[kVec];
            weights(st, w);
            d += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        }
        d = warp_sum(d);
        if (lane == 0) w_d[warp] = d;
        if (tid == 0) found = -1;
        __syncthreads();
        if (tid == 0) {
            double t = 0.0;
            for (int i = 0; i < kWarps; ++i) t += w_d[i];
            mine.sum = t;
        }
        exchange();
        double total = 0.0, before = 0.0;
        for (int r = 0; r < ctas; ++r) {
            if (r == rank) before = total;
            total += all[r].sum;
        }
        const double goal = (double)p.uniform[ob] * total;
        double upto = before;
        for (int i = 0; i < warp; ++i) upto += w_d[i];
        // the warp whose stretch holds the goal goes through it once more
        if (upto <= goal && goal < upto + w_d[warp]) {
            double at = upto;
            int hit = -1;
            for (int st = v0; st < v1 && hit < 0; st += 32) {
                double w[kVec] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (st + lane < v1) weights(st + lane, w);
                const double sum = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                double incl = sum;
                for (int o = 1; o < 32; o <<= 1) {
                    const double y = __shfl_up_sync(kAll, incl, o);
                    if (lane >= o) incl += y;
                }
                const unsigned over = __ballot_sync(kAll, at + incl > goal);
                if (over) {
                    const int l = __ffs(over) - 1;
                    int h = -1;
                    if (lane == l) {
                        double q = at + (incl - sum);
                        bool over_it = false;
#pragma unroll
                        for (int i = 0; i < kVec; ++i) {
                            q += w[i];
                            if (w[i] > 0.0 && !over_it) h = (st + lane) * kVec + i;  // (the last, should rounding have it so)
                            over_it = over_it || q > goal;
                        }
                    }
                    hit = __shfl_sync(kAll, h, l);
                }
                at += __shfl_sync(kAll, incl, 31);
            }
            if (lane == 0 && hit >= 0) found = hit;
        }
        __syncthreads();
        if (tid == 0) mine.key = (uint64_t)(uint32_t)found;
        exchange();
        for (int r = 0; r < ctas; ++r)
            if ((int)(uint32_t)all[r].key >= 0) bonus = (int)(uint32_t)all[r].key;
        if (bonus >= 0) break;
        // nothing is left (the children held all of it, and rounding kept each from being accepted): the row's likeliest token
        int id = 0x7FFFFFFF;
        for (int st = s0 + tid; st < s1; st += kThreads) {
            float x[kVec];
            load8<BF16>(row, st * kVec, V, al, x);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (x[i] == top) id = min(id, st * kVec + i);
        }
        id = __reduce_min_sync(kAll, id);
        if (lane == 0) w_k[warp] = (uint64_t)(uint32_t)id;
        __syncthreads();
        if (tid == 0) {
            uint64_t k = w_k[0];
            for (int i = 1; i < kWarps; ++i) k = w_k[i] < k ? w_k[i] : k;
            mine.key = k;
        }
        exchange();
        bonus = 0x7FFFFFFF;
        for (int r = 0; r < ctas; ++r) bonus = min(bonus, (int)(uint32_t)all[r].key);
        break;
    }
    cluster_sync();  // nobody leaves while others write to it
    if (rank != 0 || warp != 0) return;
    if (!tree_ok) a = 0;
    if (lane < p.L) p.accept_path[(size_t)b * p.L + lane] = path;
    if (lane == 0) {
        p.accept_len[b] = a;
        p.bonus[b] = bonus;
        if (p.status) p.status[b] = status;
        if (p.hist_w > 0) {
            const int w = p.hist_w;
            int k = p.hist_count[b];
            int32_t* ring = p.hist_window + (size_t)b * w;
            ring[k % w] = a;
            k += 1;
            p.hist_count[b] = k;
            const int cnt = k < w ? k : w;
            int sum = 0;
#pragma unroll 1
            for (int i = 0; i < cnt; ++i) sum += ring[i];
            p.hist_out[b] = (float)((double)sum / (double)cnt);
        }
    }
}

}  // namespace

cudaError_t verify_launch(graft_ctx* ctx, int batch, const graft_tree_out* trees, int rows, graft_dtype dt, const void* d_logits,
                          const float* d_temperature, const float* d_uniform, int32_t* d_accept_len, int32_t* d_accept_path,
                          int32_t* d_bonus, int32_t* d_status, cudaStream_t st) {
    VerifyParams p;
    p.n_nodes = trees->d_n_nodes;
    p.token = trees->d_token;
    p.parent = trees->d_parent;
    p.logits = (const uint8_t*)d_logits;
    p.temperature = d_temperature;
    p.uniform = d_uniform;
    p.accept_len = d_accept_len;
    p.accept_path = d_accept_path;
    p.bonus = d_bonus;
    p.status = d_status;
    p.rows = rows;
    p.V = ctx->cfg.V;
    p.nmax = ctx->nmax;
    p.L = ctx->cfg.L;
    p.hist_w = ctx->hist_w;
    p.hist_window = ctx->hist_window;
    p.hist_count = ctx->hist_count;
    p.hist_out = ctx->hist_out;
    int ctas = kMaxCluster;
    while (ctas > 1 && ctas * batch > 2 * ctx->num_sms) ctas >>= 1;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(ctas, batch);
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = (size_t)3 * ctx->nmax * sizeof(int32_t);
    lc.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = ctas;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&lc, dt == GRAFT_BF16 ? verify_kernel<true> : verify_kernel<false>, p);
    ctx->launches += 1;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace graft
