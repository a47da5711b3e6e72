// The acceptance walk for a target that samples (graft_verify): the tree's tokens are kept with the target's own probability, and
// what is left of its distribution is sampled at the node where none is kept.
//
// One cluster of CTAs a sequence; each CTA goes through its share of the visited node's row.  Visited rows only are read, one after
// another: which row comes next is known when the one before is summed up.
//
// What bounds it: a chain of dependent steps, one a visited node.  64 sequences, 65 nodes, V = 151,936 bf16, 13 steps in the longest walk: 78 to
// 89 us, of which 5 a step (a row of 304 KB by 8 CTAs, their sums exchanged through the cluster's shared memory) and 14 for the bonus token, whose
// row is summed in fp64 (64 operations a clock and SM) and gone through twice more.  One sequence, V = 32,000 fp32, 16 CTAs: 12 to 19 us, by the
// walk's length.  Rows read: 58 MB, 9 us at the copy's rate.
#include <float.h>

#include "common.cuh"
#include "internal.h"
#include "umma.cuh"

namespace graft {

namespace {

constexpr int kThreads = 256;  // four CTAs an SM: a sequence's cluster then spreads over as many SMs as can be
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;
constexpr int kRoots = 256;          // entries of the table of 2^(j / 256)
constexpr int kHeldWords = 2048;     // (shares of more than 65,536 pieces: bits are used again)
constexpr int kGroups = 64;          // sums that a warp keeps of its stretch of the last row
constexpr float kLeastT = 0x1p-64f;  // temperatures between 0 and this one count as it: exponents then stay in fp32's range
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
    int bring_ahead;  // the likeliest next rows are brought to L2
    int hist_w;
    int32_t* hist_window;
    int32_t* hist_count;
    float* hist_out;
};

template <bool BF16>
__device__ __forceinline__ float logit(const uint8_t* row, int v) {
    return BF16 ? __uint_as_float((uint32_t)((const uint16_t*)row)[v] << 16) : ((const float*)row)[v];
}

// A row as 16-byte pieces on 16-byte boundaries, whatever it begins on: piece s holds tokens s kE - skip .. + kE - 1, at least one of them of
// the row.
template <bool BF16>
struct Row {
    static constexpr int kE = BF16 ? 8 : 4;
    const uint4* at;
    int skip, pieces, V;
    __device__ __forceinline__ Row(const uint8_t* row, int V_) {
        const int low = (int)((uintptr_t)row & 15);
        at = (const uint4*)(row - low);
        skip = low / (BF16 ? 2 : 4);
        V = V_;
        pieces = (V + skip + kE - 1) / kE;
    }
    __device__ __forceinline__ int first(int s) const { return s * kE - skip; }
    // -inf in the place of what is not the row's
    __device__ __forceinline__ void unpack(const uint4& u, int s, bool there, float (&x)[kE]) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        const int v = first(s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (BF16) {
                x[(2 * i) % kE] = __uint_as_float(w[i] << 16);
                x[(2 * i + 1) % kE] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else
                x[i % kE] = __uint_as_float(w[i]);
        }
        if (!there || v < 0 || v + kE > V)
#pragma unroll
            for (int i = 0; i < kE; ++i) x[i] = there && v + i >= 0 && v + i < V ? x[i] : -INFINITY;
    }
};

// x as a double by integer operations (conversions run at a quarter of the rate of the arithmetic): zero and what is below 2^-126 come out up
// to 2^-126 off, which is 2^-61 in an exponent at the least temperature, and -inf as -2^128.
__device__ __forceinline__ double widen(float x) {
    const uint32_t u = __float_as_uint(x);
    return __hiloint2double((int)((u & 0x80000000u) | (((u & 0x7FFFFFFFu) >> 3) + 0x38000000u)), (int)(u << 29));
}
// 2^t in fp64 for t <= 0 or so (up to `none`, -1000 or above it: 0): t = n + j / 256 + r, |r| <= 1/512, a table of 2^(j / 256) and the exponential series to the
// third power, whose rest is below 2e-13.  The sum with 1.5 2^44 leaves 256 (n + j / 256) in its last bits.
constexpr double kFineMagic = 26388279066624.0, kFine1 = 0.69314718055994531, kFine2 = 0.24022650695910072, kFine3 = 0.05550410866482158;  // (ln 2, its square over 2, its cube over 6)
__device__ __forceinline__ double exp2_fine(double t, double none, const double* roots) {
    const double m = t + kFineMagic, r = t - (m - kFineMagic);
    const int k = __double2loint(m);
    double q = fma(r, kFine3, kFine2);
    q = fma(q, r, kFine1);
    q = fma(q, r, 1.0);
    q *= roots[k & (kRoots - 1)];
    return t > none ? __hiloint2double(__double2hiint(q) + ((k >> 8) << 20), __double2loint(q)) : 0.0;
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
__global__ void __launch_bounds__(kThreads, 4) verify_kernel(const VerifyParams p) {
    using R = Row<BF16>;
    constexpr int kE = R::kE, kAhead = 8;  // pieces that a thread has on their way
    pdl_launch_dependents();
    // (this CTA is there: others write to its shared memory once all have arrived, see the wait below)
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    extern __shared__ __align__(16) int32_t vsm[];
    int32_t* first_child = vsm;          // [nmax], 0: none (the root is nobody's child)
    int32_t* par = vsm + p.nmax;         // [nmax]
    int32_t* tok = par + p.nmax;         // [nmax]
    float* uni = (float*)(tok + p.nmax);  // [nmax]
    __shared__ uint64_t heard[2][kMaxCluster * kWarps];
    __shared__ double roots[kRoots], group[kWarps][kGroups];
    __shared__ uint32_t held[kHeldWords];  // pieces of this CTA's share that hold a token of the children
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t n_cta;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_cta));
    const int rank = (int)cluster_ctarank(), ctas = (int)n_cta, ctas_log = 31 - __clz(ctas);  // (a power of two)
    const int b = blockIdx.y;
    const size_t ob = (size_t)b * p.nmax;
    const int esz = BF16 ? 2 : 4, V = p.V;
    for (int i = tid; i < kRoots; i += kThreads) roots[i] = exp2((double)i / kRoots);
    pdl_wait();

    const int n = p.n_nodes[b];
    const float T = p.temperature ? p.temperature[b] : 1.0f;
    const bool greedy = T == 0.0f;
    const bool tree_ok = n >= 1 && n <= p.rows, t_ok = T >= 0.0f && T <= FLT_MAX;
    for (int i = tid; i < p.nmax; i += kThreads) {
        first_child[i] = 0;
        par[i] = p.parent[ob + i];
        tok[i] = p.token[ob + i];
        uni[i] = p.uniform[ob + i];
    }
    __syncthreads();
    if (tree_ok)
        for (int i = 1 + tid; i < n; i += kThreads) {  // siblings stand side by side
            const int q = par[i];
            if (q >= 0 && q < i && (i == 1 || par[i - 1] != q)) first_child[q] = i;
        }
    __syncthreads();
    const double inv_T = greedy ? 1.0 : 1.0 / (double)fmaxf(T, kLeastT), c64 = 1.4426950408889634 * inv_T;
    const float cf = (float)c64;
    // (at temperatures near fp32's largest, differences that fp32 does not hold weigh something: all comparisons take the exact sum)
    const double near_by = T > 0x1p100f ? 1e300 : (double)kNear;

    int cur = 0, a = 0, status = !tree_ok ? GRAFT_ST_BAD_TREE : !t_ok ? GRAFT_ST_BAD_LOGITS : 0, bonus = -1;
    int path = -1;  // lane l of warp 0 keeps step l
    // Every warp tells every warp of the cluster eight bytes (the same in all its lanes); `heard` by turns, so that one barrier an exchange is
    // enough (who writes to a half again has passed the barrier that all arrive at after they read it).  Then all warps work out the same.
    int turn = 0;
    const uint64_t* all = nullptr;
    const int voices = ctas * kWarps, voice = rank * kWarps + warp;
    const auto exchange = [&](uint64_t mine) {
        __syncwarp();
        if (lane < ctas) asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(mapa_u32(smem_u32(&heard[turn][voice]), lane)), "l"(mine) : "memory");
        cluster_sync();
        all = heard[turn];
        turn ^= 1;
    };
    // the sum of all warps' numbers, and of those ahead of voice v: every warp gets the same for the same v
    const auto sum_all = [&]() {
        double t = 0.0;
        for (int i = lane; i < voices; i += 32) t += __longlong_as_double((long long)all[i]);
        return warp_sum(t);
    };
    const auto sum_ahead = [&](int v) {
        double t = 0.0;
        for (int i = lane; i < v; i += 32) t += __longlong_as_double((long long)all[i]);
        return warp_sum(t);
    };
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // all CTAs of the cluster have begun
    // this CTA's share of n things begins at
    const auto share = [&](int n, int r) { return (int)(((long long)n * r) >> ctas_log); };
    while (status == 0) {
        const uint8_t* base = p.logits + ((size_t)b * p.rows + cur) * V * esz;
        const R row(base, V);
        const int s0 = share(row.pieces, rank), s1 = share(row.pieces, rank + 1);
        // f(numbers, piece) for this thread's pieces of [from, to), `step` apart; loads of kAhead pieces go ahead of the work on them
        const auto each = [&](int from, int to, int step, auto f) {
            for (int st = from; st < to; st += step * kAhead) {
                uint4 u[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) u[i] = __ldg(row.at + min(st + i * step, to - 1));
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (st + i * step >= to) break;
                    float x[kE];
                    row.unpack(u[i], st + i * step, true, x);
                    f(x, st + i * step);
                }
            }
        };
        // the first children's logits are asked for ahead of the row, and the row of the first of them, the likeliest next, is brought to L2
        const int fc = a < p.L ? first_child[cur] : 0;
        int v_c = -1;
        float z_c = 0.0f;
        if (fc > 0) {
            if (fc + lane < n && par[fc + lane] == cur) {
                v_c = tok[fc + lane];
                if (v_c >= 0 && v_c < V) z_c = logit<BF16>(base, v_c);
            }
            if (fc < p.rows && p.bring_ahead) {
                const uint8_t* ahead = base + (size_t)(fc - cur) * V * esz;
                for (int i = s0 + 8 * tid; i < s1; i += 8 * kThreads) asm volatile("prefetch.global.L2 [%0];" ::"l"(ahead + (size_t)i * 16));
            }
        }
        // the same a piece at a time, the next one on its way: passes that are made once are short code, as most of their time would go to
        // fetching it
        const auto each_short = [&](int from, int to, int step, auto f) {
            uint4 u = __ldg(row.at + max(min(from, to - 1), 0));
#pragma unroll 1
            for (int st = from; st < to; st += step) {
                const uint4 next = __ldg(row.at + min(st + step, to - 1));
                float x[kE];
                row.unpack(u, st, true, x);
                f(x, st);
                u = next;
            }
        };
        // ---- largest logit and the sum of exponentials of this CTA's share
        float m = -FLT_MAX, s = 0.0f;
        bool bad = false;
        uint64_t key = 0;
        if (greedy)
            each(s0 + tid, s1, kThreads, [&](const float (&x)[kE], int st) {
                float vm = x[0];
#pragma unroll
                for (int i = 1; i < kE; ++i) vm = fmaxf(vm, x[i]);
#pragma unroll
                for (int i = 0; i < kE; ++i) bad = bad || !(x[i] <= FLT_MAX);
                if (key == 0 || vm > m) {
                    m = vm;
                    int at = 0;
#pragma unroll
                    for (int i = kE - 1; i >= 0; --i)
                        if (x[i] == vm && row.first(st) + i >= 0 && row.first(st) + i < V) at = i;
                    key = make_key(__float_as_uint(vm), (uint32_t)(row.first(st) + at));
                }
            });
        else
            each(s0 + tid, s1, kThreads, [&](const float (&x)[kE], int st) {
                float vm = x[0];
#pragma unroll
                for (int i = 1; i < kE; ++i) vm = fmaxf(vm, x[i]);
                if (vm > m) {
                    s *= ex2_approx((m - vm) * cf);
                    m = vm;
                }
                float t = 0.0f;
#pragma unroll
                for (int i = 0; i < kE; ++i) t += ex2_approx((x[i] - m) * cf);  // (NaN and +inf: NaN)
                s += t;
            });
        float top, Zf;
        uint64_t best = 0;
        bool row_bad = false;
        if (greedy) {
            best = warp_max_key(key);
            exchange(__any_sync(kAll, bad) ? ~0ull : best);
            best = 0;
            for (int i = lane; i < voices; i += 32) best = all[i] > best ? all[i] : best;
            best = warp_max_key(best);
            row_bad = best == ~0ull;
            top = 0.0f, Zf = 1.0f;
        } else {
            const float wm = warp_max(m), ws = warp_sum(s * ex2_approx((m - wm) * cf));
            exchange((uint64_t)__float_as_uint(ws) << 32 | __float_as_uint(wm));
            float xm = -FLT_MAX;
            for (int i = lane; i < voices; i += 32) xm = fmaxf(xm, __uint_as_float((uint32_t)all[i]));
            top = warp_max(xm);
            float xs = 0.0f;
            for (int i = lane; i < voices; i += 32)
                xs += __uint_as_float((uint32_t)(all[i] >> 32)) * ex2_approx((__uint_as_float((uint32_t)all[i]) - top) * cf);
            Zf = warp_sum(xs);
        }
        // (a row without a finite entry: no exponential above zero, or as key the one of -inf)
        row_bad = row_bad || (greedy ? (uint32_t)(best >> 32) <= ord_from_float(-INFINITY) : !(Zf > 0.0f));
        if (row_bad) {
            status = GRAFT_ST_BAD_LOGITS;
            break;
        }
        // (the difference first: it is exact or nearly so, and 0 for the largest, whatever the temperature; -inf is told from the lowest
        // finite numbers at the highest ones too)
        const double zero = widen(top), none = fmax(-1000.0, (widen(-INFINITY) - zero) * c64);
        const auto weight = [&](float x) { return exp2_fine((widen(x) - zero) * c64, none, roots); };
        // ---- the children, in turn: every warp finds the same
        double Z = (double)Zf;
        bool exact = greedy;
        int next = 0, n_child = 0;
        for (;;) {
            double ahead = 0.0;
            bool again = false;
            if (fc > 0)
                for (int c0 = fc;; c0 += 32) {
                    const int c = c0 + lane;
                    const bool is = c < n && par[c] == cur;
                    const unsigned kids = __ballot_sync(kAll, is);
                    if (kids == 0) break;
                    const int v = is ? tok[c] : -1;
                    const double u = is ? (double)uni[c] : 2.0;
                    double w = 0.0;
                    if (is && v >= 0 && v < V) {
                        if (greedy)
                            w = (uint32_t)v == key_id(best) ? 1.0 : 0.0;
                        else
                            w = weight(c0 == fc ? z_c : logit<BF16>(base, v));
                        for (int e = fc; e < c; ++e)
                            if (tok[e] == v) w = 0.0;  // an earlier sibling's token is taken already
                    }
                    double sum = w;
                    for (int o = 1; o < 32; o <<= 1) {
                        const double y = __shfl_up_sync(kAll, sum, o);
                        if (lane >= o) sum += y;
                    }
                    const double left = (greedy ? 1.0 : Z) - (ahead + (sum - w));
                    const bool ok = is && w > 0.0 && u * left < w;  // (rounding may leave less than nothing behind the siblings)
                    const bool near = is && !exact && w > 0.0 && fabs(u * left - w) <= near_by * Z;
                    const unsigned oks = __ballot_sync(kAll, ok), nears = __ballot_sync(kAll, near);
                    const int f = oks ? __ffs(oks) - 1 : 32;
                    if (nears & (f >= 31 ? kAll : ((2u << f) - 1))) {
                        again = true;
                        break;
                    }
                    if (oks) {
                        next = c0 + f;
                        break;
                    }
                    ahead += __shfl_sync(kAll, sum, 31);
                    n_child = c0 + __popc(kids) - fc;
                    if (kids != kAll) break;
                }
            if (!again) break;
            // too close for sums of fp32 exponentials: the row's sum again in fp64
            double d = 0.0;
            each_short(s0 + tid, s1, kThreads, [&](const float (&x)[kE], int) {
#pragma unroll
                for (int i = 0; i < kE; ++i) d += weight(x[i]);
            });
            exchange((uint64_t)__double_as_longlong(warp_sum(d)));
            Z = sum_all();
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
        // (a piece that holds a token of the children is marked, and looks through them)
        const auto word = [&](int st) -> uint32_t& { return held[((st - s0) >> 5) & (kHeldWords - 1)]; };
        __syncthreads();
        for (int i = tid; i < min(kHeldWords, (s1 - s0 + 31) / 32); i += kThreads) held[i] = 0;
        __syncthreads();
        for (int e = tid; e < n_child; e += kThreads) {
            const int v = tok[fc + e], st = (v + row.skip) / kE;
            if (v >= 0 && v < V && st >= s0 && st < s1) atomicOr(&word(st), 1u << ((st - s0) & 31));
        }
        __syncthreads();
        const auto weights = [&](const float (&x)[kE], int st, double (&w)[kE]) {
            // (four at a time, step by step: an fp64 result takes some thirty cycles, and registers are for four)
#pragma unroll
            for (int i0 = 0; i0 < kE; i0 += 4) {
                double r[4], q[4];
                int k[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = (widen(x[i0 + i]) - zero) * c64;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i0 + i] = r[i];
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = r[i] + kFineMagic, k[i] = __double2loint(q[i]);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] -= kFineMagic;
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] -= q[i];
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = fma(r[i], kFine3, kFine2);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = fma(q[i], r[i], kFine1);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = fma(q[i], r[i], 1.0);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] *= roots[k[i] & (kRoots - 1)];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i0 + i] = w[i0 + i] > none ? __hiloint2double(__double2hiint(q[i]) + ((k[i] >> 8) << 20), __double2loint(q[i])) : 0.0;
            }
            if (st < s1 && (word(st) >> ((st - s0) & 31)) & 1)
                for (int e = 0; e < n_child; ++e) {
                    const int i0 = tok[fc + e] - row.first(st);
#pragma unroll
                    for (int i = 0; i < kE; ++i)
                        if (i == i0) w[i] = 0.0;
                }
        };
        const auto add_up = [](const double (&w)[kE]) {
            double t = (w[0] + w[1]) + (w[2] + w[3]);
            if (kE == 8) t += (w[4 % kE] + w[5 % kE]) + (w[6 % kE] + w[7 % kE]);
            return t;
        };
        // a warp's pieces follow one another, so that its sum is one stretch of the distribution
        const int own = s1 - s0, v0 = s0 + own * warp / kWarps, v1 = s0 + own * (warp + 1) / kWarps;
        // (sums of groups of it are kept, so that the place of the goal is found without going through all of it again)
        const int steps = (v1 - v0 + 31) / 32, per = (steps + kGroups - 1) / kGroups;
        if (lane + 32 < kGroups) group[warp][lane + 32] = 0.0;
        group[warp][lane] = 0.0;
        __syncwarp();
#pragma unroll 1
        for (int k = 0; k * per < steps; ++k) {
            double d = 0.0;
            each_short(v0 + 32 * per * k + lane, min(v1, v0 + 32 * per * (k + 1)), 32, [&](const float (&x)[kE], int st) {
                double w[kE];
                weights(x, st, w);
                d += add_up(w);
            });
            d = warp_sum(d);
            if (lane == 0) group[warp][k] = d;
        }
        __syncwarp();
        static_assert(kGroups == 64, "two groups a lane");
        const double g0 = group[warp][2 * lane], g1 = group[warp][2 * lane + 1];
        double upto = g0 + g1;
        for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(kAll, upto, o);
            if (lane >= o) upto += y;
        }
        exchange((uint64_t)__double_as_longlong(__shfl_sync(kAll, upto, 31)));
        const double goal = (double)uni[0] * sum_all(), mine_from = sum_ahead(voice), mine_to = voice + 1 < voices ? sum_ahead(voice + 1) : 1e300;
        // The warp whose stretch holds the goal finds the group and goes through it once more.  (No two warps do, and one does if anything
        // is left, as all have the same sums.)
        int hit = -1;
        if (mine_from <= goal && goal < mine_to) {
            const double before = upto - (g0 + g1);
            const unsigned some = __ballot_sync(kAll, g0 + g1 > 0.0), over = __ballot_sync(kAll, mine_from + upto > goal) & some;
            const int l = over ? __ffs(over) - 1 : some ? 31 - __clz(some) : 0;  // (the last with any, should rounding have it so)
            const bool second = !(g0 > 0.0) || (g1 > 0.0 && !(mine_from + before + g0 > goal));
            const int k = __shfl_sync(kAll, 2 * lane + (second ? 1 : 0), l);
            double at = __shfl_sync(kAll, mine_from + before + (second ? g0 : 0.0), l);
            int last = -1;  // token with the last weight above zero so far: the one, should rounding leave the goal behind the end
            const int from = v0 + 32 * per * k, to = min(v1, from + 32 * per);
#pragma unroll 1
            for (int st = from; st < to && hit < 0; st += 32) {
                float x[kE];
                double w[kE];
                row.unpack(__ldg(row.at + min(st + lane, to - 1)), st + lane, st + lane < to, x);
                weights(x, st + lane, w);
                const double sum = add_up(w);
                double incl = sum;
#pragma unroll 1
                for (int o = 1; o < 32; o <<= 1) {
                    const double y = __shfl_up_sync(kAll, incl, o);
                    if (lane >= o) incl += y;
                }
                const unsigned some = __ballot_sync(kAll, sum > 0.0), over = __ballot_sync(kAll, at + incl > goal) & some;
                if (some) {
                    const int l = over ? __ffs(over) - 1 : 31 - __clz(some);
                    double q = at + (incl - sum);
                    bool over_it = false;
                    int h = -1;
#pragma unroll
                    for (int e = 0; e < kE; ++e) {
                        q += w[e];
                        if (w[e] > 0.0 && !over_it) h = row.first(st + lane) + e;
                        over_it = over_it || q > goal;
                    }
                    h = __shfl_sync(kAll, h, l);
                    if (over)
                        hit = h;
                    else
                        last = h;
                }
                at += __shfl_sync(kAll, incl, 31);
            }
            if (hit < 0) hit = last;
        }
        exchange((uint64_t)(uint32_t)(hit + 1));
        int got = 0;
        for (int i = lane; i < voices; i += 32) got = max(got, (int)all[i]);
        bonus = __reduce_max_sync(kAll, got) - 1;
        if (bonus >= 0) break;
        // nothing is left (the children held all of it, and rounding kept each from being accepted): the row's likeliest token
        int id = 0x7FFFFFFF;
        each_short(s0 + tid, s1, kThreads, [&](const float (&x)[kE], int st) {
#pragma unroll
            for (int i = 0; i < kE; ++i)
                if (x[i] == top) id = min(id, row.first(st) + i);
        });
        exchange((uint64_t)(uint32_t)__reduce_min_sync(kAll, id));
        bonus = 0x7FFFFFFF;
        for (int i = lane; i < voices; i += 32) bonus = min(bonus, (int)all[i]);
        bonus = __reduce_min_sync(kAll, bonus);
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
    // (a step of the whole batch in a few microseconds' reading: there is room for rows that may not be needed)
    p.bring_ahead = (double)batch * ctx->cfg.V * (dt == GRAFT_BF16 ? 2 : 4) <= 8e6;
    p.L = ctx->cfg.L;
    p.hist_w = ctx->hist_w;
    p.hist_window = ctx->hist_window;
    p.hist_count = ctx->hist_count;
    p.hist_out = ctx->hist_out;
    // A cluster takes a step of one sequence in a few microseconds, however short its CTAs' shares are: as many CTAs as keep a piece for every
    // thread, and as are on the GPU together (four an SM)
    int ctas = kMaxCluster;
    while (ctas > 1 && ((long long)ctas * batch > 4 * ctx->num_sms || (long long)ctas * kThreads * (dt == GRAFT_BF16 ? 8 : 4) > p.V)) ctas >>= 1;
    const void* kernel = dt == GRAFT_BF16 ? (const void*)verify_kernel<true> : (const void*)verify_kernel<false>;
    if (!(ctx->verify_ready & (1 << dt))) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        ctx->verify_ready |= 1 << dt;
    }
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(ctas, batch);
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = (size_t)4 * ctx->nmax * sizeof(int32_t);
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
