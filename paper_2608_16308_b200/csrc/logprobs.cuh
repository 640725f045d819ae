// Log probabilities of the rows of logits, with entropy and top alternatives, and the gradient.
//
// One pass: every thread keeps the largest logit m that it has met, s = sum e and u = sum x e with e = 2^x, x = (l - m) log2(e) / T, and moves s and u over when m
// grows (u to u + d s, both times 2^d); states of threads, warps and the blocks of a cluster are brought to their largest m and added.  Then log sum = log s, entropy = log s - log(2) u / s.  Relative to
// m nothing overflows, whatever the logits.  Neither HBM nor the issue of instructions (half its rate) nor a pipe (exponentials 45 %) is full in bf16; what is left is the way through a round and the end of a row.  Two entries are
// multiplied and added at a time, and x is one product-and-sum with the rounded m log2(e) / T, whose rounding is made up for once per thread.  Thread blocks walk the rows, and the vectors to come, the next
// row's too, are copied ahead into slots of shared memory that belong to the thread itself (cp.async, no barrier): the sums and the selection at the end of a row leave HBM busy.
//
// 2048 rows of 32000 with the entropy, in bf16 32 us (4.1 TB/s), 37 with five alternatives, 45 with twenty, 47 without any where a third is masked (those sums are made twice); in fp32 62 with five; one row of 32000 in fp32
// with twenty 7.9 us (4.5 without): two exchanges of the cluster.
//
// Alternatives.  A thread's own logits (its unit) are known by their largest and its place.  Where at least k groups of threads have a unit of at least tau, no logit below tau is among the k largest; the
// k-th largest of the groups' largest (or a little less) is such a tau.  Only units that reach it are read a second time (they come from L2), and of their logits those that reach tau are counted against
// each other: a candidate's place is the number of those in front of it.  No order of the logits makes this long: if too many reach tau (equal ones above all), tau is searched exactly among the units, told apart by their places; the last
// resort (NaN, or k units full of the largest) is k passes.
#pragma once

#include <cooperative_groups.h>

#include "rows.cuh"

namespace dbs {

constexpr int LP_CTA = 128, LP_WARPS = LP_CTA / 32;
constexpr int LP_MAX_TOP = 64;
constexpr int LP_CANDIDATES = 256;
constexpr int LP_CLUSTER = 8;
constexpr int LP_FLIGHT = 4;                 // vectors of 16 bytes that a thread takes in one round
constexpr int LP_AHEAD = 3;                  // rounds in flight or in hand
constexpr int LP_PER_SM = 7;                 // thread blocks
constexpr int LP_SMEM = LP_AHEAD * LP_FLIGHT * LP_CTA * 16;
constexpr int LP_GROUP = 2;                  // threads of a group: 64 groups
constexpr int LP_GROUPS = LP_CTA / LP_GROUP;
constexpr int LP_CLUSTER_GROUPS = 128;       // of a cluster's row
constexpr int LP_SLACK = 4;                  // groups more than k that may reach tau
constexpr float LP_NONE = -1000.f;           // 2^LP_NONE is 0, and its product with 0 too
constexpr float LP_LOW = -1e30f;             // what -inf is taken for in sums: its probability is 0 as well, and 0 times it is 0
constexpr float LP_NEAR = 4096.f;            // |m log2(e) / T| up to which the short form of x is good
static_assert(LP_WARPS <= 32 && LP_MAX_TOP <= LP_GROUPS && LP_GROUPS == 64, "a group for every alternative, two to a lane");

struct LpArgs {
    const void *logits;
    int64_t ld;
    int32_t tokens, vocab, cluster, top, rounds;  // rounds: of a thread block's share of a row, at most
    float slope, inv_t;                       // log2(e) / T, 1 / T
    const int32_t *targets;
    float *logprob, *entropy, *stats;
    int32_t *top_ids;
    float *top_logprobs;
};

__device__ __forceinline__ float exp_2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {        // NaN where one is
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// Order of logits as of unsigned numbers: NaN first, both zeros alike; 0 is below all
__device__ __forceinline__ uint32_t order_of(float l) {
    if (l != l) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(l == 0.f ? 0.f : l);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t LP_ORDER_LEAST = 0x007FFFFFu;                    // order_of(-inf)
__device__ __forceinline__ float of_order(uint32_t k) {
    return k == 0xFFFFFFFFu ? __uint_as_float(0x7FC00000u) : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint64_t candidate(float l, uint32_t index) { return (uint64_t)order_of(l) << 32 | (0xFFFFFFFEu - index); }   // never all ones, not even of a NaN
__device__ __forceinline__ int32_t place_of(uint64_t c) { return (int32_t)(0xFFFFFFFEu - (uint32_t)c); }

// States of the lanes brought to the largest m of a warp's first `lanes` lanes (a power of two) and added; the same in each of them
struct LpState {
    float m, s, u;
    template <int LANES>
    __device__ __forceinline__ void join(float slope) {
        float top = m;
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
        const float d = m == top ? 0.f : fmaxf((m - top) * slope, LP_NONE), f = exp_2(d);
        u = (u + d * s) * f;
        s *= f;
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1) {
            s += __shfl_xor_sync(FULL, s, o);
            u += __shfl_xor_sync(FULL, u, o);
        }
        m = top;
    }
};

// One row as a thread block's share of it meets it: `head` entries up to the first 16 bytes, whole vectors, `tail` entries
template <bool F32>
struct LpRow {
    static constexpr int V = F32 ? 4 : 8;
    const uint8_t *p;
    int head, tail, from, to, vectors;       // vectors from .. to are this block's; head belongs to the first block, tail to the last
    __device__ __forceinline__ LpRow(const void *base, int64_t ld, int64_t t, int vocab, int rank, int cluster) {
        constexpr int SIZE = F32 ? 4 : 2;
        p = static_cast<const uint8_t *>(base) + t * ld * SIZE;
        const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15u) / SIZE;
        head = off ? V - off : 0;
        if (head > vocab) head = vocab;
        vectors = (vocab - head) / V;
        tail = vocab - head - vectors * V;
        const int per = cluster == 1 ? vectors : (vectors + cluster - 1) / cluster;
        from = rank * per < vectors ? rank * per : vectors;
        to = from + per < vectors ? from + per : vectors;
        if (rank != 0) head = -head;         // (its size is still needed for the places)
        if (rank != cluster - 1) tail = 0;
    }
    __device__ __forceinline__ int heads() const { return head > 0 ? head : 0; }
    __device__ __forceinline__ int place(int vector) const { return (head < 0 ? -head : head) + vector * V; }
    __device__ __forceinline__ float one(int i) const { return F32 ? reinterpret_cast<const float *>(p)[i] : bf16_lo(reinterpret_cast<const uint16_t *>(p)[i]); }
    __device__ __forceinline__ const uint4 *at(int vector) const { return reinterpret_cast<const uint4 *>(p + (int64_t)place(vector) * (F32 ? 4 : 2)); }
    __device__ __forceinline__ uint4 raw(int vector) const { return *at(vector); }
    __device__ __forceinline__ static void values(uint4 q, float v[V]) {
        if constexpr (F32) {
            v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
        } else eight_of(q, v);
    }
};

__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t max_bf16(uint32_t a, uint32_t b) {       // two at a time, NaN left out
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t max_nan_bf16(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// whether x may be l slope - ref: the rounding of ref is small, and LP_LOW slope is a number far below it
__device__ __forceinline__ bool short_form(float ref, float slope) { return fabsf(ref) <= LP_NEAR && slope <= LP_NEAR && slope >= 1e-20f; }
// largest of N vectors, NaN left out
template <bool F32, int N = 1>
__device__ __forceinline__ float largest(const uint4 (&q)[N]) {
    if constexpr (F32) {
        float l = -INFINITY;
#pragma unroll
        for (int i = 0; i < N; ++i) l = fmaxf(l, fmaxf(fmaxf(__uint_as_float(q[i].x), __uint_as_float(q[i].y)), fmaxf(__uint_as_float(q[i].z), __uint_as_float(q[i].w))));
        return l;
    } else {
        uint32_t w = max_bf16(max_bf16(q[0].x, q[0].y), max_bf16(q[0].z, q[0].w));
#pragma unroll
        for (int i = 1; i < N; ++i) w = max_bf16(w, max_bf16(max_bf16(q[i].x, q[i].y), max_bf16(q[i].z, q[i].w)));
        return fmaxf(bf16_lo(w), bf16_hi(w));
    }
}
template <bool F32>
__device__ __forceinline__ float largest(uint4 q) {
    const uint4 one[1] = {q};
    return largest<F32, 1>(one);
}
// a vector's entries two at a time; CLAMP: -inf (and what lies below `low`, in bf16 twice `low2`) as `low`
constexpr uint32_t LP_LOW2 = 0xF14AF14Au;    // LP_LOW in bf16, twice
template <bool F32, bool CLAMP>
__device__ __forceinline__ void pairs_of(uint4 q, f32x2 v[F32 ? 2 : 4], float low = LP_LOW, uint32_t low2 = LP_LOW2) {
    if constexpr (F32) {
        auto one = [&](uint32_t w) { return CLAMP ? max_nan(__uint_as_float(w), low) : __uint_as_float(w); };
        v[0] = pair(one(q.x), one(q.y));
        v[1] = pair(one(q.z), one(q.w));
    } else {
        auto two = [&](uint32_t w) { return bf16_pair(CLAMP ? max_nan_bf16(w, low2) : w); };
        v[0] = two(q.x); v[1] = two(q.y); v[2] = two(q.z); v[3] = two(q.w);
    }
}

struct LpShared {
    float m[2][LP_WARPS], s[2][LP_WARPS], u[2][LP_WARPS];       // of rows in turn
    uint32_t group[2][LP_GROUPS];
    uint64_t largest[LP_WARPS];
    uint64_t found[LP_CANDIDATES];
    uint64_t best[LP_MAX_TOP];
    uint16_t units[LP_CTA];
    int n_units[2], n_found[2];              // of rows in turn
};

// What the blocks of a cluster tell each other: their sums, their groups' largest, how many candidates they have (written once a row); and, in the first block, these
struct LpCluster {
    float m[LP_CLUSTER], s[LP_CLUSTER], u[LP_CLUSTER];
    uint32_t groups[LP_CLUSTER_GROUPS];
    int found[LP_CLUSTER];
    uint64_t best[LP_CLUSTER * LP_MAX_TOP], flat[LP_CLUSTER * LP_MAX_TOP];
};

// logits of at least tau among the units of at least tau -> sh.found (their number in sh.n_found, which may be more than there is room for).  The counts are 0 before it; all threads are behind a barrier
// that they reached behind their last reading.
template <bool F32>
__device__ __forceinline__ void lp_collect(const LpRow<F32> &row, LpShared &sh, int parity, uint64_t unit, uint64_t tau, int vocab) {
    const int tid = threadIdx.x;
    if (unit >= tau && unit) sh.units[atomicAdd(&sh.n_units[parity], 1)] = (uint16_t)tid;
    const float least = of_order((uint32_t)(tau >> 32));
    auto meet = [&](float l, int place, int of) {
        if (!tau || (l >= least && candidate(l, of) >= tau)) {
            const int i = atomicAdd(&sh.n_found[parity], 1);
            if (i < LP_CANDIDATES) sh.found[i] = candidate(l, place);
        }
    };
    if (tid < row.heads()) meet(row.one(tid), tid, tid);
    if (tid < row.tail) meet(row.one(vocab - row.tail + tid), vocab - row.tail + tid, vocab - row.tail + tid);
    __syncthreads();
    const int n_units = sh.n_units[parity], all = n_units * ((row.to - row.from + LP_CTA - 1) / LP_CTA);
    for (int i = tid; i < all; i += LP_CTA) {
        const unsigned round = (unsigned)i / (unsigned)n_units;
        const int v = row.from + (int)round * LP_CTA + sh.units[i - (int)round * n_units];
        if (v >= row.to) continue;
        const uint4 q = row.raw(v);
        if (tau && largest<F32>(q) < least) continue;
        float l[LpRow<F32>::V];
        LpRow<F32>::values(q, l);
#pragma unroll
        for (int j = 0; j < LpRow<F32>::V; ++j) meet(l[j], row.place(v) + j, row.place(v));
    }
    __syncthreads();
}

// a number that at least k of the groups' largest reach (N to a lane), and not many more: halves what lies between the least and the largest
template <int N>
__device__ __forceinline__ uint32_t lp_least(const uint32_t (&g)[N], int k) {
    uint32_t lo = g[0], hi = g[0];
#pragma unroll
    for (int i = 1; i < N; ++i) {
        lo = min(lo, g[i]);
        hi = max(hi, g[i]);
    }
    lo = __reduce_min_sync(FULL, lo);
    hi = __reduce_max_sync(FULL, hi);
    while (lo < hi) {
        const uint32_t mid = hi - (hi - lo) / 2;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popc(__ballot_sync(FULL, g[i] >= mid));
        if (n >= k) lo = mid;
        else hi = mid - 1;
        if (n >= k && n <= k + LP_SLACK) break;
    }
    // (between no logit, 0, and -inf there is none: a number from there stands for -inf, and of_order would make a NaN of it)
    return lo ? max(lo, LP_ORDER_LEAST) : 0u;
}

// the block's k largest to out(candidate, place), zeros behind them, every place from one thread.  `most`: the thread's largest, as order_of has it (0: it has none); `group`: what at least k groups' largest reach, as order_of has it.
template <bool F32, typename Out>
__device__ __forceinline__ void lp_top(const LpRow<F32> &row, LpShared &sh, int parity, uint32_t most, uint32_t group, bool plain, int k, int vocab, Out out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint64_t unit = most ? (uint64_t)most << 32 | 0xFFFFFFFFu : 0;         // (the place is needed where values do not decide)
    bool done = false;
    if (plain) {
        // (a group without logits: the search finds tau)
        if (group) lp_collect(row, sh, parity, unit, (uint64_t)group << 32, vocab);
        if (!group || sh.n_found[parity] > LP_CANDIDATES) {
            // the unit's place: of the first vector (or entry) that has its largest
            if (unit) {
                const float most = of_order((uint32_t)(unit >> 32));
                int place = tid < row.heads() && row.one(tid) == most ? tid : -1;
                for (int v = row.from + tid; place < 0 && v < row.to; v += LP_CTA)
                    if (largest<F32>(row.raw(v)) == most) place = row.place(v);
                unit = candidate(most, place < 0 ? vocab - row.tail + tid : place);
            }
            uint64_t tau = 0;
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t trial = tau | 1ull << bit;
                if (__syncthreads_count(unit >= trial) >= k) tau = trial;
            }
            if (tid == 0) sh.n_units[parity] = sh.n_found[parity] = 0;
            __syncthreads();
            lp_collect(row, sh, parity, unit, tau, vocab);
        }
        const int n = sh.n_found[parity];
        done = n <= LP_CANDIDATES;
        for (int c = tid; done && c < max(n, k); c += LP_CTA) {
            if (c >= n) {
                out(0ull, c);
                continue;
            }
            const uint64_t mine = sh.found[c];
            int before = 0;
#pragma unroll 4
            for (int i = 0; i < n; ++i) before += sh.found[i] > mine;
            if (before < k) out(mine, before);
        }
    }
    if (!done) {
        // one after the other, each the largest behind the last
        uint64_t last = ~0ull;
        for (int j = 0; j < k; ++j) {
            uint64_t b = 0;
            auto meet = [&](float l, int place) {
                const uint64_t c = candidate(l, place);
                if (c < last) b = max64(b, c);
            };
            if (last) {                       // (0: there are no more here)
                if (tid < row.heads()) meet(row.one(tid), tid);
                if (tid < row.tail) meet(row.one(vocab - row.tail + tid), vocab - row.tail + tid);
                for (int v = row.from + tid; v < row.to; v += LP_CTA) {
                    float l[LpRow<F32>::V];
                    LpRow<F32>::values(row.raw(v), l);
#pragma unroll
                    for (int i = 0; i < LpRow<F32>::V; ++i) meet(l[i], row.place(v) + i);
                }
            }
            for (int o = 16; o; o >>= 1) b = max64(b, __shfl_xor_sync(FULL, b, o));
            __syncthreads();
            if (lane == 0) sh.largest[warp] = b;
            __syncthreads();
            last = sh.largest[0];
            for (int w = 1; w < LP_WARPS; ++w) last = max64(last, sh.largest[w]);
            if (tid == 0) out(last, j);
        }
    }
}

static_assert(LP_MAX_TOP <= LP_CTA && LP_MAX_TOP <= LP_CLUSTER_GROUPS && LP_CLUSTER_GROUPS / 2 <= LP_CTA, "a thread for every candidate of a block");
template <bool F32, bool ENTROPY>
__global__ void __launch_bounds__(LP_CTA, LP_PER_SM) k_logprobs(const __grid_constant__ LpArgs a) {
    extern __shared__ __align__(16) uint4 s_slots[];
    __shared__ LpShared sh;
    constexpr int V = LpRow<F32>::V;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)(blockIdx.x % a.cluster), step = gridDim.x / a.cluster;
    uint4 *slot = s_slots + tid;              // [round][vector][thread]
    LpCluster *all = reinterpret_cast<LpCluster *>(s_slots + LP_SMEM / 16);  // (of a cluster)
    if (tid < 2) sh.n_units[tid] = sh.n_found[tid] = 0;
    pdl_wait();
    pdl_trigger();
    const float slope = a.slope;
    // rounds to come: of row t_next, the n_next-th
    int64_t t_next = blockIdx.x / a.cluster;
    int n_next = 0;
    LpRow<F32> next(a.logits, a.ld, t_next < a.tokens ? t_next : 0, a.vocab, rank, a.cluster);
    auto ahead = [&](int at) {
        if (t_next < a.tokens) {
            const int v0 = next.from + n_next * LP_FLIGHT * LP_CTA + tid;
#pragma unroll
            for (int i = 0; i < LP_FLIGHT; ++i)
                if (v0 + i * LP_CTA < next.to) copy_ahead(slot + (at * LP_FLIGHT + i) * LP_CTA, next.at(v0 + i * LP_CTA));
            if (++n_next == a.rounds) {
                n_next = 0;
                t_next += step;
                if (t_next < a.tokens) next = LpRow<F32>(a.logits, a.ld, t_next, a.vocab, rank, a.cluster);
            }
        }
        close_ahead();
    };
#pragma unroll
    for (int i = 0; i < LP_AHEAD; ++i) ahead(i);
    int at = 0, parity = 0;
    for (int64_t t = blockIdx.x / a.cluster; t < a.tokens; t += step, parity ^= 1) {
        // (a cluster: the first block has started, and is done with what the others gave it)
        if (a.cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        const LpRow<F32> row(a.logits, a.ld, t, a.vocab, rank, a.cluster);
        int target = -1;
        float at_target = 0.f;
        if (a.targets && rank == 0 && tid == 0) {
            target = a.targets[t];
            if (target >= 0 && target < a.vocab) at_target = row.one(target);
        }
        float m = -INFINITY, ref = 0.f;       // ref = fl(m slope): x = l slope - ref is off by m slope - ref
        f32x2 s = 0, u = 0;
        bool near = false;
        // the sums relative to m in place of ref, and back: 2^-r and 2^r, |r| <= 2^-13
        auto settled = [&](float sign, float s0, float u0) {
            const float r = near ? sign * fmaf(m, slope, -ref) : 0.f, y = r * 0.6931471805599453f, f = 1.f - y + 0.5f * y * y;
            return make_float2(s0 * f, (u0 - r * s0) * f);
        };
        auto meet = [&](float most) {
            if (most > m) {
                float2 v = settled(1.f, sum2(s), sum2(u));
                const float d = fmaxf((m - most) * slope, LP_NONE), f = exp_2(d);
                m = most;
                ref = most * slope;
                near = short_form(ref, slope);
                v = settled(-1.f, v.x * f, (v.y + d * v.x) * f);
                s = pair(v.x, 0.f);
                u = pair(v.y, 0.f);
            }
        };
        auto add = [&](float l) {             // any m: one that is -inf has met -inf and NaN only
            const float x = near ? fmaf(max_nan(l, LP_LOW), slope, -ref) : (l - (m == -INFINITY ? 0.f : m)) * slope, e = exp_2(x);
            s = add2(s, pair(e, 0.f));
            if (ENTROPY) u = add2(u, pair(max_nan(x, LP_NONE) * e, 0.f));
        };
        const bool any = tid < row.heads() || row.from + tid < row.to || tid < row.tail;
        if (tid < row.heads()) {
            const float l = row.one(tid);
            meet(l);
            add(l);
        }
        int left = (row.to - row.from - tid + LP_CTA - 1) / LP_CTA;         // vectors of this thread
        for (int n = 0; n < a.rounds; ++n, left -= LP_FLIGHT) {
            wait_ahead<LP_AHEAD - 1>();
            uint4 q[LP_FLIGHT];
            constexpr uint32_t NONE = F32 ? 0xFF800000u : 0xFF80FF80u;      // -inf
#pragma unroll
            for (int i = 0; i < LP_FLIGHT; ++i) q[i] = i < left ? slot[(at * LP_FLIGHT + i) * LP_CTA] : make_uint4(NONE, NONE, NONE, NONE);
            meet(largest<F32, LP_FLIGHT>(q));
            if (near) {
                f32x2 v = 0;
                auto sums = [&](auto CLAMP) {
#pragma unroll
                    for (int i = 0; i < LP_FLIGHT; ++i) {
                        if (i >= left) break;
                        f32x2 l[V / 2];
                        pairs_of<F32, decltype(CLAMP)::value>(q[i], l);
#pragma unroll
                        for (int j = 0; j < V / 2; ++j) {
                            const f32x2 x = fma2(l[j], both(slope), both(-ref));
                            const float2 xx = apart(x);
                            const f32x2 e = pair(exp_2(xx.x), exp_2(xx.y));
                            if (!decltype(CLAMP)::value) s = add2(s, e);
                            if (ENTROPY) v = fma2(x, e, v);
                        }
                    }
                };
                sums(std::false_type{});
                // -inf times its probability, 0: once more with -inf as LP_LOW (NaN stays)
                if (ENTROPY && sum2(v) != sum2(v)) {
                    v = 0;
                    sums(std::true_type{});
                }
                u = add2(u, v);
            } else {
#pragma unroll
                for (int i = 0; i < LP_FLIGHT; ++i) {
                    if (i >= left) break;
                    float l[V];
                    LpRow<F32>::values(q[i], l);
#pragma unroll
                    for (int j = 0; j < V; ++j) add(l[j]);
                }
            }
            ahead(at);
            at = at + 1 == LP_AHEAD ? 0 : at + 1;
        }
        if (tid < row.tail) {
            const float l = row.one(a.vocab - row.tail + tid);
            meet(l);
            add(l);
        }
        const float2 mine = settled(1.f, sum2(s), sum2(u));
        LpState st = {m, mine.x, mine.y};
        const uint32_t most = any ? order_of(m) : 0u;
        if (a.top) {
            uint32_t g = most;
#pragma unroll
            for (int o = 1; o < LP_GROUP; o <<= 1) g = max(g, __shfl_xor_sync(FULL, g, o));
            if (lane % LP_GROUP == 0) sh.group[parity][tid / LP_GROUP] = g;
        }
        st.join<32>(slope);
        if (lane == 0) { sh.m[parity][warp] = st.m; sh.s[parity][warp] = st.s; sh.u[parity][warp] = st.u; }
        __syncthreads();
        if (tid == 0) sh.n_units[parity ^ 1] = sh.n_found[parity ^ 1] = 0;
        st = {sh.m[parity][lane % LP_WARPS], sh.s[parity][lane % LP_WARPS], sh.u[parity][lane % LP_WARPS]};
        st.join<LP_WARPS>(slope);
        // what the row gives, once st is the whole row's
        auto nothing = [&] { return st.m == -INFINITY && st.s == 0.f; };
        auto total = [&] { return nothing() ? -INFINITY : logf(st.s); };
        auto give_sums = [&] {
            const bool none = nothing();
            const float log_sum = total();
            if (a.stats) reinterpret_cast<float2 *>(a.stats)[t] = make_float2(st.m, log_sum);
            if (ENTROPY) a.entropy[t] = none ? 0.f : log_sum - 0.6931471805599453f * (st.u / st.s);
            if (a.logprob) a.logprob[t] = target < 0 ? 0.f : target >= a.vocab ? __uint_as_float(0x7FC00000u) : none ? -INFINITY : (at_target - st.m) * a.inv_t - log_sum;
        };
        auto give = [&](uint64_t mine, int place) {
            if (!mine) return;
            if (a.top_ids) a.top_ids[t * a.top + place] = place_of(mine);
            if (a.top_logprobs) a.top_logprobs[t * a.top + place] = nothing() ? -INFINITY : (of_order((uint32_t)(mine >> 32)) - st.m) * a.inv_t - total();
        };
        // (NaN or +inf among a block's logits makes its sum NaN)
        bool ranked = false;
        if (a.cluster == 1) {
            if (tid == 0) give_sums();
            if (a.top) {
                const uint32_t g[2] = {sh.group[parity][lane], sh.group[parity][lane + 32]};
                lp_top(row, sh, parity, most, lp_least<2>(g, a.top), st.s == st.s, a.top, a.vocab, give);
            }
        } else {
            namespace cg = cooperative_groups;
            auto c = cg::this_cluster();
            const bool plain = st.s == st.s;
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (tid < a.cluster) {
                LpCluster *to = c.map_shared_rank(all, tid);
                to->m[rank] = st.m; to->s[rank] = st.s; to->u[rank] = st.u;
            }
            if (a.top) {
                // fewer and larger groups: as many for the row, whatever the cluster
                const int mine_of = LP_CLUSTER_GROUPS / a.cluster, lanes = LP_CTA / mine_of;
                uint32_t g = most;
                for (int o = 1; o < lanes; o <<= 1) g = max(g, __shfl_xor_sync(FULL, g, o));
                if (lane % lanes < a.cluster)
                    for (int r = lane % lanes; r < a.cluster; r += lanes) c.map_shared_rank(all, r)->groups[rank * mine_of + tid / lanes] = g;
            }
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
            const int r = lane % LP_CLUSTER;
            st = r < a.cluster ? LpState{all->m[r], all->s[r], all->u[r]} : LpState{-INFINITY, 0.f, 0.f};
            st.join<LP_CLUSTER>(slope);
            LpCluster *first = c.map_shared_rank(all, 0);
            uint32_t least = 0;
            if (a.top && st.s == st.s) {
                // one tau for the whole row: few candidates in any block
                uint32_t g[LP_CLUSTER_GROUPS / 32];
#pragma unroll
                for (int i = 0; i < LP_CLUSTER_GROUPS / 32; ++i) g[i] = all->groups[i * 32 + lane];
                least = lp_least(g, a.top);
            }
            if (least) {
                if (a.rounds > LP_AHEAD) lp_collect(row, sh, parity, most ? (uint64_t)most << 32 | 0xFFFFFFFFu : 0, (uint64_t)least << 32, a.vocab);
                else {
                    // (every round is still in shared memory: each thread looks through its own logits)
                    const float l_least = of_order(least);
                    auto meet_one = [&](float l, int place) {
                        if (l >= l_least) {
                            const int i = atomicAdd(&sh.n_found[parity], 1);
                            if (i < LP_CANDIDATES) sh.found[i] = candidate(l, place);
                        }
                    };
                    if (tid < row.heads()) meet_one(row.one(tid), tid);
                    if (tid < row.tail) meet_one(row.one(a.vocab - row.tail + tid), a.vocab - row.tail + tid);
                    if (most >= least)
                        for (int i = 0; row.from + tid + i * LP_CTA < row.to; ++i) {
                            const uint4 q = slot[i * LP_CTA];
                            if (!(largest<F32>(q) >= l_least)) continue;
                            float l[V];
                            LpRow<F32>::values(q, l);
#pragma unroll
                            for (int j = 0; j < V; ++j) meet_one(l[j], row.place(row.from + tid + i * LP_CTA) + j);
                        }
                    __syncthreads();
                }
                const int n = sh.n_found[parity];
                if (tid < n && n <= LP_MAX_TOP) first->best[rank * LP_MAX_TOP + tid] = sh.found[tid];
                if (tid < a.cluster) c.map_shared_rank(all, tid)->found[rank] = n;
                asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
                ranked = true;
                for (int i = 0; i < a.cluster; ++i) ranked = ranked && all->found[i] <= LP_MAX_TOP;
                if (!ranked && tid == 0) sh.n_units[parity] = sh.n_found[parity] = 0;
                __syncthreads();
            }
            if (a.top && !ranked) {
                // every block's own, then the blocks' among each other
                const uint32_t g[2] = {sh.group[parity][lane], sh.group[parity][lane + 32]};
                lp_top(row, sh, parity, most, lp_least<2>(g, a.top), plain, a.top, a.vocab, [&](uint64_t c, int place) { sh.best[place] = c; });
                __syncthreads();
                // (`found` stays as it is: another block may still be reading there that not all candidates fitted)
                if (tid < LP_MAX_TOP) first->best[rank * LP_MAX_TOP + tid] = tid < a.top ? sh.best[tid] : 0;
                asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
            }
        }
        if (a.cluster > 1 && rank == 0) {
            if (tid == 0) give_sums();
            if (a.top) {
                int n = 0;
                for (int r = 0; r < a.cluster; ++r) {
                    const int here = ranked ? all->found[r] : a.top;
                    if (tid < here) all->flat[n + tid] = all->best[r * LP_MAX_TOP + tid];
                    n += here;
                }
                __syncthreads();
                for (int i = tid; i < n; i += LP_CTA) {
                    const uint64_t mine = all->flat[i];
                    int before = 0;
#pragma unroll 8
                    for (int j = 0; j < n; ++j) before += all->flat[j] > mine;
                    if (before < a.top) give(mine, before);
                }
            }
        }
    }
}

// ---- the gradient -----------------------------------------------------------------------------
// p (c0 + c1 x) per entry, two loads of 16 or 32 bytes ahead: 2048 rows of 32000 in bf16 45 us, 5.8 TB/s; 63 of 100003 in fp32 13.4 us.  Thread blocks of 128: of 256, 50.2 us.  What is added at single entries
// (targets, alternatives) is written behind the rest by the same thread block.
struct LpGrad {
    const void *logits;
    void *dlogits;
    int64_t ld, ldd;
    int32_t tokens, vocab, top, chunks;
    float slope, inv_t;
    const int32_t *targets, *top_ids;
    const float *stats, *entropy, *dlogprob, *dentropy, *dtop;
};
constexpr int LG_ROWS_WAVES = 3, LG_ROWS_PER_SM = 8, LG_ROWS_CTA = 128, LG_ROWS_FLIGHT = 2;            // threads, eights in flight of each

template <bool F32, bool OUT32>
__global__ void __launch_bounds__(LG_ROWS_CTA) k_logprobs_backward(const __grid_constant__ LpGrad a) {
    constexpr int IN = F32 ? 4 : 2, OUT = OUT32 ? 4 : 2;
    const int tid = threadIdx.x;
    const int64_t t = blockIdx.x / a.chunks;
    const int chunk = (int)(blockIdx.x % a.chunks);
    pdl_wait();
    pdl_trigger();
    const uint8_t *in = static_cast<const uint8_t *>(a.logits) + t * a.ld * IN;
    uint8_t *out = static_cast<uint8_t *>(a.dlogits) + t * a.ldd * OUT;
    auto one = [&](int i) { return F32 ? reinterpret_cast<const float *>(in)[i] : bf16_lo(reinterpret_cast<const uint16_t *>(in)[i]); };
    auto put = [&](int i, float v) {
        if (OUT32) reinterpret_cast<float *>(out)[i] = v;
        else reinterpret_cast<uint16_t *>(out)[i] = (uint16_t)two_bf16(v, 0.f);
    };
    const int off = (int)(reinterpret_cast<uintptr_t>(out) & 15u) / OUT;
    int head = off ? 16 / OUT - off : 0;
    if (head > a.vocab) head = a.vocab;
    const int eights = (a.vocab - head) / 8, tail_at = head + eights * 8;
    const bool whole = (reinterpret_cast<uintptr_t>(in + (int64_t)head * IN) & 15u) == 0;
    // this block's eights
    const int per = (eights + a.chunks - 1) / a.chunks, from8 = min(chunk * per, eights), to8 = min(from8 + per, eights);
    uint4 q_next[LG_ROWS_FLIGHT][F32 ? 2 : 1];
    auto load = [&](int e0) {
#pragma unroll
        for (int r = 0; r < LG_ROWS_FLIGHT; ++r)
            if (e0 + r * LG_ROWS_CTA < to8) load_raw<F32>(in, head + (e0 + r * LG_ROWS_CTA) * 8, a.vocab, whole, q_next[r][0], q_next[r][F32 ? 1 : 0]);
    };
    load(from8 + tid);
    // entries at the ends of the row, and those that have a gradient of their own: read before anything is written (dlogits may be the logits)
    const bool last = chunk == a.chunks - 1;
    const int edge = chunk == 0 && tid < head ? tid : last && tid >= 32 && tid - 32 < a.vocab - tail_at ? tail_at + tid - 32 : -1;
    const float l_edge = edge >= 0 ? one(edge) : 0.f;
    // the entries that are given a gradient: every warp adds it up for itself, and thread j keeps the j-th's place and logit
    float given = 0.f, mine = 0.f, l_mine = 0.f;
    int id = -1;
    auto weight = [&](int j, int &at) {       // the target's behind the alternatives'
        at = -1;
        if (j == a.top && a.dlogprob) {
            at = a.targets[t];
            return at < 0 ? 0.f : at >= a.vocab ? __uint_as_float(0x7FC00000u) : a.dlogprob[t];
        }
        if (j < a.top) {
            at = a.top_ids[t * a.top + j];
            return at >= 0 && at < a.vocab ? a.dtop[t * a.top + j] : 0.f;
        }
        return 0.f;
    };
#pragma unroll
    for (int j0 = 0; j0 <= LP_MAX_TOP; j0 += 32) {
        int at;
        if (j0 <= a.top) given += weight(j0 + tid % 32, at);
    }
    const float2 st = reinterpret_cast<const float2 *>(a.stats)[t];
    const float dh = a.dentropy ? a.dentropy[t] : 0.f, h = a.dentropy ? a.entropy[t] : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) given += __shfl_xor_sync(FULL, given, o);
    if (tid <= a.top) {
        mine = weight(tid, id);
        // (this block's own; the ends of the row are the first one's and the last one's)
        const int from = chunk == 0 ? 0 : head + from8 * 8, to = last ? a.vocab : head + to8 * 8;
        if (id < from || id >= to) id = -1;
        // an id that is given several times belongs to the first thread that has it, which adds the weights up in the order in which they are given (the others' stores would race with its own)
        if (id >= 0) {
            l_mine = one(id);
            mine = 0.f;
            bool first = true;
#pragma unroll 8
            for (int j = 0; j < a.top; ++j)
                if (a.top_ids[t * a.top + j] == id) {
                    first = first && j >= tid;
                    mine += a.dtop[t * a.top + j];
                }
            if (a.dlogprob && a.targets[t] == id) mine += a.dlogprob[t];
            if (!first) id = -1;
        }
    }
    __syncthreads();
    const bool nothing = st.x == -INFINITY && !(st.y != st.y);
    constexpr float LN2 = 0.6931471805599453f;
    const float shift = st.y * 1.4426950408889634f;
    auto slope = [&](float v, float own) {
        const float x = (v - st.x) * a.slope - shift, p = exp_2(x);
        return nothing ? 0.f : (own - p * (given + dh * (max_nan(x, LP_NONE) * LN2 + h))) * a.inv_t;
    };
    // p (c0 + c1 x) with x = l slope - ref, two entries at a time; ref is rounded, and what that makes of p and x is in c0 and c1
    const float most = st.x * a.slope, ref = most + shift;
    const bool near = short_form(most, a.slope) && short_form(ref, a.slope);
    const float part = ref - most, low = near ? fmaf(st.x, a.slope, -most) + ((most - (ref - part)) + (shift - part)) : 0.f, y = low * LN2;
    const float k = nothing ? 0.f : -a.inv_t * (1.f - y + 0.5f * y * y);
    // -inf, and whatever else lies 1000 or so below the row's sum in units of log 2, is taken for a logit there: its p is 0, and c1 x of its size is a number that 0 can be multiplied with
    const float low_logit = near ? (ref + LP_NONE) / a.slope : 0.f;
    const uint32_t low_two = two_bf16(low_logit, low_logit);
    const f32x2 c0 = both(nothing ? 0.f : k * (given + dh * (h - y))), c1 = both(nothing ? 0.f : k * dh * LN2);
    for (int e0 = from8 + tid; e0 < to8; e0 += LG_ROWS_FLIGHT * LG_ROWS_CTA) {
        uint4 q[LG_ROWS_FLIGHT][F32 ? 2 : 1];
#pragma unroll
        for (int r = 0; r < LG_ROWS_FLIGHT; ++r)
#pragma unroll
            for (int i = 0; i < (F32 ? 2 : 1); ++i) q[r][i] = q_next[r][i];
        load(e0 + LG_ROWS_FLIGHT * LG_ROWS_CTA);
#pragma unroll
        for (int r = 0; r < LG_ROWS_FLIGHT; ++r) {
            const int e = e0 + r * LG_ROWS_CTA;
            if (e >= to8) break;
            float d[8];
            if (near) {
                f32x2 l[4];
                pairs_of<F32, true>(q[r][0], l, low_logit, low_two);
                if (F32) pairs_of<F32, true>(q[r][F32 ? 1 : 0], l + 2, low_logit, low_two);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x2 x = fma1(l[j], both(a.slope), both(-ref));
                    const float2 xx = apart(x), v = apart(mul1(pair(exp_2(xx.x), exp_2(xx.y)), fma1(x, c1, c0)));
                    d[2 * j] = v.x;
                    d[2 * j + 1] = v.y;
                }
            } else {
                if (F32) eight_of(q[r][0], q[r][F32 ? 1 : 0], d);
                else eight_of(q[r][0], d);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = slope(d[j], 0.f);
            }
            store_eight<OUT32>(out, head + e * 8, a.vocab, true, d);
        }
    }
    if (edge >= 0) put(edge, slope(l_edge, 0.f));
    __syncthreads();
    if (id >= 0) put(id, slope(l_mine, mine));
}

}  // namespace dbs
