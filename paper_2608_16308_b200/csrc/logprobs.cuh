// Log probabilities of the rows of logits, with entropy and top alternatives, and the gradient.
//
// One pass: every thread keeps the largest logit m that it has met, s = sum e and u = sum x e with e = 2^x, x = (l - m) log2(e) / T, and moves s and u over when m
// grows (u to u + d s, both times 2^d); states of threads, warps and the blocks of a cluster are joined the same way.  Then log sum = log s, entropy = log s - log(2) u / s.  Relative to m nothing overflows, whatever
// the logits.  What bounds it is HBM, with the exponential's pipe (16 a clock and SM) at two thirds of its rate for bf16.
//
// Alternatives.  A thread's own logits (its unit) are known by their largest and its place.  Where at least k groups of threads have a unit of at least tau, no logit below tau is among the k largest, so
// tau is the least of the groups' largest; only units that reach it are read a second time (they come from L2), and of their logits those that reach tau are counted against each other: a candidate's place
// is the number of those in front of it.  No order of the logits makes this long: units that share the largest value are told apart by their places, tau is searched exactly if too many are
// left, and the last resort (NaN, or k units full of the largest) is k passes.
#pragma once

#include <cooperative_groups.h>

#include "rows.cuh"

namespace dbs {

constexpr int LP_CTA = 512, LP_WARPS = LP_CTA / 32;
constexpr int LP_MAX_TOP = 64;
constexpr int LP_CANDIDATES = LP_CTA;        // a thread ranks one
constexpr int LP_CLUSTER = 8;
constexpr int LP_FLIGHT = 4;                 // loads of 16 bytes in flight per thread
constexpr float LP_NONE = -1000.f;           // 2^LP_NONE is 0, and its product with 0 too
static_assert(LP_WARPS <= 32 && LP_MAX_TOP <= LP_CTA / 8, "groups of eight lanes and more");

struct LpArgs {
    const void *logits;
    int64_t ld;
    int32_t tokens, vocab, cluster, top;
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
__device__ __forceinline__ float of_order(uint32_t k) {
    return k == 0xFFFFFFFFu ? __uint_as_float(0x7FC00000u) : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint64_t candidate(float l, uint32_t index) { return (uint64_t)order_of(l) << 32 | (0xFFFFFFFEu - index); }   // never all ones, not even of a NaN
__device__ __forceinline__ int32_t place_of(uint64_t c) { return (int32_t)(0xFFFFFFFEu - (uint32_t)c); }

struct LpState {
    float m, s, u;
    __device__ __forceinline__ void join(float m2, float s2, float u2, float slope) {
        const float top = fmaxf(m, m2);
        const float d = m == top ? 0.f : fmaxf((m - top) * slope, LP_NONE), d2 = m2 == top ? 0.f : fmaxf((m2 - top) * slope, LP_NONE);
        const float f = exp_2(d), f2 = exp_2(d2);
        u = (u + d * s) * f + (u2 + d2 * s2) * f2;
        s = s * f + s2 * f2;
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
        const int per = (vectors + cluster - 1) / cluster;
        from = rank * per < vectors ? rank * per : vectors;
        to = from + per < vectors ? from + per : vectors;
        if (rank != 0) head = -head;         // (its size is still needed for the places)
        if (rank != cluster - 1) tail = 0;
    }
    __device__ __forceinline__ int heads() const { return head > 0 ? head : 0; }
    __device__ __forceinline__ int place(int vector) const { return (head < 0 ? -head : head) + vector * V; }
    __device__ __forceinline__ float one(int i) const { return F32 ? reinterpret_cast<const float *>(p)[i] : bf16_lo(reinterpret_cast<const uint16_t *>(p)[i]); }
    __device__ __forceinline__ uint4 raw(int vector) const { return *reinterpret_cast<const uint4 *>(p + (int64_t)place(vector) * (F32 ? 4 : 2)); }
    __device__ __forceinline__ static void values(uint4 q, float v[V]) {
        if constexpr (F32) {
            v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
        } else eight_of(q, v);
    }
};

__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t min64(uint64_t a, uint64_t b) { return a < b ? a : b; }

struct LpShared {
    float m[LP_WARPS], s[LP_WARPS], u[LP_WARPS];
    uint64_t group[LP_WARPS];
    uint64_t found[LP_CANDIDATES];
    uint64_t best[LP_CLUSTER][LP_MAX_TOP];   // of every block of the cluster, in the first one
    float cm[LP_CLUSTER], cs[LP_CLUSTER], cu[LP_CLUSTER];
    uint16_t units[LP_CTA];
    int n_units, n_found;
};

// logits of at least tau among the units of at least tau -> sh.found (their number in sh.n_found, which may be more than there is room for)
template <bool F32>
__device__ __forceinline__ void lp_collect(const LpRow<F32> &row, LpShared &sh, uint64_t unit, uint64_t tau, int vocab) {
    const int tid = threadIdx.x;
    if (tid == 0) sh.n_units = sh.n_found = 0;
    __syncthreads();
    if (unit >= tau && unit) sh.units[atomicAdd(&sh.n_units, 1)] = (uint16_t)tid;
    auto meet = [&](float l, int place, int of) {
        if (candidate(l, of) >= tau) {
            const int i = atomicAdd(&sh.n_found, 1);
            if (i < LP_CANDIDATES) sh.found[i] = candidate(l, place);
        }
    };
    if (tid < row.heads()) meet(row.one(tid), tid, tid);
    if (tid < row.tail) meet(row.one(vocab - row.tail + tid), vocab - row.tail + tid, vocab - row.tail + tid);
    __syncthreads();
    const int per = (row.to - row.from + LP_CTA - 1) / LP_CTA, all = sh.n_units * per;
    for (int i = tid; i < all; i += LP_CTA) {
        const int v = row.from + i / sh.n_units * LP_CTA + sh.units[i % sh.n_units];
        if (v >= row.to) continue;
        float l[LpRow<F32>::V];
        LpRow<F32>::values(row.raw(v), l);
#pragma unroll
        for (int j = 0; j < LpRow<F32>::V; ++j) meet(l[j], row.place(v) + j, row.place(v));
    }
    __syncthreads();
}

// the block's k largest into best[0 .. k), zeros behind them
template <bool F32>
__device__ __forceinline__ void lp_top(const LpRow<F32> &row, LpShared &sh, uint64_t unit, bool plain, int k, int vocab, uint64_t *best) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < k) best[tid] = 0;
    bool done = false;
    if (plain) {
        uint64_t g = unit, least;
        const int lanes = k <= LP_WARPS ? 32 : k <= 2 * LP_WARPS ? 16 : 8;
        for (int o = 1; o < lanes; o <<= 1) g = max64(g, __shfl_xor_sync(FULL, g, o));
        for (int o = lanes; o < 32; o <<= 1) g = min64(g, __shfl_xor_sync(FULL, g, o));
        if (lane == 0) sh.group[warp] = g;
        __syncthreads();
        least = sh.group[0];
        for (int w = 1; w < LP_WARPS; ++w) least = min64(least, sh.group[w]);
        // (a group without logits: the search below finds tau)
        if (least) lp_collect(row, sh, unit, least, vocab);
        if (!least || sh.n_found > LP_CANDIDATES) {
            least = 0;
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t trial = least | 1ull << bit;
                if (__syncthreads_count(unit >= trial) >= k) least = trial;
            }
            lp_collect(row, sh, unit, least, vocab);
        }
        done = sh.n_found <= LP_CANDIDATES;
        if (done && tid < sh.n_found) {
            const uint64_t mine = sh.found[tid];
            int before = 0;
            for (int i = 0; i < sh.n_found; ++i) before += sh.found[i] > mine;
            if (before < k) best[before] = mine;
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
            if (tid < row.heads()) meet(row.one(tid), tid);
            if (tid < row.tail) meet(row.one(vocab - row.tail + tid), vocab - row.tail + tid);
            for (int v = row.from + tid; v < row.to; v += LP_CTA) {
                float l[LpRow<F32>::V];
                LpRow<F32>::values(row.raw(v), l);
#pragma unroll
                for (int i = 0; i < LpRow<F32>::V; ++i) meet(l[i], row.place(v) + i);
            }
            for (int o = 16; o; o >>= 1) b = max64(b, __shfl_xor_sync(FULL, b, o));
            __syncthreads();
            if (lane == 0) sh.group[warp] = b;
            __syncthreads();
            last = sh.group[0];
            for (int w = 1; w < LP_WARPS; ++w) last = max64(last, sh.group[w]);
            if (tid == 0) best[j] = last;
            if (!last) break;                 // (no more logits here; the same in every thread)
        }
    }
    __syncthreads();
}

template <bool F32>
__global__ void __launch_bounds__(LP_CTA, 2) k_logprobs(const __grid_constant__ LpArgs a) {
    __shared__ LpShared sh;
    constexpr int V = LpRow<F32>::V;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)(blockIdx.x % a.cluster);
    const int64_t t = blockIdx.x / a.cluster;
    if (a.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    pdl_wait();
    pdl_trigger();
    const LpRow<F32> row(a.logits, a.ld, t, a.vocab, rank, a.cluster);
    int target = -1;
    float at_target = 0.f;
    if (a.targets && rank == 0 && tid == 0) {
        target = a.targets[t];
        if (target >= 0 && target < a.vocab) at_target = row.one(target);
    }
    const float slope = a.slope;
    LpState st = {-INFINITY, 0.f, 0.f};
    int unit_at = tid < row.heads() ? tid : row.from + tid < row.to ? row.place(row.from + tid) : tid < row.tail ? a.vocab - row.tail + tid : -1;
    auto meet = [&](float most, int place) {
        if (most > st.m) {
            const float d = fmaxf((st.m - most) * slope, LP_NONE), f = exp_2(d);
            st.u = (st.u + d * st.s) * f;
            st.s *= f;
            st.m = most;
            unit_at = place;
        }
    };
    auto add = [&](float l) {
        const float x = (l - (st.m == -INFINITY ? 0.f : st.m)) * slope, e = exp_2(x);
        st.s += e;
        st.u += max_nan(x, LP_NONE) * e;
    };
    if (tid < row.heads()) {
        const float l = row.one(tid);
        meet(l, tid);
        add(l);
    }
    for (int v0 = row.from + tid; v0 < row.to; v0 += LP_FLIGHT * LP_CTA) {
        uint4 q[LP_FLIGHT];
#pragma unroll
        for (int i = 0; i < LP_FLIGHT; ++i)
            if (v0 + i * LP_CTA < row.to) q[i] = row.raw(v0 + i * LP_CTA);
#pragma unroll
        for (int i = 0; i < LP_FLIGHT; ++i) {
            if (v0 + i * LP_CTA >= row.to) break;
            float l[V];
            LpRow<F32>::values(q[i], l);
            float most = l[0];
#pragma unroll
            for (int j = 1; j < V; ++j) most = fmaxf(most, l[j]);
            meet(most, row.place(v0 + i * LP_CTA));
#pragma unroll
            for (int j = 0; j < V; ++j) add(l[j]);
        }
    }
    if (tid < row.tail) {
        const float l = row.one(a.vocab - row.tail + tid);
        meet(l, a.vocab - row.tail + tid);
        add(l);
    }
    const uint64_t unit = unit_at < 0 ? 0 : candidate(st.m, unit_at);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(FULL, st.m, o), s2 = __shfl_xor_sync(FULL, st.s, o), u2 = __shfl_xor_sync(FULL, st.u, o);
        st.join(m2, s2, u2, slope);
    }
    if (lane == 0) { sh.m[warp] = st.m; sh.s[warp] = st.s; sh.u[warp] = st.u; }
    __syncthreads();
    st = {sh.m[0], sh.s[0], sh.u[0]};
    for (int w = 1; w < LP_WARPS; ++w) st.join(sh.m[w], sh.s[w], sh.u[w], slope);
    uint64_t *best = sh.best[0];
    if (a.top) {
        // (behind the sums: NaN or +inf among the block's logits makes its sum NaN)
        if (rank) best = sh.found;            // (the first block's room is for all)
        lp_top(row, sh, unit, st.s == st.s, a.top, a.vocab, rank ? sh.best[1] : sh.best[0]);
        if (rank) best = sh.best[1];
    }
    if (a.cluster > 1) {
        namespace cg = cooperative_groups;
        auto c = cg::this_cluster();
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (rank) {
            LpShared *first = c.map_shared_rank(&sh, 0);
            if (tid == 0) { first->cm[rank] = st.m; first->cs[rank] = st.s; first->cu[rank] = st.u; }
            if (tid < a.top) first->best[rank][tid] = best[tid];
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank) return;
        for (int r = 1; r < a.cluster; ++r) st.join(sh.cm[r], sh.cs[r], sh.cu[r], slope);
    }
    const bool nothing = st.m == -INFINITY && st.s == 0.f;
    const float total = nothing ? -INFINITY : logf(st.s);
    if (tid == 0) {
        if (a.stats) reinterpret_cast<float2 *>(a.stats)[t] = make_float2(st.m, total);
        if (a.entropy) a.entropy[t] = nothing ? 0.f : total - 0.6931471805599453f * (st.u / st.s);
        if (a.logprob) a.logprob[t] = target < 0 ? 0.f : target >= a.vocab ? __uint_as_float(0x7FC00000u) : nothing ? -INFINITY : (at_target - st.m) * a.inv_t - total;
    }
    // the blocks' alternatives among each other
    const int all = a.top * a.cluster;
    for (int i = tid; i < all; i += LP_CTA) {
        const uint64_t mine = sh.best[i / a.top][i % a.top];
        if (!mine) continue;
        int before = i % a.top;
        for (int r = 0; r < a.cluster; ++r)
            if (r != i / a.top)
                for (int j = 0; j < a.top && sh.best[r][j] > mine; ++j) ++before;
        if (before >= a.top) continue;
        if (a.top_ids) a.top_ids[t * a.top + before] = place_of(mine);
        if (a.top_logprobs) a.top_logprobs[t * a.top + before] = nothing ? -INFINITY : (of_order((uint32_t)(mine >> 32)) - st.m) * a.inv_t - total;
    }
}

// ---- the gradient -----------------------------------------------------------------------------
struct LpGrad {
    const void *logits;
    void *dlogits;
    int64_t ld, ldd;
    int32_t tokens, vocab, top, chunks;
    float slope, inv_t;
    const int32_t *targets, *top_ids;
    const float *stats, *entropy, *dlogprob, *dentropy, *dtop;
};
constexpr int LG2_CTA = 256, LG2_ROUNDS = 2;                     // eights of a thread
constexpr int LG2_EIGHTS = LG2_CTA * LG2_ROUNDS;                 // of a block

template <bool F32, bool OUT32>
__global__ void __launch_bounds__(LG2_CTA) k_logprobs_backward(const __grid_constant__ LpGrad a) {
    __shared__ float s_given;
    __shared__ int s_id[LP_MAX_TOP + 1];
    __shared__ float s_weight[LP_MAX_TOP + 1];
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
    const int first = chunk * LG2_EIGHTS + tid;
    float l[LG2_ROUNDS][8];
#pragma unroll
    for (int r = 0; r < LG2_ROUNDS; ++r) {
        const int e = first + r * LG2_CTA;
        if (e < eights) {
            uint4 x, y;
            load_raw<F32>(in, head + e * 8, a.vocab, whole, x, y);
            if (F32) eight_of(x, y, l[r]);
            else eight_of(x, l[r]);
        }
    }
    // entries at the ends of the row, and those that have a gradient of their own: read before anything is written (dlogits may be the logits)
    const bool last = chunk == a.chunks - 1;
    const int edge = chunk == 0 && tid < head ? tid : last && tid >= 32 && tid - 32 < a.vocab - tail_at ? tail_at + tid - 32 : -1;
    const float l_edge = edge >= 0 ? one(edge) : 0.f;
    if (tid <= a.top) {
        int id = -1;
        float w = 0.f;
        if (tid == a.top) {
            if (a.dlogprob) {
                id = a.targets[t];
                w = id < 0 ? 0.f : id >= a.vocab ? __uint_as_float(0x7FC00000u) : a.dlogprob[t];
            }
        } else if (a.dtop) {
            id = a.top_ids[t * a.top + tid];
            if (id >= 0 && id < a.vocab) w = a.dtop[t * a.top + tid];
        }
        s_id[tid] = id >= 0 && id < a.vocab ? id : -1;
        s_weight[tid] = w;
    }
    const float2 st = reinterpret_cast<const float2 *>(a.stats)[t];
    const float dh = a.dentropy ? a.dentropy[t] : 0.f, h = a.dentropy ? a.entropy[t] : 0.f;
    __syncthreads();
    float mine = 0.f, l_mine = 0.f;
    int id = -1;
    if (tid <= a.top) {
        id = s_id[tid];
        // (this block's own: the ends of the row are the first one's and the last one's)
        const int at = head + chunk * LG2_EIGHTS * 8, from = chunk == 0 ? 0 : min(at, tail_at), to = last ? a.vocab : min(at + LG2_EIGHTS * 8, tail_at);
        if (id < from || id >= to) id = -1;
        if (id >= 0) {
            l_mine = one(id);
            for (int j = 0; j <= a.top; ++j)
                if (s_id[j] == id) mine += s_weight[j];
        }
    }
    if (tid == 0) {
        float g = 0.f;
        for (int j = 0; j <= a.top; ++j) g += s_weight[j];
        s_given = g;
    }
    __syncthreads();
    const bool nothing = st.x == -INFINITY && !(st.y != st.y);
    const float given = s_given;
    constexpr float LN2 = 0.6931471805599453f;
    const float shift = st.y * 1.4426950408889634f;
    auto slope = [&](float v, float own) {
        const float x = (v - st.x) * a.slope - shift, p = exp_2(x);
        return nothing ? 0.f : (own - p * (given + dh * (max_nan(x, LP_NONE) * LN2 + h))) * a.inv_t;
    };
#pragma unroll
    for (int r = 0; r < LG2_ROUNDS; ++r) {
        const int e = first + r * LG2_CTA;
        if (e < eights) {
            float d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = slope(l[r][j], 0.f);
            store_eight<OUT32>(out, head + e * 8, a.vocab, true, d);
        }
    }
    if (edge >= 0) put(edge, slope(l_edge, 0.f));
    __syncthreads();
    if (id >= 0) put(id, slope(l_mine, mine));
}

}  // namespace dbs
