// A block joins the residual stream: out = r + scale drop(gate * norm_block(b)), h = norm_next(out), and the gradient of that.
//
// A row is owned by a team of warps, one or two times eight columns a thread: the values stay on the chip between the sums over the row (one for each norm, two for a layer norm; backwards one
// for each norm) and every array is read and written once.  A warp is a team for short rows, a thread block holds several teams then; rows of more than 4096 columns are shared out to a cluster
// whose blocks add up through each other's shared memory.  Teams walk the tokens.  The rows to come are copied ahead into slots of shared memory that belong to the thread itself (cp.async, no
// barrier): a sum over the row would else leave HBM idle.  Weights, gate, scales and biases of a thread's columns lie beside them in fp32, multiplied with one another once: what is left is HBM and, with
// dropout, nearly as many instructions; so products and sums go two entries at a time.
//
// Sums over the tokens (gradients of weights, biases and a shared gate) are held by the threads of a column and written once per team; a second kernel adds the teams up in a
// fixed order.  With a shared gate g and weight w both gradients follow from one sum: A = sum drop(G) xhat gives dw = scale g A and dg = scale (w A + c B), B = sum drop(G).
#pragma once

#include <cooperative_groups.h>

#include "rows.cuh"

namespace dbs {

constexpr int JOIN_COLS = 4096;              // of a row in one thread block; more: a cluster
constexpr int JOIN_CLUSTER = 8;
constexpr int64_t JOIN_MAX_N = JOIN_COLS * JOIN_CLUSTER;
constexpr int JOIN_AHEAD = 2;                // rows in flight or in hand, per team
constexpr int JOIN_SUMS_COLS = 32, JOIN_SUMS_CTA = 256;
// threads at most: of kernels with two eights a thread, and with one
template <int E> constexpr int join_cta() { return JOIN_COLS / 8 / E; }

struct JoinPlan {
    int eights;                              // of a thread: 1, 2
    int warps, teams, cluster;               // warps of a team in a thread block, teams in it, blocks to a row
    int clusters;                            // in the grid
};

struct JoinArgs {
    Rows r, b, gate, out, h;                 // forward (gate: rows, else gate_vec)
    Rows dh, dout, dr, db, dgate;            // backward (out: what the forward call left)
    const void *w_block, *c_block, *gate_vec, *w_next, *c_next;
    int32_t params_f32, pieces, params;      // pieces of 16 bytes of an eight, in a slot and for its columns
    float *stats;
    Drop drop;
    float scale, eps_block, eps_next, inv_n;
    int32_t norm_block, norm_next, tokens, n, warps, teams;
    float *parts;                            // [team][sum][ldp]
    int64_t ldp;
};

// an eight of row t into its slot (pieces `step` apart)
template <bool F32>
__device__ __forceinline__ void row_ahead(const Rows &r, int64_t t, int col, int n, uint4 *slot, int step) {
    const void *row = row_at<F32>(r, t);
    if (r.aligned && col + 8 <= n) {
        const uint8_t *p = static_cast<const uint8_t *>(row) + (int64_t)col * (F32 ? 4 : 2);
        copy_ahead(slot, p);
        if (F32) copy_ahead(slot + step, p + 16);
    } else {
        uint4 a, b;
        load_raw<F32>(row, col, n, false, a, b);
        slot[0] = a;
        if (F32) slot[step] = b;
    }
}
template <bool F32>
__device__ __forceinline__ void row_here(const uint4 *slot, int step, f32x2 v[4]) {
    if (F32) pairs_of_eight(slot[0], slot[step], v);
    else pairs_of_eight(slot[0], v);
}
__device__ __forceinline__ void row_here(bool f32, const uint4 *slot, int step, f32x2 v[4]) {
    if (f32) row_here<true>(slot, step, v);
    else row_here<false>(slot, step, v);
}
__device__ __forceinline__ float vector_one(const void *p, bool f32, int i) {
    return f32 ? static_cast<const float *>(p)[i] : __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
}
// factors of eight columns in fp32, the product of what is given (null: 1); zeros behind the row's end
__device__ __forceinline__ void columns_here(uint4 *to, int step, int col, int n, bool f32, float scale, const void *v, const void *w) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = col + j < n ? scale : 0.f;
        if (col + j < n && v) x[j] *= vector_one(v, f32, col + j);
        if (col + j < n && w) x[j] *= vector_one(w, f32, col + j);
    }
    to[0] = fp32_four(x);
    to[step] = fp32_four(x + 4);
}

struct JoinTeam {
    int lane, warp, warps, team, teams, rank, cluster, parity, room;
    float *sums;                             // [parity][team][2][room]: zeros behind the warps'
    __device__ __forceinline__ JoinTeam(const JoinArgs &a, float *s) {
        lane = threadIdx.x & 31;
        const int w = threadIdx.x >> 5;
        warps = a.warps;
        teams = a.teams;
        team = w / warps;
        warp = w - team * warps;
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
        parity = 0;
        sums = s;
        room = (warps * cluster + 3) & ~3;
        for (int i = threadIdx.x; i < 4 * teams * room; i += blockDim.x) s[i] = 0.f;
        // (a cluster: every block has started before its shared memory is written)
        if (cluster > 1) meet();
        else __syncthreads();
    }
    __device__ __forceinline__ int64_t first() const { return (int64_t)(blockIdx.x / cluster) * teams + team; }
    __device__ __forceinline__ int64_t step() const { return (int64_t)(gridDim.x / cluster) * teams; }
    __device__ __forceinline__ static void meet() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
    // Sums over the row, the same in every thread of it.  Two buffers in turn: who writes one again has passed a barrier that its readers reached behind their reading.
    template <int K>
    __device__ __forceinline__ void add(float (&v)[K]) {
#pragma unroll
        for (int o = 16; o; o >>= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(FULL, v[k], o);
        const int all = warps * cluster;
        if (all == 1) return;
        float *s = sums + (parity * teams + team) * 2 * room;
        parity ^= 1;
        if (cluster == 1) {
            if (lane == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) s[k * room + warp] = v[k];
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(warps * 32) : "memory");
        } else {
            namespace cg = cooperative_groups;
            auto c = cg::this_cluster();
            if (lane < cluster) {
                float *to = c.map_shared_rank(s, lane);
#pragma unroll
                for (int k = 0; k < K; ++k) to[k * room + rank * warps + warp] = v[k];
            }
            meet();
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float4 x = *reinterpret_cast<const float4 *>(s + k * room);
            v[k] = (x.x + x.y) + (x.z + x.w);
            for (int i = 4; i < all; i += 4) {
                x = *reinterpret_cast<const float4 *>(s + k * room + i);
                v[k] += (x.x + x.y) + (x.z + x.w);
            }
        }
    }
};

// mean and 1 / deviation of the row whose entries the threads hold (zeros behind its end)
template <int E>
__device__ __forceinline__ float2 norm_stats(JoinTeam &tm, const f32x2 (&v)[E][4], const int (&cnt)[E], int norm, float eps, float inv_n) {
    if (norm == DBSPMSPV_NORM_NONE) return make_float2(0.f, 1.f);
    float mean = 0.f, s[1];
    f32x2 p = 0;
    if (norm == DBSPMSPV_NORM_LAYER) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j) p = add2(p, v[e][j]);
        s[0] = sum2(p);
        tm.add(s);
        mean = s[0] * inv_n;
        p = 0;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2 d = add2(v[e][j], both(-mean));
            p = fma2(d, d, p);
        }
    s[0] = sum2(p);
    if (norm == DBSPMSPV_NORM_LAYER)
#pragma unroll
        for (int e = 0; e < E; ++e)          // (the zeros behind the end have no difference: once more without them)
            if (cnt[e] < 8) {
                s[0] = 0.f;
#pragma unroll
                for (int i = 0; i < E; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 x = apart(v[i][j]);
                        if (2 * j < cnt[i]) s[0] += (x.x - mean) * (x.x - mean);
                        if (2 * j + 1 < cnt[i]) s[0] += (x.y - mean) * (x.y - mean);
                    }
                break;
            }
    tm.add(s);
    return make_float2(mean, rsqrtf(s[0] * inv_n + eps));
}

// Shared memory: the slots [ahead][eight][piece][thread], the columns' factors [eight][piece][thread], the teams' sums
inline size_t join_smem(const JoinPlan &p, int pieces, int params) {
    return (size_t)(JOIN_AHEAD * pieces + params) * p.eights * p.warps * p.teams * 32 * 16 + (size_t)4 * p.teams * ((p.warps * p.cluster + 3) & ~3) * 4;
}

// What both kernels begin with: this thread's columns, slots and factors
template <int E>
struct JoinThread {
    uint4 *slots, *factors;
    int step, pieces, params, col[E], cnt[E];
    __device__ __forceinline__ JoinThread(const JoinArgs &a, uint4 *s_dyn, const JoinTeam &tm) {
        step = blockDim.x;
        pieces = a.pieces;
        params = a.params;
        slots = s_dyn + threadIdx.x;
        factors = slots + JOIN_AHEAD * E * a.pieces * step;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            col[e] = (((tm.rank * E + e) * tm.warps + tm.warp) * 32 + tm.lane) * 8;
            cnt[e] = max(0, min(8, a.n - col[e]));
        }
        for (int i = 0; i < JOIN_AHEAD * E * a.pieces; ++i) slots[i * step] = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ uint4 *slot(int at, int e, int piece) const { return slots + ((at * E + e) * pieces + piece) * step; }
    __device__ __forceinline__ uint4 *factor(int e, int piece) const { return factors + (e * params + piece) * step; }
};

// factors: gate * w_block * scales (or without a gate that has rows), w_next, then (BIAS) c_block * gate * scales, c_next
template <bool SF32, bool BF32, int E, bool BIAS>
__global__ void __launch_bounds__(join_cta<E>(), E == 1 ? 2 : 3) k_join(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint4 s_dyn[];
    JoinTeam tm(a, reinterpret_cast<float *>(s_dyn + (size_t)(JOIN_AHEAD * a.pieces + a.params) * E * blockDim.x));
    const JoinThread<E> me(a, s_dyn, tm);
    const int n = a.n, step = me.step;
    constexpr int RP = SF32 ? 2 : 1, BP = BF32 ? 2 : 1;
    pdl_wait();
    pdl_trigger();
    const int64_t first = tm.first(), walk = tm.step();
    auto ahead = [&](int64_t t, int at) {
        if (t < a.tokens)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (me.cnt[e] == 0) continue;
                if (a.r.p) row_ahead<SF32>(a.r, t, me.col[e], n, me.slot(at, e, 0), step);
                if (a.b.p) row_ahead<BF32>(a.b, t, me.col[e], n, me.slot(at, e, RP), step);
                if (a.gate.p) {
                    if (a.params_f32) row_ahead<true>(a.gate, t, me.col[e], n, me.slot(at, e, RP + BP), step);
                    else row_ahead<false>(a.gate, t, me.col[e], n, me.slot(at, e, RP + BP), step);
                }
            }
        close_ahead();
    };
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i) ahead(first + i * walk, i);
    const Numbers num = numbers_of(a.drop);
    const float scale = a.drop.random ? a.scale * a.drop.scale : a.scale;
    Columns cols[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        cols[e] = columns_of(num, (uint32_t)me.col[e] >> 3);
        columns_here(me.factor(e, 0), step, me.col[e], n, a.params_f32, scale, a.w_block, a.gate_vec);
        columns_here(me.factor(e, 2), step, me.col[e], n, a.params_f32, 1.f, a.w_next, nullptr);
        if (BIAS) {
            columns_here(me.factor(e, 4), step, me.col[e], n, a.params_f32, a.c_block ? scale : 0.f, a.c_block, a.gate_vec);
            columns_here(me.factor(e, 6), step, me.col[e], n, a.params_f32, a.c_next ? 1.f : 0.f, a.c_next, nullptr);
        }
    }
    int at = 0;
    for (int64_t t = first; t < a.tokens; t += walk) {
        wait_ahead<JOIN_AHEAD - 1>();
        f32x2 v[E][4], x[E][4], w[4];
        float2 sb = make_float2(0.f, 1.f);
        if (a.b.p) {
#pragma unroll
            for (int e = 0; e < E; ++e) row_here<BF32>(me.slot(at, e, RP), step, v[e]);
            sb = norm_stats<E>(tm, v, me.cnt, a.norm_block, a.eps_block, a.inv_n);
            const f32x2 inv = both(sb.y), shift = both(-sb.x * sb.y);
#pragma unroll
            for (int e = 0; e < E; ++e) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[e][j] = fma2(v[e][j], inv, shift);
                if (BIAS) {
                    f32x2 c[4];
                    row_here<true>(me.factor(e, 0), step, w);
                    row_here<true>(me.factor(e, 4), step, c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[e][j] = fma2(v[e][j], w[j], c[j]);
                }
                if (a.gate.p) {
                    row_here(a.params_f32, me.slot(at, e, RP + BP), step, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[e][j] = mul2(v[e][j], w[j]);
                }
                if (a.drop.random) drop_eight(a.drop, num, cols[e], (uint32_t)t, v[e]);
                row_here<SF32>(me.slot(at, e, 0), step, x[e]);
                if (!BIAS) row_here<true>(me.factor(e, 0), step, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[e][j] = BIAS ? add2(v[e][j], x[e][j]) : fma2(v[e][j], w[j], x[e][j]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) row_here<SF32>(me.slot(at, e, 0), step, x[e]);
        }
        ahead(t + JOIN_AHEAD * walk, at);
        at = at + 1 == JOIN_AHEAD ? 0 : at + 1;
        if (a.out.p)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (me.cnt[e]) store_eight<SF32>(const_cast<void *>(row_at<SF32>(a.out, t)), me.col[e], n, me.cnt[e] == 8 && a.out.aligned, x[e]);
        if (!a.h.p && !a.stats) continue;
        const float2 sn = norm_stats<E>(tm, x, me.cnt, a.norm_next, a.eps_next, a.inv_n);
        if (a.stats && tm.rank == 0 && tm.warp == 0 && tm.lane == 0) reinterpret_cast<float4 *>(a.stats)[t] = make_float4(sb.x, sb.y, sn.x, sn.y);
        if (a.h.p) {
            const f32x2 inv = both(sn.y), shift = both(-sn.x * sn.y);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (me.cnt[e] == 0) continue;
                f32x2 c[4];
                row_here<true>(me.factor(e, 2), step, w);
                if (BIAS) row_here<true>(me.factor(e, 6), step, c);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x2 y = fma2(x[e][j], inv, shift);
                    x[e][j] = BIAS ? fma2(y, w[j], c[j]) : mul2(y, w[j]);
                }
                store_eight<false>(const_cast<void *>(row_at<false>(a.h, t)), me.col[e], n, me.cnt[e] == 8 && a.h.aligned, x[e]);
            }
        }
    }
}

// factors: w_next, gate * w_block * scales (or without a gate that has rows), then c_block * scales for the gradient of such a gate.  Sums over a team's tokens: dw_next, A, then (BIAS) dc_next, B.
template <bool SF32, bool BF32, int E, bool BIAS>
__global__ void __launch_bounds__(join_cta<E>(), E == 1 ? 1 : 2) k_join_backward(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint4 s_dyn[];
    constexpr int SP = SF32 ? 2 : 1, BP = BF32 ? 2 : 1, SUMS = BIAS ? 4 : 2;
    JoinTeam tm(a, reinterpret_cast<float *>(s_dyn + (size_t)(JOIN_AHEAD * a.pieces + a.params) * E * blockDim.x));
    const JoinThread<E> me(a, s_dyn, tm);
    const int n = a.n, step = me.step;
    pdl_wait();
    pdl_trigger();
    const int64_t first = tm.first(), walk = tm.step();
    const bool block = a.parts || a.db.p || a.dgate.p;
    // pieces: dh, dout, out, b, gate
    constexpr int DOUT = 1, OUT = DOUT + SP, B = OUT + SP, GATE = B + BP;
    auto ahead = [&](int64_t t, int at) {
        if (t < a.tokens)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (me.cnt[e] == 0) continue;
                if (a.dh.p) row_ahead<false>(a.dh, t, me.col[e], n, me.slot(at, e, 0), step);
                if (a.dout.p) row_ahead<SF32>(a.dout, t, me.col[e], n, me.slot(at, e, DOUT), step);
                if (a.out.p) row_ahead<SF32>(a.out, t, me.col[e], n, me.slot(at, e, OUT), step);
                if (a.b.p) row_ahead<BF32>(a.b, t, me.col[e], n, me.slot(at, e, B), step);
                if (a.gate.p) {
                    if (a.params_f32) row_ahead<true>(a.gate, t, me.col[e], n, me.slot(at, e, GATE), step);
                    else row_ahead<false>(a.gate, t, me.col[e], n, me.slot(at, e, GATE), step);
                }
            }
        close_ahead();
    };
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i) ahead(first + i * walk, i);
    const Numbers num = numbers_of(a.drop);
    const float scale = a.drop.random ? a.scale * a.drop.scale : a.scale;
    Columns cols[E];
    f32x2 sum[SUMS][E][4];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        cols[e] = columns_of(num, (uint32_t)me.col[e] >> 3);
        columns_here(me.factor(e, 0), step, me.col[e], n, a.params_f32, 1.f, a.w_next, nullptr);
        columns_here(me.factor(e, 2), step, me.col[e], n, a.params_f32, scale, a.w_block, a.gate_vec);
        if (a.dgate.p) columns_here(me.factor(e, 4), step, me.col[e], n, a.params_f32, a.c_block ? scale : 0.f, a.c_block, nullptr);
#pragma unroll
        for (int k = 0; k < SUMS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[k][e][j] = 0;
    }
    int at = 0;
    for (int64_t t = first; t < a.tokens; t += walk) {
        const float4 st = a.stats ? reinterpret_cast<const float4 *>(a.stats)[t] : make_float4(0.f, 1.f, 0.f, 1.f);
        wait_ahead<JOIN_AHEAD - 1>();
        f32x2 g[E][4], u[E][4], w[4];
        // g: normalised out, u: dh * w_next
        const f32x2 inv_out = both(st.w), shift_out = both(-st.z * st.w);
        f32x2 p0 = 0, p1 = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            row_here<false>(me.slot(at, e, 0), step, u[e]);
            row_here<SF32>(me.slot(at, e, OUT), step, g[e]);
            row_here<true>(me.factor(e, 0), step, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[e][j] = fma2(g[e][j], inv_out, shift_out);
                sum[0][e][j] = fma2(u[e][j], g[e][j], sum[0][e][j]);
                if (BIAS) sum[2][e][j] = add2(u[e][j], sum[2][e][j]);
                u[e][j] = mul2(u[e][j], w[j]);
                p0 = fma2(u[e][j], g[e][j], p0);
                p1 = add2(u[e][j], p1);
            }
        }
        f32x2 slope = both(1.f), along = 0, mean = 0;
        if (a.norm_next != DBSPMSPV_NORM_NONE && a.dh.p) {
            float s[2] = {sum2(p0), sum2(p1)};
            tm.add(s);
            slope = inv_out;
            along = both(-st.w * (s[0] * a.inv_n));
            if (a.norm_next == DBSPMSPV_NORM_LAYER) mean = both(-st.w * (s[1] * a.inv_n));
        }
        // g: G, then drop(G), then that times gate, w and scales;  u: the normalised b
        const f32x2 inv_b = both(st.y), shift_b = both(-st.x * st.y);
        p0 = p1 = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            row_here<SF32>(me.slot(at, e, DOUT), step, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) g[e][j] = add2(w[j], fma2(u[e][j], slope, fma2(g[e][j], along, mean)));
            if (me.cnt[e] && a.dr.p) store_eight<SF32>(const_cast<void *>(row_at<SF32>(a.dr, t)), me.col[e], n, me.cnt[e] == 8 && a.dr.aligned, g[e]);
            if (!block) continue;
            if (a.drop.random) drop_eight(a.drop, num, cols[e], (uint32_t)t, g[e]);
            row_here<BF32>(me.slot(at, e, B), step, u[e]);
#pragma unroll
            for (int j = 0; j < 4; ++j) u[e][j] = fma2(u[e][j], inv_b, shift_b);
            if (a.gate.p) {
                if (a.dgate.p && me.cnt[e]) {
                    f32x2 d[4];
                    row_here<true>(me.factor(e, 2), step, w);
                    row_here<true>(me.factor(e, 4), step, d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = mul2(g[e][j], fma2(u[e][j], w[j], d[j]));
                    if (a.params_f32) store_eight<true>(const_cast<void *>(row_at<true>(a.dgate, t)), me.col[e], n, me.cnt[e] == 8 && a.dgate.aligned, d);
                    else store_eight<false>(const_cast<void *>(row_at<false>(a.dgate, t)), me.col[e], n, me.cnt[e] == 8 && a.dgate.aligned, d);
                }
                row_here(a.params_f32, me.slot(at, e, GATE), step, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[e][j] = mul2(g[e][j], w[j]);
            }
            row_here<true>(me.factor(e, 2), step, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum[1][e][j] = fma2(g[e][j], u[e][j], sum[1][e][j]);
                if (BIAS) sum[3][e][j] = add2(g[e][j], sum[3][e][j]);
                g[e][j] = mul2(g[e][j], w[j]);
                p0 = fma2(g[e][j], u[e][j], p0);
                p1 = add2(g[e][j], p1);
            }
        }
        ahead(t + JOIN_AHEAD * walk, at);
        at = at + 1 == JOIN_AHEAD ? 0 : at + 1;
        if (!a.db.p) continue;
        slope = both(1.f);
        along = mean = 0;
        if (a.norm_block != DBSPMSPV_NORM_NONE) {
            float s[2] = {sum2(p0), sum2(p1)};
            tm.add(s);
            slope = inv_b;
            along = both(-st.y * (s[0] * a.inv_n));
            if (a.norm_block == DBSPMSPV_NORM_LAYER) mean = both(-st.y * (s[1] * a.inv_n));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (me.cnt[e] == 0) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) g[e][j] = fma2(g[e][j], slope, fma2(u[e][j], along, mean));
            if (a.db.f32) store_eight<true>(const_cast<void *>(row_at<true>(a.db, t)), me.col[e], n, me.cnt[e] == 8 && a.db.aligned, g[e]);
            else store_eight<false>(const_cast<void *>(row_at<false>(a.db, t)), me.col[e], n, me.cnt[e] == 8 && a.db.aligned, g[e]);
        }
    }
    if (!a.parts) return;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (me.cnt[e])
#pragma unroll
            for (int k = 0; k < SUMS; ++k) store_eight<true>(a.parts + (first * SUMS + k) * a.ldp, me.col[e], (int)a.ldp, true, sum[k][e]);
}

// The teams' sums added up, and what follows from them
struct JoinSums {
    const float *parts;
    int64_t ldp;
    int32_t teams, n, params_f32;
    float scale;
    const void *w_block, *c_block, *gate_vec;
    float *dw_block, *dc_block, *dgate, *dw_next, *dc_next;
};
template <bool BIAS>
__global__ void __launch_bounds__(JOIN_SUMS_CTA) k_join_sums(const __grid_constant__ JoinSums a) {
    constexpr int SUMS = BIAS ? 4 : 2, X = JOIN_SUMS_COLS / 4, Y = JOIN_SUMS_CTA / X;
    __shared__ float4 s_sum[Y][SUMS][X];
    const int x = threadIdx.x % X, y = threadIdx.x / X;
    const int64_t at = (int64_t)blockIdx.x * JOIN_SUMS_COLS + 4 * x;
    pdl_wait();
    pdl_trigger();
    float4 v[SUMS];
#pragma unroll
    for (int k = 0; k < SUMS; ++k) v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < a.ldp)                           // (rows of the parts are whole eights)
#pragma unroll 4
        for (int i = y; i < a.teams; i += Y)
#pragma unroll
            for (int k = 0; k < SUMS; ++k) {
                const float4 p = *reinterpret_cast<const float4 *>(a.parts + ((int64_t)i * SUMS + k) * a.ldp + at);
                v[k].x += p.x; v[k].y += p.y; v[k].z += p.z; v[k].w += p.w;
            }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) s_sum[y][k][x] = v[k];
    __syncthreads();
    const int col = blockIdx.x * JOIN_SUMS_COLS + threadIdx.x;
    if (threadIdx.x >= JOIN_SUMS_COLS || col >= a.n) return;
    float s[SUMS];
#pragma unroll
    for (int k = 0; k < SUMS; ++k) {
        s[k] = 0.f;
        for (int i = 0; i < Y; ++i) s[k] += reinterpret_cast<const float *>(&s_sum[i][k][0])[threadIdx.x];
    }
    s[1] *= a.scale;
    const float g = a.gate_vec ? vector_one(a.gate_vec, a.params_f32, col) : 1.f;
    if (a.dw_next) a.dw_next[col] = s[0];
    if (a.dw_block) a.dw_block[col] = s[1] * g;
    if (BIAS) s[SUMS - 1] *= a.scale;
    if (BIAS && a.dc_next) a.dc_next[col] = s[SUMS - 2];
    if (BIAS && a.dc_block) a.dc_block[col] = s[SUMS - 1] * g;
    if (a.dgate) {
        float d = a.w_block ? s[1] * vector_one(a.w_block, a.params_f32, col) : s[1];
        if (BIAS && a.c_block) d += s[SUMS - 1] * vector_one(a.c_block, a.params_f32, col);
        a.dgate[col] = d;
    }
}

}  // namespace dbs
