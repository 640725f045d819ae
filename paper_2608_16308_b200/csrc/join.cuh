// A block joins the residual stream: out = r + scale drop(gate * norm_block(b)), h = norm_next(out), and the gradient of that.
//
// A row is owned by a team of warps, eight columns a thread: the values stay on the chip between the sums over the row (one for each norm, two for a layer norm; backwards one
// for each norm) and every array is read and written once.  A warp is a team for rows of up to 256 columns, a thread block holds up to eight teams; rows of more than JOIN_WARPS warps
// are shared out to a cluster whose blocks add up through each other's shared memory.  Teams walk the tokens, and the rows to come are copied ahead into slots of shared memory that belong to the thread
// itself (cp.async, no barrier): what bounds a long batch is HBM, and a sum over the row would else leave it idle.
//
// Sums over the tokens (gradients of weights, biases and a shared gate) are held by the threads of a column and written once per team; a second kernel adds the teams up in a
// fixed order.  With a shared gate g and weight w both gradients follow from one sum: A = sum q xhat gives dw = g A and dg = w A + c B, B = sum q.
#pragma once

#include <cooperative_groups.h>

#include "rows.cuh"

namespace dbs {

constexpr int JOIN_WARPS = 16;               // of a row in one thread block; more: a cluster
constexpr int JOIN_CLUSTER = 8;
constexpr int64_t JOIN_MAX_N = JOIN_WARPS * JOIN_CLUSTER * 256;
constexpr int JOIN_AHEAD = 3;                // rows in flight or in hand, per team
constexpr int JOIN_CTA = JOIN_WARPS * 32;
constexpr int JOIN_SUMS_X = 32, JOIN_SUMS_Y = 16;

struct JoinPlan {
    int warps, teams, cluster;               // warps of a team in a thread block, teams in it, blocks to a row
    int clusters;                            // in the grid
};

struct JoinArgs {
    Rows r, b, gate, out, h;                 // forward (gate: rows, else gate_vec)
    Rows dh, dout, dr, db, dgate;            // backward (out: what the forward call left)
    const void *w_block, *c_block, *gate_vec, *w_next, *c_next;
    int32_t params_f32, params_aligned;
    float *stats;
    Drop drop;
    float scale, eps_block, eps_next, inv_n;
    int32_t norm_block, norm_next, tokens, n, warps, teams, pieces;
    float *parts;                            // [team][sum][ldp]
    int64_t ldp;
};

__device__ __forceinline__ void copy_ahead(void *smem, const void *p) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p) : "memory");
}
__device__ __forceinline__ void close_ahead() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void wait_ahead() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// the thread's eight entries of row t into its slot (pieces `step` apart)
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
__device__ __forceinline__ void row_here(const uint4 *slot, int step, float v[8]) {
    if (F32) eight_of(slot[0], slot[step], v);
    else eight_of(slot[0], v);
}
__device__ __forceinline__ void vector_eight(const void *p, bool f32, bool aligned, int col, int n, float v[8]) {
    uint4 a, b;
    const bool whole = aligned && col + 8 <= n;
    if (f32) {
        load_raw<true>(p, col, n, whole, a, b);
        eight_of(a, b, v);
    } else {
        load_raw<false>(p, col, n, whole, a, b);
        eight_of(a, v);
    }
}

struct JoinTeam {
    int lane, warp, warps, team, teams, rank, cluster, parity;
    float *sums;                             // [parity][team][2][cluster * warps]
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
    }
    __device__ __forceinline__ int col() const { return ((rank * warps + warp) * 32 + lane) * 8; }
    __device__ __forceinline__ int64_t first() const { return (int64_t)(blockIdx.x / cluster) * teams + team; }
    __device__ __forceinline__ int64_t step() const { return (int64_t)(gridDim.x / cluster) * teams; }
    // Sums over the row, the same in every thread of it.  Two buffers in turn: who writes one again has passed a barrier that its readers reached behind their reading.
    template <int K>
    __device__ __forceinline__ void add(float (&v)[K]) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(FULL, v[k], o);
        const int all = warps * cluster;
        if (all == 1) return;
        float *s = sums + (parity * teams + team) * 2 * all;
        parity ^= 1;
        if (cluster == 1) {
            if (lane == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) s[k * all + warp] = v[k];
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(warps * 32) : "memory");
        } else {
            namespace cg = cooperative_groups;
            auto c = cg::this_cluster();
            if (lane < cluster) {
                float *to = c.map_shared_rank(s, lane);
#pragma unroll
                for (int k = 0; k < K; ++k) to[k * all + rank * warps + warp] = v[k];
            }
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float x = 0.f;
            for (int i = lane; i < all; i += 32) x += s[k * all + i];
#pragma unroll
            for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
            v[k] = x;
        }
    }
};

// mean and 1 / deviation of the row whose entries the threads hold (zeros behind its end)
__device__ __forceinline__ float2 norm_stats(JoinTeam &tm, const float v[8], int cnt, int norm, float eps, float inv_n) {
    if (norm == DBSPMSPV_NORM_NONE) return make_float2(0.f, 1.f);
    float mean = 0.f, s[1];
    if (norm == DBSPMSPV_NORM_LAYER) {
        s[0] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += v[j];
        tm.add(s);
        mean = s[0] * inv_n;
    }
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float d = j < cnt ? v[j] - mean : 0.f;
        s[0] += d * d;
    }
    tm.add(s);
    return make_float2(mean, rsqrtf(s[0] * inv_n + eps));
}

// Shared memory: the slots [ahead][piece][thread], then the teams' sums
inline size_t join_smem(const JoinPlan &p, int pieces) { return (size_t)JOIN_AHEAD * pieces * p.warps * p.teams * 32 * 16 + (size_t)2 * p.teams * 2 * p.warps * p.cluster * 4; }

template <bool SF32, bool BF32>
__global__ void __launch_bounds__(JOIN_CTA, 2) k_join(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t s_dyn[];
    const int step = blockDim.x;
    uint4 *slot = reinterpret_cast<uint4 *>(s_dyn) + threadIdx.x;
    JoinTeam tm(a, reinterpret_cast<float *>(reinterpret_cast<uint4 *>(s_dyn) + (size_t)JOIN_AHEAD * a.pieces * step));
    const int n = a.n, col = tm.col(), cnt = n - col < 0 ? 0 : n - col > 8 ? 8 : n - col;
    const bool live = cnt > 0, full = cnt == 8;
    constexpr int RP = SF32 ? 2 : 1, BP = BF32 ? 2 : 1;
    for (int i = 0; i < JOIN_AHEAD * a.pieces; ++i) slot[i * step] = make_uint4(0u, 0u, 0u, 0u);
    // (a cluster: every block has started before its shared memory is written)
    if (tm.cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    pdl_wait();
    pdl_trigger();
    const Numbers num = numbers_of(a.drop);
    const int64_t first = tm.first(), walk = tm.step();
    auto ahead = [&](int64_t t, int s) {
        if (live && t < a.tokens) {
            uint4 *p = slot + s * a.pieces * step;
            if (a.r.p) row_ahead<SF32>(a.r, t, col, n, p, step);
            if (a.b.p) {
                row_ahead<BF32>(a.b, t, col, n, p + RP * step, step);
                if (a.gate.p) {
                    if (a.params_f32) row_ahead<true>(a.gate, t, col, n, p + (RP + BP) * step, step);
                    else row_ahead<false>(a.gate, t, col, n, p + (RP + BP) * step, step);
                }
            }
        }
        close_ahead();
    };
#pragma unroll
    for (int s = 0; s < JOIN_AHEAD; ++s) ahead(first + s * walk, s);
    int at = 0;
    for (int64_t t = first; t < a.tokens; t += walk) {
        wait_ahead<JOIN_AHEAD - 1>();
        uint4 *p = slot + at * a.pieces * step;
        float x[8], v[8];
        row_here<SF32>(p, step, x);
        float2 sb = make_float2(0.f, 1.f);
        if (a.b.p) {
            row_here<BF32>(p + RP * step, step, v);
            sb = norm_stats(tm, v, cnt, a.norm_block, a.eps_block, a.inv_n);
            if (live) {
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (v[j] - sb.x) * sb.y;
                if (a.w_block) {
                    vector_eight(a.w_block, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] *= q[j];
                }
                if (a.c_block) {
                    vector_eight(a.c_block, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += q[j];
                }
                if (a.gate.p || a.gate_vec) {
                    if (a.gate_vec) vector_eight(a.gate_vec, a.params_f32, a.params_aligned, col, n, q);
                    else if (a.params_f32) row_here<true>(p + (RP + BP) * step, step, q);
                    else row_here<false>(p + (RP + BP) * step, step, q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] *= q[j];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= a.scale;
                if (a.drop.random) drop_eight(a.drop, num, (uint32_t)col >> 3, (uint32_t)t, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = j < cnt ? x[j] + v[j] : 0.f;
            }
        }
        ahead(t + JOIN_AHEAD * walk, at);
        at = at + 1 == JOIN_AHEAD ? 0 : at + 1;
        if (live && a.out.p) store_eight<SF32>(const_cast<void *>(row_at<SF32>(a.out, t)), col, n, full && a.out.aligned, x);
        if (!a.h.p && !a.stats) continue;
        const float2 sn = norm_stats(tm, x, cnt, a.norm_next, a.eps_next, a.inv_n);
        if (a.stats && tm.rank == 0 && tm.warp == 0 && tm.lane == 0) reinterpret_cast<float4 *>(a.stats)[t] = make_float4(sb.x, sb.y, sn.x, sn.y);
        if (live && a.h.p) {
            float q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (x[j] - sn.x) * sn.y;
            if (a.w_next) {
                vector_eight(a.w_next, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= q[j];
            }
            if (a.c_next) {
                vector_eight(a.c_next, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] += q[j];
            }
            store_eight<false>(const_cast<void *>(row_at<false>(a.h, t)), col, n, full && a.h.aligned, x);
        }
    }
}

// Sums over tokens of a team: dw_next, A, then (BIAS) dc_next, B
template <bool SF32, bool BF32, bool BIAS>
__global__ void __launch_bounds__(JOIN_CTA, 2) k_join_backward(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t s_dyn[];
    constexpr int SP = SF32 ? 2 : 1, BP = BF32 ? 2 : 1, SUMS = BIAS ? 4 : 2;
    const int step = blockDim.x;
    uint4 *slot = reinterpret_cast<uint4 *>(s_dyn) + threadIdx.x;
    JoinTeam tm(a, reinterpret_cast<float *>(reinterpret_cast<uint4 *>(s_dyn) + (size_t)JOIN_AHEAD * a.pieces * step));
    const int n = a.n, col = tm.col(), cnt = n - col < 0 ? 0 : n - col > 8 ? 8 : n - col;
    const bool live = cnt > 0, full = cnt == 8;
    for (int i = 0; i < JOIN_AHEAD * a.pieces; ++i) slot[i * step] = make_uint4(0u, 0u, 0u, 0u);
    if (tm.cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    pdl_wait();
    pdl_trigger();
    const Numbers num = numbers_of(a.drop);
    const int64_t first = tm.first(), walk = tm.step();
    const bool block = a.parts || a.db.p || a.dgate.p;
    // pieces: dh, dout, out, b, gate
    constexpr int DOUT = 1, OUT = DOUT + SP, B = OUT + SP, GATE = B + BP;
    auto ahead = [&](int64_t t, int s) {
        if (live && t < a.tokens) {
            uint4 *p = slot + s * a.pieces * step;
            if (a.dh.p) row_ahead<false>(a.dh, t, col, n, p, step);
            if (a.dout.p) row_ahead<SF32>(a.dout, t, col, n, p + DOUT * step, step);
            if (a.out.p) row_ahead<SF32>(a.out, t, col, n, p + OUT * step, step);
            if (a.b.p) row_ahead<BF32>(a.b, t, col, n, p + B * step, step);
            if (a.gate.p) {
                if (a.params_f32) row_ahead<true>(a.gate, t, col, n, p + GATE * step, step);
                else row_ahead<false>(a.gate, t, col, n, p + GATE * step, step);
            }
        }
        close_ahead();
    };
#pragma unroll
    for (int s = 0; s < JOIN_AHEAD; ++s) ahead(first + s * walk, s);
    float sum[SUMS][8];
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[k][j] = 0.f;
    int at = 0;
    for (int64_t t = first; t < a.tokens; t += walk) {
        const float4 st = a.stats ? reinterpret_cast<const float4 *>(a.stats)[t] : make_float4(0.f, 1.f, 0.f, 1.f);
        wait_ahead<JOIN_AHEAD - 1>();
        uint4 *p = slot + at * a.pieces * step;
        float g[8], u[8], q[8];
        row_here<false>(p, step, u);
        row_here<SF32>(p + OUT * step, step, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            g[j] = (g[j] - st.z) * st.w;
            sum[0][j] += u[j] * g[j];
            if (BIAS) sum[2][j] += u[j];
        }
        if (a.w_next && live) {
            vector_eight(a.w_next, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] *= q[j];
        }
        if (a.norm_next != DBSPMSPV_NORM_NONE && a.dh.p) {
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[0] += u[j] * g[j];
                s[1] += u[j];
            }
            tm.add(s);
            const float along = s[0] * a.inv_n, mean = a.norm_next == DBSPMSPV_NORM_LAYER ? s[1] * a.inv_n : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = st.w * (u[j] - mean - g[j] * along);
        }
        row_here<SF32>(p + DOUT * step, step, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] += u[j];
        if (live && a.dr.p) store_eight<SF32>(const_cast<void *>(row_at<SF32>(a.dr, t)), col, n, full && a.dr.aligned, g);
        if (block) {
            // g: q, then q * gate * w;  u: the normalised b
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = j < cnt ? g[j] * a.scale : 0.f;
            if (a.drop.random) drop_eight(a.drop, num, (uint32_t)col >> 3, (uint32_t)t, g);
            row_here<BF32>(p + B * step, step, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = (u[j] - st.x) * st.y;
            if (a.gate.p) {
                if (a.dgate.p && live) {
                    float d[8];
                    if (a.w_block) vector_eight(a.w_block, a.params_f32, a.params_aligned, col, n, d);
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] = a.w_block ? d[j] * u[j] : u[j];
                    if (a.c_block) {
                        vector_eight(a.c_block, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
                        for (int j = 0; j < 8; ++j) d[j] += q[j];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] *= g[j];
                    if (a.params_f32) store_eight<true>(const_cast<void *>(row_at<true>(a.dgate, t)), col, n, full && a.dgate.aligned, d);
                    else store_eight<false>(const_cast<void *>(row_at<false>(a.dgate, t)), col, n, full && a.dgate.aligned, d);
                }
                if (a.params_f32) row_here<true>(p + GATE * step, step, q);
                else row_here<false>(p + GATE * step, step, q);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] *= q[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum[1][j] += g[j] * u[j];
                if (BIAS) sum[3][j] += g[j];
            }
            if (a.db.p) {
                if (live && a.gate_vec) {
                    vector_eight(a.gate_vec, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] *= q[j];
                }
                if (live && a.w_block) {
                    vector_eight(a.w_block, a.params_f32, a.params_aligned, col, n, q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] *= q[j];
                }
                if (a.norm_block != DBSPMSPV_NORM_NONE) {
                    float s[2] = {0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        s[0] += g[j] * u[j];
                        s[1] += g[j];
                    }
                    tm.add(s);
                    const float along = s[0] * a.inv_n, mean = a.norm_block == DBSPMSPV_NORM_LAYER ? s[1] * a.inv_n : 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = st.y * (g[j] - mean - u[j] * along);
                }
                if (live) {
                    if (a.db.f32) store_eight<true>(const_cast<void *>(row_at<true>(a.db, t)), col, n, full && a.db.aligned, g);
                    else store_eight<false>(const_cast<void *>(row_at<false>(a.db, t)), col, n, full && a.db.aligned, g);
                }
            }
        }
        ahead(t + JOIN_AHEAD * walk, at);
        at = at + 1 == JOIN_AHEAD ? 0 : at + 1;
    }
    if (a.parts && live) {
        float *to = a.parts + first * SUMS * a.ldp + col;
#pragma unroll
        for (int k = 0; k < SUMS; ++k) {
            float4 *v = reinterpret_cast<float4 *>(to + k * a.ldp);
            v[0] = make_float4(sum[k][0], sum[k][1], sum[k][2], sum[k][3]);
            v[1] = make_float4(sum[k][4], sum[k][5], sum[k][6], sum[k][7]);
        }
    }
}

// The teams' sums added up, and what follows from them
struct JoinSums {
    const float *parts;
    int64_t ldp;
    int32_t teams, n, params_f32;
    const void *w_block, *c_block, *gate_vec;
    float *dw_block, *dc_block, *dgate, *dw_next, *dc_next;
};
__device__ __forceinline__ float vector_one(const void *p, bool f32, int i) {
    return f32 ? static_cast<const float *>(p)[i] : __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
}
template <bool BIAS>
__global__ void __launch_bounds__(JOIN_SUMS_X *JOIN_SUMS_Y) k_join_sums(const __grid_constant__ JoinSums a) {
    constexpr int SUMS = BIAS ? 4 : 2;
    __shared__ float s_sum[JOIN_SUMS_Y][SUMS][JOIN_SUMS_X];
    const int x = threadIdx.x % JOIN_SUMS_X, y = threadIdx.x / JOIN_SUMS_X, col = blockIdx.x * JOIN_SUMS_X + x;
    pdl_wait();
    pdl_trigger();
    float v[SUMS];
#pragma unroll
    for (int k = 0; k < SUMS; ++k) v[k] = 0.f;
    if (col < a.n)
#pragma unroll 4
        for (int i = y; i < a.teams; i += JOIN_SUMS_Y)
#pragma unroll
            for (int k = 0; k < SUMS; ++k) v[k] += a.parts[((int64_t)i * SUMS + k) * a.ldp + col];
#pragma unroll
    for (int k = 0; k < SUMS; ++k) s_sum[y][k][x] = v[k];
    __syncthreads();
    if (y || col >= a.n) return;
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
        for (int i = 1; i < JOIN_SUMS_Y; ++i) v[k] += s_sum[i][k][x];
    const float g = a.gate_vec ? vector_one(a.gate_vec, a.params_f32, col) : 1.f;
    if (a.dw_next) a.dw_next[col] = v[0];
    if (a.dw_block) a.dw_block[col] = v[1] * g;
    if (BIAS && a.dc_next) a.dc_next[col] = v[SUMS - 2];
    if (BIAS && a.dc_block) a.dc_block[col] = v[SUMS - 1] * g;
    if (a.dgate) {
        float d = a.w_block ? v[1] * vector_one(a.w_block, a.params_f32, col) : v[1];
        if (BIAS && a.c_block) d += v[SUMS - 1] * vector_one(a.c_block, a.params_f32, col);
        a.dgate[col] = d;
    }
}

}  // namespace dbs
