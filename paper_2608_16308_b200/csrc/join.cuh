// A block joins the residual stream: out = r + scale drop(gate * norm_block(b)), h = norm_next(out), and the gradient of that.
//
// A row is owned by a team of warps; a warp takes 256 or 512 columns of it, eight or twice eight a lane: the values stay on the chip between the sums over the row (one for each norm, two for a layer norm;
// backwards one for each norm) and every array is read and written once.  A warp is a team for short rows, a thread block holds several teams then; rows of more than 4096 columns are shared out to a
// cluster whose blocks send their sums into each other's shared memory.  Teams walk the tokens.  The rows to come are copied ahead into shared memory of the warp (cp.async): a sum over the row would else
// leave HBM idle.  Weights, gate, scales and biases of the columns lie beside them in fp32, multiplied with one another once.  What is left is the way through a row, whose sums a team
// waits for with one row in hand (half of an SM's issue rate and of HBM's); products and sums go two entries at a time, and where all rows are whole eights on 16 bytes (WHOLE) a row's address is one product-and-sum and its copy one instruction.
// Other rows: of one on 16 bytes the last eight is copied in words and stored entry by entry; one that is not is copied and written in words of 4 bytes, side by side across the warp, and in shared memory moved by half a word
// where it begins between two.
//
// Sums over the tokens (gradients of weights, biases and a shared gate) are held by the threads of a column and written once per team; a second kernel adds the teams up in a
// fixed order.  With a shared gate g and weight w both gradients follow from one sum: A = sum drop(G) xhat gives dw = scale g A and dg = scale (w A + c B), B = sum drop(G).
#pragma once

#include <type_traits>

#include "rows.cuh"

namespace dbs {

constexpr int JOIN_COLS = 4096;              // of a row in one thread block; more: a cluster
constexpr int JOIN_CLUSTER = 8;
constexpr int64_t JOIN_MAX_N = JOIN_COLS * JOIN_CLUSTER;
constexpr int JOIN_AHEAD = 2;                // rows in flight or in hand, per team
constexpr int JOIN_SUMS_CTA = 512;
constexpr int JOIN_WAIT = 1 << 20;           // tries of a wait for a cluster's sums, before it gives up: about two seconds
// threads at most (two eights a lane, or rows of up to 2048 columns); of gradients with sums of biases (one eight a lane)
__host__ __device__ constexpr int join_cta(bool sums_of_biases) { return sums_of_biases ? JOIN_COLS / 8 : JOIN_COLS / 16; }

struct JoinPlan {
    int eights;                              // of a lane: 1, 2
    int warps, teams, cluster;               // warps of a team in a thread block, teams in it, blocks to a row
    int clusters;                            // in the grid
};

struct JoinArgs {
    Rows r, b, gate, out, h;                 // forward (gate: rows, else gate_vec)
    Rows dh, dout, dr, db, dgate;            // backward (out: what the forward call left)
    const void *w_block, *c_block, *gate_vec, *w_next, *c_next;
    int32_t params_f32, room, params;        // bytes that a warp's eights of one row take in shared memory; pieces of 16 bytes of factors for an eight
    float *stats;
    Drop drop;
    float scale, eps_block, eps_next, inv_n;
    int32_t norm_block, norm_next, tokens, n, warps, teams;
    float *parts;                            // [team][sum][ldp]
    int64_t ldp;
};

// the same where all rows are whole eights on 16 bytes: `mine` is the lane's place in row 0.  (An eight behind the row's end is 0 bytes long: no branch.)
template <bool F32>
__device__ __forceinline__ void row_ahead(const uint8_t *mine, uint32_t stride, uint32_t t, const WarpEight &w, uint8_t *to) {
    const uint8_t *p = mine + (uint64_t)t * stride;
    copy_ahead(to + w.lane * 16, p, w.cnt * 2);
    if (F32) copy_ahead(to + 512 + w.lane * 16, p + 16, w.cnt * 2);
}
// and where all rows are whole eights on 16 bytes
template <bool F32>
__device__ __forceinline__ void row_out(uint8_t *mine, uint32_t stride, uint32_t t, const f32x2 v[4]) {
    uint8_t *p = mine + (uint64_t)t * stride;
    if (F32) {
        ulonglong2 *q = reinterpret_cast<ulonglong2 *>(p);
        q[0] = make_ulonglong2(v[0], v[1]);
        q[1] = make_ulonglong2(v[2], v[3]);
    } else *reinterpret_cast<uint4 *>(p) = bf16_eight(v);
}

__device__ __forceinline__ float vector_one(const void *p, bool f32, int i) {
    return f32 ? static_cast<const float *>(p)[i] : __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
}
// Eight entries each of K vectors of parameters as they lie, of SIDE eights.  All loads stand side by side, without a branch between them: a short call waits for memory once.
struct Eight {
    uint4 a, b;
};
template <int SIDE, int K>
__device__ __forceinline__ void vectors_here(const void *(&p)[K], bool f32, const WarpEight *w, int n, Eight (&q)[SIDE][K]) {
    const void *some = nullptr;              // (in the place of one that is not there)
    uintptr_t low = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        some = some ? some : p[k];
        low |= reinterpret_cast<uintptr_t>(p[k]);
    }
    if (!some) {
#pragma unroll
        for (int i = 0; i < SIDE * K; ++i) q[i / K][i % K] = Eight{make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
        return;
    }
    bool whole = (low & 15u) == 0;
#pragma unroll
    for (int i = 0; i < SIDE; ++i) whole = whole && w[i].cnt == 8;
    auto load = [&](auto F32, auto WHOLE) {
#pragma unroll
        for (int i = 0; i < SIDE; ++i)
#pragma unroll
            for (int k = 0; k < K; ++k) load_raw<decltype(F32)::value>(p[k] ? p[k] : some, w[i].mine(), n, decltype(WHOLE)::value, q[i][k].a, q[i][k].b);
    };
    if (f32) whole ? load(std::true_type{}, std::true_type{}) : load(std::true_type{}, std::false_type{});
    else whole ? load(std::false_type{}, std::true_type{}) : load(std::false_type{}, std::false_type{});
}
__device__ __forceinline__ void vector_values(const Eight &q, const void *p, bool f32, float v[8]) {
    if (f32) eight_of(q.a, q.b, v);
    else eight_of(q.a, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p ? v[j] : 1.f;
}
// factors of eight columns in fp32: scale and two vectors (null: ones) multiplied; zeros behind the row's end
__device__ __forceinline__ void columns_here(uint4 *to, int col, int n, bool f32, float scale, const Eight &v, const void *has_v, const Eight &w, const void *has_w) {
    float x[8], y[8];
    vector_values(v, has_v, f32, x);
    vector_values(w, has_w, f32, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = col + j < n ? scale * x[j] * y[j] : 0.f;
    to[0] = fp32_four(x);
    to[32] = fp32_four(x + 4);
}
__device__ __forceinline__ void factors_here(const uint4 *at, f32x2 v[4]) {
    const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(at), b = *reinterpret_cast<const ulonglong2 *>(at + 32);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}

// Sums over the row.  In a thread block they meet at a barrier of the team's; in a cluster every warp sends its own to each block's shared memory, where an mbarrier counts the bytes (no fence, which would wait
// for the rows written meanwhile).  Two buffers in turn: who writes one again has passed a barrier that its readers reached behind their reading.
__host__ __device__ inline int join_sums_room(int warps, int cluster) { return warps * cluster < 8 ? 8 : (warps * cluster + 3) & ~3; }
// CLUSTERS: whether there can be any (one eight a lane and no sums of biases: rows of up to 2048 columns, of which a thread block has a team or more)
template <bool CLUSTERS>
struct JoinTeam {
    int lane, warp, warps, team, teams, rank, cluster, room;
    bool alone;                              // a warp has the whole row
    int last;                                // the last warp of the row with columns; their number, and that of the others
    float cols_last, inv_last, cols;
    uint32_t turn;                           // sums so far; from LOST on a wait of this warp's for its cluster has run out: it neither sends nor waits any more, and what it would have summed is NaN
    static constexpr uint32_t LOST = 1u << 31;
    float *sums;                             // [buffer][team][2][room]: zeros behind the warps'; then, of a cluster, its barriers
    __device__ __forceinline__ JoinTeam(const JoinArgs &a, float *s, int columns) {
        lane = threadIdx.x & 31;
        const int w = threadIdx.x >> 5;
        warps = a.warps;
        teams = a.teams;
        team = w / warps;
        warp = w - team * warps;
        rank = 0;
        cluster = 1;
        if (CLUSTERS) {
            asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
            asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
        }
        turn = 0;
        sums = s;
        room = join_sums_room(warps, cluster);
        alone = warps * cluster == 1;
        last = (a.n - 1) / columns;
        cols = columns;
        cols_last = a.n - last * columns;
        inv_last = 1.f / cols_last;
        for (int i = threadIdx.x; i < 4 * teams * room; i += blockDim.x) s[i] = 0.f;
        if (CLUSTERS && cluster > 1) {
            if (threadIdx.x < 2) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(barrier(threadIdx.x)) : "memory");
            // (every block's barriers are there before another one sends)
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            meet();
        } else __syncthreads();
    }
    __device__ __forceinline__ int64_t first() const { return (int64_t)(blockIdx.x / cluster) * teams + team; }
    __device__ __forceinline__ int64_t step() const { return (int64_t)(gridDim.x / cluster) * teams; }
    __device__ __forceinline__ static void meet() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
    __device__ __forceinline__ uint32_t barrier(int i) const { return (uint32_t)__cvta_generic_to_shared(sums + 4 * teams * room) + 8 * i; }
    template <int K>
    __device__ __forceinline__ static void add_warp(float (&v)[K]) {
#pragma unroll
        for (int o = 16; o; o >>= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(FULL, v[k], o);
    }
    // (One that exits before the others are done would be sent to behind its end: the cluster's barrier waits until all its threads have come here or exited.)
    __device__ __forceinline__ void give_up() {
        turn |= LOST;
        asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");
    }
    // every warp's K numbers to every warp of the row: [number][room], warps in the order of their columns.  False: a wait ran out.
    template <int K>
    __device__ __forceinline__ bool exchange(const float (&v)[K], const float *&s, int tries = JOIN_WAIT) {
        const int buffer = turn & 1, phase = (turn >> 1) & 1;
        float *to = sums + (buffer * teams + team) * 2 * room;
        s = to;
        ++turn;
        if (!CLUSTERS || cluster == 1) {
            if (lane == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) to[k * room + warp] = v[k];
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(warps * 32) : "memory");
            return true;
        }
        const bool on = turn < LOST;          // (a barrier whose phase was given up takes no second arrival)
        if (threadIdx.x == 0 && on) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(barrier(buffer)), "r"(warps * cluster * K * 4) : "memory");
        if (lane < cluster && on) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                uint32_t there, bar;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(to + k * room + rank * warps + warp)), "r"(lane));
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(barrier(buffer)), "r"(lane));
                asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(there), "r"(__float_as_uint(v[k])), "r"(bar) : "memory");
            }
        }
        uint32_t ok = 0;
        for (int i = on ? 0 : tries; i < tries && !ok; ++i)
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(barrier(buffer)), "r"(phase) : "memory");
        if (__all_sync(FULL, ok)) return true;
        if (on) give_up();
        return false;
    }
    // the same sums in every thread of the row; NaN where a wait ran out
    template <int K>
    __device__ __forceinline__ void add(float (&v)[K]) {
        add_warp(v);
        if (alone) return;
        const float *s;
        const bool ok = exchange(v, s);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float4 x = *reinterpret_cast<const float4 *>(s + k * room), y = *reinterpret_cast<const float4 *>(s + k * room + 4);
            v[k] = ((x.x + x.y) + (x.z + x.w)) + ((y.x + y.y) + (y.z + y.w));
            for (int i = 8; i < warps * cluster; i += 4) {
                const float4 z = *reinterpret_cast<const float4 *>(s + k * room + i);
                v[k] += (z.x + z.y) + (z.z + z.w);
            }
            if (!ok) v[k] = __uint_as_float(0x7FC00000u);
        }
    }
    // Mean of the row and the sum of the squared differences from it, from each warp's own: those of its entries from its own mean, and of that mean from the row's (Chan, Golub and LeVeque, 1979).
    __device__ __forceinline__ float2 spread(float sum, float squares, float inv_n) {
        if (alone) return make_float2(sum * inv_n, squares);
        const float *s, v[2] = {sum, squares};
        const bool ok = exchange(v, s);
        float mean = 0.f, all = 0.f;
        for (int i = 0; i <= last; ++i) mean += s[i];
        mean *= inv_n;
        for (int i = 0; i <= last; ++i) {
            const float d = s[i] * (i < last ? 1.f / cols : inv_last) - mean;
            all += s[room + i] + (i < last ? cols : cols_last) * d * d;
        }
        return ok ? make_float2(mean, all) : make_float2(__uint_as_float(0x7FC00000u), 0.f);
    }
};

// mean and 1 / deviation of the row whose entries the threads hold (zeros behind its end)
template <int E, bool WHOLE, typename Team>
__device__ __forceinline__ float2 norm_stats(Team &tm, const f32x2 (&v)[E][4], const WarpEight (&w)[E], int norm, float eps, float inv_n) {
    float s[1];
    f32x2 p[2] = {0, 0};
    if (norm == DBSPMSPV_NORM_RMS) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j % 2] = fma2(v[e][j], v[e][j], p[j % 2]);
        s[0] = sum2(add2(p[0], p[1]));
        tm.add(s);
        return make_float2(0.f, rsqrtf(s[0] * inv_n + eps));
    }
    if (norm != DBSPMSPV_NORM_LAYER) return make_float2(0.f, 1.f);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j % 2] = add2(p[j % 2], v[e][j]);
    s[0] = sum2(add2(p[0], p[1]));
    Team::add_warp(s);
    const float sum = s[0];
    const int place = w[0].col / (256 * E);
    const f32x2 minus = both(-sum * (place < tm.last ? 1.f / (256 * E) : place == tm.last ? tm.inv_last : 0.f));
    s[0] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        f32x2 q = 0;
        const int cnt = w[e].cnt;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x2 d = add2(v[e][j], minus);
            if (!WHOLE && cnt < 8) {
                const float2 x = apart(d);
                d = pair(2 * j < cnt ? x.x : 0.f, 2 * j + 1 < cnt ? x.y : 0.f);
            }
            q = fma2(d, d, q);
        }
        s[0] += WHOLE && cnt == 0 ? 0.f : sum2(q);                           // (zeros behind the row's end have no difference from the mean)
    }
    Team::add_warp(s);
    const float2 all = tm.spread(sum, s[0], inv_n);
    return make_float2(all.x, rsqrtf(all.y * inv_n + eps));
}

// the row's sums of u * xhat and, behind a layer norm, of u
template <typename Team>
__device__ __forceinline__ float2 slope_sums(Team &tm, int norm, f32x2 along, f32x2 mean) {
    if (norm == DBSPMSPV_NORM_LAYER) {
        float s[2] = {sum2(along), sum2(mean)};
        tm.add(s);
        return make_float2(s[0], s[1]);
    }
    float s[1] = {sum2(along)};
    tm.add(s);
    return make_float2(s[0], 0.f);
}

// A warp's shared memory: the rows [ahead][eight][array], the columns' factors [eight][piece][lane], room for rows that are written in words.  Behind the warps': the teams' sums, barriers.
__host__ __device__ inline int join_warp_bytes(int eights, int room, int params, bool whole) { return JOIN_AHEAD * room + eights * params * 512 + (whole ? 0 : 1024); }
inline size_t join_smem(const JoinPlan &p, int room, int params, bool whole) {
    return (size_t)join_warp_bytes(p.eights, room, params, whole) * p.warps * p.teams + (size_t)4 * p.teams * join_sums_room(p.warps, p.cluster) * 4 + 16;
}

// What both kernels begin with: the warp's columns and its shared memory
template <int E, bool WHOLE>
struct JoinWarp {
    uint8_t *rows, *spare;
    uint4 *factors;
    int room;
    WarpEight w[E];
    template <typename Team>
    __device__ __forceinline__ JoinWarp(const JoinArgs &a, uint8_t *s_dyn, const Team &tm) {
        room = a.room;
        rows = s_dyn + (threadIdx.x >> 5) * join_warp_bytes(E, a.room, a.params, WHOLE);
        factors = reinterpret_cast<uint4 *>(rows + JOIN_AHEAD * room) + tm.lane;
        spare = rows + JOIN_AHEAD * room + E * a.params * 512;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            w[e].lane = tm.lane;
            w[e].col = ((tm.rank * tm.warps + tm.warp) * E + e) * 256;
            w[e].cnt = max(0, min(8, a.n - w[e].mine()));
        }
        for (int i = tm.lane; i < JOIN_AHEAD * room / 16; i += 32) reinterpret_cast<uint4 *>(rows)[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
    }
    __device__ __forceinline__ uint4 *factor(int e, int params, int piece) const { return factors + (e * params + piece) * 32; }
    // the lane's place in row 0
    template <bool F32>
    __device__ __forceinline__ uint8_t *mine(const Rows &r) const { return static_cast<uint8_t *>(r.p) + (int64_t)w[0].mine() * (F32 ? 4 : 2); }
};

// 4096 rows of 4096 in bf16, root mean squares on both sides, a gate, dropout: 29.3 us, 4.58 TB/s (HBM copies 6.46): 294 warp instructions a warp and 256 columns at 2.0 of 4 a clock and SM, a quarter of them the generator's (24 us
// without dropout and gate).
// 1, 8 rows: 5.5 us, the calling thread.
// factors: gate * w_block * scales (or without a gate that has rows), w_next, then (BIAS) c_block * gate * scales, c_next
// FORM: rows of any kind; whole eights on 16 bytes; those, and r, b, out and h are all there (4096 x 4096 with their tests in the loop 32.8 us, 29.4 without).
enum { JOIN_ANY = 0, JOIN_WHOLE = 1, JOIN_ALL = 2 };
template <bool SF32, bool BF32, int E, bool BIAS, int FORM, bool GATES>
__global__ void __launch_bounds__(join_cta(false), E == 1 ? 4 : 3) k_join(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t s_dyn[];
    constexpr bool WHOLE = FORM != JOIN_ANY, ALL = FORM == JOIN_ALL;
    constexpr int SZ = SF32 ? 4 : 2, BZ = BF32 ? 4 : 2, PARAMS = BIAS ? 8 : 4;
    // where a lane's eights of r, b and the gate lie in a row's shared memory
    constexpr int AT_R = 0, AT_B = E * eight_room<SF32, WHOLE>(), AT_G = AT_B + E * eight_room<BF32, WHOLE>();
    JoinTeam<(E == 2)> tm(a, reinterpret_cast<float *>(s_dyn + join_warp_bytes(E, a.room, PARAMS, WHOLE) * (blockDim.x >> 5)), 256 * E);
    const JoinWarp<E, WHOLE> me(a, s_dyn, tm);
    const int n = a.n;
    pdl_wait();
    pdl_trigger();
    const uint32_t tokens = a.tokens, walk = (uint32_t)tm.step(), first = (uint32_t)tm.first();
    const uint8_t *my_r = me.template mine<SF32>(a.r), *my_b = me.template mine<BF32>(a.b);
    uint8_t *my_out = me.template mine<SF32>(a.out), *my_h = me.template mine<false>(a.h);
    const bool has_r = ALL || a.r.p, has_b = ALL || a.b.p, has_out = ALL || a.out.p, has_h = ALL || a.h.p;
    auto ahead = [&](uint32_t t, uint8_t *to) {
        if (t < tokens)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (WHOLE) {
                    if (has_r) row_ahead<SF32>(my_r + e * 256 * SZ, a.r.step, t, me.w[e], to + AT_R + e * eight_room<SF32, WHOLE>());
                    if (has_b) row_ahead<BF32>(my_b + e * 256 * BZ, a.b.step, t, me.w[e], to + AT_B + e * eight_room<BF32, WHOLE>());
                } else {
                    if (has_r) row_ahead<SF32>(a.r, t, me.w[e], n, to + AT_R + e * eight_room<SF32, WHOLE>());
                    if (has_b) row_ahead<BF32>(a.b, t, me.w[e], n, to + AT_B + e * eight_room<BF32, WHOLE>());
                }
                if (GATES) {
                    if (a.params_f32) row_ahead<true>(a.gate, t, me.w[e], n, to + AT_G + e * eight_room<true, false>());
                    else row_ahead<false>(a.gate, t, me.w[e], n, to + AT_G + e * eight_room<false, false>());
                }
            }
        close_ahead();
    };
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i) ahead(first + i * walk, me.rows + i * me.room);
    const Numbers num = numbers_of(a.drop);
    const float scale = a.drop.random ? a.scale * a.drop.scale : a.scale;
    Columns cols[E];
    // (both eights' vectors side by side, but for biases, which would not fit the registers)
    constexpr int SIDE = BIAS ? 1 : E;
#pragma unroll
    for (int e0 = 0; e0 < E; e0 += SIDE) {
        const void *given[BIAS ? 5 : 3] = {a.w_block, a.w_next, a.gate_vec};
        if constexpr (BIAS) {
            given[3] = a.c_block;
            given[4] = a.c_next;
        }
        Eight q[SIDE][BIAS ? 5 : 3];
        vectors_here(given, a.params_f32, me.w + e0, n, q);
#pragma unroll
        for (int i = 0; i < SIDE; ++i) {
            const int e = e0 + i, col = me.w[e].mine();
            cols[e] = columns_of(num, (uint32_t)col >> 3);
            columns_here(me.factor(e, PARAMS, 0), col, n, a.params_f32, scale, q[i][0], a.w_block, q[i][2], a.gate_vec);
            columns_here(me.factor(e, PARAMS, 2), col, n, a.params_f32, 1.f, q[i][1], a.w_next, q[i][1], nullptr);
            if constexpr (BIAS) {
                columns_here(me.factor(e, PARAMS, 4), col, n, a.params_f32, a.c_block ? scale : 0.f, q[i][3], a.c_block, q[i][2], a.gate_vec);
                columns_here(me.factor(e, PARAMS, 6), col, n, a.params_f32, a.c_next ? 1.f : 0.f, q[i][4], a.c_next, q[i][4], nullptr);
            }
        }
    }
    uint8_t *at = me.rows;
    for (uint32_t t = first; t < tokens; t += walk) {
        wait_ahead<JOIN_AHEAD - 1>();
        if (!WHOLE) __syncwarp();             // (words are other lanes')
        f32x2 v[E][4], x[E][4], w[4];
        float2 sb = make_float2(0.f, 1.f);
        if (has_b) {
#pragma unroll
            for (int e = 0; e < E; ++e) row_here<BF32, WHOLE>(a.b, t, me.w[e], at + AT_B + e * eight_room<BF32, WHOLE>(), v[e]);
            sb = norm_stats<E, WHOLE>(tm, v, me.w, a.norm_block, a.eps_block, a.inv_n);
            const f32x2 inv = both(sb.y), shift = both(-sb.x * sb.y);
#pragma unroll
            for (int e = 0; e < E; ++e) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[e][j] = fma2(v[e][j], inv, shift);
                if (BIAS) {
                    f32x2 c[4];
                    factors_here(me.factor(e, PARAMS, 0), w);
                    factors_here(me.factor(e, PARAMS, 4), c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[e][j] = fma2(v[e][j], w[j], c[j]);
                }
                if (GATES) {
                    if (a.params_f32) row_here<true, false>(a.gate, t, me.w[e], at + AT_G + e * eight_room<true, false>(), w);
                    else row_here<false, false>(a.gate, t, me.w[e], at + AT_G + e * eight_room<false, false>(), w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[e][j] = mul2(v[e][j], w[j]);
                }
            }
            if (a.drop.random) drop_eights<E, true>(a.drop, num, cols, t, v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                row_here<SF32, WHOLE>(a.r, t, me.w[e], at + AT_R + e * eight_room<SF32, WHOLE>(), x[e]);
                if (!BIAS) factors_here(me.factor(e, PARAMS, 0), w);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[e][j] = BIAS ? add2(v[e][j], x[e][j]) : fma2(v[e][j], w[j], x[e][j]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) row_here<SF32, WHOLE>(a.r, t, me.w[e], at + AT_R + e * eight_room<SF32, WHOLE>(), x[e]);
        }
        if (!WHOLE) __syncwarp();
        ahead(t + JOIN_AHEAD * walk, at);
        at = at == me.rows ? me.rows + me.room : me.rows;
        static_assert(JOIN_AHEAD == 2, "two rows in turn");
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (WHOLE) {
                if (has_out && me.w[e].cnt) row_out<SF32>(my_out + e * 256 * SZ, a.out.step, t, x[e]);
            } else if (has_out) row_out<SF32>(a.out, t, me.w[e], n, x[e], me.spare);
        }
        if (!has_h && !a.stats) continue;
        const float2 sn = norm_stats<E, WHOLE>(tm, x, me.w, a.norm_next, a.eps_next, a.inv_n);
        if (a.stats && tm.rank == 0 && tm.warp == 0 && tm.lane == 0) reinterpret_cast<float4 *>(a.stats)[t] = make_float4(sb.x, sb.y, sn.x, sn.y);
        if (!has_h) continue;
        const f32x2 inv = both(sn.y), shift = both(-sn.x * sn.y);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            f32x2 c[4];
            factors_here(me.factor(e, PARAMS, 2), w);
            if (BIAS) factors_here(me.factor(e, PARAMS, 6), c);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x2 y = fma2(x[e][j], inv, shift);
                x[e][j] = BIAS ? fma2(y, w[j], c[j]) : mul2(y, w[j]);
            }
            if (WHOLE) {
                if (me.w[e].cnt) row_out<false>(my_h + e * 512, a.h.step, t, x[e]);
            } else row_out<false>(a.h, t, me.w[e], n, x[e], me.spare);
        }
    }
}

// 4096 rows of 4096 as above: 46.8 us with the sums behind it, 4.3 TB/s; 413 warp instructions a warp and 256 columns at 2.06 a clock and SM from 16 warps, whose registers (128) the
// sums over tokens take.
// factors: w_next, gate * w_block * scales (or without a gate that has rows), c_block * scales for the gradient of such a gate.  Sums over a team's tokens: dw_next, A, then (BIAS) dc_next, B.
template <bool SF32, bool BF32, int E, bool BIAS, bool WHOLE, bool GATES>
__global__ void __launch_bounds__(join_cta(BIAS), BIAS ? 1 : 2) k_join_backward(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t s_dyn[];
    constexpr int SZ = SF32 ? 4 : 2, BZ = BF32 ? 4 : 2, SUMS = BIAS ? 4 : 2;
    constexpr int S8 = eight_room<SF32, WHOLE>(), B8 = eight_room<BF32, WHOLE>(), H8 = eight_room<false, WHOLE>();
    constexpr int AT_DOUT = E * H8, AT_OUT = AT_DOUT + E * S8, AT_B = AT_OUT + E * S8, AT_G = AT_B + E * B8;
    JoinTeam<(E == 2 || BIAS)> tm(a, reinterpret_cast<float *>(s_dyn + join_warp_bytes(E, a.room, a.params, WHOLE) * (blockDim.x >> 5)), 256 * E);
    const JoinWarp<E, WHOLE> me(a, s_dyn, tm);
    const int n = a.n;
    pdl_wait();
    pdl_trigger();
    const uint32_t tokens = a.tokens, walk = (uint32_t)tm.step(), first = (uint32_t)tm.first();
    const bool block = WHOLE || a.parts || a.db.p || a.dgate.p;
    const uint8_t *my_dh = me.template mine<false>(a.dh), *my_dout = me.template mine<SF32>(a.dout), *my_out = me.template mine<SF32>(a.out), *my_b = me.template mine<BF32>(a.b);
    uint8_t *my_dr = me.template mine<SF32>(a.dr), *my_db = a.db.f32 ? me.template mine<true>(a.db) : me.template mine<false>(a.db);
    auto ahead = [&](uint32_t t, uint8_t *to) {
        if (t < tokens)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (WHOLE) {
                    row_ahead<false>(my_dh + e * 512, a.dh.step, t, me.w[e], to + e * H8);
                    row_ahead<SF32>(my_dout + e * 256 * SZ, a.dout.step, t, me.w[e], to + AT_DOUT + e * S8);
                    row_ahead<SF32>(my_out + e * 256 * SZ, a.out.step, t, me.w[e], to + AT_OUT + e * S8);
                    if (a.b.p) row_ahead<BF32>(my_b + e * 256 * BZ, a.b.step, t, me.w[e], to + AT_B + e * B8);
                } else {
                    if (a.dh.p) row_ahead<false>(a.dh, t, me.w[e], n, to + e * H8);
                    if (a.dout.p) row_ahead<SF32>(a.dout, t, me.w[e], n, to + AT_DOUT + e * S8);
                    if (a.out.p) row_ahead<SF32>(a.out, t, me.w[e], n, to + AT_OUT + e * S8);
                    if (a.b.p) row_ahead<BF32>(a.b, t, me.w[e], n, to + AT_B + e * B8);
                }
                if (GATES) {
                    if (a.params_f32) row_ahead<true>(a.gate, t, me.w[e], n, to + AT_G + e * eight_room<true, false>());
                    else row_ahead<false>(a.gate, t, me.w[e], n, to + AT_G + e * eight_room<false, false>());
                }
            }
        close_ahead();
    };
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i) ahead(first + i * walk, me.rows + i * me.room);
    const Numbers num = numbers_of(a.drop);
    const float scale = a.drop.random ? a.scale * a.drop.scale : a.scale;
    Columns cols[E];
    f32x2 sum[SUMS][E][4];
    const void *given[GATES ? 4 : 3] = {a.w_block, a.w_next, a.gate_vec};
    if constexpr (GATES) given[3] = a.c_block;
    Eight q[E][GATES ? 4 : 3];
    vectors_here(given, a.params_f32, me.w, n, q);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int col = me.w[e].mine();
        cols[e] = columns_of(num, (uint32_t)col >> 3);
        columns_here(me.factor(e, a.params, 0), col, n, a.params_f32, 1.f, q[e][1], a.w_next, q[e][1], nullptr);
        columns_here(me.factor(e, a.params, 2), col, n, a.params_f32, scale, q[e][0], a.w_block, q[e][2], a.gate_vec);
        if constexpr (GATES)
            if (a.dgate.p) columns_here(me.factor(e, a.params, 4), col, n, a.params_f32, a.c_block ? scale : 0.f, q[e][3], a.c_block, q[e][3], nullptr);
#pragma unroll
        for (int k = 0; k < SUMS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[k][e][j] = 0;
    }
    const float4 *stats = reinterpret_cast<const float4 *>(a.stats);
    float4 st_next = stats && first < tokens ? stats[first] : make_float4(0.f, 1.f, 0.f, 1.f);
    uint8_t *at = me.rows;
    for (uint32_t t = first; t < tokens; t += walk) {
        const float4 st = st_next;
        if (stats && t + walk < tokens) st_next = stats[t + walk];
        wait_ahead<JOIN_AHEAD - 1>();
        if (!WHOLE) __syncwarp();
        f32x2 g[E][4], u[E][4], w[4];
        // g: normalised out, u: dh * w_next
        const f32x2 inv_out = both(st.w), shift_out = both(-st.z * st.w);
        f32x2 p0 = 0, p1 = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            row_here<false, WHOLE>(a.dh, t, me.w[e], at + e * H8, u[e]);
            row_here<SF32, WHOLE>(a.out, t, me.w[e], at + AT_OUT + e * S8, g[e]);
            factors_here(me.factor(e, a.params, 0), w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[e][j] = fma1(g[e][j], inv_out, shift_out);
                sum[0][e][j] = fma1(u[e][j], g[e][j], sum[0][e][j]);
                if (BIAS) sum[2][e][j] = add1(u[e][j], sum[2][e][j]);
                u[e][j] = mul1(u[e][j], w[j]);
                p0 = fma1(u[e][j], g[e][j], p0);
            }
            if (a.norm_next == DBSPMSPV_NORM_LAYER)
#pragma unroll
                for (int j = 0; j < 4; ++j) p1 = add1(u[e][j], p1);
        }
        f32x2 slope = both(1.f), along = 0, mean = 0;
        if (a.norm_next != DBSPMSPV_NORM_NONE && (WHOLE || a.dh.p)) {
            const float2 s = slope_sums(tm, a.norm_next, p0, p1);
            slope = inv_out;
            along = both(-st.w * (s.x * a.inv_n));
            mean = both(-st.w * (s.y * a.inv_n));
        }
        // g: G, then drop(G), then that times gate, w and scales;  u: the normalised b
        const f32x2 inv_b = both(st.y), shift_b = both(-st.x * st.y);
        p0 = p1 = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            row_here<SF32, WHOLE>(a.dout, t, me.w[e], at + AT_DOUT + e * S8, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) g[e][j] = add1(w[j], fma1(u[e][j], slope, fma1(g[e][j], along, mean)));
            if (WHOLE) {
                if (me.w[e].cnt) row_out<SF32>(my_dr + e * 256 * SZ, a.dr.step, t, g[e]);
            } else if (a.dr.p) row_out<SF32>(a.dr, t, me.w[e], n, g[e], me.spare);
        }
        if (block && a.drop.random) drop_eights<E, true>(a.drop, num, cols, t, g);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (!block) continue;
            row_here<BF32, WHOLE>(a.b, t, me.w[e], at + AT_B + e * B8, u[e]);
#pragma unroll
            for (int j = 0; j < 4; ++j) u[e][j] = fma1(u[e][j], inv_b, shift_b);
            if (GATES) {
                if (GATES && a.dgate.p) {
                    f32x2 d[4];
                    factors_here(me.factor(e, a.params, 2), w);
                    factors_here(me.factor(e, a.params, 4), d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = mul1(g[e][j], fma1(u[e][j], w[j], d[j]));
                    if (a.params_f32) row_out<true>(a.dgate, t, me.w[e], n, d, me.spare);
                    else row_out<false>(a.dgate, t, me.w[e], n, d, me.spare);
                }
                if (a.params_f32) row_here<true, false>(a.gate, t, me.w[e], at + AT_G + e * eight_room<true, false>(), w);
                else row_here<false, false>(a.gate, t, me.w[e], at + AT_G + e * eight_room<false, false>(), w);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[e][j] = mul1(g[e][j], w[j]);
            }
            factors_here(me.factor(e, a.params, 2), w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum[1][e][j] = fma1(g[e][j], u[e][j], sum[1][e][j]);
                if (BIAS) sum[3][e][j] = add1(g[e][j], sum[3][e][j]);
                g[e][j] = mul1(g[e][j], w[j]);
                p0 = fma1(g[e][j], u[e][j], p0);
            }
            if (a.norm_block == DBSPMSPV_NORM_LAYER)
#pragma unroll
                for (int j = 0; j < 4; ++j) p1 = add1(g[e][j], p1);
        }
        if (!WHOLE) __syncwarp();
        ahead(t + JOIN_AHEAD * walk, at);
        at = at == me.rows ? me.rows + me.room : me.rows;
        if (!WHOLE && !a.db.p) continue;
        slope = both(1.f);
        along = mean = 0;
        if (a.norm_block != DBSPMSPV_NORM_NONE) {
            const float2 s = slope_sums(tm, a.norm_block, p0, p1);
            slope = inv_b;
            along = both(-st.y * (s.x * a.inv_n));
            mean = both(-st.y * (s.y * a.inv_n));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
            for (int j = 0; j < 4; ++j) g[e][j] = fma1(g[e][j], slope, fma1(u[e][j], along, mean));
            if (WHOLE) {
                if (me.w[e].cnt == 0) continue;
                if (a.db.f32) row_out<true>(my_db + e * 1024, a.db.step, t, g[e]);
                else row_out<false>(my_db + e * 512, a.db.step, t, g[e]);
            } else if (a.db.f32) row_out<true>(a.db, t, me.w[e], n, g[e], me.spare);
            else row_out<false>(a.db, t, me.w[e], n, g[e], me.spare);
        }
    }
    if (a.parts)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (me.w[e].cnt)
#pragma unroll
                for (int k = 0; k < SUMS; ++k) store_eight<true>(a.parts + (first * (int64_t)SUMS + k) * a.ldp, me.w[e].mine(), (int)a.ldp, true, sum[k][e]);
}

// The teams' sums added up, and what follows from them: COLS columns a thread block, four a lane, teams side by side.  32 columns are whole lines of the parts, 8 are sectors; these for rows of
// fewer than 2048 columns, which make few thread blocks (with the gradient in front of it, 4000 rows of 1000: 21.7 -> 20.8 us, but 4096 of 4096: 46.9 -> 50.2).
struct JoinSums {
    const float *parts;
    int64_t ldp;
    int32_t teams, n, params_f32;
    float scale;
    const void *w_block, *c_block, *gate_vec;
    float *dw_block, *dc_block, *dgate, *dw_next, *dc_next;
};
template <bool BIAS, int COLS>
__global__ void __launch_bounds__(JOIN_SUMS_CTA) k_join_sums(const __grid_constant__ JoinSums a) {
    constexpr int SUMS = BIAS ? 4 : 2, X = COLS / 4, Y = JOIN_SUMS_CTA / X, WARPS = JOIN_SUMS_CTA / 32;
    __shared__ float4 s_warp[WARPS][SUMS][X];
    __shared__ float s_sum[SUMS][COLS];
    const int tid = threadIdx.x, x = tid % X, y = tid / X;
    const int64_t at = (int64_t)blockIdx.x * COLS + 4 * x;
    pdl_wait();
    pdl_trigger();
    float4 v[SUMS];
#pragma unroll
    for (int k = 0; k < SUMS; ++k) v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < a.ldp)                           // (rows of the parts are whole eights)
#pragma unroll 5
        for (int i = y; i < a.teams; i += Y)
#pragma unroll
            for (int k = 0; k < SUMS; ++k) {
                const float4 p = *reinterpret_cast<const float4 *>(a.parts + ((int64_t)i * SUMS + k) * a.ldp + at);
                v[k].x += p.x; v[k].y += p.y; v[k].z += p.z; v[k].w += p.w;
            }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) {
#pragma unroll
        for (int o = X; o < 32; o <<= 1) {
            v[k].x += __shfl_xor_sync(FULL, v[k].x, o);
            v[k].y += __shfl_xor_sync(FULL, v[k].y, o);
            v[k].z += __shfl_xor_sync(FULL, v[k].z, o);
            v[k].w += __shfl_xor_sync(FULL, v[k].w, o);
        }
        if (tid % 32 < X) s_warp[tid / 32][k][x] = v[k];
    }
    __syncthreads();
    if (tid < SUMS * COLS) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) t += reinterpret_cast<const float *>(s_warp[i])[tid];
        (&s_sum[0][0])[tid] = t;
    }
    __syncthreads();
    const int col = blockIdx.x * COLS + tid;
    if (tid >= COLS || col >= a.n) return;
    float s[SUMS];
#pragma unroll
    for (int k = 0; k < SUMS; ++k) s[k] = s_sum[k][tid];
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
