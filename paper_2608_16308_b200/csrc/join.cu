// The join of a block with the residual stream: entry points, and how rows are shared out (kernels: join.cuh).  No handle: the current device, and nothing that lasts longer than a call.
#include <math.h>

#include <type_traits>

#include "internal.cuh"
#include "join.cuh"
#include "rows.cuh"

namespace dbs {

// ---- joins -----------------------------------------------------------------------------------
// Threads that an SM holds of the joins' kernels, by their registers (forwards; backwards)
static int join_threads(int eights, bool backward) { return backward ? 512 : eights == 2 ? 768 : 1024; }
static int eight_bytes(bool f32, bool whole) { return f32 ? (whole ? eight_room<true, true>() : eight_room<true, false>()) : (whole ? eight_room<false, true>() : eight_room<false, false>()); }
static JoinPlan join_plan(int sms, int64_t tokens, int64_t n, int eights, int room, int params, bool whole, bool backward) {
    JoinPlan p;
    const int warps = (int)ceil64(n, (int64_t)256 * eights), most = JOIN_COLS / 256 / eights;
    p.eights = eights;
    p.cluster = (int)ceil64(warps, most);
    p.warps = (int)ceil64(warps, p.cluster);
    p.teams = 1;
    // several short rows to a thread block, once there is a block for every SM
    while (p.cluster == 1 && 2 * p.teams * p.warps <= 8 && tokens >= (int64_t)2 * p.teams * sms) p.teams *= 2;
    const int by_registers = join_threads(eights, backward) / (p.warps * p.teams * 32), by_memory = (int)((227 * 1024) / (join_smem(p, room, params, whole) + 1024));
    int per_sm = by_registers < by_memory ? by_registers : by_memory;
    per_sm = per_sm < 1 ? 1 : per_sm > 24 ? 24 : per_sm;
    const int64_t want = ceil64(tokens, p.teams), blocks = (int64_t)sms * per_sm / p.cluster;
    p.clusters = (int)(want < blocks ? want : blocks < 1 ? 1 : blocks);
    return p;
}
// Two eights a lane share what a sum over the row costs; rows of up to 1024 columns have too few for that
static int join_eights(int64_t n, bool sums_of_biases) { return n > 1024 && !sums_of_biases ? 2 : 1; }
// whether every row is whole eights on 16 bytes (and its place one product of 32 bits)
template <typename... R> static bool all_whole(int64_t n, const R &...r) { return n % 8 == 0 && ((r.p && r.aligned && r.ld * (r.f32 ? 4 : 2) <= (int64_t)UINT32_MAX) && ...); }
static bool norm_ok(int norm) { return norm >= DBSPMSPV_NORM_NONE && norm <= DBSPMSPV_NORM_LAYER; }
static bool opts_ok(const dbspmspv_join_opts *o) {
    return o && norm_ok(o->norm_block) && norm_ok(o->norm_next) && o->eps_block >= 0.f && o->eps_next >= 0.f && isfinite(o->eps_block) && isfinite(o->eps_next) && isfinite(o->scale) &&
           o->drop >= 0.f && o->drop <= 1.f;
}
static JoinArgs join_args(const dbspmspv_join_opts &o, int32_t tokens, int64_t n, const JoinPlan &p, int room, int params) {
    JoinArgs a = {};
    a.params_f32 = o.params_f32 != 0;
    a.scale = o.scale; a.eps_block = o.eps_block; a.eps_next = o.eps_next; a.inv_n = (float)(1.0 / (double)n);
    a.norm_block = o.norm_block; a.norm_next = o.norm_next;
    a.tokens = tokens; a.n = (int32_t)n; a.warps = p.warps; a.teams = p.teams; a.room = room; a.params = params;
    return a;
}
// Room for the sums of any gradient call of this size: the most teams that any of them has (those with the least shared memory, bf16 throughout)
static int64_t join_room(int sms, int64_t tokens, int64_t n) {
    int64_t most = 0;
    for (int eights = 1; eights <= 2; ++eights) {
        const JoinPlan p = join_plan(sms, tokens, n, eights, eights * 4 * eight_bytes(false, true), 4, true, true);
        const int64_t teams = (int64_t)p.clusters * p.teams;
        if (teams > most) most = teams;
    }
    return most * 4 * ceil64(n, 8) * 8 * 4;
}
// A kernel for the options that are known when it is compiled
template <typename F> static auto by_types(const dbspmspv_join_opts *o, bool whole, F f) {
    using T = std::true_type;
    using N = std::false_type;
    if (whole) return o->stream_f32 ? (o->block_f32 ? f(T{}, T{}, T{}) : f(T{}, N{}, T{})) : (o->block_f32 ? f(N{}, T{}, T{}) : f(N{}, N{}, T{}));
    return o->stream_f32 ? (o->block_f32 ? f(T{}, T{}, N{}) : f(T{}, N{}, N{})) : (o->block_f32 ? f(N{}, T{}, N{}) : f(N{}, N{}, N{}));
}

}  // namespace dbs

extern "C" {

void dbspmspv_default_join_opts(dbspmspv_join_opts *o) {
    if (!o) return;
    *o = dbspmspv_join_opts{};
    o->norm_block = DBSPMSPV_NORM_NONE;
    o->norm_next = DBSPMSPV_NORM_RMS;
    o->eps_block = o->eps_next = 1e-5f;
    o->scale = 1.f;
}

int dbspmspv_join(const dbspmspv_join_opts *o, int32_t tokens, int64_t n, const void *r, int64_t ldr, const void *b, int64_t ldb, const void *w_block, const void *c_block, const void *gate,
                  int64_t ldg, const void *w_next, const void *c_next, const uint64_t *random, void *out, int64_t ldo, void *h, int64_t ldh, float *stats, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (!opts_ok(o) || tokens < 0 || n < 1) return DBSPMSPV_ERR_INVALID_ARG;
    if (n > JOIN_MAX_N) return DBSPMSPV_ERR_UNSUPPORTED;
    if (tokens > 0 && ((!r && !b) || (!out && !h) || (b && o->drop > 0.f && !random))) return DBSPMSPV_ERR_INVALID_ARG;
    if ((o->norm_block == DBSPMSPV_NORM_NONE && (w_block || c_block)) || (o->norm_next == DBSPMSPV_NORM_NONE && (w_next || c_next))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!rows_ok(r, ldr, n) || !rows_ok(b, ldb, n) || !rows_ok(out, ldo, n) || !rows_ok(h, ldh, n) || (gate && ldg != 0 && ldg < n)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(o->stream_f32 ? 4 : 2, r, out) || !on_bytes(o->block_f32 ? 4 : 2, b) || !on_bytes(o->params_f32 ? 4 : 2, w_block, c_block, gate, w_next, c_next) || !on_bytes(2, h) ||
        !on_bytes(16, stats) || !on_bytes(8, random))
        return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    if (!on_current_device(r ? r : b, dev) || !on_current_device(out ? out : h, dev)) return DBSPMSPV_ERR_INVALID_ARG;
    const bool bias = (b && c_block) || c_next, rows = b && gate && ldg;
    const Rows R = rows_of(r, ldr, o->stream_f32), BR = rows_of(b, ldb, o->block_f32), OUT = rows_of(out, ldo, o->stream_f32), H = rows_of(h, ldh, false), G = rows_of(rows ? gate : nullptr, ldg, o->params_f32);
    const bool whole = all_whole(n, R, BR, OUT, H) && (!rows || G.aligned);
    const int params = bias ? 8 : 4, eights = join_eights(n, false);
    const int room = eights * (eight_bytes(o->stream_f32, whole) + eight_bytes(o->block_f32, whole) + (rows ? eight_bytes(o->params_f32, false) : 0));
    const JoinPlan p = join_plan(sms, tokens, n, eights, room, params, whole, false);
    JoinArgs a = join_args(*o, tokens, n, p, room, params);
    a.r = R; a.b = BR; a.out = OUT; a.h = H;
    if (b) {
        a.gate = G;
        a.gate_vec = rows ? nullptr : gate;
        a.w_block = w_block; a.c_block = c_block;
        a.drop = drop_of(o->drop, random);
    }
    a.w_next = w_next; a.c_next = c_next; a.stats = stats;
    if (!b) a.norm_block = DBSPMSPV_NORM_NONE;
    auto kernel = by_types(o, whole, [&](auto S, auto BL, auto W) {
        constexpr bool s = decltype(S)::value, l = decltype(BL)::value, w = decltype(W)::value;
        return eights == 2 ? (bias ? k_join<s, l, 2, true, w> : k_join<s, l, 2, false, w>) : (bias ? k_join<s, l, 1, true, w> : k_join<s, l, 1, false, w>);
    });
    return launch_rows(kernel, p.clusters * p.cluster, p.warps * p.teams * 32, p.cluster, join_smem(p, room, params, whole), static_cast<cudaStream_t>(stream), a);
}

int dbspmspv_join_workspace(const dbspmspv_join_opts *o, int32_t tokens, int64_t n, int64_t *bytes) {
    using namespace dbs;
    if (!opts_ok(o) || tokens < 0 || n < 1 || !bytes) return DBSPMSPV_ERR_INVALID_ARG;
    if (n > JOIN_MAX_N) return DBSPMSPV_ERR_UNSUPPORTED;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    *bytes = tokens ? join_room(sms, tokens, n) : 0;
    return DBSPMSPV_OK;
}

int dbspmspv_join_backward(const dbspmspv_join_opts *o, int32_t tokens, int64_t n, const void *out, int64_t ldo, const void *b, int64_t ldb, const float *stats, const void *w_block,
                           const void *c_block, const void *gate, int64_t ldg, const void *w_next, const uint64_t *random, const void *dh, int64_t lddh, const void *dout, int64_t lddo, void *dr,
                           int64_t lddr, void *db, int64_t lddb, float *dw_block, float *dc_block, void *dgate, int64_t lddg, float *dw_next, float *dc_next, void *workspace,
                           int64_t workspace_bytes, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (!opts_ok(o) || tokens < 0 || n < 1 || workspace_bytes < 0) return DBSPMSPV_ERR_INVALID_ARG;
    if (n > JOIN_MAX_N) return DBSPMSPV_ERR_UNSUPPORTED;
    const bool nb = o->norm_block != DBSPMSPV_NORM_NONE, nn = o->norm_next != DBSPMSPV_NORM_NONE, rows = gate && ldg;
    if ((!nb && (w_block || c_block || dw_block || dc_block)) || (!nn && (w_next || dw_next || dc_next)) || (dgate && !gate)) return DBSPMSPV_ERR_INVALID_ARG;
    const bool block = db || dw_block || dc_block || dgate, sums = dw_block || dc_block || dw_next || dc_next || (dgate && !rows);
    if (tokens > 0) {
        if ((!dh && !dout) || (nn && dh && !out) || (block && (nb || dgate) && !b) || ((nb || nn) && !stats) || (block && o->drop > 0.f && !random)) return DBSPMSPV_ERR_INVALID_ARG;
        if (!dr && !block && !sums) return DBSPMSPV_ERR_INVALID_ARG;
    }
    if (!rows_ok(out, ldo, n) || !rows_ok(b, ldb, n) || (rows && ldg < n) || !rows_ok(dh, lddh, n) || !rows_ok(dout, lddo, n) || !rows_ok(dr, lddr, n) || !rows_ok(db, lddb, n) ||
        (dgate && rows && lddg < n))
        return DBSPMSPV_ERR_INVALID_ARG;
    const int pt = o->params_f32 ? 4 : 2;
    if (!on_bytes(o->stream_f32 ? 4 : 2, out, dout, dr) || !on_bytes(o->block_f32 ? 4 : 2, b) || !on_bytes(pt, w_block, c_block, gate, w_next) || !on_bytes(2, dh) ||
        !on_bytes(o->dblock_f32 ? 4 : 2, db) || !on_bytes(4, dw_block, dc_block, dw_next, dc_next) || !on_bytes(rows ? pt : 4, dgate) || !on_bytes(16, stats, workspace) || !on_bytes(8, random))
        return DBSPMSPV_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens == 0) {
        for (float *v : {dw_block, dc_block, dw_next, dc_next, rows ? nullptr : static_cast<float *>(dgate)})
            if (v) DBS_CUDA(cudaMemsetAsync(v, 0, (size_t)n * 4, st));
        return DBSPMSPV_OK;
    }
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    if (!on_current_device(dh ? dh : dout, dev) || (dr && !on_current_device(dr, dev))) return DBSPMSPV_ERR_INVALID_ARG;
    if (sums && (!workspace || workspace_bytes < join_room(sms, tokens, n))) return DBSPMSPV_ERR_INVALID_ARG;
    const bool bias = dc_block || dc_next || (dgate && !rows && c_block), gates = rows && block;
    const Rows DH = rows_of(dh, lddh, false), DOUT = rows_of(dout, lddo, o->stream_f32), DR = rows_of(dr, lddr, o->stream_f32), OUT = rows_of(nn && dh ? out : nullptr, ldo, o->stream_f32);
    const Rows BR = rows_of(block && (nb || dgate) ? b : nullptr, ldb, o->block_f32), DB = rows_of(db, lddb, o->dblock_f32);
    const Rows G = rows_of(gates ? gate : nullptr, ldg, o->params_f32), DG = rows_of(gates ? dgate : nullptr, lddg, o->params_f32);
    const bool whole = all_whole(n, DH, DOUT, DR, OUT, BR, DB) && (!gates || (G.aligned && DG.aligned));
    const int params = gates && dgate ? 6 : 4, eights = join_eights(n, bias);
    const int room = eights * (eight_bytes(false, whole) + 2 * eight_bytes(o->stream_f32, whole) + eight_bytes(o->block_f32, whole) + (gates ? eight_bytes(o->params_f32, false) : 0));
    const JoinPlan p = join_plan(sms, tokens, n, eights, room, params, whole, true);
    JoinArgs a = join_args(*o, tokens, n, p, room, params);
    a.dh = DH; a.dout = DOUT; a.dr = DR; a.out = OUT; a.b = BR; a.db = DB; a.gate = G; a.dgate = DG;
    if (block) {
        a.gate_vec = rows ? nullptr : gate;
        a.w_block = w_block; a.c_block = c_block;
        a.drop = drop_of(o->drop, random);
    }
    a.w_next = w_next; a.stats = const_cast<float *>(stats);
    a.parts = sums ? static_cast<float *>(workspace) : nullptr;
    a.ldp = ceil64(n, 8) * 8;
    auto kernel = by_types(o, whole, [&](auto S, auto BL, auto W) {
        constexpr bool s = decltype(S)::value, l = decltype(BL)::value, w = decltype(W)::value;
        return bias ? k_join_backward<s, l, 1, true, w> : eights == 2 ? k_join_backward<s, l, 2, false, w> : k_join_backward<s, l, 1, false, w>;
    });
    s = launch_rows(kernel, p.clusters * p.cluster, p.warps * p.teams * 32, p.cluster, join_smem(p, room, params, whole), st, a);
    if (s != DBSPMSPV_OK || !sums) return s;
    JoinSums j = {a.parts, a.ldp, p.clusters * p.teams, (int32_t)n, a.params_f32, a.drop.random ? o->scale * a.drop.scale : o->scale, w_block, c_block, rows ? nullptr : gate,
                  dw_block, dc_block, rows ? nullptr : static_cast<float *>(dgate), dw_next, dc_next};
    return launch_rows(bias ? k_join_sums<true> : k_join_sums<false>, (int)ceil64(n, JOIN_SUMS_COLS), JOIN_SUMS_CTA, 1, 0, st, j);
}

}  // extern "C"
