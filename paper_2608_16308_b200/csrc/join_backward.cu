// The join of a block with the residual stream, gradient: entry points (kernels: join.cuh; how rows are shared out: join_plan.cuh).  No handle: the current device, and nothing that lasts longer than a call.
#include "join_plan.cuh"

extern "C" {

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
    if (sums && (!workspace || workspace_bytes < join_room(sms, tokens, n))) return DBSPMSPV_ERR_INVALID_ARG;
    const bool bias = dc_block || dc_next || (dgate && !rows && c_block), gates = rows && block;
    const Rows DH = rows_of(dh, lddh, false), DOUT = rows_of(dout, lddo, o->stream_f32), DR = rows_of(dr, lddr, o->stream_f32), OUT = rows_of(nn && dh ? out : nullptr, ldo, o->stream_f32);
    const Rows BR = rows_of(block && (nb || dgate) ? b : nullptr, ldb, o->block_f32), DB = rows_of(db, lddb, o->dblock_f32);
    const Rows G = rows_of(gates ? gate : nullptr, ldg, o->params_f32), DG = rows_of(gates ? dgate : nullptr, lddg, o->params_f32);
    const void *kept = first_of(OUT.p, BR.p, stats);
    if ((kept && !on_current_device(kept, dev)) || !on_current_device(first_of(dh, dout), dev) || !on_current_device(first_of(dr, db, dw_block, dc_block, dgate, dw_next, dc_next), dev))
        return DBSPMSPV_ERR_INVALID_ARG;
    const bool whole = dh && dout && dr && db && nn && all_whole(n, DH, DOUT, DR, OUT, BR, DB) && (!gates || (G.aligned && DG.aligned));
    const int params = gates && dgate ? 6 : 4, eights = join_eights(sms, tokens, n, bias);
    const int room = eights * (eight_bytes(false, whole) + 2 * eight_bytes(o->stream_f32, whole) + eight_bytes(o->block_f32, whole) + (gates ? eight_bytes(o->params_f32, false) : 0));
    JoinPlan p = join_plan(sms, tokens, n, eights, room, params, whole, true, bias);
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
    auto kernel = by_types(o, [&](auto S, auto BL) {
        constexpr bool s = decltype(S)::value, l = decltype(BL)::value;
        auto form = [&](auto W, auto GA) {
            constexpr bool w = decltype(W)::value, g = decltype(GA)::value;
            return bias ? k_join_backward<s, l, 1, true, w, g> : eights == 2 ? k_join_backward<s, l, 2, false, w, g> : k_join_backward<s, l, 1, false, w, g>;
        };
        using T = std::true_type;
        using N = std::false_type;
        return whole ? (gates ? form(T{}, T{}) : form(T{}, N{})) : (gates ? form(N{}, T{}) : form(N{}, N{}));
    });
    if ((s = fit_clusters(reinterpret_cast<const void *>(kernel), dev, p, join_smem(p, room, params, whole))) != DBSPMSPV_OK) return s;
    s = launch_rows(dev, kernel, p.clusters * p.cluster, p.warps * p.teams * 32, p.cluster, join_smem(p, room, params, whole), st, a);
    if (s != DBSPMSPV_OK || !sums) return s;
    JoinSums j = {a.parts, a.ldp, p.clusters * p.teams, (int32_t)n, a.params_f32, a.drop.random ? o->scale * a.drop.scale : o->scale, w_block, c_block, rows ? nullptr : gate,
                  dw_block, dc_block, rows ? nullptr : static_cast<float *>(dgate), dw_next, dc_next};
    const int cols = n < 2048 ? 8 : 32;
    auto add_up = cols == 32 ? (bias ? k_join_sums<true, 32> : k_join_sums<false, 32>) : (bias ? k_join_sums<true, 8> : k_join_sums<false, 8>);
    return launch_rows(dev, add_up, (int)ceil64(n, cols), JOIN_SUMS_CTA, 1, 0, st, j);
}

}  // extern "C"
