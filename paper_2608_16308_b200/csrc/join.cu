// The join of a block with the residual stream: entry points (kernels: join.cuh; how rows are shared out: join_plan.cuh).  No handle: the current device, and nothing that lasts longer than a call.
#include "join_plan.cuh"

namespace dbs {

// Two blocks of a cluster exchange numbers a few times; one of them may keep silent.  Counts the exchanges that gave up, and 100 for one that went wrong.
static __global__ void __launch_bounds__(32) k_join_wait(const __grid_constant__ JoinArgs a, int tries, int silent, int32_t *gave_up) {
    extern __shared__ __align__(16) uint8_t s_dyn[];
    pdl_wait();
    JoinTeam<true> tm(a, reinterpret_cast<float *>(s_dyn), 256);
    if (tm.rank == silent) tm.give_up();
    int n = 0;
    for (int i = 0; i < 4; ++i) {
        const float *s, v[2] = {(float)(tm.rank + 1), (float)i};
        if (!tm.exchange(v, s, tries)) ++n;
        else if (s[0] != 1.f || s[1] != 2.f || s[tm.room] != i || s[tm.room + 1] != i) n += 100;
        __syncwarp();
    }
    if (tm.lane == 0) gave_up[tm.rank] = n;
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
    if (!on_current_device(first_of(r, b), dev) || !on_current_device(first_of(out, h), dev)) return DBSPMSPV_ERR_INVALID_ARG;
    const bool bias = (b && c_block) || c_next, rows = b && gate && ldg;
    const Rows R = rows_of(r, ldr, o->stream_f32), BR = rows_of(b, ldb, o->block_f32), OUT = rows_of(out, ldo, o->stream_f32), H = rows_of(h, ldh, false), G = rows_of(rows ? gate : nullptr, ldg, o->params_f32);
    const bool all = r && b && out && h, whole = all_whole(n, R, BR, OUT, H) && (!rows || (all && G.aligned));
    const int params = bias ? 8 : 4, eights = join_eights(sms, tokens, n, false);
    const int room = eights * (eight_bytes(o->stream_f32, whole) + eight_bytes(o->block_f32, whole) + (rows ? eight_bytes(o->params_f32, false) : 0));
    JoinPlan p = join_plan(sms, tokens, n, eights, room, params, whole, false, bias);
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
    auto kernel = by_types(o, [&](auto S, auto BL) {
        constexpr bool s = decltype(S)::value, l = decltype(BL)::value;
        auto form = [&](auto F, auto GA) {
            constexpr int f = decltype(F)::value;
            constexpr bool g = decltype(GA)::value;
            return eights == 2 ? (bias ? k_join<s, l, 2, true, f, g> : k_join<s, l, 2, false, f, g>) : (bias ? k_join<s, l, 1, true, f, g> : k_join<s, l, 1, false, f, g>);
        };
        using Any = std::integral_constant<int, JOIN_ANY>;
        using Whole = std::integral_constant<int, JOIN_WHOLE>;
        using All = std::integral_constant<int, JOIN_ALL>;
        if (!whole) return rows ? form(Any{}, std::true_type{}) : form(Any{}, std::false_type{});
        if (!all) return form(Whole{}, std::false_type{});
        return rows ? form(All{}, std::true_type{}) : form(All{}, std::false_type{});
    });
    if ((s = fit_clusters(reinterpret_cast<const void *>(kernel), dev, p, join_smem(p, room, params, whole))) != DBSPMSPV_OK) return s;
    return launch_rows(dev, kernel, p.clusters * p.cluster, p.warps * p.teams * 32, p.cluster, join_smem(p, room, params, whole), static_cast<cudaStream_t>(stream), a);
}

int dbspmspv_test_cluster_wait(int32_t max_tries, int32_t silent, int32_t *gave_up, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (max_tries < 1 || max_tries > 4096 || silent < -1 || silent > 1 || !gave_up || !on_bytes(4, gave_up)) return DBSPMSPV_ERR_INVALID_ARG;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    if (!on_current_device(gave_up, dev)) return DBSPMSPV_ERR_INVALID_ARG;
    JoinArgs a = {};
    a.n = 512; a.warps = a.teams = 1;
    return launch_rows(dev, k_join_wait, 2, 32, 2, 4 * join_sums_room(1, 2) * 4 + 16, static_cast<cudaStream_t>(stream), a, max_tries, silent, gave_up);
}

}  // extern "C"
