// How the rows of a join are shared out to warps, thread blocks and clusters, and what its entry points have in common.
#pragma once

#include <math.h>

#include <type_traits>

#include "internal.cuh"
#include "join.cuh"
#include "rows.cuh"

namespace dbs {

// Threads that an SM holds of the joins' kernels, by their registers
inline int join_threads(int eights, bool backward) { return !backward ? (eights == 2 ? 768 : 1024) : 512; }
inline int eight_bytes(bool f32, bool whole) { return f32 ? (whole ? eight_room<true, true>() : eight_room<true, false>()) : (whole ? eight_room<false, true>() : eight_room<false, false>()); }
inline JoinPlan join_plan(int sms, int64_t tokens, int64_t n, int eights, int room, int params, bool whole, bool backward, bool biases) {
    JoinPlan p;
    const int warps = (int)ceil64(n, (int64_t)256 * eights), most = join_cta(backward && biases) / 32;
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
// no more clusters than run at once: the others' rows would wait for the first to be through with all of theirs (1500 rows of 11008, clusters of three: 53.2 -> 47.6 us)
inline int fit_clusters(const void *kernel, int dev, JoinPlan &p, size_t smem) {
    if (p.cluster == 1) return DBSPMSPV_OK;
    int most;
    const int s = clusters_at_once(kernel, dev, p.warps * p.teams * 32, p.cluster, smem, &most);
    if (s == DBSPMSPV_OK && p.clusters > most) p.clusters = most;
    return s;
}
// Two eights a lane share what a sum over the row costs: from 1024 columns on where no more than a quarter of the lanes has none and there are more rows than SMs hold at once (333 rows of 1037: 8.3 us with two,
// 7.5 with one; 4000 rows of 1000, gradient: 24.5 and 21.7), and from 2048 on in any case.  Gradients with sums of biases have no registers for two.  (One without such sums: 2048 columns at most, which
// are a thread block's; its kernels know no clusters.)
inline int join_eights(int sms, int64_t tokens, int64_t n, bool sums_of_biases) {
    if (sums_of_biases || n <= 1024) return 1;
    return n > 2048 || (4 * n >= 3 * (ceil64(n, 512) * 512) && tokens > 2 * sms) ? 2 : 1;
}
// whether every row of what is there is whole eights on 16 bytes (and its place one product of 32 bits)
template <typename... R> inline bool all_whole(int64_t n, const R &...r) { return n % 8 == 0 && ((!r.p || (r.aligned && r.ld * (r.f32 ? 4 : 2) <= (int64_t)UINT32_MAX)) && ...); }
inline bool norm_ok(int norm) { return norm >= DBSPMSPV_NORM_NONE && norm <= DBSPMSPV_NORM_LAYER; }
inline bool opts_ok(const dbspmspv_join_opts *o) {
    return o && norm_ok(o->norm_block) && norm_ok(o->norm_next) && o->eps_block >= 0.f && o->eps_next >= 0.f && isfinite(o->eps_block) && isfinite(o->eps_next) && isfinite(o->scale) &&
           o->drop >= 0.f && o->drop <= 1.f;
}
inline JoinArgs join_args(const dbspmspv_join_opts &o, int32_t tokens, int64_t n, const JoinPlan &p, int room, int params) {
    JoinArgs a = {};
    a.params_f32 = o.params_f32 != 0;
    a.scale = o.scale; a.eps_block = o.eps_block; a.eps_next = o.eps_next; a.inv_n = (float)(1.0 / (double)n);
    a.norm_block = o.norm_block; a.norm_next = o.norm_next;
    a.tokens = tokens; a.n = (int32_t)n; a.warps = p.warps; a.teams = p.teams; a.room = room; a.params = params;
    return a;
}
// Room for the sums of any gradient call of this size: the most teams that any of them has (those with the least shared memory, bf16 throughout)
inline int64_t join_room(int sms, int64_t tokens, int64_t n) {
    int64_t most = 0;
    for (int form = 0; form < 3; ++form) {
        const bool biases = form == 2;
        const int eights = form == 1 ? 2 : 1;
        if (form == 0 && n > 2048) continue;
        const JoinPlan p = join_plan(sms, tokens, n, eights, eights * 4 * eight_bytes(false, true), 4, true, true, biases);
        const int64_t teams = (int64_t)p.clusters * p.teams;
        if (teams > most) most = teams;
    }
    return most * 4 * ceil64(n, 8) * 8 * 4;
}
// A kernel for the types that are known when it is compiled: f(stream in fp32, block in fp32)
template <typename F> inline auto by_types(const dbspmspv_join_opts *o, F f) {
    using T = std::true_type;
    using N = std::false_type;
    return o->stream_f32 ? (o->block_f32 ? f(T{}, T{}) : f(T{}, N{})) : (o->block_f32 ? f(N{}, T{}) : f(N{}, N{}));
}

}  // namespace dbs
