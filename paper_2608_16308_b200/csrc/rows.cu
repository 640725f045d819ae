// What stands between the layers of a network and behind the last one: the join of a block with the residual stream, dropout, log probabilities.
// Entry points; kernels: join.cuh, logprobs.cuh.  No handle: the current device, and nothing that lasts longer than a call.
#include <math.h>

#include <type_traits>

#include "internal.cuh"
#include "join.cuh"
#include "logprobs.cuh"
#include "rows.cuh"

namespace dbs {

// ---- dropout ---------------------------------------------------------------------------------
// A thread takes the same eight columns of DR_ROWS rows, whose loads do not wait for one another; thread blocks are as wide as the rows, if these are narrow.
constexpr int DR_CTA = 256, DR_ROWS = 4;
struct DropArgs {
    Rows x, y;
    Drop drop;
    int32_t tokens, n, wide, chunks;         // threads along the columns (a power of two), thread blocks along a row
};
template <bool F32>
__global__ void __launch_bounds__(DR_CTA) k_dropout(const __grid_constant__ DropArgs a) {
    const int tall = DR_CTA / a.wide, x = threadIdx.x & (a.wide - 1), y = threadIdx.x / a.wide;
    const int64_t eight = (int64_t)(blockIdx.x % a.chunks) * a.wide + x, t0 = (int64_t)(blockIdx.x / a.chunks) * tall * DR_ROWS + y;
    pdl_wait();
    pdl_trigger();
    if (eight * 8 >= a.n) return;
    const int col = (int)eight * 8;
    const bool whole = a.n - col >= 8;
    uint4 p[DR_ROWS], q[DR_ROWS];
#pragma unroll
    for (int r = 0; r < DR_ROWS; ++r)
        if (t0 + r * tall < a.tokens) load_raw<F32>(row_at<F32>(a.x, t0 + r * tall), col, a.n, whole && a.x.aligned, p[r], q[r]);
    const Numbers num = numbers_of(a.drop);
    const Columns cols = columns_of(num, (uint32_t)eight);
#pragma unroll
    for (int r = 0; r < DR_ROWS; ++r) {
        const int64_t t = t0 + r * tall;
        if (t >= a.tokens) break;
        void *to = const_cast<void *>(row_at<F32>(a.y, t));
        if (a.drop.random) {
            f32x2 v[4];
            if (F32) pairs_of_eight(p[r], q[r], v);
            else pairs_of_eight(p[r], v);
            drop_eight(a.drop, num, cols, (uint32_t)t, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = mul2(v[j], both(a.drop.scale));
            store_eight<F32>(to, col, a.n, whole && a.y.aligned, v);
        } else store_raw<F32>(to, col, a.n, whole && a.y.aligned, p[r], q[r]);
    }
}

static int64_t ceil64(int64_t a, int64_t b) { return (a + b - 1) / b; }
template <typename... P> static bool on_bytes(uintptr_t bytes, P... p) { return (((reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0) && ...); }
static bool rows_ok(const void *p, int64_t ld, int64_t width) { return !p || ld >= width; }

// Threads that an SM holds of the joins' kernels, by their registers
constexpr int JOIN_FORWARD_THREADS = 768, JOIN_BACKWARD_THREADS = 512;

// ---- joins -----------------------------------------------------------------------------------
static JoinPlan join_plan(int sms, int64_t tokens, int64_t n, int eights, int pieces, int params, int threads_per_sm) {
    JoinPlan p;
    const int warps = (int)ceil64(n, (int64_t)256 * eights), most = JOIN_COLS / 256 / eights;
    p.eights = eights;
    p.cluster = 1;
    while (p.cluster * most < warps) p.cluster *= 2;
    p.warps = (int)ceil64(warps, p.cluster);
    p.teams = 1;
    // several short rows to a thread block, once there is a block for every SM
    while (p.cluster == 1 && 2 * p.teams * p.warps <= 8 && tokens >= (int64_t)2 * p.teams * sms) p.teams *= 2;
    const int by_registers = threads_per_sm / (p.warps * p.teams * 32), by_memory = (int)((227 * 1024) / (join_smem(p, pieces, params) + 1024));
    int per_sm = by_registers < by_memory ? by_registers : by_memory;
    per_sm = per_sm < 1 ? 1 : per_sm > 24 ? 24 : per_sm;
    const int64_t want = ceil64(tokens, p.teams), room = (int64_t)sms * per_sm / p.cluster;
    p.clusters = (int)(want < room ? want : room < 1 ? 1 : room);
    return p;
}
// Two eights a thread share what a sum over the row costs; rows of up to 1024 columns have too few for that
static int join_eights(int64_t n, bool sums_of_biases) { return n > 1024 && !sums_of_biases ? 2 : 1; }
static bool norm_ok(int norm) { return norm >= DBSPMSPV_NORM_NONE && norm <= DBSPMSPV_NORM_LAYER; }
static bool opts_ok(const dbspmspv_join_opts *o) {
    return o && norm_ok(o->norm_block) && norm_ok(o->norm_next) && o->eps_block >= 0.f && o->eps_next >= 0.f && isfinite(o->eps_block) && isfinite(o->eps_next) && isfinite(o->scale) &&
           o->drop >= 0.f && o->drop <= 1.f;
}
static JoinArgs join_args(const dbspmspv_join_opts &o, int32_t tokens, int64_t n, const JoinPlan &p, int pieces, int params) {
    JoinArgs a = {};
    a.params_f32 = o.params_f32 != 0;
    a.scale = o.scale; a.eps_block = o.eps_block; a.eps_next = o.eps_next; a.inv_n = (float)(1.0 / (double)n);
    a.norm_block = o.norm_block; a.norm_next = o.norm_next;
    a.tokens = tokens; a.n = (int32_t)n; a.warps = p.warps; a.teams = p.teams; a.pieces = pieces; a.params = params;
    return a;
}
// Room for the sums of any gradient call of this size: a team per token at most, and never more than fit the GPU with the fewest pieces
static int64_t join_room(int sms, int64_t tokens, int64_t n) {
    int64_t most = 0;
    for (int eights = 1; eights <= 2; ++eights) {
        const JoinPlan p = join_plan(sms, tokens, n, eights, 1, 4, JOIN_BACKWARD_THREADS);
        const int64_t teams = (int64_t)p.clusters * p.teams;
        if (teams > most) most = teams;
    }
    return most * 4 * ceil64(n, 8) * 8 * 4;
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
    const int gate_pieces = b && gate && ldg ? (o->params_f32 ? 2 : 1) : 0, pieces = (o->stream_f32 ? 2 : 1) + (o->block_f32 ? 2 : 1) + gate_pieces;
    const bool bias = (b && c_block) || c_next;
    const int params = bias ? 8 : 4, eights = join_eights(n, false);
    const JoinPlan p = join_plan(sms, tokens, n, eights, pieces, params, JOIN_FORWARD_THREADS);
    JoinArgs a = join_args(*o, tokens, n, p, pieces, params);
    a.r = rows_of(r, ldr, o->stream_f32); a.b = rows_of(b, ldb, o->block_f32); a.out = rows_of(out, ldo, o->stream_f32); a.h = rows_of(h, ldh, false);
    if (b) {
        if (gate_pieces) a.gate = rows_of(gate, ldg, o->params_f32);
        else a.gate_vec = gate;
        a.w_block = w_block; a.c_block = c_block;
        a.drop = drop_of(o->drop, random);
    }
    a.w_next = w_next; a.c_next = c_next; a.stats = stats;
    if (!b) a.norm_block = DBSPMSPV_NORM_NONE;
    auto pick = [&](auto E, auto B) {
        constexpr int E_ = decltype(E)::value;
        constexpr bool B_ = decltype(B)::value;
        return o->stream_f32 ? (o->block_f32 ? k_join<true, true, E_, B_> : k_join<true, false, E_, B_>) : (o->block_f32 ? k_join<false, true, E_, B_> : k_join<false, false, E_, B_>);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    auto kernel = eights == 2 ? (bias ? pick(Two{}, std::true_type{}) : pick(Two{}, std::false_type{})) : (bias ? pick(One{}, std::true_type{}) : pick(One{}, std::false_type{}));
    return launch_rows(kernel, p.clusters * p.cluster, p.warps * p.teams * 32, p.cluster, join_smem(p, pieces, params), static_cast<cudaStream_t>(stream), a);
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
    const int gate_pieces = rows && block ? (o->params_f32 ? 2 : 1) : 0, pieces = 1 + 2 * (o->stream_f32 ? 2 : 1) + (o->block_f32 ? 2 : 1) + gate_pieces;
    const bool bias = dc_block || dc_next || (dgate && !rows && c_block);
    const int params = gate_pieces && dgate ? 6 : 4, eights = join_eights(n, bias);
    const JoinPlan p = join_plan(sms, tokens, n, eights, pieces, params, JOIN_BACKWARD_THREADS);
    JoinArgs a = join_args(*o, tokens, n, p, pieces, params);
    a.dh = rows_of(dh, lddh, false); a.dout = rows_of(dout, lddo, o->stream_f32); a.dr = rows_of(dr, lddr, o->stream_f32);
    if (nn && dh) a.out = rows_of(out, ldo, o->stream_f32);
    if (block) {
        if (nb || dgate) a.b = rows_of(b, ldb, o->block_f32);
        if (rows) a.gate = rows_of(gate, ldg, o->params_f32);
        else a.gate_vec = gate;
        if (rows) a.dgate = rows_of(dgate, lddg, o->params_f32);
        a.w_block = w_block; a.c_block = c_block;
        a.db = rows_of(db, lddb, o->dblock_f32);
        a.drop = drop_of(o->drop, random);
    }
    a.w_next = w_next; a.stats = const_cast<float *>(stats);
    a.parts = sums ? static_cast<float *>(workspace) : nullptr;
    a.ldp = ceil64(n, 8) * 8;
    auto pick = [&](auto E, auto B) {
        constexpr int E_ = decltype(E)::value;
        constexpr bool B_ = decltype(B)::value;
        return o->stream_f32 ? (o->block_f32 ? k_join_backward<true, true, E_, B_> : k_join_backward<true, false, E_, B_>)
                             : (o->block_f32 ? k_join_backward<false, true, E_, B_> : k_join_backward<false, false, E_, B_>);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    auto kernel = bias ? pick(One{}, std::true_type{}) : eights == 2 ? pick(Two{}, std::false_type{}) : pick(One{}, std::false_type{});
    s = launch_rows(kernel, p.clusters * p.cluster, p.warps * p.teams * 32, p.cluster, join_smem(p, pieces, params), st, a);
    if (s != DBSPMSPV_OK || !sums) return s;
    JoinSums j = {a.parts, a.ldp, p.clusters * p.teams, (int32_t)n, a.params_f32, a.drop.random ? o->scale * a.drop.scale : o->scale, w_block, c_block, rows ? nullptr : gate,
                  dw_block, dc_block, rows ? nullptr : static_cast<float *>(dgate), dw_next, dc_next};
    return launch_rows(bias ? k_join_sums<true> : k_join_sums<false>, (int)ceil64(n, JOIN_SUMS_COLS), JOIN_SUMS_CTA, 1, 0, st, j);
}

int dbspmspv_dropout(const void *x, int64_t ldx, int f32, int32_t tokens, int64_t n, float drop, const uint64_t *random, void *y, int64_t ldy, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (tokens < 0 || n < 1 || n > INT32_MAX || !(drop >= 0.f && drop <= 1.f) || ldx < n || ldy < n) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens > 0 && (!x || !y || (drop > 0.f && !random))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(f32 ? 4 : 2, x, y) || !on_bytes(8, random)) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    if (!on_current_device(x, dev) || !on_current_device(y, dev)) return DBSPMSPV_ERR_INVALID_ARG;
    DropArgs a = {rows_of(x, ldx, f32), rows_of(y, ldy, f32), drop_of(drop, random), tokens, (int32_t)n, 1, 1};
    const int64_t eights = ceil64(n, 8);
    while (a.wide < DR_CTA && a.wide < eights) a.wide *= 2;
    a.chunks = (int32_t)ceil64(eights, a.wide);
    const int64_t blocks = a.chunks * ceil64(tokens, (int64_t)(DR_CTA / a.wide) * DR_ROWS);
    if (blocks > INT32_MAX) return DBSPMSPV_ERR_UNSUPPORTED;
    return launch_rows(f32 ? k_dropout<true> : k_dropout<false>, (int)blocks, DR_CTA, 1, 0, static_cast<cudaStream_t>(stream), a);
}

int dbspmspv_logprobs(const void *logits, int64_t ldl, int logits_f32, int32_t tokens, int32_t vocab, float temperature, const int32_t *targets, float *logprob, float *entropy, float *stats,
                      int32_t top, int32_t *top_ids, float *top_logprobs, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (tokens < 0 || vocab < 1 || !(temperature > 0.f) || !isfinite(temperature) || top < 0 || top > LP_MAX_TOP || top > vocab || ldl < vocab) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens > 0 && (!logits || (logprob && !targets) || (top && !top_ids && !top_logprobs))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(logits_f32 ? 4 : 2, logits) || !on_bytes(4, targets, logprob, entropy, top_ids, top_logprobs) || !on_bytes(8, stats)) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    if (!on_current_device(logits, dev)) return DBSPMSPV_ERR_INVALID_ARG;
    LpArgs a = {logits, ldl, tokens, vocab, 1, top, 0, (float)(1.4426950408889634 / (double)temperature), (float)(1.0 / (double)temperature), logprob ? targets : nullptr, logprob, entropy, stats, top_ids, top_logprobs};
    // a row is shared out while there are SMs without one and every block has a vector for each of its threads
    const int64_t vectors = vocab / (logits_f32 ? 4 : 8);
    while (a.cluster < LP_CLUSTER && (int64_t)2 * a.cluster * tokens <= (int64_t)sms * LP_PER_SM && vectors >= (int64_t)2 * a.cluster * LP_CTA) a.cluster *= 2;
    a.rounds = (int32_t)ceil64(ceil64(vectors, a.cluster), LP_CTA * LP_FLIGHT);
    const int64_t room = (int64_t)sms * LP_PER_SM, clusters = a.cluster > 1 || tokens < room ? tokens : room;
    auto kernel = logits_f32 ? (entropy ? k_logprobs<true, true> : k_logprobs<true, false>) : (entropy ? k_logprobs<false, true> : k_logprobs<false, false>);
    return launch_rows(kernel, (int)clusters * a.cluster, LP_CTA, a.cluster, LP_SMEM, static_cast<cudaStream_t>(stream), a);
}

int dbspmspv_logprobs_backward(const void *logits, int64_t ldl, int logits_f32, int32_t tokens, int32_t vocab, float temperature, const int32_t *targets, const float *stats, const float *entropy,
                               int32_t top, const int32_t *top_ids, const float *dlogprob, const float *dentropy, const float *dtop, void *dlogits, int64_t ldd, int dlogits_f32,
                               dbspmspv_stream_t stream) {
    using namespace dbs;
    if (tokens < 0 || vocab < 1 || !(temperature > 0.f) || !isfinite(temperature) || top < 0 || top > LP_MAX_TOP || top > vocab || ldl < vocab || ldd < vocab) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens > 0 && (!logits || !dlogits || !stats || (dlogprob && !targets) || (dentropy && !entropy) || (dtop && (!top || !top_ids)))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(logits_f32 ? 4 : 2, logits) || !on_bytes(dlogits_f32 ? 4 : 2, dlogits) || !on_bytes(4, targets, entropy, top_ids, dlogprob, dentropy, dtop) || !on_bytes(8, stats))
        return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    if (!on_current_device(logits, dev) || !on_current_device(dlogits, dev)) return DBSPMSPV_ERR_INVALID_ARG;
    // a row is shared out until there are LG_ROWS_WAVES rounds of thread blocks, or two loads left to a thread
    const int64_t most = ceil64(vocab, (int64_t)8 * LG_ROWS_CTA * LG_ROWS_FLIGHT), want = ceil64((int64_t)sms * 5 * LG_ROWS_WAVES, tokens), chunks = want < most ? want : most;
    if (chunks * tokens > INT32_MAX) return DBSPMSPV_ERR_UNSUPPORTED;
    LpGrad a = {logits, dlogits, ldl, ldd, tokens, vocab, dtop ? top : 0, (int32_t)chunks, (float)(1.4426950408889634 / (double)temperature), (float)(1.0 / (double)temperature),
                targets, top_ids, stats, entropy, dlogprob, dentropy, dtop};
    auto kernel = logits_f32 ? (dlogits_f32 ? k_logprobs_backward<true, true> : k_logprobs_backward<true, false>)
                             : (dlogits_f32 ? k_logprobs_backward<false, true> : k_logprobs_backward<false, false>);
    return launch_rows(kernel, (int)(chunks * tokens), LG_ROWS_CTA, 1, 0, static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"
