// Dropout, and log probabilities behind the last layer: entry points (kernels of the latter: logprobs.cuh).  No handle: the current device, and nothing that lasts longer than a call.
#include <math.h>

#include "internal.cuh"
#include "logprobs.cuh"
#include "rows.cuh"

namespace dbs {

// temperatures whose inverse, times log2(e), fp32 holds
static bool temperature_ok(float t) { return t > 0.f && isfinite(t) && isfinite((float)(1.4426950408889634 / (double)t)); }

// ---- dropout ---------------------------------------------------------------------------------
// Bounded by HBM and, in bf16, by the generator's instructions as well: 2048 x 11008 18.8 us, 4.8 TB/s (15.0 where nothing is dropped; fp32 29.0 us, 6.2 TB/s).
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
    const Columns cols[1] = {columns_of(num, (uint32_t)eight)};
#pragma unroll
    for (int r = 0; r < DR_ROWS; ++r) {
        const int64_t t = t0 + r * tall;
        if (t >= a.tokens) break;
        void *to = const_cast<void *>(row_at<F32>(a.y, t));
        if (a.drop.random) {
            f32x2 v[1][4];
            if (F32) pairs_of_eight(p[r], q[r], v[0]);
            else pairs_of_eight(p[r], v[0]);
            drop_eights<1, false>(a.drop, num, cols, (uint32_t)t, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[0][j] = mul2(v[0][j], both(a.drop.scale));
            store_eight<F32>(to, col, a.n, whole && a.y.aligned, v[0]);
        } else store_raw<F32>(to, col, a.n, whole && a.y.aligned, p[r], q[r]);
    }
}

// Rows that do not begin on 16 bytes: words of 4 bytes side by side across the warp, on the way in and out (2048 x 11008, rows of 11009: 62 -> 29 us; 32 bits, 1024 rows: 43 -> 20).  A warp has DR_ROWS rows of its columns in flight.
template <bool F32>
__global__ void __launch_bounds__(DR_CTA) k_dropout_words(const __grid_constant__ DropArgs a) {
    constexpr int ROOM = eight_room<F32, false>();
    __shared__ __align__(16) uint8_t s_rows[DR_CTA / 32][DR_ROWS * ROOM + 1024];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t unit = (int64_t)blockIdx.x * (DR_CTA / 32) + warp;
    uint8_t *rows = s_rows[warp];
    WarpEight w;
    w.lane = lane;
    w.col = (int)(unit % a.chunks) * 256;
    w.cnt = max(0, min(8, a.n - w.mine()));
    const int64_t t0 = unit / a.chunks * DR_ROWS;
    pdl_wait();
    pdl_trigger();
#pragma unroll
    for (int r = 0; r < DR_ROWS; ++r)
        if (t0 + r < a.tokens) row_ahead<F32>(a.x, t0 + r, w, a.n, rows + r * ROOM);
    close_ahead();
    const Numbers num = numbers_of(a.drop);
    const Columns cols[1] = {columns_of(num, (uint32_t)w.mine() >> 3)};
    wait_ahead<0>();
    __syncwarp();
#pragma unroll
    for (int r = 0; r < DR_ROWS; ++r) {
        const int64_t t = t0 + r;
        if (t >= a.tokens) break;
        f32x2 v[1][4];
        row_here<F32, false>(a.x, t, w, rows + r * ROOM, v[0]);
        drop_eights<1, false>(a.drop, num, cols, (uint32_t)t, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[0][j] = mul2(v[0][j], both(a.drop.scale));
        row_out<F32>(a.y, t, w, a.n, v[0], rows + DR_ROWS * ROOM);
    }
}

}  // namespace dbs

extern "C" {

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
    if (a.drop.random && !(a.x.aligned && a.y.aligned)) {
        a.chunks = (int32_t)ceil64(n, 256);
        const int64_t blocks = ceil64(a.chunks * ceil64(tokens, DR_ROWS), DR_CTA / 32);
        if (blocks > INT32_MAX) return DBSPMSPV_ERR_UNSUPPORTED;
        return launch_rows(dev, f32 ? k_dropout_words<true> : k_dropout_words<false>, (int)blocks, DR_CTA, 1, 0, static_cast<cudaStream_t>(stream), a);
    }
    const int64_t eights = ceil64(n, 8);
    while (a.wide < DR_CTA && a.wide < eights) a.wide *= 2;
    a.chunks = (int32_t)ceil64(eights, a.wide);
    const int64_t blocks = a.chunks * ceil64(tokens, (int64_t)(DR_CTA / a.wide) * DR_ROWS);
    if (blocks > INT32_MAX) return DBSPMSPV_ERR_UNSUPPORTED;
    return launch_rows(dev, f32 ? k_dropout<true> : k_dropout<false>, (int)blocks, DR_CTA, 1, 0, static_cast<cudaStream_t>(stream), a);
}

int dbspmspv_logprobs(const void *logits, int64_t ldl, int logits_f32, int32_t tokens, int32_t vocab, float temperature, const int32_t *targets, float *logprob, float *entropy, float *stats,
                      int32_t top, int32_t *top_ids, float *top_logprobs, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (tokens < 0 || vocab < 1 || !temperature_ok(temperature) || top < 0 || top > LP_MAX_TOP || top > vocab || ldl < vocab) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens > 0 && (!logits || (logprob && !targets) || (top && !top_ids && !top_logprobs))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(logits_f32 ? 4 : 2, logits) || !on_bytes(4, targets, logprob, entropy, top_ids, top_logprobs) || !on_bytes(8, stats)) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    const void *first = first_of(logprob, entropy, stats, top_ids, top_logprobs);
    if (!on_current_device(logits, dev) || (first && !on_current_device(first, dev))) return DBSPMSPV_ERR_INVALID_ARG;
    LpArgs a = {logits, ldl, tokens, vocab, 1, top, 0, (float)(1.4426950408889634 / (double)temperature), (float)(1.0 / (double)temperature), logprob ? targets : nullptr, logprob, entropy, stats, top_ids, top_logprobs};
    // a row is shared out while there are SMs without one and every block has a vector for each of its threads
    const int64_t vectors = vocab / (logits_f32 ? 4 : 8);
    while (a.cluster < LP_CLUSTER && (int64_t)2 * a.cluster * tokens <= (int64_t)sms * LP_PER_SM && vectors >= (int64_t)2 * a.cluster * LP_CTA) a.cluster *= 2;
    a.rounds = (int32_t)ceil64(ceil64(vectors, a.cluster), LP_CTA * LP_FLIGHT);
    const int64_t room = (int64_t)sms * LP_PER_SM, clusters = a.cluster > 1 || tokens < room ? tokens : room;
    auto kernel = logits_f32 ? (entropy ? k_logprobs<true, true> : k_logprobs<true, false>) : (entropy ? k_logprobs<false, true> : k_logprobs<false, false>);
    return launch_rows(dev, kernel, (int)clusters * a.cluster, LP_CTA, a.cluster, LP_SMEM + (a.cluster > 1 ? sizeof(LpCluster) : 0), static_cast<cudaStream_t>(stream), a);
}

int dbspmspv_logprobs_backward(const void *logits, int64_t ldl, int logits_f32, int32_t tokens, int32_t vocab, float temperature, const int32_t *targets, const float *stats, const float *entropy,
                               int32_t top, const int32_t *top_ids, const float *dlogprob, const float *dentropy, const float *dtop, void *dlogits, int64_t ldd, int dlogits_f32,
                               dbspmspv_stream_t stream) {
    using namespace dbs;
    if (tokens < 0 || vocab < 1 || !temperature_ok(temperature) || top < 0 || top > LP_MAX_TOP || top > vocab || ldl < vocab || ldd < vocab) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens > 0 && (!logits || !dlogits || !stats || (dlogprob && !targets) || (dentropy && !entropy) || (dtop && (!top || !top_ids)))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(logits_f32 ? 4 : 2, logits) || !on_bytes(dlogits_f32 ? 4 : 2, dlogits) || !on_bytes(4, targets, entropy, top_ids, dlogprob, dentropy, dtop) || !on_bytes(8, stats))
        return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    int dev, sms, s;
    if ((s = current_device(&dev, &sms)) != DBSPMSPV_OK) return s;
    if (!on_current_device(logits, dev) || !on_current_device(dlogits, dev)) return DBSPMSPV_ERR_INVALID_ARG;
    // a row is shared out until there are LG_ROWS_WAVES rounds of thread blocks, but few rows to one round; and until two loads are left to a thread
    const int64_t most = ceil64(vocab, (int64_t)8 * LG_ROWS_CTA * LG_ROWS_FLIGHT), at_once = (int64_t)sms * LG_ROWS_PER_SM;
    const int64_t want = tokens < at_once / 2 ? at_once / tokens : ceil64(at_once * LG_ROWS_WAVES, tokens), chunks = want < most ? want : most;
    if (chunks * tokens > INT32_MAX) return DBSPMSPV_ERR_UNSUPPORTED;
    LpGrad a = {logits, dlogits, ldl, ldd, tokens, vocab, dtop ? top : 0, (int32_t)chunks, (float)(1.4426950408889634 / (double)temperature), (float)(1.0 / (double)temperature),
                targets, top_ids, stats, entropy, dlogprob, dentropy, dtop};
    auto kernel = logits_f32 ? (dlogits_f32 ? k_logprobs_backward<true, true> : k_logprobs_backward<true, false>)
                             : (dlogits_f32 ? k_logprobs_backward<false, true> : k_logprobs_backward<false, false>);
    return launch_rows(dev, kernel, (int)(chunks * tokens), LG_ROWS_CTA, 1, 0, static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"
