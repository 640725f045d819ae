// Dense products of the pruned layers on the tensor cores (tcgen05.mma, accumulators in TMEM), for more tokens than the
// kernel over active columns serves (linear_columns.cuh) and for the gradients.
//
// From a handful of tokens on every weight is reached, and a layer pruned without a pattern to half has no form that the
// tensor cores could skip anything of: the product of the matrix with zeros in the pruned places is the fast one.  All three products
//
//   forward          Y [token][row]     = X [token][column]  times  W [row][column] over the columns
//   gradient of x    dX [token][column] = dZ [token][row]    times  W [row][column] over the rows
//   gradient of W    dW [column][row]   = X [token][column]  times  dZ [token][row] over the tokens (stored places only)
//
// read the operands as they lie -- tokens row by row, W in the strips of the copy by columns ([strip of 64 rows][column][row], 128
// bytes per column and strip).  64 rows of bf16 are the 128 bytes of one swizzle row, so a strip is an operand tile with the rows
// along M/N for the forward product and along K for the gradient of x; nothing is transposed or laid out again.
//
//   * Tile 128 x 256, K in blocks of 64, four stages of 48 KB filled by TMA (edges are zero-filled by the tensor maps), one thread
//     issues the loads, one the products, four warps empty the accumulators.  Two accumulators of 256 TMEM columns take turns, so
//     the epilogue of one tile runs under the products of the next.
//   * Gated: the tile's 256 columns are 128 rows of the gate and the same 128 of the other layer; both sums of an output
//     meet in one thread.
//   * Gradient of W: M are the columns and N the rows, so that the lanes of a warp hold 32 neighbouring columns of one row and the
//     stored ones among them are neighbours in the values' array: one popc gives each its place.
//   * Few tiles: the C thread blocks of a cluster share K and add their sums up through distributed shared memory, in rank order.
//
// Sums are fp32 in TMEM; what is handed on in bf16 is rounded once.  Every wait is bounded.
#pragma once

#include <cooperative_groups.h>
#include <cuda.h>

#include "internal.cuh"
#include "staging.cuh"

namespace dbs {

constexpr int LG_M = 128, LG_N = 256, LG_K = 64;
constexpr int LG_A_BYTES = LG_M * LG_K * 2, LG_B_BYTES = LG_N * LG_K * 2, LG_STAGE_BYTES = LG_A_BYTES + LG_B_BYTES;
constexpr int LG_STAGES = 4;
constexpr int LG_SMEM = LG_STAGES * LG_STAGE_BYTES + 1024;     // (the swizzle's pattern repeats every 1024 bytes: the stages begin on a multiple)
constexpr int LG_WARPS = 6;                                    // loads, products, four for the accumulators
constexpr int LG_CTA = LG_WARPS * 32;
constexpr int LG_CHUNK = 16;                                   // accumulator columns that a thread takes at a time
static_assert(LG_N * LG_M * 4 <= LG_STAGES * LG_STAGE_BYTES, "a tile's sums, for the other thread blocks of a cluster, lie in the stages");

enum LgForm { LG_FORWARD = 0, LG_GATED = 1, LG_DX = 2, LG_DW = 3 };

struct LgMaps { CUtensorMap a[2], b[2]; };                     // (the second ones: the second layer of a gated block)

struct LgArgs {
    int tiles_m, tiles_n;           // tiles of one product
    int products;                   // LG_DW: 2 for the two layers of a gated block, as one list of tiles
    int k_blocks;                   // of one layer
    int layers;                     // LG_DX: the layers whose products are added up, one behind the other along K
    int64_t tokens, width;          // rows and columns of y (LG_DW: rows of W = columns of dZ)
    void *y;
    int64_t ldy;
    int y_f32, act;
    const uint16_t *bias, *residual;
    int64_t ldr;
    uint16_t *z, *u;                // in front of the activation; the other projection (may be null)
    int64_t ldz;
    uint16_t *dw[2];
    const uint2 *index[2];          // [row][word of 32 columns]: stored columns, place of the first of them
    int index_words;
    int32_t *status;
};

// ---- activations -------------------------------------------------------------------------
__device__ __forceinline__ float lin_act(float z, int act) {
    switch (act) {
        case DBSPMSPV_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
        case DBSPMSPV_ACT_SILU: return z / (1.f + expf(-z));
        case DBSPMSPV_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678f));
        default: return z;
    }
}
__device__ __forceinline__ float lin_act_slope(float z, int act) {
    switch (act) {
        case DBSPMSPV_ACT_RELU: return z > 0.f ? 1.f : 0.f;
        case DBSPMSPV_ACT_SILU: { const float p = 1.f / (1.f + expf(-z)); return p * (1.f + z * (1.f - p)); }
        case DBSPMSPV_ACT_GELU: return 0.5f * (1.f + erff(z * 0.70710678f)) + z * (0.39894228f * expf(-0.5f * z * z));
        default: return 1.f;
    }
}
__device__ __forceinline__ uint32_t lin_bf16(float v) { return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v)); }
__device__ __forceinline__ float lin_f32(uint32_t half) { return __uint_as_float(half << 16); }

// ---- instructions ------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_load16(uint32_t addr, float (&v)[LG_CHUNK]) {
    uint32_t r[LG_CHUNK];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr));
#pragma unroll
    for (int i = 0; i < LG_CHUNK; ++i) v[i] = __uint_as_float(r[i]);
}
// (the loaded registers are named, so that nothing that uses them moves in front of the wait)
__device__ __forceinline__ void tc_load_wait(float (&v)[LG_CHUNK]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                   "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]) :: "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory"); }

// Descriptor of an operand tile in shared memory under the 128-byte swizzle.  K along the swizzle rows: 64 of K per row, eight rows of M/N 1024
// bytes on (the other stride is not used).  M/N along them: eight of K 1024 bytes on, the next 64 of M/N behind the block's 64 of K.
__device__ __forceinline__ uint64_t lg_desc(uint32_t addr, bool mn_major) {
    const uint64_t leading = mn_major ? LG_K * 128 : 16;
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (leading >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__host__ __device__ constexpr uint32_t lg_idesc(bool a_mn, bool b_mn) {        // fp32 sums, bf16 operands
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)a_mn << 15 | (uint32_t)b_mn << 16 | (uint32_t)(LG_N >> 3) << 17 | (uint32_t)(LG_M >> 4) << 24;
}

// Bounded wait that also gives up when another thread of the block has (s_fail).
__device__ __forceinline__ bool lg_wait(uint64_t *bar, uint32_t parity, volatile int *fail, int32_t *status) {
    for (int i = 0; i < MBAR_WAIT_LIMIT; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*fail) return false;
    }
    *fail = 1;
    *status = DBSPMSPV_ERR_TIMEOUT;
    return false;
}

// ---- what becomes of 16 neighbouring sums of one token -----------------------------------
__device__ __forceinline__ void lg_store16(uint16_t *p, const float (&v)[LG_CHUNK], int count) {
    if (count == LG_CHUNK && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
        uint32_t w[LG_CHUNK / 2];
#pragma unroll
        for (int i = 0; i < LG_CHUNK / 2; ++i) w[i] = lin_bf16(v[2 * i]) | lin_bf16(v[2 * i + 1]) << 16;
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
#pragma unroll
        for (int i = 0; i < LG_CHUNK; ++i)
            if (i < count) p[i] = (uint16_t)lin_bf16(v[i]);
    }
}
__device__ __forceinline__ void lg_add16(const uint16_t *p, float (&v)[LG_CHUNK], int count) {
    if (count == LG_CHUNK && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
        const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
        const uint32_t w[LG_CHUNK / 2] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < LG_CHUNK / 2; ++i) { v[2 * i] += __uint_as_float(w[i] << 16); v[2 * i + 1] += __uint_as_float(w[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < LG_CHUNK; ++i)
            if (i < count) v[i] += lin_f32(p[i]);
    }
}
__device__ __forceinline__ void lg_act16(float (&v)[LG_CHUNK], int act) {
    if (act == DBSPMSPV_ACT_NONE) return;
    if (act == DBSPMSPV_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < LG_CHUNK; ++i) v[i] = lin_act(v[i], DBSPMSPV_ACT_RELU);
    } else if (act == DBSPMSPV_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < LG_CHUNK; ++i) v[i] = lin_act(v[i], DBSPMSPV_ACT_SILU);
    } else {
#pragma unroll
        for (int i = 0; i < LG_CHUNK; ++i) v[i] = lin_act(v[i], DBSPMSPV_ACT_GELU);
    }
}
// outputs [col, col + 16) of token `t`; v: the sums, u: the other layer's (gated)
template <int FORM>
__device__ __forceinline__ void lg_finish(const LgArgs &a, int64_t t, int64_t col, float (&v)[LG_CHUNK], const float (&u)[LG_CHUNK]) {
    if (t >= a.tokens || col >= a.width) return;
    const int count = a.width - col < LG_CHUNK ? (int)(a.width - col) : LG_CHUNK;
    if (FORM == LG_FORWARD && a.bias) lg_add16(a.bias + col, v, count);
    if (FORM != LG_DX && a.z) lg_store16(a.z + t * a.ldz + col, v, count);
    if (FORM != LG_DX) lg_act16(v, a.act);
    if (FORM == LG_GATED) {
        if (a.u) lg_store16(a.u + t * a.ldz + col, u, count);
#pragma unroll
        for (int i = 0; i < LG_CHUNK; ++i) v[i] *= u[i];
    }
    if (FORM == LG_FORWARD && a.residual) lg_add16(a.residual + t * a.ldr + col, v, count);
    if (FORM == LG_FORWARD && a.y_f32) {
        float *p = static_cast<float *>(a.y) + t * a.ldy + col;
#pragma unroll
        for (int i = 0; i < LG_CHUNK; ++i)
            if (i < count) p[i] = v[i];
    } else {
        lg_store16(static_cast<uint16_t *>(a.y) + t * a.ldy + col, v, count);
    }
}

// Tiles in the order they are taken: those of one weight tile side by side, so that its weights come from L2 after the first.
struct LgTile { int m, n, product; };
__device__ __forceinline__ LgTile lg_tile(const LgArgs &a, int i) {
    const int per = a.tiles_m * a.tiles_n;
    LgTile t;
    t.product = i / per;
    i -= t.product * per;
    t.n = i / a.tiles_m;
    t.m = i - t.n * a.tiles_m;
    return t;
}

template <int FORM, int C>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(LG_CTA, 1)
k_linear_gemm(const __grid_constant__ LgMaps maps, const __grid_constant__ LgArgs a) {
    namespace cg = cooperative_groups;
    constexpr bool A_MN = FORM == LG_DW, B_MN = FORM != LG_DX;
    extern __shared__ uint8_t s_raw[];
    __shared__ __align__(8) uint64_t s_full[LG_STAGES], s_empty[LG_STAGES], s_done[2], s_free[2];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_fail;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t stages = (smem_addr(s_raw) + 1023u) & ~1023u;
    const int rank = C > 1 ? (int)(blockIdx.x % C) : 0;
    const int first = (int)(blockIdx.x / C), step = (int)(gridDim.x / C), n_tiles = a.tiles_m * a.tiles_n * a.products;
    const int kb_all = a.k_blocks * a.layers, kb0 = (int)((int64_t)kb_all * rank / C), kb1 = (int)((int64_t)kb_all * (rank + 1) / C);
    if (tid == 0) {
        for (int s = 0; s < LG_STAGES; ++s) { mbar_init(&s_full[s], 1); mbar_init(&s_empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&s_done[s], 1); mbar_init(&s_free[s], 4); }
        s_fail = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_wait();
    if (warp == 0) {
        if (lane == 0) {                                               // ---- loads
            int it = 0;
            bool ok = true;
            for (int i = first; i < n_tiles && ok; i += step) {
                const LgTile t = lg_tile(a, i);
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int s = it % LG_STAGES, layer = kb >= a.k_blocks, k = kb - layer * a.k_blocks;
                    if (it >= LG_STAGES && !lg_wait(&s_empty[s], (uint32_t)((it / LG_STAGES - 1) & 1), &s_fail, a.status)) { ok = false; break; }
                    const uint32_t pa = stages + s * LG_STAGE_BYTES, pb = pa + LG_A_BYTES, bar = smem_addr(&s_full[s]);
                    mbar_arrive_expect_tx(&s_full[s], LG_STAGE_BYTES);
                    if (FORM == LG_DW) {
#pragma unroll
                        for (int q = 0; q < LG_M / 64; ++q) tma_load_2d(pa + q * 8192, &maps.a[0], t.m * LG_M + q * 64, k * LG_K, bar);
#pragma unroll
                        for (int q = 0; q < LG_N / 64; ++q) tma_load_2d(pb + q * 8192, &maps.b[t.product], t.n * LG_N + q * 64, k * LG_K, bar);
                    } else {
                        tma_load_2d(pa, &maps.a[layer], k * LG_K, t.m * LG_M, bar);
                        if (FORM == LG_DX) tma_load_3d(pb, &maps.b[layer], 0, t.n * LG_N, k, bar);
                        else if (FORM == LG_FORWARD) tma_load_3d(pb, &maps.b[0], 0, k * LG_K, t.n * (LG_N / DC_ROWS), bar);
                        else {
                            tma_load_3d(pb, &maps.b[0], 0, k * LG_K, t.n * (LG_N / DC_ROWS / 2), bar);
                            tma_load_3d(pb + LG_B_BYTES / 2, &maps.b[1], 0, k * LG_K, t.n * (LG_N / DC_ROWS / 2), bar);
                        }
                    }
                }
            }
            if (!ok)                                                   // gave up: the copies in flight land before the block ends
                for (int q = it < LG_STAGES ? 0 : it - LG_STAGES; q < it; ++q) (void)mbar_wait_bounded(&s_full[q % LG_STAGES], (uint32_t)((q / LG_STAGES) & 1), 1 << 16);
        }
    } else if (warp == 1) {
        if (lane == 0) {                                               // ---- products
            int it = 0, n = 0;
            bool ok = true;
            for (int i = first; i < n_tiles && ok; i += step, ++n) {
                const uint32_t d = tmem + (uint32_t)(n & 1) * LG_N;
                if (n >= 2 && !lg_wait(&s_free[n & 1], (uint32_t)((n / 2 - 1) & 1), &s_fail, a.status)) { ok = false; break; }
                tc_fence_after();
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int s = it % LG_STAGES;
                    if (!lg_wait(&s_full[s], (uint32_t)((it / LG_STAGES) & 1), &s_fail, a.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t pa = stages + s * LG_STAGE_BYTES, pb = pa + LG_A_BYTES;
#pragma unroll
                    for (int k = 0; k < LG_K / 16; ++k)
                        tc_mma(d, lg_desc(pa + k * (A_MN ? 2048 : 32), A_MN), lg_desc(pb + k * (B_MN ? 2048 : 32), B_MN), lg_idesc(A_MN, B_MN), kb > kb0 || k > 0);
                    tc_commit(&s_empty[s]);
                }
                if (ok) tc_commit(&s_done[n & 1]);
            }
            if (!ok && it > 0)                                         // gave up: the products in flight end before the accumulators are given back
                (void)mbar_wait_bounded(&s_empty[(it - 1) % LG_STAGES], (uint32_t)(((it - 1) / LG_STAGES) & 1), 1 << 16);
        }
    } else {                                                           // ---- accumulators: warp w reads the lanes 32 (w % 4) ...
        const int quad = warp & 3;
        const uint32_t mine = tmem + ((uint32_t)(quad * 32) << 16);
        int n = 0;
        for (int i = first; i < n_tiles; i += step, ++n) {
            const LgTile t = lg_tile(a, i);
            if (!lg_wait(&s_done[n & 1], (uint32_t)((n / 2) & 1), &s_fail, a.status)) break;
            __syncwarp();
            tc_fence_after();
            const uint32_t d = mine + (uint32_t)(n & 1) * LG_N;
            if constexpr (FORM == LG_DW) {
                const int word = t.m * (LG_M / 32) + quad;
                const uint2 *index = a.index[t.product] + word;
                uint16_t *dw = a.dw[t.product];
                const int64_t row0 = (int64_t)t.n * LG_N;
                const uint32_t below = (1u << lane) - 1u;
                for (int c = 0; c < LG_N; c += LG_CHUNK) {
                    uint2 e[LG_CHUNK];
#pragma unroll
                    for (int k = 0; k < LG_CHUNK; ++k) {
                        e[k] = make_uint2(0u, 0u);
                        if (word < a.index_words && row0 + c + k < a.width) e[k] = __ldg(index + (row0 + c + k) * a.index_words);
                    }
                    float v[LG_CHUNK];
                    tc_load16(d + c, v);
                    tc_load_wait(v);
#pragma unroll
                    for (int k = 0; k < LG_CHUNK; ++k)
                        if ((e[k].x >> lane) & 1u) dw[(size_t)e[k].y + __popc(e[k].x & below)] = (uint16_t)lin_bf16(v[k]);
                    __syncwarp();
                }
            } else if constexpr (C == 1) {
                const int64_t token = (int64_t)t.m * LG_M + quad * 32 + lane;
                constexpr int OUT = FORM == LG_GATED ? LG_N / 2 : LG_N;
                if ((int64_t)t.m * LG_M + quad * 32 < a.tokens) {
                    for (int c = 0; c < OUT; c += LG_CHUNK) {
                        float v[LG_CHUNK], u[LG_CHUNK];
                        tc_load16(d + c, v);
                        if (FORM == LG_GATED) { tc_load16(d + OUT + c, u); tc_load_wait(u); }
                        tc_load_wait(v);
                        lg_finish<FORM>(a, token, (int64_t)t.n * OUT + c, v, u);
                        __syncwarp();
                    }
                }
            } else {
                // this block's sums into its own shared memory, [column][token]: every copy has landed and every product has been made
                const uint32_t at = stages + (uint32_t)(quad * 32 + lane) * 4;
                if ((int64_t)t.m * LG_M + quad * 32 < a.tokens) {
                    for (int c = 0; c < LG_N; c += LG_CHUNK) {
                        float v[LG_CHUNK];
                        tc_load16(d + c, v);
                        tc_load_wait(v);
#pragma unroll
                        for (int k = 0; k < LG_CHUNK; ++k)
                            asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + (uint32_t)(c + k) * (LG_M * 4)), "f"(v[k]) : "memory");
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_free[n & 1]);
        }
    }
    __syncwarp();
    if constexpr (C > 1 && FORM != LG_DW) {
        // (one tile per cluster)  Rank r adds up the C sums of its share of the columns and finishes them.
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (warp >= 2 && !s_fail && first < n_tiles) {
            const LgTile t = lg_tile(a, first);
            const int quad = warp & 3;
            constexpr int OUT = FORM == LG_GATED ? LG_N / 2 : LG_N;
            const uint32_t at = stages + (uint32_t)(quad * 32 + lane) * 4;
            const int64_t token = (int64_t)t.m * LG_M + quad * 32 + lane;
            if ((int64_t)t.m * LG_M + quad * 32 < a.tokens) {
                for (int c = rank * LG_CHUNK; c < OUT; c += C * LG_CHUNK) {
                    float v[LG_CHUNK], u[LG_CHUNK];
#pragma unroll
                    for (int k = 0; k < LG_CHUNK; ++k) v[k] = u[k] = 0.f;
#pragma unroll
                    for (int r = 0; r < C; ++r) {
                        uint32_t far;
                        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(at), "r"(r));
#pragma unroll
                        for (int k = 0; k < LG_CHUNK; ++k) {
                            float f;
                            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(far + (uint32_t)(c + k) * (LG_M * 4)) : "memory");
                            v[k] += f;
                            if (FORM == LG_GATED) {
                                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(far + (uint32_t)(OUT + c + k) * (LG_M * 4)) : "memory");
                                u[k] += f;
                            }
                        }
                    }
                    lg_finish<FORM>(a, token, (int64_t)t.n * OUT + c, v, u);
                }
            }
        }
        __syncwarp();
        cluster.sync();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

}  // namespace dbs
