// Dense products of the pruned layers on the tensor cores (tcgen05.mma, accumulators in TMEM), for more tokens than the
// kernel over active columns serves (linear_columns.cuh) and for the gradients.
//
// From a handful of tokens on every weight is reached, and a layer pruned without a pattern to half has no form that the
// tensor cores could skip anything of: the product of the matrix with zeros in the pruned places is the fast one.  All three products
//
//   forward          Y^T [row][token]    = W [row][column]     times  X [token][column] over the columns
//   gradient of x    dX^T [column][token] = W [row][column]    times  dZ [token][row] over the rows
//   gradient of W    dW^T [column][row]  = X [token][column]   times  dZ [token][row] over the tokens (stored places only)
//
// read the operands as they lie -- tokens row by row, W in the strips of the copy by columns ([strip of 64 rows][column][row], 128
// bytes per column and strip).  64 rows of bf16 are the 128 bytes of one swizzle row, so a strip is an operand tile with the rows
// along M for the forward product and along K for the gradient of x; nothing is transposed or laid out again.
//
//   * M (the lanes of an accumulator) is the dimension that lies side by side in the output, and tokens are N, so that few tokens
//     are a narrow tile.  Tiles are 128 x NT.
//   * One thread issues the loads (TMA; edges are zero-filled by the tensor maps), one the products, eight warps empty the accumulators.
//     Two accumulators take turns, so the epilogue of one tile runs under the products of the next.
//   * Epilogue: the sums of a few tokens at a time go through shared memory, [token][lane], and are finished from there, eight neighbours of a
//     token per thread: 16 bytes a load or store, 256 bytes side by side, the residual fetched in front of the exchange.
//     (A lane's own values, 2 bytes at a time, by four warps: 11008 x 4096 gated, 2048 tokens, both projections kept 373 us, 280 through shared memory.)
//   What bounds it: many tokens, the tensor cores under the power limit (11008 x 4096 gated, 2048 tokens: 300 us, 1230 TFLOP/s of dense product, 260 us in short bursts;
//   cuBLAS reaches 1356 and in short bursts 1628 on 8192^3, this kernel there 1430); few tokens, HBM on the copy (the same layers, 6 tokens: 30 us, 180 MB at 6 TB/s).
//   * CG = 2: the two thread blocks of a cluster work on one 256 x 256 tile, each with half of either operand in its shared memory:
//     32 KB per block of K and SM where one block alone would need 48.
//   * Gated: M are 64 rows of the gate and the same 64 of the other layer; both sums of an output meet in that exchange.
//   * Gradient of W: the lanes of a warp hold 32 neighbouring columns of one row, and the stored ones among them are neighbours in the
//     values' array: one popc gives each its place.
//   * C > 1, few tiles: the C thread blocks of a cluster share K and add their sums up through distributed shared memory, in rank order.
//
// Sums are fp32 in TMEM; what is handed on in bf16 is rounded once.  Every wait for a barrier in shared memory is bounded; those of the hardware's own (TMEM, clusters, the kernel in front) end with the blocks they wait for.
#pragma once

#include <cooperative_groups.h>
#include <cuda.h>

#include "internal.cuh"
#include "linear_plan.h"
#include "staging.cuh"

namespace dbs {

constexpr int LG_A_BYTES = LG_M * LG_K * 2;
constexpr int LG_FINISH = 8;                                   // warps that empty the accumulators, two for each quarter of the lanes
constexpr int LG_FINISH_DW = 16;                               // ... for the gradient of W, whose values go one by one: twice as many
__host__ __device__ constexpr int lg_threads(bool dw) { return (2 + (dw ? LG_FINISH_DW : LG_FINISH)) * 32; }       // (and one warp each for the loads and the products)

// Stages of a form: a block of K of both operands.  Narrow tiles (few tokens, bound by HBM) leave room for two thread blocks per SM.
__host__ __device__ constexpr int lg_stage_bytes(int cg, int nt) { return LG_A_BYTES + nt / cg * LG_K * 2; }
__host__ __device__ constexpr int lg_stages(int cg, int nt) { return nt <= 16 ? 5 : cg == 2 ? 6 : 4; }
// Tokens whose sums are exchanged at a time, and how many such buffers there are
__host__ __device__ constexpr int lg_tokens(int nt) { return nt <= 64 ? 16 : 32; }
__host__ __device__ constexpr int lg_buffers(int nt) { return nt == 64 ? 1 : 2; }
__host__ __device__ constexpr int lg_exchange(int nt) { return lg_tokens(nt) * lg_buffers(nt) * LG_M * 4; }
// (the swizzle's pattern repeats every 1024 bytes: the stages begin on a multiple)
__host__ __device__ constexpr int lg_smem(int cg, int nt) { return lg_stages(cg, nt) * lg_stage_bytes(cg, nt) + lg_exchange(nt) + 1024; }

enum LgForm { LG_FORWARD = 0, LG_GATED = 1, LG_DX = 2, LG_DW = 3 };

struct LgMaps { CUtensorMap a[2], b[2]; };                     // (the second ones: the second layer of a gated block)

struct LgArgs {
    int tiles_m, tiles_n;           // tiles of one product: of the output's width (LG_DW: of its columns), of the tokens (LG_DW: of its rows)
    int products;                   // LG_DW: 2 for the two layers of a gated block, as one list of tiles
    int k_blocks;                   // of one layer
    int layers;                     // LG_DX: the layers whose products are added up, one behind the other along K
    int64_t tokens, width;          // rows and columns of y (LG_DW: width = rows of W)
    void *y;
    int64_t ldy;
    int y_f32, act;
    const uint16_t *bias, *residual;
    int64_t ldr;
    uint16_t *z, *u;                // in front of the activation; the other projection (may be null)
    int64_t ldz;
    int aligned;                    // every row of y, z, u and the residual begins on 16 bytes
    uint16_t *dw[2];
    uint32_t stored[2];             // their weights (for the range-checked build)
    const uint2 *index[2];          // [word of 32 columns][row]: stored columns, place of the first of them
    int index_words;
    int32_t *status;
};

// ---- activations -------------------------------------------------------------------------
// 1 / (1 + exp(-z)) by the exponential of -|z|: the other one is infinite from -88.7 on, where z times the result is still a normal number.
__device__ __forceinline__ float lin_sigmoid(float z) {
    const float e = expf(-fabsf(z));
    return (z < 0.f ? e : 1.f) / (1.f + e);
}
// Phi(z).  (By erfc: 1 + erf cancels on the left, off by 10 % at -5 and nothing left from -5.5 on.)
__device__ __forceinline__ float lin_phi(float z) { return 0.5f * erfcf(z * -0.70710678f); }
__device__ __forceinline__ float lin_act(float z, int act) {
    switch (act) {
        case DBSPMSPV_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
        case DBSPMSPV_ACT_SILU: return z * lin_sigmoid(z);
        case DBSPMSPV_ACT_GELU: return z * lin_phi(z);
        default: return z;
    }
}
// The same by the fast exponential and divide, for what is rounded to bf16 or stands in an epilogue: off by (1.2 |z| + 8) 2^-23 of the result at most.
// (expf and a full divide took a quarter of the epilogue's instructions.)
__device__ __forceinline__ float lin_sigmoid_fast(float z) {
    const float e = __expf(-fabsf(z));
    return __fdividef(z < 0.f ? e : 1.f, 1.f + e);
}
__device__ __forceinline__ float lin_silu_fast(float z) { return z * lin_sigmoid_fast(z); }
__device__ __forceinline__ uint32_t lin_bf16(float v) { return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v)); }
__device__ __forceinline__ uint32_t lin_pair(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ float lin_f32(uint32_t half) { return __uint_as_float(half << 16); }

// ---- instructions ------------------------------------------------------------------------
template <int CG>
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t idesc, bool add) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %4, p;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// arrives on the barrier (CG = 2: on the one at the same place in both thread blocks) when every product issued so far has been made
template <int CG>
__device__ __forceinline__ void tc_commit(uint64_t *bar) {
    if (CG == 1) asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// (load and wait in one statement: nothing may touch the registers in between)
__device__ __forceinline__ void tc_load16(uint32_t addr, float (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, int rank) {
    uint32_t far;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(addr), "r"(rank));
    return far;
}
// (relaxed, as PTX has it for handing tensor memory to another thread: what is handed on is the accumulator, whose loads have ended (wait::ld of the whole warp), ordered by the tcgen05 fences
// before this arrival and behind the wait; nothing else is read behind it.  A release would wait for the warp's stores to global memory.)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t far) { asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(far) : "memory"); }
__device__ __forceinline__ float4 ld_cluster(uint32_t far) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(far) : "memory");
    return v;
}
__device__ __forceinline__ float ld_cluster1(uint32_t far) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(far) : "memory");
    return v;
}
__device__ __forceinline__ void ld_shared(uint32_t addr, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 4)
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3]) : "r"(addr + i * 4) : "memory");
}
__device__ __forceinline__ void st_shared(uint32_t addr, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
// the warps that empty the accumulators meet; with a vote: whether `ok` holds in all of them
__device__ __forceinline__ void finish_sync() { asm volatile("bar.sync 1, %0;" ::"n"(LG_FINISH * 32) : "memory"); }
__device__ __forceinline__ bool finish_all(bool ok) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"((uint32_t)ok), "n"(LG_FINISH * 32) : "memory");
    return all != 0;
}
__device__ __forceinline__ void store_if(bool p, uint16_t *at, uint32_t v) {       // (predicated: no branch per element)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %0, 0;\n\t@p st.global.b16 [%1], %2;\n\t}" ::"r"((uint32_t)p), "l"(at), "h"((uint16_t)v) : "memory");
}

// Descriptor of an operand tile in shared memory under the 128-byte swizzle.  K along the swizzle rows: 64 of K per row, eight rows of M/N 1024
// bytes on (the other stride is not used).  M/N along them: eight of K 1024 bytes on, the next 64 of M/N behind the block's 64 of K.
// The upper word is a constant, the lower one counts addresses in 16 bytes: the next 16 of K are an addition away.
constexpr uint32_t LG_DESC_HIGH = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t lg_desc_low(uint32_t addr, bool mn_major) { return ((addr >> 4) & 0x3FFFu) | (uint32_t)((mn_major ? LG_K * 128 : 16) >> 4) << 16; }
__host__ __device__ constexpr uint32_t lg_idesc(int m, int n, bool a_mn, bool b_mn) {        // fp32 sums, bf16 operands
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)a_mn << 15 | (uint32_t)b_mn << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
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

// The same for the two threads that everything waits for: they look again at once.
__device__ __forceinline__ bool lg_spin(uint64_t *bar, uint32_t parity, volatile int *fail, int32_t *status) {
    for (int i = 0; i < (1 << 26); ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
        if (ok) return true;
        if ((i & 255) == 255 && *fail) return false;
    }
    *fail = 1;
    *status = DBSPMSPV_ERR_TIMEOUT;
    return false;
}

// ---- what becomes of neighbouring sums of one token --------------------------------------
__device__ __forceinline__ void lg_act(float (&v)[8], int act) {
    if (act == DBSPMSPV_ACT_NONE) return;
    if (act == DBSPMSPV_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lin_act(v[i], DBSPMSPV_ACT_RELU);
    } else if (act == DBSPMSPV_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lin_silu_fast(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lin_act(v[i], DBSPMSPV_ACT_GELU);
    }
}
// Half words [from, from + 8) of the sixteen in c[0 .. 7], two to a word; from = 0 .. 8
__device__ __forceinline__ void lg_shift(uint32_t (&c)[9], int from, uint32_t (&w)[4]) {
    c[8] = 0u;                                                         // (not read)
#pragma unroll
    for (int i = 0; i < 5; ++i) c[i] = from & 8 ? c[i + 4] : c[i];
#pragma unroll
    for (int i = 0; i < 6; ++i) c[i] = from & 4 ? c[i + 2] : c[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) c[i] = from & 2 ? c[i + 1] : c[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = from & 1 ? __funnelshift_r(c[i], c[i + 1], 16) : c[i];
}
// Columns col .. col + 7 of a row of `width` bf16, two to a word; past the row's end 0.  `aligned`: rows begin on 16 bytes, and col is a multiple of eight.  Elsewhere the sixteen that lie
// on 16 bytes around them are loaded, where all of them belong to the row.
__device__ __forceinline__ void lg_get(const uint16_t *row, int64_t col, int64_t width, bool aligned, uint32_t (&w)[4]) {
    const uint16_t *p = row + col;
    if (aligned && col + 8 <= width) {
        const uint4 q = *reinterpret_cast<const uint4 *>(p);
        w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    } else if (!aligned && col >= 8 && col + 16 <= width) {
        const int s = (int)((reinterpret_cast<uintptr_t>(p) >> 1) & 7u);
        const uint4 q = *reinterpret_cast<const uint4 *>(p - s), r = *reinterpret_cast<const uint4 *>(p - s + 8);
        uint32_t c[9] = {q.x, q.y, q.z, q.w, r.x, r.y, r.z, r.w, 0u};
        lg_shift(c, s, w);
    } else {
        const int64_t count = width - col;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (2 * i < count ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < count ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
}
__device__ __forceinline__ float lg_half(const uint32_t (&w)[4], int i) { return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); }

// Columns 8 j .. 8 j + 7 of a tile's part of a row (`row` points to its first column, `width` of its columns exist; none: nothing is stored), a thread each, the G threads of a
// row side by side in the warp.  A row that does not begin on 16 bytes is stored in the eights that do: a thread takes the end of its neighbour's
// values and the beginning of its own; the first one has the end of the last one's, and stores both edges in pieces of 8, 4 and 2 bytes.  (All threads of the warp call it together.)
template <int G, bool ALIGNED>
__device__ __forceinline__ void lg_put(uint16_t *row, int j, int width, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = lin_pair(v[2 * i], v[2 * i + 1]);
    const int s = ALIGNED ? 0 : (int)((reinterpret_cast<uintptr_t>(row) >> 1) & 7u);
    if (!ALIGNED) {
        uint32_t c[9];
        const int before = ((threadIdx.x & 31) & ~(G - 1)) | ((j - 1) & (G - 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) { c[i] = __shfl_sync(0xFFFFFFFFu, w[i], before); c[i + 4] = w[i]; }
        lg_shift(c, 8 - s, w);
    }
    auto one_by_one = [&](uint16_t *p, int lo, int hi) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k >= lo && k < hi) p[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
    };
    uint16_t *p = row + 8 * j - s;
    const int hi = width - (8 * j - s) < 8 ? width - (8 * j - s) : 8;
    if (ALIGNED || s == 0 || j > 0) {
        if (hi == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else one_by_one(p, 0, hi);
    } else {
        if (hi == 8 && width > 0) {                                    // places s .. 7 of the first eight
            if (s & 1) p[s] = (uint16_t)((s & 4 ? (s & 2 ? w[3] : w[2]) : (s & 2 ? w[1] : w[0])) >> 16);
            const int e = s + (s & 1);
            if (e & 2) *reinterpret_cast<uint32_t *>(p + e) = e & 4 ? w[3] : w[1];
            if (e <= 4) *reinterpret_cast<uint2 *>(p + 4) = make_uint2(w[2], w[3]);
        } else one_by_one(p, s, hi);
        p = row + 8 * G - s;                                           // places 0 .. s - 1 of the eight behind the last one
        if (width >= 8 * G) {
            if (s & 4) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
            if (s & 2) *reinterpret_cast<uint32_t *>(p + (s & 4)) = s & 4 ? w[2] : w[0];
            if (s & 1) p[s - 1] = (uint16_t)(s & 4 ? (s & 2 ? w[3] : w[2]) : (s & 2 ? w[1] : w[0]));
        } else one_by_one(p, 0, width - (8 * G - s) < s ? width - (8 * G - s) : s);
    }
}

// The tokens t0 + q * every below `end`, CT of them at a time, of the tile's output columns from col0 on, by thread e of LG_FINISH * 32, which keeps its eight columns.
// exchange(c) brings the sums of the tokens q = c .. c + CT - 1 to where read(q, lane, v) finds eight of them (false: gave up).  The residual is fetched a
// round ahead, the first one in front of the wait for the sums (4096 x 11008, 2048 tokens, 155 -> 149 us).
template <int FORM, int CT, bool ALIGNED, class Exchange, class Read>
__device__ __forceinline__ void lg_out_as(const LgArgs &a, int64_t t0, int every, int64_t end, int64_t col0, int e, Exchange exchange, Read read) {
    constexpr int OUT = FORM == LG_GATED ? LG_M / 2 : LG_M, G = OUT / 8, PASS = LG_FINISH * 32 / G, ITEMS = CT > PASS ? CT / PASS : 1;
    static_assert(CT % PASS == 0 || CT < PASS, "");
    const int q0 = e / G, j = e % G, part = a.width - col0 < OUT ? (int)(a.width - col0) : OUT, count = part - 8 * j < 8 ? part - 8 * j : 8;
    uint32_t bias[4], res[ITEMS][4], next[ITEMS][4];
    auto fetch = [&](int c) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int64_t t = t0 + (int64_t)(c + k * PASS + q0) * every;
            if (q0 < CT && t < end && count > 0) lg_get(a.residual + t * a.ldr, col0 + 8 * j, a.width, ALIGNED, next[k]);
        }
    };
    if (FORM == LG_FORWARD && a.bias && count > 0) lg_get(a.bias, col0 + 8 * j, a.width, false, bias);
    if (FORM == LG_FORWARD && a.residual) fetch(0);
    for (int c = 0; t0 + (int64_t)c * every < end; c += CT) {
        if (FORM == LG_FORWARD && a.residual) {
#pragma unroll
            for (int k = 0; k < ITEMS; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) res[k][i] = next[k][i];
            fetch(c + CT);
        }
        if (!exchange(c)) return;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int q = q0 < CT ? k * PASS + q0 : 0;
            const int64_t t = t0 + (int64_t)(c + q) * every;
            const int width = q0 < CT && t < end ? part : 0;           // (a thread without a token stores nothing, but the other rows' threads may need it)
            if (ALIGNED && width <= 8 * j) continue;
            float v[8], u[8];
            read(c + q, 8 * j, v);
            if (FORM == LG_GATED) read(c + q, OUT + 8 * j, u);
            if (FORM == LG_FORWARD && a.bias) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += lg_half(bias, i);
            }
            if (FORM != LG_DX && a.z) lg_put<G, ALIGNED>(a.z + t * a.ldz + col0, j, width, v);
            if (FORM != LG_DX) lg_act(v, a.act);
            if (FORM == LG_GATED) {
                if (a.u) lg_put<G, ALIGNED>(a.u + t * a.ldz + col0, j, width, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= u[i];
            }
            if (FORM == LG_FORWARD && a.residual) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += lg_half(res[k], i);
            }
            if (FORM == LG_FORWARD && a.y_f32) {
                float *p = static_cast<float *>(a.y) + t * a.ldy + col0 + 8 * j;
                if (ALIGNED && width - 8 * j >= 8) {
                    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
                    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (8 * j + i < width) p[i] = v[i];
                }
            } else lg_put<G, ALIGNED>(static_cast<uint16_t *>(a.y) + t * a.ldy + col0, j, width, v);
        }
    }
}

template <int FORM, int CT, class Exchange, class Read>
__device__ __forceinline__ void lg_out(const LgArgs &a, int64_t t0, int every, int64_t end, int64_t col0, int e, Exchange exchange, Read read) {
    if (a.aligned) lg_out_as<FORM, CT, true>(a, t0, every, end, col0, e, exchange, read);
    else lg_out_as<FORM, CT, false>(a, t0, every, end, col0, e, exchange, read);
}

// Tiles in the order they are taken: the token tiles of one weight tile side by side, so that its weights come from L2 after the first.
struct LgTile { int m, n, product; };
__device__ __forceinline__ LgTile lg_tile(const LgArgs &a, int i) {
    const int per = a.tiles_m * a.tiles_n;
    LgTile t;
    t.product = i / per;
    i -= t.product * per;
    t.m = i / a.tiles_n;
    t.n = i - t.m * a.tiles_n;
    return t;
}

// Range-checked build: a place of the index that lies behind the last weight is recorded and skipped.
__device__ __forceinline__ bool lg_in_range(const LgArgs &a, int product, uint32_t at) {
#ifdef DBS_BOUNDS_CHECK
    if (at >= a.stored[product]) { *a.status = DBSPMSPV_ERR_INTERNAL; return false; }
#endif
    return true;
}

// CG thread blocks of a cluster per tile of CG * 128 x NT; C of them (CG = 1) share its K.
template <int FORM, int CG, int NT, int C>
__global__ void __cluster_dims__(CG * C, 1, 1) __launch_bounds__(lg_threads(FORM == LG_DW), NT <= 64 ? 2 : 1)
k_linear_gemm(const __grid_constant__ LgMaps maps, const __grid_constant__ LgArgs a) {
    namespace cg = cooperative_groups;
    static_assert(CG == 1 || (CG == 2 && C == 1 && NT == 256), "");
    static_assert(FORM != LG_DW || NT == 256, "");
    constexpr bool A_MN = FORM != LG_DX, B_MN = FORM == LG_DW;
    constexpr int STAGES = lg_stages(CG, NT), STAGE_BYTES = lg_stage_bytes(CG, NT), NB = NT / CG;     // NB: rows of operand B in this block's shared memory
    constexpr int FINISH = FORM == LG_DW ? LG_FINISH_DW : LG_FINISH;
    constexpr int TMEM_COLS = 2 * NT < 32 ? 32 : 2 * NT;
    constexpr int OUT = FORM == LG_GATED ? LG_M / 2 : LG_M;                                           // output columns of this block's tile
    static_assert(C == 1 || NT * LG_M * 4 <= STAGES * STAGE_BYTES, "a tile's sums, for the other thread blocks of the cluster, lie in the stages");
    extern __shared__ uint8_t s_raw[];
    __shared__ __align__(8) uint64_t s_full[STAGES], s_empty[STAGES], s_done[2], s_free[2];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_fail;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t stages = (smem_addr(s_raw) + 1023u) & ~1023u, exchange = stages + STAGES * STAGE_BYTES;
    const int rank = C > 1 ? (int)(blockIdx.x % C) : 0, half = CG > 1 ? (int)(blockIdx.x & 1) : 0;
    const int first = (int)(blockIdx.x / (CG * C)), step = (int)(gridDim.x / (CG * C)), n_tiles = a.tiles_m * a.tiles_n * a.products;
    const int kb_all = a.k_blocks * a.layers, kb0 = (int)((int64_t)kb_all * rank / C), kb1 = (int)((int64_t)kb_all * (rank + 1) / C);
    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&s_full[s], 1); mbar_init(&s_empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&s_done[s], 1); mbar_init(&s_free[s], FINISH * CG); }
        s_fail = 0;
        fence_barrier_init();
    }
    if (warp == 0 && lane < 4) asm volatile("prefetch.tensormap [%0];" ::"l"(lane & 2 ? &maps.b[lane & 1] : &maps.a[lane & 1]) : "memory");
    if (warp == 1) {
        if (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "n"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "n"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        }
    }
    tc_fence_before();
    if (CG > 1) cg::this_cluster().sync();                             // (the other block's barriers are there)
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_wait();
    if (warp == 0) {
        if (lane == 0) {                                               // ---- loads
            int issued = 0, s = 0;
            uint32_t phase = 1;                                        // (a barrier that nobody has arrived on: the phase before its first counts as complete)
            bool ok = true;
            for (int i = first; i < n_tiles && ok; i += step) {
                const LgTile t = lg_tile(a, i);
                const int m0 = (t.m * CG + half) * OUT, n0 = t.n * NT + half * NB;    // (gated: 64 rows of both layers)
                int layer = kb0 >= a.k_blocks, k = kb0 - layer * a.k_blocks;
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!lg_spin(&s_empty[s], phase, &s_fail, a.status)) { ok = false; break; }
                    const uint32_t pa = stages + s * STAGE_BYTES, pb = pa + LG_A_BYTES;
                    // (both blocks' copies are counted by the first one's barrier)
                    const uint32_t bar = CG > 1 ? cluster_addr(smem_addr(&s_full[s]), 0) : smem_addr(&s_full[s]);
                    if (half == 0) mbar_arrive_expect_tx(&s_full[s], CG * STAGE_BYTES);
                    if (FORM == LG_DW) {
#pragma unroll
                        for (int q = 0; q < LG_M / 64; ++q) tma_load_2d<CG>(pa + q * 8192, &maps.a[0], m0 + q * 64, k * LG_K, bar);
#pragma unroll
                        for (int q = 0; q < NB / 64; ++q) tma_load_2d<CG>(pb + q * 8192, &maps.b[t.product], n0 + q * 64, k * LG_K, bar);
                    } else {
                        if (FORM == LG_DX) tma_load_3d<CG>(pa, &maps.a[layer], 0, m0, k, bar);
                        else if (FORM == LG_FORWARD) tma_load_3d<CG>(pa, &maps.a[0], 0, k * LG_K, m0 / DC_ROWS, bar);
                        else {
                            tma_load_3d<CG>(pa, &maps.a[0], 0, k * LG_K, m0 / DC_ROWS, bar);
                            tma_load_3d<CG>(pa + LG_A_BYTES / 2, &maps.a[1], 0, k * LG_K, m0 / DC_ROWS, bar);
                        }
                        tma_load_2d<CG>(pb, &maps.b[layer], k * LG_K, n0, bar);
                    }
                    ++issued;
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                    if (++k == a.k_blocks) { k = 0; ++layer; }
                }
            }
            pdl_trigger();                                             // (the next kernel's blocks may begin where this one's end; what they read waits for all of this one)
            // Every stage is given back before the block may leave: the products' thread of a pair arrives in both blocks, and nothing may arrive in shared memory of a block that is gone.
            // (The accumulators' barriers do not tell: which of two commits arrives first in the other block is not said.  Stages that were never filled count as given back.)
            for (int q = 0; q < STAGES && ok; ++q) {
                ok = lg_spin(&s_empty[s], phase, &s_fail, a.status);
                if (++s == STAGES) { s = 0; phase ^= 1; }
            }
            if (!ok) {                                                 // gave up: the copies in flight land before the block ends
                if (CG == 1)
                    for (int q = issued < STAGES ? 0 : issued - STAGES; q < issued; ++q) (void)mbar_wait_bounded(&s_full[q % STAGES], (uint32_t)((q / STAGES) & 1), 1 << 16);
                else                                                   // (the barrier that counts them may be the other block's: far longer than a copy takes)
                    for (int q = 0; q < 2000; ++q) __nanosleep(1000);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && half == 0) {                                  // ---- products
            constexpr uint32_t idesc = lg_idesc(CG * LG_M, NT, A_MN, B_MN);
            const uint32_t low_a = lg_desc_low(stages, A_MN), low_b = lg_desc_low(stages + LG_A_BYTES, B_MN);
            int s = 0, n = 0, last = -1;
            uint32_t phase = 0;
            bool ok = true;
            for (int i = first; i < n_tiles && ok; i += step, ++n) {
                const uint32_t d = tmem + (uint32_t)(n & 1) * NT;
                if (n >= 2 && !lg_spin(&s_free[n & 1], (uint32_t)((n / 2 - 1) & 1), &s_fail, a.status)) { ok = false; break; }
                tc_fence_after();
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!lg_spin(&s_full[s], phase, &s_fail, a.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t pa = low_a + s * (STAGE_BYTES >> 4), pb = low_b + s * (STAGE_BYTES >> 4);
#pragma unroll
                    for (int k = 0; k < LG_K / 16; ++k)
                        tc_mma<CG>(d, pa + k * ((A_MN ? 2048 : 32) >> 4), pb + k * ((B_MN ? 2048 : 32) >> 4), LG_DESC_HIGH, idesc, kb > kb0 || k > 0);
                    tc_commit<CG>(&s_empty[s]);
                    last = s;
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                }
                if (ok) tc_commit<CG>(&s_done[n & 1]);
            }
            if (!ok && last >= 0)                                      // gave up: the products in flight end before the accumulators are given back
                (void)mbar_wait_bounded(&s_empty[last], phase ^ (last == STAGES - 1 ? 1u : 0u), 1 << 16);
        }
    } else {                                                           // ---- accumulators: warp w reads the lanes 32 (w % 4) ...
        const int quad = warp & 3, group = (warp - 2) >> 2, e = tid - 64;
        const uint32_t mine = tmem + ((uint32_t)(quad * 32) << 16);
        int n = 0, turn = 0;
        uint2 ahead[NT / FINISH / 8 + 1];                              // (gradient of W)
        for (int i = first; i < n_tiles; i += step, ++n) {
            const LgTile t = lg_tile(a, i);
            const uint32_t d = mine + (uint32_t)(n & 1) * NT;
            if constexpr (FORM == LG_DW && C > 1) {
                // this block's sums into its own shared memory, [row][lane]
                if (!__all_sync(0xFFFFFFFFu, lg_wait(&s_done[n & 1], (uint32_t)((n / 2) & 1), &s_fail, a.status))) break;
                tc_fence_after();
                for (int c = group * 16; c < NT; c += FINISH / 4 * 16) {
                    float v[16];
                    tc_load16(d + c, v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) st_shared(stages + (uint32_t)((c + k) * LG_M + quad * 32 + lane) * 4, v[k]);
                }
            } else if constexpr (FORM == LG_DW) {
                // (the index of a warp's rows is fetched a tile ahead, the first one while the products run; it is read from the warp's own part of shared memory, two rows to a load
                // that all lanes share)
                constexpr int ROWS = NT / (FINISH / 4);
                uint16_t *dw = a.dw[t.product];
                const uint32_t below = (1u << lane) - 1u, own = exchange + (uint32_t)(warp - 2) * (ROWS * 8);
                uint2 x[ROWS / 32];
                auto fetch = [&](const LgTile &t) {
                    const int word = (t.m * CG + half) * (LG_M / 32) + quad;
                    const int64_t row0 = (int64_t)t.n * NT + group * ROWS;
                    const uint2 *index = a.index[t.product] + (int64_t)word * a.width;
#pragma unroll
                    for (int q = 0; q < ROWS / 32; ++q) ahead[q] = word < a.index_words && row0 + q * 32 + lane < a.width ? __ldg(index + row0 + q * 32 + lane) : make_uint2(0u, 0u);
                };
                if (n == 0) fetch(t);
#pragma unroll
                for (int q = 0; q < ROWS / 32; ++q) x[q] = ahead[q];
                if (i + step < n_tiles) fetch(lg_tile(a, i + step));
                __syncwarp();
#pragma unroll
                for (int q = 0; q < ROWS / 32; ++q) asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(own + (uint32_t)(q * 32 + lane) * 8), "r"(x[q].x), "r"(x[q].y) : "memory");
                __syncwarp();
                if (!__all_sync(0xFFFFFFFFu, lg_wait(&s_done[n & 1], (uint32_t)((n / 2) & 1), &s_fail, a.status))) break;
                tc_fence_after();
#pragma unroll 1
                for (int r = 0; r < ROWS; r += 16) {
                    float v[16];
                    uint32_t at[16], bits[16];                         // (all places first: the stores keep their order)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(bits[2 * k]), "=r"(at[2 * k]), "=r"(bits[2 * k + 1]), "=r"(at[2 * k + 1]) : "r"(own + (uint32_t)(r + 2 * k) * 8));
                        at[2 * k] += __popc(bits[2 * k] & below);
                        at[2 * k + 1] += __popc(bits[2 * k + 1] & below);
                    }
                    tc_load16(d + group * ROWS + r, v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t w = lin_pair(v[2 * k], v[2 * k + 1]);
                        store_if(((bits[2 * k] >> lane) & 1u) && lg_in_range(a, t.product, at[2 * k]), dw + at[2 * k], w & 0xFFFFu);
                        store_if(((bits[2 * k + 1] >> lane) & 1u) && lg_in_range(a, t.product, at[2 * k + 1]), dw + at[2 * k + 1], w >> 16);
                    }
                }
            } else {
                const int64_t t0 = (int64_t)t.n * NT, end = t0 + NT < a.tokens ? t0 + NT : a.tokens;
                auto done = [&] { return (bool)__all_sync(0xFFFFFFFFu, lg_wait(&s_done[n & 1], (uint32_t)((n / 2) & 1), &s_fail, a.status)); };
                if constexpr (C > 1) {
                    // this block's sums into its own shared memory, [token][lane]: every copy has landed and every product has been made
                    if (!done()) break;
                    tc_fence_after();
                    for (int c = group * 16; t0 + c < end; c += 32) {
                        float v[16];
                        tc_load16(d + c, v);
#pragma unroll
                        for (int k = 0; k < 16; ++k) st_shared(stages + (uint32_t)((c + k) * LG_M + quad * 32 + lane) * 4, v[k]);
                    }
                } else {
                    constexpr int CT = lg_tokens(NT), BUFFERS = lg_buffers(NT);
                    bool ok = true;
                    uint32_t buffer = exchange;
                    lg_out<FORM, CT>(a, t0, 1, end, (int64_t)(t.m * CG + half) * OUT, e, [&](int c) {
                        if (c == 0) {
                            ok = finish_all(done());                   // (all of them go on to the exchange, or none)
                            if (!ok) return false;
                            tc_fence_after();
                        } else if (BUFFERS == 1) finish_sync();        // (everybody has read the tokens before)
                        if (BUFFERS > 1) buffer = exchange + (uint32_t)(turn++ & 1) * (CT * LG_M * 4);
                        if (group * 16 < CT) {
                            float v[16];
                            tc_load16(d + c + group * 16, v);
#pragma unroll
                            for (int k = 0; k < 16; ++k) st_shared(buffer + (uint32_t)((group * 16 + k) * LG_M + quad * 32 + lane) * 4, v[k]);
                        }
                        finish_sync();
                        return true;
                    }, [&](int q, int l, float (&v)[8]) { ld_shared(buffer + (uint32_t)((q & (CT - 1)) * LG_M + l) * 4, v); });
                    if (!ok) break;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(cluster_addr(smem_addr(&s_free[n & 1]), CG > 1 ? 0 : rank));
        }
    }
    __syncwarp();
    if constexpr (C > 1 && FORM != LG_DW) {
        // (one tile per cluster)  Rank r adds up the C sums of every C-th token and finishes them.
        cg::this_cluster().sync();
        if (warp >= 2 && !s_fail && first < n_tiles) {
            const LgTile t = lg_tile(a, first);
            constexpr int CT = NT / C < lg_tokens(NT) ? NT / C : lg_tokens(NT);
            const int64_t t0 = (int64_t)t.n * NT, end = t0 + NT < a.tokens ? t0 + NT : a.tokens, col0 = (int64_t)t.m * OUT;
            const int e = tid - 64;
            // (through shared memory once more: a thread's eight sums from every rank directly are 32 bytes a lane of remote memory, 29.3 -> 33.4 us for the gradient of x and W at 64 tokens)
            lg_out<FORM, CT>(a, t0 + rank, C, end, col0, e, [&](int c) {
                finish_sync();                                         // (everybody has read the tokens before)
                for (int i = e; i < CT * LG_M / 4; i += LG_FINISH * 32) {
                    const int q = i / (LG_M / 4), l = i % (LG_M / 4) * 4;
                    float4 part[C];
#pragma unroll
                    for (int r = 0; r < C; ++r) part[r] = ld_cluster(cluster_addr(stages, r) + (uint32_t)((rank + (c + q) * C) * LG_M + l) * 4);
                    float4 v = part[0];
#pragma unroll
                    for (int r = 1; r < C; ++r) { v.x += part[r].x; v.y += part[r].y; v.z += part[r].z; v.w += part[r].w; }
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(exchange + (uint32_t)(q * LG_M + l) * 4), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
                }
                finish_sync();
                return true;
            }, [&](int q, int l, float (&v)[8]) { ld_shared(exchange + (uint32_t)((q & (CT - 1)) * LG_M + l) * 4, v); });
        }
        __syncwarp();
    }
    if constexpr (C > 1 && FORM == LG_DW) {
        // Rank r adds up the C sums of every C-th row and stores them; a warp has its 32 columns, eight rows at a time.
        cg::this_cluster().sync();
        if (warp >= 2 && !s_fail && first < n_tiles) {
            const LgTile t = lg_tile(a, first);
            const int quad = warp & 3, group = (warp - 2) >> 2, word = t.m * (LG_M / 32) + quad;
            const int64_t row0 = (int64_t)t.n * NT;
            const uint2 *index = a.index[t.product] + (int64_t)word * a.width;
            const uint32_t below = (1u << lane) - 1u, from = stages + (uint32_t)(quad * 32 + lane) * 4;
            uint16_t *dw = a.dw[t.product];
            for (int r0 = rank + C * group; r0 < NT && row0 + r0 < a.width && word < a.index_words; r0 += C * (FINISH / 4) * 8) {
                uint2 x[8];
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int r = r0 + k * C * (FINISH / 4);
                    x[k] = r < NT && row0 + r < a.width ? __ldg(index + row0 + r) : make_uint2(0u, 0u);
                    float part[C];
#pragma unroll
                    for (int q = 0; q < C; ++q) part[q] = ld_cluster1(cluster_addr(from, q) + (uint32_t)(r < NT ? r : 0) * (LG_M * 4));
                    v[k] = part[0];
#pragma unroll
                    for (int q = 1; q < C; ++q) v[k] += part[q];
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t at = x[k].y + __popc(x[k].x & below);
                    store_if(((x[k].x >> lane) & 1u) && lg_in_range(a, t.product, at), dw + at, lin_bf16(v[k]));
                }
            }
        }
        __syncwarp();
    }
    tc_fence_before();
    if (CG * C > 1) cg::this_cluster().sync();                         // (nobody reads this block's shared memory or works on its accumulators any more)
    else __syncthreads();
    tc_fence_after();
    if (warp == 1) {
        if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TMEM_COLS));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TMEM_COLS));
    }
}

}  // namespace dbs
