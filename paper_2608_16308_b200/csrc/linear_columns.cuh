// Linear and gated layers for single tokens (and a few): y = act(W x + bias) + residual, y = act(W_gate x) * (W_up x).
//
// One pass over the columns that the token reaches, from the copy by columns ([strip of 64 rows][column][row], see
// decode_columns.cuh): what the call cannot do without is 2 bytes per weight of those columns.  A cluster of C thread blocks owns a
// strip; a warp blocks its own share of x, keeps the entries that are not zero as a list (column and bf16 value in a word) in shared memory and goes on to
// their columns, 16 bytes a lane, all loads independent.  The sums of warps and ranks meet in shared memory, in a fixed order, and the
// thread of a row finishes it there, so that neither a second pass over y nor an atomic is needed.
//   * A gated call reads the same list against both layers' strips: both sums of a row end in one thread.
//   * Several tokens are several rows of the grid: their columns overlap in L2 (the rule on tokens is in linear.cu).
// The products are those of the matrix with zeros in the pruned places: a zero entry of x adds nothing (the weights are finite), one
// that is not finite reaches every row.
#pragma once

#include <cooperative_groups.h>

#include "linear_gemm.cuh"

namespace dbs {

constexpr int LC_WARPS = 16;             // (eight or four, and more thread blocks: no faster)
constexpr int LC_CTA = LC_WARPS * 32;
constexpr int LC_PIECE = 64;             // entries of x that a warp blocks side by side
static_assert(DC_ROWS == 64, "eight lanes with eight rows each share a column");

// entries of a warp's list, at most; the ranks and warps take the pieces of x in turn
__host__ __device__ inline int64_t lc_warp_entries(int64_t n, int c) {
    const int64_t pieces = (n + LC_PIECE - 1) / LC_PIECE;
    return (pieces + (int64_t)c * LC_WARPS - 1) / ((int64_t)c * LC_WARPS) * LC_PIECE;
}

struct LcArgs {
    const uint16_t *x;
    int64_t ldx, n, m;
    const uint4 *w[2];
    const uint16_t *bias, *residual;
    int64_t ldr;
    void *y;
    int64_t ldy;
    int y_f32, act;
    uint16_t *z, *u;
    int64_t ldz;
};

// Shared memory: the warps' lists, their sums [layer][warp][row], the sums of every rank [rank][layer][row]
__host__ __device__ inline int64_t lc_smem(int64_t n, int layers, int c) { return LC_WARPS * lc_warp_entries(n, c) * 4 + (LC_WARPS + c) * layers * DC_ROWS * 4; }

// Long lists of two layers are walked two rounds at a time: the loads of the second do not wait for the sums of the first (gated, calls of one size one behind the other, 11008 x 4096: 36.6 -> 31.7 us;
// 4096 x 11008: 32.2 -> 30.3; but 1037 x 515, eight tokens: 8.2 -> 9.5, and one layer gains nothing.  Among other calls the first takes 33.3 us, 5.4 TB/s).
constexpr int LC_LONG_LIST = 128;        // entries of a warp, where none of x is zero
template <int LAYERS, int C, int ROUNDS>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(LC_CTA, 2)
k_linear_cols(const __grid_constant__ LcArgs a, int strips) {
    namespace cg = cooperative_groups;
    constexpr int ILP = 8 / LAYERS;                                   // columns in flight per lane: 4 KB per warp
    extern __shared__ __align__(16) uint8_t s_dyn[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = C > 1 ? (int)(blockIdx.x % C) : 0, unit = (int)(blockIdx.x / C);
    const int64_t token = unit / strips;
    // (What differs is what the compiler makes of the loop under 64 registers.  Behind the remainder, the gated kernels of short lists spill 24 to 64 bytes and keep all loads of a round in flight; behind the
    // product they fit, and wait for memory twice as long: stalls for it 4.6 in place of 2.5 per instruction, 1000 x 2000 8.4 in place of 7.0 us.  Those of long lists spill up to
    // 112 bytes behind the remainder and none behind the product: 4096 x 11008 32.7 and 30.3 us.)
    const int strip = ROUNDS == 1 ? unit % strips : unit - (int)token * strips;
    // (a cluster: every block has started before its shared memory is written; met again behind the weights)
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    pdl_wait();
    const uint16_t *x = a.x + token * a.ldx;
    float (*s_part)[LC_WARPS][DC_ROWS] = reinterpret_cast<float (*)[LC_WARPS][DC_ROWS]>(s_dyn + (size_t)LC_WARPS * lc_warp_entries(a.n, C) * 4);
    float (*s_sum)[LAYERS][DC_ROWS] = reinterpret_cast<float (*)[LAYERS][DC_ROWS]>(s_part + LAYERS);
    uint32_t *list = reinterpret_cast<uint32_t *>(s_dyn) + (size_t)warp * lc_warp_entries(a.n, C);
    int n = 0;
    {
        const bool aligned = (reinterpret_cast<uintptr_t>(x) & 3u) == 0;
        for (int64_t j0 = ((int64_t)warp * C + rank) * LC_PIECE; j0 < a.n; j0 += (int64_t)LC_WARPS * C * LC_PIECE) {
            const int64_t j = j0 + 2 * lane;
            uint32_t v = 0;
            if (aligned && j + 1 < a.n) v = *reinterpret_cast<const uint32_t *>(x + j);
            else {
                if (j < a.n) v = x[j];
                if (j + 1 < a.n) v |= (uint32_t)x[j + 1] << 16;
            }
            const bool lo = v & 0x7FFFu, hi = v & 0x7FFF0000u;
            const uint32_t ml = __ballot_sync(FULL, lo), mh = __ballot_sync(FULL, hi), below = (1u << lane) - 1u;
            int at = n + __popc(ml & below) + __popc(mh & below);
            if (lo) list[at++] = (uint32_t)j | v << 16;
            if (hi) list[at] = (uint32_t)(j + 1) | (v & 0xFFFF0000u);
            n += __popc(ml) + __popc(mh);
        }
        __syncwarp();
    }
    pdl_trigger();
    {
        const uint4 *w[LAYERS];
#pragma unroll
        for (int l = 0; l < LAYERS; ++l) w[l] = a.w[l] + (size_t)strip * a.n * (DC_ROWS / 8) + (lane & 7);
        float acc[LAYERS][8];
#pragma unroll
        for (int l = 0; l < LAYERS; ++l)
#pragma unroll
            for (int r = 0; r < 8; ++r) acc[l][r] = 0.f;
#pragma unroll ROUNDS
        for (int k0 = 0; k0 < n; k0 += 4 * ILP) {
            uint4 v[LAYERS][ILP];
            float xv[ILP];
#pragma unroll
            for (int q = 0; q < ILP; ++q) {
                const int k = k0 + q * 4 + (lane >> 3);
                xv[q] = 0.f;
#pragma unroll
                for (int l = 0; l < LAYERS; ++l) v[l][q] = make_uint4(0u, 0u, 0u, 0u);
                if (k < n) {
                    const uint32_t e = list[k];
                    xv[q] = __uint_as_float(e & 0xFFFF0000u);
#pragma unroll
                    for (int l = 0; l < LAYERS; ++l) v[l][q] = __ldcs(w[l] + (size_t)(e & 0xFFFFu) * (DC_ROWS / 8));
                }
            }
#pragma unroll
            for (int q = 0; q < ILP; ++q)
#pragma unroll
                for (int l = 0; l < LAYERS; ++l) {
                    const uint32_t p[4] = {v[l][q].x, v[l][q].y, v[l][q].z, v[l][q].w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        acc[l][2 * r] += __uint_as_float(p[r] << 16) * xv[q];
                        acc[l][2 * r + 1] += __uint_as_float(p[r] & 0xFFFF0000u) * xv[q];
                    }
                }
        }
        // sums over the four column slots of the warp: two halving exchanges leave two rows per lane
        const bool h16 = lane & 16, h8 = lane & 8;
#pragma unroll
        for (int l = 0; l < LAYERS; ++l) {
            float a4[4], a2[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) a4[i] = (h16 ? acc[l][i + 4] : acc[l][i]) + __shfl_xor_sync(FULL, h16 ? acc[l][i] : acc[l][i + 4], 16);
#pragma unroll
            for (int i = 0; i < 2; ++i) a2[i] = (h8 ? a4[i + 2] : a4[i]) + __shfl_xor_sync(FULL, h8 ? a4[i] : a4[i + 2], 8);
            *reinterpret_cast<float2 *>(&s_part[l][warp][(lane & 7) * 8 + (h16 ? 4 : 0) + (h8 ? 2 : 0)]) = make_float2(a2[0], a2[1]);
        }
    }
    __syncthreads();
    float sum = 0.f;                                                  // thread (layer, row)
    const int layer = tid / DC_ROWS, r = tid % DC_ROWS;
    if (layer < LAYERS) {
#pragma unroll
        for (int k = 0; k < LC_WARPS; ++k) sum += s_part[layer][k][r];
    }
    if (C > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (layer < LAYERS) cluster.map_shared_rank(&s_sum[0][0][0], 0)[(rank * LAYERS + layer) * DC_ROWS + r] = sum;
        cluster.sync();
        if (rank != 0) return;
    } else if (LAYERS > 1) {
        if (layer < LAYERS) s_sum[0][layer][r] = sum;
        __syncthreads();
    }
    const int64_t row = (int64_t)strip * DC_ROWS + tid;
    if (tid >= DC_ROWS || row >= a.m) return;
    float z = sum, up = 0.f;
    if (C > 1 || LAYERS > 1) {
        z = 0.f;
#pragma unroll
        for (int q = 0; q < C; ++q) {
            z += s_sum[q][0][tid];
            if (LAYERS > 1) up += s_sum[q][LAYERS - 1][tid];
        }
    }
    if (a.bias) z += lin_f32(a.bias[row]);
    if (a.z) a.z[token * a.ldz + row] = (uint16_t)lin_bf16(z);
    float y = lin_act(z, a.act);
    if (LAYERS > 1) {
        if (a.u) a.u[token * a.ldz + row] = (uint16_t)lin_bf16(up);
        y *= up;
    }
    if (a.residual) y += lin_f32(a.residual[token * a.ldr + row]);
    if (a.y_f32) static_cast<float *>(a.y)[token * a.ldy + row] = y;
    else static_cast<uint16_t *>(a.y)[token * a.ldy + row] = (uint16_t)lin_bf16(y);
}

}  // namespace dbs
