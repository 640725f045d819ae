// Linear and gated feed-forward layers over pruned bf16 weights, from one token to a prompt, with their gradients
// (Section 4.3's layers with what stands around their product in a network): entry points, the choice of kernel, and the
// small kernels beside the products.  The products: linear_columns.cuh (single tokens), linear_gemm.cuh (tensor cores).
#include <cub/cub.cuh>

#include "call_graph.cuh"
#include "internal.cuh"
#include "microkernels.cuh"
#include "linear_columns.cuh"
#include "linear_gemm.cuh"
#include "linear_plan.h"

namespace dbs {

constexpr int LIN_COLS_MAX_SMEM = 200 * 1024;
// Tokens that a call over active columns takes one by one, side by side in the grid; more go to the tensor cores.
constexpr int LIN_COLS_MAX_TOKENS = 2;
constexpr int64_t LIN_COLS_MAX_WEIGHTS = 16ll << 20;

// ---- at create ------------------------------------------------------------------------------
// Stored columns of a row, 32 to a word, from the copy by columns; a warp takes the 32 rows of half a strip.
__global__ void k_linear_words(const uint16_t *w, int64_t m, int64_t n, int words, uint2 *index, int32_t *count) {
    const int64_t warp = (blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    const int64_t half = warp / words, row = half * 32 + lane;
    const int word = (int)(warp % words);
    if (row >= m) return;
    const uint16_t *p = w + ((row / DC_ROWS) * n + (int64_t)word * 32) * DC_ROWS + row % DC_ROWS;
    uint32_t bits = 0;
    for (int c = 0; c < 32; ++c)
        if ((int64_t)word * 32 + c < n && p[(int64_t)c * DC_ROWS] != DC_ABSENT) bits |= 1u << c;
    index[word * m + row].x = bits;
    count[row * words + word] = __popc(bits);
}
// (counted row by row, kept word by word: a tile of the gradient takes the rows of one word side by side)
__global__ void k_linear_places(int64_t m, int words, const int32_t *first, uint2 *index) {
    const int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
    if (i < m * words) index[i].y = (uint32_t)first[i % m * words + i / m];
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
    static EncodeTiled f = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) { (void)cudaGetLastError(); p = nullptr; }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}
// bf16, the first dimension 64 entries of a box (the 128 bytes of a swizzle row); places outside are read as zeros
static int encode(CUtensorMap *map, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box) {
    const cuuint32_t ones[3] = {1, 1, 1};
    EncodeTiled f = encode_tiled();
    if (!f) return DBSPMSPV_ERR_CUDA;
    return f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? DBSPMSPV_OK : DBSPMSPV_ERR_CUDA;
}
// `rows` rows of `width` entries, ld entries apart; a box holds 64 entries of box_rows rows
static int encode_rows(CUtensorMap *map, const uint16_t *p, int64_t rows, int64_t width, int64_t ld, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    return encode(map, p, 2, dims, strides, box);
}
// the copy by columns: 64 rows of a strip, `cols` columns, `strips` strips
static int encode_weights(CUtensorMap *map, const dbspmspv_handle_s *h, int cols, int strips) {
    const cuuint64_t dims[3] = {(cuuint64_t)DC_ROWS, (cuuint64_t)h->d.n, (cuuint64_t)((h->d.m + DC_ROWS - 1) / DC_ROWS)};
    const cuuint64_t strides[2] = {DC_ROWS * 2, (cuuint64_t)h->d.n * DC_ROWS * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)cols, (cuuint32_t)strips};
    return encode(map, h->lin_w, 3, dims, strides, box);
}
int linear_handle_maps(dbspmspv_handle_s *h) {
    int s = encode_weights(&h->lin_maps[0], h, LG_K, LG_M / DC_ROWS);
    if (s == DBSPMSPV_OK) s = encode_weights(&h->lin_maps[1], h, LG_K, LG_M / DC_ROWS / 2);
    if (s == DBSPMSPV_OK) s = encode_weights(&h->lin_maps[2], h, LG_M, 1);
    return s;
}

// Behind the copy by columns: the index of the stored weights by row.
int build_linear_index(dbspmspv_handle_s *h, cudaStream_t st) {
    const int64_t m = h->d.m, n = h->d.n;
    const int words = (int)((n + 31) / 32);
    const int64_t items = m * words;
    uint2 *index = nullptr;
    int32_t *count = nullptr, *first = nullptr;
    void *tmp = nullptr;
    size_t bytes = 0;
    int s = DBSPMSPV_OK;
    if (cudaMalloc(&index, (size_t)items * sizeof(uint2)) != cudaSuccess) { (void)cudaGetLastError(); return DBSPMSPV_ERR_ALLOC; }
    h->lin_index = index;
    h->lin_words = words;
    if (cub::DeviceScan::ExclusiveSum(nullptr, bytes, count, first, items, st) != cudaSuccess) return DBSPMSPV_ERR_CUDA;
    if (cudaMalloc(&count, (size_t)items * 4) != cudaSuccess || cudaMalloc(&first, (size_t)items * 4) != cudaSuccess || cudaMalloc(&tmp, bytes ? bytes : 1) != cudaSuccess) s = DBSPMSPV_ERR_ALLOC;
    if (s == DBSPMSPV_OK) {
        const int64_t threads = (m + 31) / 32 * words * 32;
        k_linear_words<<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(h->lin_w, m, n, words, index, count);
        if (cub::DeviceScan::ExclusiveSum(tmp, bytes, count, first, items, st) != cudaSuccess) s = DBSPMSPV_ERR_CUDA;
        k_linear_places<<<(unsigned)((items + 255) / 256), 256, 0, st>>>(m, words, first, index);
        if (cudaStreamSynchronize(st) != cudaSuccess) s = DBSPMSPV_ERR_CUDA;
    }
    cudaFree(count); cudaFree(first); cudaFree(tmp);
    if (s != DBSPMSPV_OK) (void)cudaGetLastError();
    return s;
}

// ---- beside the products --------------------------------------------------------------------
// (rows of a workspace buffer begin on 16 bytes and are padded to a multiple of eight entries)
__device__ __forceinline__ void lin_store8(uint16_t *row, int64_t j, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = lin_pair(v[2 * k], v[2 * k + 1]);
    *reinterpret_cast<uint4 *>(row + j) = make_uint4(w[0], w[1], w[2], w[3]);
}

// x whose rows TMA cannot address, with rows that it can, by thread blocks `block` of `blocks`
struct LinPack {
    const uint16_t *x;
    int64_t ldx, tokens, n;
    uint16_t *out;
    int64_t ldo;
};
__device__ __forceinline__ void lin_pack(const LinPack &a, int64_t block, int64_t blocks) {
    const int64_t per = a.ldo / 8, total = a.tokens * per;
    for (int64_t i = block * blockDim.x + threadIdx.x; i < total; i += blocks * blockDim.x) {
        const int64_t t = i / per, j = (i - t * per) * 8;
        uint32_t w[4];
        lg_get(a.x + t * a.ldx, j, a.n, false, w);
        *reinterpret_cast<uint4 *>(a.out + t * a.ldo + j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__global__ void k_linear_pack(const __grid_constant__ LinPack a) {
    pdl_wait();
    lin_pack(a, blockIdx.x, gridDim.x);
    pdl_trigger();
}

// What the products of a gradient take: dz = dy act'(z), or dg = dy u act'(g) and du = dy act(g), rounded to bf16 (the tensor cores' operands; the
// roundings are independent, so a sum over rows or tokens is off by about 2^-9 of its own size, as much as its own rounding to bf16), and the bias' gradient
// from the unrounded ones.  Bound by HBM: 2 bytes for each of dy, z, u, dz.  The thread blocks from pack_from on pack x meanwhile.
constexpr int LS_CTA = 256;
constexpr int LS_COLS = 32;              // columns of a thread block that adds up the bias' gradient: four threads, 64 tokens side by side
struct LsArgs {
    const uint16_t *dy, *z, *u;
    int64_t lddy, ldz, tokens, m;
    int act;
    uint16_t *d0, *d1;              // null: not wanted
    int64_t ldd;
    float *dbias;
    int aligned;                    // every row of dy, z and u begins on 16 bytes
    int pack_from;
    LinPack pack;
};
__device__ __forceinline__ void ls_unpack(const uint32_t (&w)[4], float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = lg_half(w, k);
}
// eight neighbours of one token: dy becomes du (gated) or dz; d: dg
template <bool GATED>
__device__ __forceinline__ void ls_eight(const LsArgs &a, float (&dy)[8], const float (&z)[8], const float (&u)[8], float (&d)[8]) {
    if (a.act == DBSPMSPV_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float p = lin_sigmoid_fast(z[k]), slope = p * (1.f + z[k] * (1.f - p));
            if (GATED) { d[k] = dy[k] * u[k] * slope; dy[k] *= z[k] * p; } else dy[k] *= slope;
        }
    } else if (a.act == DBSPMSPV_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float p = lin_phi(z[k]), slope = p + z[k] * (0.39894228f * __expf(-0.5f * z[k] * z[k]));
            if (GATED) { d[k] = dy[k] * u[k] * slope; dy[k] *= z[k] * p; } else dy[k] *= slope;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool relu = a.act == DBSPMSPV_ACT_RELU;
            const float slope = relu && !(z[k] > 0.f) ? 0.f : 1.f;
            if (GATED) { d[k] = dy[k] * u[k] * slope; dy[k] *= relu ? lin_act(z[k], DBSPMSPV_ACT_RELU) : z[k]; } else dy[k] *= slope;
        }
    }
}
template <bool GATED>
__global__ void __launch_bounds__(LS_CTA) k_linear_slopes(const __grid_constant__ LsArgs a) {
    pdl_wait();
    if ((int)blockIdx.x >= a.pack_from) {
        lin_pack(a.pack, (int)blockIdx.x - a.pack_from, (int)gridDim.x - a.pack_from);
    } else {
        // (two at a time: what is loaded for both is under way before either is worked on)
        const int64_t per = (a.m + 7) / 8, total = a.tokens * per, step = (int64_t)a.pack_from * LS_CTA;
        for (int64_t i0 = blockIdx.x * (int64_t)LS_CTA + threadIdx.x; i0 < total; i0 += 2 * step) {
            uint32_t wy[2][4], wz[2][4] = {}, wu[2][4] = {};
            int64_t t[2], j[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int64_t i = i0 + q * step;
                t[q] = i / per;
                j[q] = (i - t[q] * per) * 8;
                if (i < total) {
                    lg_get(a.dy + t[q] * a.lddy, j[q], a.m, a.aligned, wy[q]);
                    if (GATED || a.z) lg_get(a.z + t[q] * a.ldz, j[q], a.m, a.aligned, wz[q]);
                    if (GATED) lg_get(a.u + t[q] * a.ldz, j[q], a.m, a.aligned, wu[q]);
                }
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if (i0 + q * step >= total) break;
                float dy[8], z[8], u[8], d[8];
                ls_unpack(wy[q], dy);
                ls_unpack(wz[q], z);
                ls_unpack(wu[q], u);
                if (GATED || a.z) ls_eight<GATED>(a, dy, z, u, d);
                if (GATED) lin_store8(a.d0 + t[q] * a.ldd, j[q], d);
                lin_store8((GATED ? a.d1 : a.d0) + t[q] * a.ldd, j[q], dy);
            }
        }
    }
    pdl_trigger();
}
// With the bias' gradient: a thread block takes LS_COLS columns of all tokens; its sums meet in a fixed order.
__global__ void __launch_bounds__(LS_CTA) k_linear_bias(const __grid_constant__ LsArgs a) {
    constexpr int G = LS_COLS / 8, LANES = LS_CTA / G;
    __shared__ float s_sum[LS_CTA / 32][LS_COLS];
    const int tid = threadIdx.x;
    pdl_wait();
    if ((int)blockIdx.x >= a.pack_from) {
        lin_pack(a.pack, (int)blockIdx.x - a.pack_from, (int)gridDim.x - a.pack_from);
        pdl_trigger();
        return;
    }
    const int64_t j = (int64_t)blockIdx.x * LS_COLS + (tid % G) * 8;
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.f;
    for (int64_t t0 = tid / G; t0 < a.tokens && j < a.m; t0 += 4 * LANES) {
        uint32_t wy[4][4] = {}, wz[4][4] = {};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t t = t0 + q * LANES;
            if (t < a.tokens) {
                lg_get(a.dy + t * a.lddy, j, a.m, a.aligned, wy[q]);
                if (a.z) lg_get(a.z + t * a.ldz, j, a.m, a.aligned, wz[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t t = t0 + q * LANES;
            if (t >= a.tokens) break;
            float dy[8], z[8], none[8];
            ls_unpack(wy[q], dy);
            ls_unpack(wz[q], z);
            if (a.z) ls_eight<false>(a, dy, z, z, none);
            if (a.d0) lin_store8(a.d0 + t * a.ldd, j, dy);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += dy[k];
        }
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
#pragma unroll
        for (int o = G; o < 32; o <<= 1) sum[k] += __shfl_xor_sync(FULL, sum[k], o);
        if ((tid & 31) < G) s_sum[tid >> 5][(tid % G) * 8 + k] = sum[k];
    }
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * LS_COLS + tid;
    if (tid < LS_COLS && col < a.m) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < LS_CTA / 32; ++k) v += s_sum[k][tid];
        a.dbias[col] = v;
    }
    pdl_trigger();
}

// ---- launches -------------------------------------------------------------------------------
static int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
static bool tma_rows(const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld & 7) == 0; }

template <int FORM, int CG, int NT, int C>
static int add_gemm_as(dbspmspv_handle_s *h, CallList &calls, const LgMaps &maps, const LgArgs &a, int grid) {
    bool &done = h->lin_configured[FORM][CG - 1][NT / 64][C];
    if (!done) {
        DBS_CUDA(cudaFuncSetAttribute(k_linear_gemm<FORM, CG, NT, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, lg_smem(CG, NT)));
        done = true;
    }
    calls.add(k_linear_gemm<FORM, CG, NT, C>, grid, lg_threads(FORM == LG_DW), lg_smem(CG, NT), calls.n > 0, maps, a);
    return DBSPMSPV_OK;
}
template <int FORM>
static int add_gemm(dbspmspv_handle_s *h, CallList &calls, const LgMaps &maps, const LgArgs &a, LgPlan p) {
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n * a.products;
    if (tiles >= (1ll << 27)) return DBSPMSPV_ERR_UNSUPPORTED;
    const int slots = h->sm_count * (p.nt <= 64 ? 2 : 1) / p.cg, grid = (int)(tiles < slots ? tiles : slots) * p.cg;
    if (p.cg == 2) return add_gemm_as<FORM, 2, 256, 1>(h, calls, maps, a, grid);
    if constexpr (FORM == LG_DW) {
        switch (p.c) {
            case 1: return add_gemm_as<FORM, 1, 256, 1>(h, calls, maps, a, grid);
            case 2: return add_gemm_as<FORM, 1, 256, 2>(h, calls, maps, a, (int)tiles * 2);
            case 4: return add_gemm_as<FORM, 1, 256, 4>(h, calls, maps, a, (int)tiles * 4);
            default: return add_gemm_as<FORM, 1, 256, 8>(h, calls, maps, a, (int)tiles * 8);
        }
    } else {
#define LG_CASE(NT, C) if (p.nt == NT && p.c == C) return add_gemm_as<FORM, 1, NT, C>(h, calls, maps, a, C > 1 ? (int)tiles * C : grid);
        LG_TILES(LG_CASE)
#undef LG_CASE
        return DBSPMSPV_ERR_CUDA;
    }
}
// whether every row of the outputs and of the residual begins on 16 bytes (LgArgs::aligned)
static int aligned_rows(const LgArgs &a) {
    auto fits = [](const void *p, int64_t ld, int64_t item) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * item % 16 == 0); };
    return fits(a.y, a.ldy, a.y_f32 ? 4 : 2) && fits(a.z, a.ldz, 2) && fits(a.u, a.ldz, 2) && fits(a.residual, a.ldr, 2);
}
template <int LAYERS, int C, int ROUNDS = 1>
static int add_columns_c(dbspmspv_handle_s *h, CallList &calls, const LcArgs &a, int strips, int tokens) {
    if constexpr (LAYERS == 2 && ROUNDS == 1)
        if (lc_warp_entries(a.n, C) >= LC_LONG_LIST) return add_columns_c<LAYERS, C, 2>(h, calls, a, strips, tokens);
    bool &done = h->lin_cols_configured[LAYERS + ROUNDS - 2][C];
    if (!done) {
        DBS_CUDA(cudaFuncSetAttribute(k_linear_cols<LAYERS, C, ROUNDS>, cudaFuncAttributeMaxDynamicSharedMemorySize, LIN_COLS_MAX_SMEM));
        done = true;
    }
    calls.add(k_linear_cols<LAYERS, C, ROUNDS>, strips * C * tokens, LC_CTA, (size_t)lc_smem(a.n, LAYERS, C), false, a, strips);
    return DBSPMSPV_OK;
}
// Thread blocks of a strip: doubled, up to eight, until there are more of them than SMs.  (4096 x 11008, half active, 1 / 2 / 4 / 8 blocks: 20.3 / 14.4 / 12.0 / 14.9 us; 12288 x 4096,
// dense: 19.4 / 23.2 / 22.9 / 31.8.)
static int columns_cluster(const dbspmspv_handle_s *h, int64_t tokens) {
    const int64_t units = (h->d.m + DC_ROWS - 1) / DC_ROWS * tokens;
    int c = 1;
    while (c < 8 && units * c <= h->sm_count) c *= 2;
    return c;
}
template <int LAYERS>
static int add_columns(dbspmspv_handle_s *h, CallList &calls, const LcArgs &a, int tokens) {
    const int strips = (int)((a.m + DC_ROWS - 1) / DC_ROWS);
    switch (columns_cluster(h, tokens)) {
        case 1: return add_columns_c<LAYERS, 1>(h, calls, a, strips, tokens);
        case 2: return add_columns_c<LAYERS, 2>(h, calls, a, strips, tokens);
        case 4: return add_columns_c<LAYERS, 4>(h, calls, a, strips, tokens);
        default: return add_columns_c<LAYERS, 8>(h, calls, a, strips, tokens);
    }
}
// Whether a forward call goes over the columns: up to LIN_COLS_MAX_TOKENS tokens; and small layers whose x would have to be packed for the tensor cores (a kernel more), as long as the tokens'
// passes over the weights are few bytes (1037 x 515, eight tokens: 5.8 against 8.5 us; 2751 x 1025, five: 6.0 / 8.9, six are past it; gated 1037 x 515, eight: 6.1 / 8.7,
// but 1500 x 1500, three: 11.2 / 8.8).
static bool over_columns(const dbspmspv_handle_s *h, int layers, int64_t tokens, bool packed) {
    if (h->d.n > 65536 || lc_smem(h->d.n, layers, columns_cluster(h, tokens)) > LIN_COLS_MAX_SMEM) return false;
    return tokens <= LIN_COLS_MAX_TOKENS || (packed && tokens <= 16 && tokens * layers * layers * h->d.m * h->d.n <= LIN_COLS_MAX_WEIGHTS);
}

// ---- workspace: x as TMA can read it, then the products' operands of a gradient ---------------
struct LinRoom {
    uint8_t *at;
    int64_t left;
    uint16_t *take(int64_t rows, int64_t ld) {
        const int64_t bytes = round_up(rows * ld * 2, 256);
        if (!at || left < bytes) return nullptr;
        uint8_t *p = at;
        at += bytes;
        left -= bytes;
        return reinterpret_cast<uint16_t *>(p);
    }
};
static int64_t workspace_bytes(const dbspmspv_handle_s *h, int layers, int64_t tokens, bool backward) {
    int64_t b = 0;
    if (backward || !over_columns(h, layers, tokens, false)) b += round_up(tokens * round_up(h->d.n, 8) * 2, 256);
    if (backward) b += layers * round_up(tokens * round_up(h->d.m, 8) * 2, 256);
    return b;
}

// x as the tensor maps can address it: as it lies (p.out null), or packed into the workspace by a kernel to come
static int usable_x(const dbspmspv_handle_s *h, const uint16_t **x, int64_t *ldx, int tokens, LinRoom &room, LinPack *p) {
    *p = LinPack{};
    if (tma_rows(*x, *ldx)) return DBSPMSPV_OK;
    const int64_t n = h->d.n, ld = round_up(n, 8);
    uint16_t *out = room.take(tokens, ld);
    if (!out) return DBSPMSPV_ERR_INVALID_ARG;
    *p = LinPack{*x, *ldx, tokens, n, out, ld};
    *x = out;
    *ldx = ld;
    return DBSPMSPV_OK;
}
static int pack_blocks(const dbspmspv_handle_s *h, const LinPack &p) {
    if (!p.out) return 0;
    const int64_t g = (p.tokens * (p.ldo / 8) + LS_CTA - 1) / LS_CTA, most = 16 * h->sm_count;
    return (int)(g < most ? g : most);
}

static bool has_linear(const dbspmspv_handle_s *h) { return h->d.dtype == DBSPMSPV_BF16 && h->lin_ready; }

struct LinForward {
    const uint16_t *x;
    int64_t ldx;
    int tokens;
    const uint16_t *bias;
    int act;
    const uint16_t *residual;
    int64_t ldr;
    void *y;
    int64_t ldy;
    int y_f32;
    uint16_t *z, *u;
    int64_t ldz;
};
// one layer, or (up != null) the gate and the other layer of a gated block
static int forward(dbspmspv_handle_s *h, dbspmspv_handle_s *up, LinForward f, LinRoom room, cudaStream_t st) {
    const Device &d = h->d;
    CallList calls;
    int s = DBSPMSPV_OK;
    if (over_columns(h, up ? 2 : 1, f.tokens, !tma_rows(f.x, f.ldx))) {
        LcArgs a = {};
        a.x = f.x; a.ldx = f.ldx; a.n = d.n; a.m = d.m;
        a.w[0] = reinterpret_cast<const uint4 *>(h->lin_w);
        a.w[1] = up ? reinterpret_cast<const uint4 *>(up->lin_w) : nullptr;
        a.bias = f.bias; a.residual = f.residual; a.ldr = f.ldr; a.y = f.y; a.ldy = f.ldy; a.y_f32 = f.y_f32; a.act = f.act;
        a.z = f.z; a.u = f.u; a.ldz = f.ldz;
        s = up ? add_columns<2>(h, calls, a, f.tokens) : add_columns<1>(h, calls, a, f.tokens);
    } else {
        LinPack pack;
        if ((s = usable_x(h, &f.x, &f.ldx, f.tokens, room, &pack)) != DBSPMSPV_OK) return s;
        if (pack.out) calls.add(k_linear_pack, pack_blocks(h, pack), LS_CTA, 0, false, pack);
        const int out = up ? LG_M / 2 : LG_M;
        const int64_t kb = ceil64(d.n, LG_K);
        LgArgs a = {};
        a.tokens = f.tokens; a.width = d.m;
        a.y = f.y; a.ldy = f.ldy; a.y_f32 = f.y_f32; a.act = f.act; a.bias = f.bias; a.residual = f.residual; a.ldr = f.ldr;
        a.z = f.z; a.u = f.u; a.ldz = f.ldz; a.aligned = aligned_rows(a); a.status = &d.ws.ctr->status;
        const LgPlan p = plan_gemm(h->sm_count, f.tokens, d.m, out, kb, !!a.z + !!a.u + !!a.residual, a.aligned);
        LgMaps maps = {};
        maps.a[0] = up ? h->lin_maps[1] : h->lin_maps[0];
        if (up) maps.a[1] = up->lin_maps[1];
        if ((s = encode_rows(&maps.b[0], f.x, f.tokens, d.n, f.ldx, p.nt / p.cg)) != DBSPMSPV_OK) return s;
        a.tiles_m = (int)ceil64(d.m, p.cg * out); a.tiles_n = (int)ceil64(f.tokens, p.nt); a.products = 1; a.layers = 1; a.k_blocks = (int)kb;
        s = up ? add_gemm<LG_GATED>(h, calls, maps, a, p) : add_gemm<LG_FORWARD>(h, calls, maps, a, p);
    }
    return s == DBSPMSPV_OK ? submit_calls(h, calls, st) : s;
}

struct LinBackward {
    const uint16_t *x;
    int64_t ldx;
    int tokens, act;
    const uint16_t *z, *u;
    int64_t ldz;
    const uint16_t *dy;
    int64_t lddy;
    uint16_t *dx;
    int64_t lddx;
    uint16_t *dw[2];
    float *dbias;
};
static int backward(dbspmspv_handle_s *h, dbspmspv_handle_s *up, LinBackward b, LinRoom room, cudaStream_t st) {
    const Device &d = h->d;
    CallList calls;
    int s = DBSPMSPV_OK;
    const bool want_w = b.dw[0] || b.dw[1], products = b.dx || want_w;
    const int layers = up ? 2 : 1;
    LinPack pack = {};
    if (want_w && (s = usable_x(h, &b.x, &b.ldx, b.tokens, room, &pack)) != DBSPMSPV_OK) return s;
    const uint16_t *dz[2] = {b.dy, nullptr};
    int64_t ldd = b.lddy;
    const bool as_it_is = !up && b.act == DBSPMSPV_ACT_NONE && tma_rows(b.dy, b.lddy);
    if ((products && !as_it_is) || b.dbias) {
        LsArgs a = {};
        a.dy = b.dy; a.lddy = b.lddy; a.z = b.act == DBSPMSPV_ACT_NONE && !up ? nullptr : b.z; a.u = b.u; a.ldz = b.ldz;
        a.tokens = b.tokens; a.m = d.m; a.act = b.act; a.dbias = b.dbias;
        if (products && !as_it_is) {
            ldd = round_up(d.m, 8);
            a.ldd = ldd;
            dz[0] = a.d0 = room.take(b.tokens, ldd);
            if (up) dz[1] = a.d1 = room.take(b.tokens, ldd);
            if (!a.d0 || (up && !a.d1)) return DBSPMSPV_ERR_INVALID_ARG;
        }
        const int64_t g = b.dbias ? ceil64(d.m, LS_COLS) : ceil64(b.tokens * ceil64(d.m, 8), LS_CTA), most = b.dbias ? g : 8 * h->sm_count;
        a.pack_from = (int)(g < most ? g : most);
        a.pack = pack;
        a.aligned = tma_rows(b.dy, b.lddy) && (!a.z || tma_rows(a.z, b.ldz)) && (!up || tma_rows(b.u, b.ldz));
        calls.add(b.dbias ? k_linear_bias : up ? k_linear_slopes<true> : k_linear_slopes<false>, a.pack_from + pack_blocks(h, pack), LS_CTA, 0, false, a);
    } else if (pack.out) {
        calls.add(k_linear_pack, pack_blocks(h, pack), LS_CTA, 0, false, pack);
    }
    LgArgs a = {};
    a.status = &d.ws.ctr->status;
    if (b.dx) {
        const int64_t kb = ceil64(d.m, DC_ROWS);
        a.tokens = b.tokens; a.width = d.n; a.y = b.dx; a.ldy = b.lddx; a.aligned = aligned_rows(a);
        const LgPlan p = plan_gemm(h->sm_count, b.tokens, d.n, LG_M, kb * layers, 0, a.aligned);
        LgMaps maps = {};
        for (int l = 0; l < layers; ++l) {
            maps.a[l] = l ? up->lin_maps[2] : h->lin_maps[2];
            if ((s = encode_rows(&maps.b[l], dz[l], b.tokens, d.m, ldd, p.nt / p.cg)) != DBSPMSPV_OK) return s;
        }
        a.tiles_m = (int)ceil64(d.n, p.cg * LG_M); a.tiles_n = (int)ceil64(b.tokens, p.nt); a.products = 1; a.layers = layers; a.k_blocks = (int)kb;
        if ((s = add_gemm<LG_DX>(h, calls, maps, a, p)) != DBSPMSPV_OK) return s;
    }
    if (want_w) {
        LgMaps maps = {};
        if ((s = encode_rows(&maps.a[0], b.x, b.tokens, d.n, b.ldx, LG_K)) != DBSPMSPV_OK) return s;
        a.products = 0;
        for (int l = 0; l < layers; ++l) {
            if (!b.dw[l]) continue;
            if ((s = encode_rows(&maps.b[a.products], dz[l], b.tokens, d.m, ldd, LG_K)) != DBSPMSPV_OK) return s;
            a.dw[a.products] = b.dw[l];
            a.stored[a.products] = (uint32_t)(l ? up : h)->nnz;
            a.index[a.products++] = (l ? up : h)->lin_index;
        }
        const LgPlan p = plan_weights(h->sm_count, b.tokens, d.m, d.n, a.products);
        const int64_t kb = ceil64(b.tokens, LG_K);
        a.tiles_m = (int)ceil64(d.n, p.cg * LG_M); a.tiles_n = (int)ceil64(d.m, p.nt); a.layers = 1; a.k_blocks = (int)kb;
        a.tokens = b.tokens; a.width = d.m; a.index_words = h->lin_index ? h->lin_words : up->lin_words;
        if ((s = add_gemm<LG_DW>(h, calls, maps, a, p)) != DBSPMSPV_OK) return s;
    }
    return submit_calls(h, calls, st);
}

static bool act_ok(int act) { return act >= DBSPMSPV_ACT_NONE && act <= DBSPMSPV_ACT_GELU; }
static bool stride_ok(const void *p, int64_t ld, int64_t width) { return !p || ld >= width; }
template <typename... P> static bool on_bytes(uintptr_t bytes, P... p) { return (((reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0) && ...); }
static const uint16_t *in(const void *p) { return static_cast<const uint16_t *>(p); }
static uint16_t *out(void *p) { return static_cast<uint16_t *>(p); }
static LinRoom room(void *p, int64_t bytes) { return LinRoom{static_cast<uint8_t *>(p), bytes}; }

}  // namespace dbs

extern "C" {

int dbspmspv_linear_workspace(dbspmspv_handle_t h, dbspmspv_handle_t up, int32_t tokens, int backward, int64_t *bytes) {
    if (!h || !bytes || tokens < 0) return DBSPMSPV_ERR_INVALID_ARG;
    if (!dbs::has_linear(h) || (up && !dbs::has_linear(up))) return DBSPMSPV_ERR_UNSUPPORTED;
    *bytes = dbs::workspace_bytes(h, up ? 2 : 1, tokens, backward != 0);
    return DBSPMSPV_OK;
}

int dbspmspv_linear(dbspmspv_handle_t h, const void *x, int64_t ldx, int32_t tokens, const void *bias, int act, const void *residual, int64_t ldr, void *y, int64_t ldy,
                    int y_f32, void *z, int64_t ldz, void *workspace, int64_t workspace_bytes, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (!h || tokens < 0 || workspace_bytes < 0 || !act_ok(act) || (tokens > 0 && (!x || !y))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_handle_device(h)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!has_linear(h)) return DBSPMSPV_ERR_UNSUPPORTED;
    const int64_t m = h->d.m, n = h->d.n;
    if (ldx < n || ldy < m || !stride_ok(residual, ldr, m) || !stride_ok(z, ldz, m)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(16, workspace) || !on_bytes(2, x, bias, residual, z) || !on_bytes(y_f32 ? 4 : 2, y)) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    h->last_stream = st;
    return forward(h, nullptr, {in(x), ldx, tokens, in(bias), act, in(residual), ldr, y, ldy, y_f32 != 0, out(z), nullptr, ldz}, room(workspace, workspace_bytes), st);
}

int dbspmspv_gated(dbspmspv_handle_t gate, dbspmspv_handle_t up, const void *x, int64_t ldx, int32_t tokens, int act, void *y, int64_t ldy, void *g, void *u, int64_t ldgu,
                   void *workspace, int64_t workspace_bytes, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (!gate || !up || tokens < 0 || workspace_bytes < 0 || !act_ok(act) || (tokens > 0 && (!x || !y))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_handle_device(gate) || !on_handle_device(up)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!has_linear(gate) || !has_linear(up)) return DBSPMSPV_ERR_UNSUPPORTED;
    const int64_t m = gate->d.m, n = gate->d.n;
    if (up->d.m != m || up->d.n != n) return DBSPMSPV_ERR_INVALID_ARG;
    if (ldx < n || ldy < m || !stride_ok(g, ldgu, m) || !stride_ok(u, ldgu, m)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(16, workspace) || !on_bytes(2, x, y, g, u)) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens == 0) return DBSPMSPV_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    gate->last_stream = up->last_stream = st;
    return forward(gate, up, {in(x), ldx, tokens, nullptr, act, nullptr, 0, y, ldy, 0, out(g), out(u), ldgu}, room(workspace, workspace_bytes), st);
}

int dbspmspv_linear_backward(dbspmspv_handle_t h, const void *x, int64_t ldx, int32_t tokens, int act, const void *z, int64_t ldz, const void *dy, int64_t lddy, void *dx,
                             int64_t lddx, void *dw, float *dbias, void *workspace, int64_t workspace_bytes, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (!h || tokens < 0 || workspace_bytes < 0 || !act_ok(act)) return DBSPMSPV_ERR_INVALID_ARG;
    if (tokens > 0 && (!dy || (dw && !x) || (act != DBSPMSPV_ACT_NONE && !z))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_handle_device(h)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!has_linear(h) || (dw && !h->lin_index)) return DBSPMSPV_ERR_UNSUPPORTED;
    const int64_t m = h->d.m, n = h->d.n;
    if ((dw && ldx < n) || lddy < m || (act != DBSPMSPV_ACT_NONE && ldz < m) || !stride_ok(dx, lddx, n)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(16, workspace) || !on_bytes(2, x, z, dy, dx, dw) || !on_bytes(4, dbias)) return DBSPMSPV_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    h->last_stream = st;
    if (tokens == 0) {
        if (dw) DBS_CUDA(cudaMemsetAsync(dw, 0, (size_t)h->nnz * 2, st));
        if (dbias) DBS_CUDA(cudaMemsetAsync(dbias, 0, (size_t)m * 4, st));
        return DBSPMSPV_OK;
    }
    return backward(h, nullptr, {in(x), ldx, tokens, act, in(z), nullptr, ldz, in(dy), lddy, out(dx), lddx, {out(dw), nullptr}, dbias}, room(workspace, workspace_bytes), st);
}

int dbspmspv_gated_backward(dbspmspv_handle_t gate, dbspmspv_handle_t up, const void *x, int64_t ldx, int32_t tokens, int act, const void *g, const void *u, int64_t ldgu,
                            const void *dy, int64_t lddy, void *dx, int64_t lddx, void *dw_gate, void *dw_up, void *workspace, int64_t workspace_bytes, dbspmspv_stream_t stream) {
    using namespace dbs;
    if (!gate || !up || tokens < 0 || workspace_bytes < 0 || !act_ok(act)) return DBSPMSPV_ERR_INVALID_ARG;
    const bool want_w = dw_gate || dw_up;
    if (tokens > 0 && (!dy || !g || !u || (want_w && !x))) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_handle_device(gate) || !on_handle_device(up)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!has_linear(gate) || !has_linear(up) || (dw_gate && !gate->lin_index) || (dw_up && !up->lin_index)) return DBSPMSPV_ERR_UNSUPPORTED;
    const int64_t m = gate->d.m, n = gate->d.n;
    if (up->d.m != m || up->d.n != n) return DBSPMSPV_ERR_INVALID_ARG;
    if ((want_w && ldx < n) || lddy < m || ldgu < m || !stride_ok(dx, lddx, n)) return DBSPMSPV_ERR_INVALID_ARG;
    if (!on_bytes(16, workspace) || !on_bytes(2, x, g, u, dy, dx, dw_gate, dw_up)) return DBSPMSPV_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    gate->last_stream = up->last_stream = st;
    if (tokens == 0) {
        if (dw_gate) DBS_CUDA(cudaMemsetAsync(dw_gate, 0, (size_t)gate->nnz * 2, st));
        if (dw_up) DBS_CUDA(cudaMemsetAsync(dw_up, 0, (size_t)up->nnz * 2, st));
        return DBSPMSPV_OK;
    }
    return backward(gate, up, {in(x), ldx, tokens, act, in(g), in(u), ldgu, in(dy), lddy, out(dx), lddx, {out(dw_gate), out(dw_up)}, nullptr}, room(workspace, workspace_bytes), st);
}

}  // extern "C"
