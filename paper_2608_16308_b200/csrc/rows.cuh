// Rows of bf16 or fp32 taken eight columns a thread: what the joins, dropout and log probabilities share.
#pragma once

#include <cuda_bf16.h>

#include "internal.cuh"
#include "microkernels.cuh"

namespace dbs {

// A row operand: base, stride between rows in entries, whether every row begins on 16 bytes (set by the host).
struct Rows {
    void *p;
    int64_t ld;
    int32_t f32, aligned;
};
inline Rows rows_of(const void *p, int64_t ld, bool f32) {
    return Rows{const_cast<void *>(p), ld, f32, (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * (f32 ? 4 : 2)) % 16 == 0};
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {          // to nearest even
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}
__device__ __forceinline__ void eight_of(uint4 q, float v[8]) {
    v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
    v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
}
__device__ __forceinline__ void eight_of(uint4 a, uint4 b, float v[8]) {
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
}
__device__ __forceinline__ uint4 bf16_eight(const float v[8]) { return make_uint4(two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])); }

// Columns col to col + 7 of a row of n (col < n), zeros behind its end.  `whole`: all eight are there and begin on 16 bytes.
template <bool F32>
__device__ __forceinline__ void load_raw(const void *row, int col, int n, bool whole, uint4 &a, uint4 &b) {
    if (F32) {
        const uint32_t *p = static_cast<const uint32_t *>(row) + col;
        if (whole) {
            a = *reinterpret_cast<const uint4 *>(p);
            b = *reinterpret_cast<const uint4 *>(p + 4);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = col + j < n ? p[j] : 0u;
            a = make_uint4(w[0], w[1], w[2], w[3]);
            b = make_uint4(w[4], w[5], w[6], w[7]);
        }
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(row) + col;
        if (whole) a = *reinterpret_cast<const uint4 *>(p);
        else {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = col + j < n ? p[j] : 0u;
            a = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
}
template <bool F32>
__device__ __forceinline__ void store_raw(void *row, int col, int n, bool whole, uint4 a, uint4 b) {
    if (F32) {
        uint32_t *p = static_cast<uint32_t *>(row) + col;
        if (whole) {
            *reinterpret_cast<uint4 *>(p) = a;
            *reinterpret_cast<uint4 *>(p + 4) = b;
        } else {
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < n) p[j] = w[j];
        }
    } else {
        uint16_t *p = static_cast<uint16_t *>(row) + col;
        if (whole) *reinterpret_cast<uint4 *>(p) = a;
        else {
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < n) p[j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
        }
    }
}
__device__ __forceinline__ uint4 fp32_four(const float *v) { return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])); }
template <bool F32>
__device__ __forceinline__ void store_eight(void *row, int col, int n, bool whole, const float v[8]) {
    if (F32) store_raw<true>(row, col, n, whole, fp32_four(v), fp32_four(v + 4));
    else store_raw<false>(row, col, n, whole, bf16_eight(v), uint4{});
}
template <bool F32>
__device__ __forceinline__ const void *row_at(const Rows &r, int64_t t) {
    return static_cast<const uint8_t *>(r.p) + t * r.ld * (F32 ? 4 : 2);
}

// ---- dropout ---------------------------------------------------------------------------------
// Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, 2011): ten rounds of two 32 x 32 -> 64 bit products and their exclusive ors.
struct Drop {
    const uint64_t *random;   // seed, offset; null: nothing is dropped
    uint32_t below;           // P << 16 (P < 65536)
    int32_t all;              // P = 65536: everything is dropped
    float scale;              // 65536 / (65536 - P)
};
struct Numbers {
    uint32_t k0, k1, c2, c3;
};
__device__ __forceinline__ Numbers numbers_of(const Drop &d) {
    if (!d.random) return Numbers{};
    const uint64_t seed = d.random[0], offset = d.random[1];
    return Numbers{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
}
__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, const Numbers &s) {
    uint32_t c2 = s.c2, c3 = s.c3, k0 = s.k0, k1 = s.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)q;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}
// v[j] scaled, or 0 where entry 8 * eight + j of the token is dropped: its 16 bits are below P exactly if the word that begins with them is below P << 16
__device__ __forceinline__ void drop_eight(const Drop &d, const Numbers &s, uint32_t eight, uint32_t token, float v[8]) {
    const uint4 q = philox(eight, token, s);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t bits = j % 2 ? w[j / 2] : w[j / 2] << 16;
        v[j] = bits >= d.below && !d.all ? v[j] * d.scale : 0.f;
    }
}

// ---- the host's side ----------------------------------------------------------------------------
inline Drop drop_of(float p, const void *random) {
    const int32_t below = (int32_t)((double)p * 65536.0 + 0.5);
    if (below == 0) return Drop{};
    return Drop{static_cast<const uint64_t *>(random), below >= 65536 ? 0u : (uint32_t)below << 16, below >= 65536, below >= 65536 ? 0.f : 65536.f / (65536 - below)};
}

// Whether `p` is memory that kernels of the current device may use as theirs: not the host's own, not another device's.
inline bool on_current_device(const void *p, int dev) {
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return a.type == cudaMemoryTypeManaged || a.type == cudaMemoryTypeHost || (a.type == cudaMemoryTypeDevice && a.device == dev);
}

// SMs of the current device, asked for once per device
inline int current_device(int *dev, int *sms) {
    static int known[64];
    DBS_CUDA(cudaGetDevice(dev));
    if (*dev < 0 || *dev >= 64) return DBSPMSPV_ERR_UNSUPPORTED;
    int n = __atomic_load_n(&known[*dev], __ATOMIC_RELAXED);
    if (!n) {
        DBS_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, *dev));
        __atomic_store_n(&known[*dev], n, __ATOMIC_RELAXED);
    }
    *sms = n;
    return DBSPMSPV_OK;
}

// One launch in clusters of `cluster` thread blocks, set up while the kernel in front of it drains (every kernel launched so begins with pdl_wait).
template <typename... P, typename... A>
inline int launch_rows(void (*kernel)(P...), int blocks, int threads, int cluster, size_t smem, cudaStream_t st, const A &...args) {
    if (smem > 48 * 1024) DBS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(blocks);
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    c.attrs = attr;
    c.numAttrs = cluster > 1 ? 2 : 1;
    DBS_CUDA(cudaLaunchKernelEx(&c, kernel, args...));
    return DBSPMSPV_OK;
}

}  // namespace dbs
