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
    uint32_t step;            // ... in bytes (its low 32 bits)
};
inline Rows rows_of(const void *p, int64_t ld, bool f32) {
    return Rows{const_cast<void *>(p), ld, f32, (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * (f32 ? 4 : 2)) % 16 == 0, (uint32_t)(ld * (f32 ? 4 : 2))};
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
// Two fp32 in a register pair: sm_100 multiplies and adds them with one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
    f32x2 p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ f32x2 both(float v) { return pair(v, v); }
__device__ __forceinline__ float2 apart(f32x2 p) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// The same one after the other.  Where registers are short the pairs cost more moves than they save (gradient of a join, 4096 x 4096: 61.1 us in pairs, 58.1 one by one; forwards 33.0 and 33.6).
__device__ __forceinline__ f32x2 fma1(f32x2 a, f32x2 b, f32x2 c) {
    const float2 x = apart(a), y = apart(b), z = apart(c);
    return pair(fmaf(x.x, y.x, z.x), fmaf(x.y, y.y, z.y));
}
__device__ __forceinline__ f32x2 mul1(f32x2 a, f32x2 b) {
    const float2 x = apart(a), y = apart(b);
    return pair(x.x * y.x, x.y * y.y);
}
__device__ __forceinline__ f32x2 add1(f32x2 a, f32x2 b) {
    const float2 x = apart(a), y = apart(b);
    return pair(x.x + y.x, x.y + y.y);
}
__device__ __forceinline__ float sum2(f32x2 p) {
    const float2 v = apart(p);
    return v.x + v.y;
}
__device__ __forceinline__ f32x2 as_pair(uint32_t lo, uint32_t hi) { return pair(__uint_as_float(lo), __uint_as_float(hi)); }
__device__ __forceinline__ f32x2 bf16_pair(uint32_t w) { return pair(bf16_lo(w), bf16_hi(w)); }

__device__ __forceinline__ void pairs_of_eight(uint4 q, f32x2 v[4]) { v[0] = bf16_pair(q.x); v[1] = bf16_pair(q.y); v[2] = bf16_pair(q.z); v[3] = bf16_pair(q.w); }
__device__ __forceinline__ void pairs_of_eight(uint4 a, uint4 b, f32x2 v[4]) { v[0] = as_pair(a.x, a.y); v[1] = as_pair(a.z, a.w); v[2] = as_pair(b.x, b.y); v[3] = as_pair(b.z, b.w); }
__device__ __forceinline__ uint32_t two_bf16(f32x2 p) { const float2 v = apart(p); return two_bf16(v.x, v.y); }
__device__ __forceinline__ uint4 bf16_eight(const f32x2 v[4]) { return make_uint4(two_bf16(v[0]), two_bf16(v[1]), two_bf16(v[2]), two_bf16(v[3])); }
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
template <bool F32>
__device__ __forceinline__ void store_eight(void *row, int col, int n, bool whole, const f32x2 v[4]) {
    if (F32) {
        const float2 a = apart(v[0]), b = apart(v[1]), c = apart(v[2]), d = apart(v[3]);
        store_raw<true>(row, col, n, whole, make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y)),
                        make_uint4(__float_as_uint(c.x), __float_as_uint(c.y), __float_as_uint(d.x), __float_as_uint(d.y)));
    } else store_raw<false>(row, col, n, whole, bf16_eight(v), uint4{});
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

// Copies into shared memory that a thread makes for itself: group by group, and no barrier where it reads them itself
__device__ __forceinline__ void copy_ahead(void *smem, const void *p) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p) : "memory");
}
// ... of which `bytes` are read and the rest is zeros
__device__ __forceinline__ void copy_ahead(void *smem, const void *p, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_word_ahead(void *smem, const void *p, uint32_t bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p), "r"(bytes) : "memory");
}
__device__ __forceinline__ void close_ahead() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void wait_ahead() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// ---- rows in a warp's shared memory --------------------------------------------------------------
// A lane's eight lies at 16 * lane; fp32: the first four there and the others 512 bytes behind (WHOLE), or all at 32 * lane.  What is not WHOLE has 16 bytes more: rows that begin between two words.
template <bool F32, bool WHOLE> __host__ __device__ constexpr int eight_room() { return (F32 ? 1024 : 512) + (WHOLE ? 0 : 16); }
// whether row t of bf16 begins between two words
__device__ __forceinline__ int between(const Rows &r, int64_t t) { return ((int)(reinterpret_cast<uintptr_t>(r.p) >> 1) ^ ((int)t & (int)r.ld)) & 1; }

struct WarpEight {
    int lane, col, cnt;                      // the warp's first column; the lane's entries, 0 to 8
    __device__ __forceinline__ int mine() const { return col + lane * 8; }
};
// The warp's eights of row t, columns from w.col on, towards shared memory at `to`.  Copies say how many bytes they read, so the row's end needs no loads of its own, for which the warp, and then its team, would wait
// (4000 rows of 4001 in bf16, gradient: 163 us with them, 129 without; 1000 columns off 16 bytes 50 and 36).  A row that begins between two words is copied from the word's begin: two bytes of what lies in front of it come along, but not in front of row 0.
template <bool F32>
__device__ __forceinline__ void row_ahead(const Rows &r, int64_t t, const WarpEight &w, int n, uint8_t *to) {
    const uint8_t *row = static_cast<const uint8_t *>(row_at<F32>(r, t));
    const int here = min(256, n - w.col);    // entries of the warp
    if (here <= 0) return;
    if (r.aligned) {
        const uint8_t *p = row + (int64_t)w.mine() * (F32 ? 4 : 2);
        uint8_t *at = to + w.lane * (F32 ? 32 : 16);
        if (w.cnt == 8) {
            copy_ahead(at, p);
            if (F32) copy_ahead(at + 16, p + 16);
        } else if (w.cnt) {
#pragma unroll
            for (int k = 0; k < (F32 ? 8 : 4); ++k) copy_word_ahead(at + 4 * k, p + 4 * k, max(0, min(4, w.cnt * (F32 ? 4 : 2) - 4 * k)));
        }
        return;
    }
    if (F32) {
        const uint8_t *p = row + (int64_t)w.col * 4;
#pragma unroll
        for (int i = w.lane; i < 256; i += 32) copy_word_ahead(to + i * 4, p + i * 4, i < here ? 4 : 0);
        return;
    }
    // entry e of the words is the row's w.col + e - odd
    const int odd = between(r, t), end = n - w.col + odd;
    const uint8_t *p = row + (int64_t)w.col * 2 - 2 * odd;
    const bool front = odd && w.col == 0 && t == 0 && w.lane == 0;
    if (front) reinterpret_cast<uint16_t *>(to)[1] = *reinterpret_cast<const uint16_t *>(row);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = w.lane + 32 * k;
        if (k || !front) copy_word_ahead(to + i * 4, p + i * 4, max(0, min(4, 2 * (end - 2 * i))));
    }
    if (odd && w.lane == 0) copy_word_ahead(to + 512, p + 512, max(0, min(4, 2 * (end - 256))));
}
// the lane's eight, zeros behind the row's end
template <bool F32, bool WHOLE>
__device__ __forceinline__ void row_here(const Rows &r, int64_t t, const WarpEight &w, const uint8_t *at, f32x2 v[4]) {
    if (F32) {
        const uint4 *p = reinterpret_cast<const uint4 *>(at + w.lane * (WHOLE ? 16 : 32));
        pairs_of_eight(p[0], p[WHOLE ? 32 : 1], v);
    } else {
        uint4 q = *reinterpret_cast<const uint4 *>(at + w.lane * 16);
        if (!WHOLE && !r.aligned && between(r, t)) {
            const uint32_t next = *reinterpret_cast<const uint32_t *>(at + w.lane * 16 + 16);
            q = make_uint4(__funnelshift_r(q.x, q.y, 16), __funnelshift_r(q.y, q.z, 16), __funnelshift_r(q.z, q.w, 16), __funnelshift_r(q.w, next, 16));
        }
        pairs_of_eight(q, v);
    }
    if (!WHOLE && w.cnt < 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 x = apart(v[j]);
            v[j] = pair(2 * j < w.cnt ? x.x : 0.f, 2 * j + 1 < w.cnt ? x.y : 0.f);
        }
    }
}
// the warp's eights to row t; `room`: 1024 bytes of the warp's shared memory
template <bool F32>
__device__ __forceinline__ void row_out(const Rows &r, int64_t t, const WarpEight &w, int n, const f32x2 v[4], uint8_t *room) {
    void *row = const_cast<void *>(row_at<F32>(r, t));
    if (r.aligned) {
        if (w.cnt) store_eight<F32>(row, w.mine(), n, w.cnt == 8, v);
        return;
    }
    const int here = min(256, n - w.col);
    if (F32) {
        f32x2 *mine = reinterpret_cast<f32x2 *>(room + w.lane * 32);
#pragma unroll
        for (int j = 0; j < 4; ++j) mine[j] = v[j];
        __syncwarp();
        uint32_t *p = static_cast<uint32_t *>(row) + w.col;
#pragma unroll
        for (int i = w.lane; i < 256; i += 32)
            if (i < here) p[i] = reinterpret_cast<const uint32_t *>(room)[i];
    } else {
        *reinterpret_cast<uint4 *>(room + w.lane * 16) = bf16_eight(v);
        __syncwarp();
        const int odd = between(r, t);
        uint16_t *p = static_cast<uint16_t *>(row) + w.col;
        // word i of the row holds entries 2 i - odd and the next of the warp's share; an entry without a neighbour goes by itself
        const uint16_t *from = reinterpret_cast<const uint16_t *>(room);
        const uint32_t *words = reinterpret_cast<const uint32_t *>(room);
        uint32_t *to = reinterpret_cast<uint32_t *>(p - odd);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = w.lane + 32 * k, e = 2 * i - odd;
            if (e >= 0 && e + 1 < here) to[i] = odd ? __funnelshift_r(words[i - 1], words[i], 16) : words[i];
        }
        if (here > 0 && odd && w.lane == 0) p[0] = from[0];
        if (here > 0 && w.lane == 1 && ((here + odd) & 1)) p[here - 1] = from[here - 1];
    }
    __syncwarp();
}
// ---- dropout ---------------------------------------------------------------------------------
// Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, 2011): ten rounds of two 32 x 32 -> 64 bit products and their exclusive ors.
struct Drop {
    const uint64_t *random;   // seed, offset; null: nothing is dropped
    uint32_t above;           // a word is kept if it is above this: (P << 16) - 1, and all ones for P = 65536
    float scale;              // 65536 / (65536 - P)
};
// What rows and columns have in common: keys of the rounds, and the first one's products with the offset
struct Numbers {
    uint32_t k0, k1, c3, first, second;
};
constexpr uint32_t PHILOX_M0 = 0xD2511F53u, PHILOX_M1 = 0xCD9E8D57u, PHILOX_W0 = 0x9E3779B9u, PHILOX_W1 = 0xBB67AE85u;
__device__ __forceinline__ Numbers numbers_of(const Drop &d) {
    if (!d.random) return Numbers{};
    const uint64_t seed = d.random[0], offset = d.random[1], q = (uint64_t)(uint32_t)offset * PHILOX_M1;
    return Numbers{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)(offset >> 32), (uint32_t)(q >> 32) ^ (uint32_t)seed, (uint32_t)q};
}
// The counter is (eight, token, offset): what depends on the columns alone is worked out once for all tokens, three of the six products in the first three rounds among it (a fourth is the token's alone)
struct Columns {
    uint32_t a, b, c, d;
};
__device__ __forceinline__ Columns columns_of(const Numbers &s, uint32_t eight) {
    const uint64_t p1 = (uint64_t)eight * PHILOX_M0, q2 = (uint64_t)((uint32_t)(p1 >> 32) ^ s.c3 ^ s.k1) * PHILOX_M1;
    const uint64_t p3 = (uint64_t)((uint32_t)(q2 >> 32) ^ s.second ^ (s.k0 + PHILOX_W0)) * PHILOX_M0;
    return Columns{(uint32_t)p1 ^ (s.k1 + PHILOX_W1), (uint32_t)q2 ^ (s.k0 + 2 * PHILOX_W0), (uint32_t)(p3 >> 32) ^ (s.k1 + 2 * PHILOX_W1), (uint32_t)p3};
}
// the numbers of E eights of a token
template <int E, bool KEYS_ANEW>
__device__ __forceinline__ void philox(const Numbers &s, const Columns (&w)[E], uint32_t token, uint4 (&out)[E]) {
    const uint64_t p2 = (uint64_t)(s.first ^ token) * PHILOX_M0;
    uint32_t c0[E], c1[E], c2[E], c3[E], k0 = s.k0 + 3 * PHILOX_W0, k1 = s.k1 + 3 * PHILOX_W1;
    // (the keys of the rounds are added up again for every token: kept, they would take fourteen registers that the joins' kernels do not have; gradient of 4096 x 4096 68 -> 62 us)
    if (KEYS_ANEW) asm volatile("" : "+r"(k0), "+r"(k1));
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const uint64_t q3 = (uint64_t)((uint32_t)(p2 >> 32) ^ w[e].a) * PHILOX_M1;
        c0[e] = (uint32_t)(q3 >> 32) ^ w[e].b;
        c1[e] = (uint32_t)q3;
        c2[e] = w[e].c ^ (uint32_t)p2;
        c3[e] = w[e].d;
    }
#pragma unroll
    for (int r = 3; r < 10; ++r) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint64_t p = (uint64_t)c0[e] * PHILOX_M0, q = (uint64_t)c2[e] * PHILOX_M1;
            c0[e] = (uint32_t)(q >> 32) ^ c1[e] ^ k0;
            c1[e] = (uint32_t)q;
            c2[e] = (uint32_t)(p >> 32) ^ c3[e] ^ k1;
            c3[e] = (uint32_t)p;
        }
        k0 += PHILOX_W0;
        k1 += PHILOX_W1;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = make_uint4(c0[e], c1[e], c2[e], c3[e]);
}
// v with zeros where entries of the token are dropped (what makes up for them is the caller's to multiply): 16 bits are below P exactly if the word that begins with them is below P << 16
template <int E, bool KEYS_ANEW>
__device__ __forceinline__ void drop_eights(const Drop &d, const Numbers &s, const Columns (&w)[E], uint32_t token, f32x2 (&v)[E][4]) {
    uint4 q[E];
    philox<E, KEYS_ANEW>(s, w, token, q);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const uint32_t bits[4] = {q[e].x, q[e].y, q[e].z, q[e].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 x = apart(v[e][j]);
            v[e][j] = pair(bits[j] << 16 > d.above ? x.x : 0.f, bits[j] > d.above ? x.y : 0.f);
        }
    }
}

// ---- the host's side ----------------------------------------------------------------------------
inline int64_t ceil64(int64_t a, int64_t b) { return (a + b - 1) / b; }
template <typename... P> inline bool on_bytes(uintptr_t bytes, P... p) { return (((reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0) && ...); }
inline bool rows_ok(const void *p, int64_t ld, int64_t width) { return !p || ld >= width; }

inline Drop drop_of(float p, const void *random) {
    const int32_t below = (int32_t)((double)p * 65536.0 + 0.5);
    if (below == 0) return Drop{};
    if (below >= 65536) return Drop{static_cast<const uint64_t *>(random), 0xFFFFFFFFu, 0.f};
    return Drop{static_cast<const uint64_t *>(random), ((uint32_t)below << 16) - 1u, 65536.f / (65536 - below)};
}

template <typename... P> inline const void *first_of(P... p) {                     // of those that are there
    const void *all[] = {static_cast<const void *>(p)...};
    for (const void *q : all)
        if (q) return q;
    return nullptr;
}
// Whether `p` is memory that kernels of the current device can reach: its own, managed, or the host's if that is pinned; not the host's other memory, not another device's.
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

// Lets a kernel have all of an SM's shared memory, once per kernel and device (the call takes the thread half a microsecond, a launch two).  The kernels that were told are kept in a small table; one that
// finds no place there is told again.
inline int allow_smem(const void *kernel, int dev) {
    constexpr int PLACES = 256, TRIES = 8;
    static const void *told[64][PLACES];
    const size_t first = (reinterpret_cast<uintptr_t>(kernel) >> 4) * 2654435761u >> 8;
    const void **free = nullptr;
    for (int i = 0; i < TRIES && !free; ++i) {
        const void **at = &told[dev][(first + i) % PLACES], *known = __atomic_load_n(at, __ATOMIC_ACQUIRE);
        if (known == kernel) return DBSPMSPV_OK;
        if (!known) free = at;
    }
    cudaFuncAttributes f;
    DBS_CUDA(cudaFuncGetAttributes(&f, kernel));
    DBS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)f.sharedSizeBytes));
    const void *none = nullptr;
    if (free) __atomic_compare_exchange_n(free, &none, kernel, false, __ATOMIC_RELEASE, __ATOMIC_RELAXED);
    return DBSPMSPV_OK;
}

// Clusters that the device holds at once (an SM that is left over in its part of the chip takes none: 142 clusters of three where 148 SMs have room for as many blocks, and six more would wait for the others
// to end).  Asked for once: kept with 48 bits of what was asked in a small table, newer answers over older ones.
inline int clusters_at_once(const void *kernel, int dev, int threads, int cluster, size_t smem, int *most) {
    constexpr int PLACES = 256;
    static uint64_t known[PLACES];
    uint64_t key = reinterpret_cast<uintptr_t>(kernel);
    for (uint64_t part : {(uint64_t)dev, (uint64_t)threads, (uint64_t)cluster, (uint64_t)smem}) key = (key ^ part) * 0x9E3779B97F4A7C15ull, key ^= key >> 29;
    uint64_t *at = &known[(key >> 8) % PLACES];
    const uint64_t was = __atomic_load_n(at, __ATOMIC_RELAXED);
    if (was && (was & ~0xFFFFull) == (key & ~0xFFFFull)) {
        *most = (int)(was & 0xFFFFu);
        return DBSPMSPV_OK;
    }
    const int s = allow_smem(kernel, dev);
    if (s != DBSPMSPV_OK) return s;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(cluster);
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim = {(unsigned)cluster, 1, 1};
    c.attrs = &attr;
    c.numAttrs = 1;
    int n = 0;
    DBS_CUDA(cudaOccupancyMaxActiveClusters(&n, kernel, &c));
    n = n < 1 ? 1 : n > 0xFFFF ? 0xFFFF : n;
    __atomic_store_n(at, (key & ~0xFFFFull) | (uint64_t)n, __ATOMIC_RELAXED);
    *most = n;
    return DBSPMSPV_OK;
}

// One launch in clusters of `cluster` thread blocks, set up while the kernel in front of it drains (every kernel launched so begins with pdl_wait).
template <typename... P, typename... A>
inline int launch_rows(int dev, void (*kernel)(P...), int blocks, int threads, int cluster, size_t smem, cudaStream_t st, const A &...args) {
    if (smem > 16 * 1024) {
        const int s = allow_smem(reinterpret_cast<const void *>(kernel), dev);
        if (s != DBSPMSPV_OK) return s;
    }
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
