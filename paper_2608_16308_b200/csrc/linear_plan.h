// How the tensor-core products of the linear layers are cut into tiles.  Host code without CUDA, so that a test can ask it for every size.
#pragma once

#include <stdint.h>

namespace dbs {

constexpr int LG_M = 128, LG_K = 64;     // output columns of a thread block's tile; a block of K

// CG thread blocks per tile of CG * 128 x nt, or C that share a tile's K.
struct LgPlan { int cg, nt, c; };

// Tiles of one thread block, (nt, C): the kernels that are built beside the pairs.  (No tile of 128 tokens: one of 64 has at least its rounds, since twice as many blocks fit, the same time
// per block of K and half the emptying.)
#define LG_TILES(X) X(16, 1) X(16, 2) X(16, 4) X(16, 8) X(64, 1) X(64, 2) X(64, 4) X(64, 8) X(256, 1) X(256, 2) X(256, 4) X(256, 8)

static inline int64_t ceil64(int64_t v, int64_t by) { return (v + by - 1) / by; }

// Thread blocks that have to share K.  The tensor cores cut off what an addition leaves below the accumulator's last bit, so a sum of one sign loses 5.5e-9 of itself per term (16,384 terms 6.5e-5,
// 131,072 terms 7.2e-4, 2 M terms 1.2e-2; those of a library's product are the same), which beyond half a million terms is more than a rounding to bf16.  So an accumulator takes 131,072 at most
// as long as there are clusters to share them (a million terms); their sums are added up in fp32.
constexpr int64_t LG_SUM_BLOCKS = 131072 / LG_K;
static inline int least_shares(int64_t kb) {
    int c = 1;
    while (c < 8 && kb > c * LG_SUM_BLOCKS) c *= 2;
    return c;
}

// The cut of a product whose tiles are `out` output columns wide (one thread block's) and `kb` blocks of K long; `arrays` beside y are read or written with the outputs.  Blocks of K follow each other at 0.34 us
// in a thread block, whatever the width of its tile and whether it shares its SM; a tile is emptied under the products of the next, the last one is not; emptying it, and adding up the sums of C thread
// blocks, cost more the wider it is.  Measured on seven layers (700 x 5000 to 11008 x 4096), 20 to 1000 tokens, eleven cuts each: the one
// chosen here is 0.7 % behind the best on average, 7 % at most, and the worst of the eleven is two to four times as slow (4096 x 4096, 256 tokens: 17 to 35 us).  With three arrays whose rows begin anywhere (5803 x 558,
// 587 tokens) tiles of 64 tokens take 30 us, of 256 39.
static inline LgPlan plan_gemm(int sm_count, int64_t tokens, int64_t width, int out, int64_t kb, int arrays, bool aligned) {
    struct { LgPlan p; int slots; } const all[] = {{{2, 256, 1}, sm_count / 2}, {{1, 16, 1}, 2 * sm_count}, {{1, 64, 1}, 2 * sm_count}, {{1, 256, 1}, sm_count}};
    const double each = (aligned ? 0.3 + 0.5 * arrays : 1.3 + 1.2 * arrays) * out / LG_M;      // us to empty 64 tokens of a tile
    LgPlan best = all[0].p;
    const int shares = least_shares(kb);
    double least = 0.;
    for (const auto &q : all) {
        if ((q.p.nt == 16) != (tokens <= 16)) continue;               // (a layer's weights go through once: a narrow tile only where all tokens fit in)
        if (q.p.cg == 2 && shares > 1) continue;
        const int64_t tiles = ceil64(width, q.p.cg * out) * ceil64(tokens, q.p.nt);
        for (int c = shares; c <= (q.p.cg == 1 ? 8 : 1); c *= 2) {
            // (a cluster is placed within a part of the GPU: the larger it is, the more SMs stay without one)
            if (c > shares && (kb < 2 * c || tiles * c >= q.slots - c * c / 2)) break;
            const double products = (double)ceil64(kb, c) * 0.34, rounds = (double)ceil64(tiles * c, q.slots), empty = each * q.p.nt / 64. / (c == 1 ? 1. : c == 2 ? 1.4 : c == 4 ? 2. : 2.8);
            const double cost = products + empty + (rounds - 1.) * (products > empty ? products : empty) + (c > 1 ? 0.2 * c * (1. + q.p.nt / 64.) : 0.);
            if (least == 0. || cost < least) { least = cost; best = q.p; best.c = c; }
        }
    }
    return best;
}

// The gradient of the weights of `products` m x n layers: pairs where they fill the GPU; else thread blocks of one tile share the tokens while SMs would stay idle and each has four blocks of tokens or more (whole
// gradient, shared out / not: 1024 x 1024, 2048 tokens 24 / 30 us, 1000 tokens 19.6 / 20.1; 250 x 300, 2000 tokens 21 / 27; 944 x 1835, 1378 tokens 39 / 39).
static inline LgPlan plan_weights(int sm_count, int64_t tokens, int64_t m, int64_t n, int products) {
    LgPlan p = {2, 256, 1};
    const int64_t kb = ceil64(tokens, LG_K);
    const int shares = least_shares(kb);
    if (shares > 1 || ceil64(n, 2 * LG_M) * ceil64(m, p.nt) * products * 4 < sm_count / 2 * 3) {
        p.cg = 1;
        p.c = shares;
        const int64_t tiles = ceil64(n, LG_M) * ceil64(m, p.nt) * products;
        while (p.c < 8 && tiles * p.c * 2 < sm_count - 2 * p.c * p.c && kb >= 8 * p.c) p.c *= 2;
    }
    return p;
}

}  // namespace dbs
