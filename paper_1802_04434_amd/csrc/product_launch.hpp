// Host side of the products of 16-bit matrices (product_kernels.hpp): how one is cut, and its launches.
#pragma once
#include <cmath>

#include "api_common.hpp"
#include "product_kernels.hpp"

namespace product {

constexpr size_t kMaxBlocks = (size_t)1 << 23;      // of 256 threads: a launch has fewer than 2^32

inline size_t rounded(size_t n, size_t to) { return (n + to - 1) / to * to; }
inline size_t tiles_of(size_t n, int tile) { return (n + 64 * (size_t)tile - 1) / (64 * (size_t)tile); }

// tiles of 64 times `tile` squared, the sum over k in `splits` parts; half: of a symmetric result only those on and above the diagonal
struct Plan {
    int tile;
    size_t splits;
    bool half = false;
    bool few = false;          // steps, so few that a block holds one at a time
};

inline size_t bands_of(size_t tiles) { return (tiles + kHigh - 1) / kHigh; }

// What a product takes with a plan, from products of 64 to 8192 squared by 64 to 16384, as they lie and down k alike: us a step of 64 of k with few blocks on the card
// and with as many as fit, and us a block besides, for its first loads and for writing the result.  Two launches cost 3 us more, and the partial sums their bytes, written, read
// and joined at 2.5 TB/s.  us by tiles of 256 / 128 / 64 squared: 4096 cubed 103 / 121 / 200, 2048 cubed 40.6 / 21.6 / 30.3, 1024 cubed 23.5 / 9.6 / 6.2.
struct Shape {
    int tile;
    double fit, empty, alone, full, starts, ends;      // empty: blocks a compute unit up to which a step takes as long as alone
};
constexpr Shape kShapes[] = {{4, 1, 0, 0.90, 1.40, 3.0, 9.0}, {2, 2, 0, 0.38, 0.87, 2.5, 2.5}, {1, 4, 0.5, 0.25, 0.80, 2.2, 1.0}};

inline double cost_of(size_t M, size_t N, size_t K, size_t count, const Plan &plan) {
    const Shape &s = kShapes[plan.tile == 4 ? 0 : plan.tile == 2 ? 1 : 2];
    const size_t steps = (K + kStep - 1) / kStep, side = tiles_of(M, s.tile), tiles = plan.half ? side * (side + 1) / 2 : side * tiles_of(N, s.tile);
    const double blocks = (double)(tiles * count * plan.splits), each = (double)((steps + plan.splits - 1) / plan.splits);
    auto round = [&](double load) {       // blocks a compute unit
        const double crowd = std::fmax(0.0, (load - s.empty) / (s.fit - s.empty));
        return each * (s.alone + (s.full - s.alone) * crowd) + s.starts + (plan.half ? 1.5 : 1.0) * s.ends * std::fmax(0.25, load / s.fit);
    };
    const double rounds = std::floor(blocks / (256 * s.fit)), rest = blocks / 256 - rounds * s.fit;
    double us = rounds * round(s.fit) + (rest > 0 ? round(rest) : 0);
    if (plan.splits > 1) us += 3.0 + (double)(count * plan.splits * M * N) * 8 / 5e6;
    return us;
}

// Up to four steps, where more blocks than four a compute unit write their results (a softmax's statistics are little to write), a block holds one step at a time.  us, so / otherwise: gradients of 8192 rows against
// 128000 x 256 2,578 / 2,784, 128000 x 64 1,741 / 1,996, 48 of 250 x 700 orthogonalised 199 / 247; but a loss of 4096 rows against 32000 x 256 156 / 124, one matrix of 256 x 256 91 / 84.
constexpr size_t kFewSteps = 4, kFewBlocks = 1024;

inline Plan plan_of(size_t M, size_t N, size_t K, size_t count, bool may_split, bool symmetric = false, bool written = true) {
    const size_t steps = (K + kStep - 1) / kStep;
    Plan best{1, 1};
    double least = 1e300;
    auto consider = [&](const Plan &plan) {
        const double us = cost_of(M, N, K, count, plan);
        if (us < least) least = us, best = plan;
    };
    const size_t small = tiles_of(M, 1) * tiles_of(N, 1) * count;
    if (written && small <= kMaxBlocks && (steps == 1 || (steps <= kFewSteps && small > kFewBlocks))) return {1, 1, false, true};
    for (const Shape &s : kShapes) {
        const size_t tiles = tiles_of(M, s.tile) * tiles_of(N, s.tile) * count;
        consider({s.tile, 1});
        if (symmetric && tiles > count) consider({s.tile, 1, true});
        // no more parts than fill the card once
        for (size_t splits = 2; may_split && splits * 2 <= steps && tiles * splits <= (size_t)(256 * s.fit); splits *= 2) consider({s.tile, splits});
    }
    return best;
}

// bytes of partial sums
inline size_t parts_bytes(const Plan &plan, size_t count, size_t M, size_t N) { return plan.splits > 1 ? count * plan.splits * M * N * sizeof(float) : 0; }

struct Product {
    Operand a, b;
    size_t count, M, N, steps;
    float *parts;              // as many as the plan asks for
    bool twofold = false;      // operands are sums of two
    size_t tail = kStep;       // k of the last step
};

template <typename E, bool A_DOWN, bool B_DOWN, typename End>
int run(const Plan &plan, const Product &p, const typename End::Args &end, hipStream_t stream) {
    const size_t tiles_m = tiles_of(p.M, plan.tile), tiles_n = tiles_of(p.N, plan.tile), bands = plan.half ? bands_of(tiles_m) : 0;
    const size_t blocks = (bands ? half_tiles((uint32_t)tiles_m, (uint32_t)bands) : tiles_m * tiles_n) * plan.splits * p.count;
    if (blocks > kMaxBlocks) return SS_ERR_ARG;
    const TilesArgs<typename End::Args> args{p.a, p.b, (uint32_t)p.M, (uint32_t)p.N, (uint32_t)(p.twofold ? 3 * p.steps : p.steps), (uint32_t)p.tail, (uint32_t)p.steps, (uint32_t)tiles_m, (uint32_t)tiles_n, (uint32_t)plan.splits, (uint32_t)bands, p.parts, end};
    const auto kernel = plan.few         ? tiles_kernel<E, A_DOWN, B_DOWN, 1, End, End::kStrips>
                        : plan.tile == 4 ? tiles_kernel<E, A_DOWN, B_DOWN, 4, End>
                        : plan.tile == 2 ? tiles_kernel<E, A_DOWN, B_DOWN, 2, End>
                                         : tiles_kernel<E, A_DOWN, B_DOWN, 1, End>;
    const int rc = host::launch(kernel, blocks, 0, stream, args, 256);
    if (rc != SS_OK || plan.splits == 1) return rc;
    if constexpr (End::kParts) {
        const uint64_t across = (p.N + 7) / 8, eights = across * p.M * p.count;
        uint32_t slices = 1;      // until there is a block for each compute unit, or two parts for a lane
        while (slices < 64 && eights * slices < 256 * 256 && 4 * slices <= plan.splits) slices *= 2;
        const uint64_t blocks_of = (eights * slices + 255) / 256;
        if (blocks_of > kMaxBlocks) return SS_ERR_ARG;
        const JoinArgs<typename End::Args> join{p.parts, (uint32_t)p.M, (uint32_t)p.N, (uint32_t)plan.splits, (uint32_t)across, eights, slices, end};
        return host::launch(join_kernel<End>, blocks_of, 0, stream, join, 256);
    }
    return SS_ERR_ARG;
}

// parts of one scratch buffer, one after the other at multiples of 256 bytes
struct Layout {
    size_t bytes = 0;
    size_t take(size_t n) {
        const size_t at = bytes;
        bytes += rounded(n, 256);
        return at;
    }
};

}  // namespace product
