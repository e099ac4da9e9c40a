// Host side of the products of 16-bit matrices (product_kernels.hpp): how one is cut, and its launches.
#pragma once
#include <cmath>

#include "api_common.hpp"
#include "product_kernels.hpp"

namespace product {

constexpr size_t kMaxBlocks = (size_t)1 << 23;      // of 256 threads: a launch has fewer than 2^32

inline size_t rounded(size_t n, size_t to) { return (n + to - 1) / to * to; }
inline size_t tiles_of(size_t n, int tile) { return (n + 64 * (size_t)tile - 1) / (64 * (size_t)tile); }

// tiles of 64 times `tile` squared, the sum over k in `splits` parts
struct Plan {
    int tile;
    size_t splits;
};

inline Plan plan_of(size_t, size_t, size_t, size_t, bool) { return Plan{2, 1}; }

// bytes of partial sums
inline size_t parts_bytes(const Plan &plan, size_t count, size_t M, size_t N) { return plan.splits > 1 ? count * plan.splits * M * N * sizeof(float) : 0; }

struct Product {
    Operand a, b;
    size_t count, M, N, steps;
    float *parts;              // as many as the plan asks for
};

template <typename E, bool A_DOWN, bool B_DOWN, typename End>
int run(const Plan &plan, const Product &p, const typename End::Args &end, hipStream_t stream) {
    const size_t tiles_m = tiles_of(p.M, plan.tile), tiles_n = tiles_of(p.N, plan.tile), blocks = tiles_m * tiles_n * plan.splits * p.count;
    if (blocks > kMaxBlocks) return SS_ERR_ARG;
    const TilesArgs<typename End::Args> args{p.a, p.b, (uint32_t)p.M, (uint32_t)p.N, (uint32_t)p.steps, (uint32_t)tiles_m, (uint32_t)tiles_n, (uint32_t)plan.splits, p.parts, end};
    const int rc = host::launch(tiles_kernel<E, A_DOWN, B_DOWN, 2, End>, blocks, 0, stream, args, 256);
    if (rc != SS_OK || plan.splits == 1) return rc;
    if constexpr (End::kStrips) {
        const uint64_t across = (p.N + 7) / 8, eights = across * p.M * p.count;
        if ((eights + 255) / 256 > kMaxBlocks) return SS_ERR_ARG;
        const JoinArgs<typename End::Args> join{p.parts, (uint32_t)p.M, (uint32_t)p.N, (uint32_t)plan.splits, (uint32_t)across, eights, end};
        return host::launch(join_kernel<End>, (eights + 255) / 256, 0, stream, join, 256);
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
