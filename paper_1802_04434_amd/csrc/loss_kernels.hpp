// Softmax cross entropy over a large vocabulary, z = h w^T, and its gradient, neither of which keeps z.
//
// Forward: the tiles of z stay in registers; of each row a tile leaves its largest entry m and the sum of exp(z - m), and
// whoever has the target's column leaves that entry.  One kernel joins them: lse = M + log(sum of s exp(m - M)).
// Backward: with lse in hand exp(z - lse) is the softmax, so that D = dloss (softmax - target) is computed tile by tile once more, a
// piece of the vocabulary at a time, rounded to bf16 for the products dh += D w and dw = D^T h.
#pragma once
#include "product_kernels.hpp"

#pragma clang fp contract(off)

namespace loss {

using product::f32x16;
using product::f32x4;
using product::u32x4;

constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }

// ------------------------------------------------------------- forward ----

struct Part {
    float top, sum;
};

template <bool RAGGED>
struct StatsEnd {
    static constexpr bool kStrips = false, kParts = false, kRagged = RAGGED;
    struct Args {
        Part *parts;               // (half a tile's columns, row)
        float *picked;             // the target's logit, by row
        const int64_t *target;
        int64_t first;             // token of column 0
        uint32_t part0;            // the first part of this piece
    };
    // A wave's 32 T rows by 32 T columns of z; a row is in lanes r and r + 32, four columns of each eight
    template <int T>
    static __device__ __forceinline__ void finish(const Args &a, const f32x16 (&c)[T][T], uint32_t m, uint32_t n, uint32_t part, uint32_t M, uint32_t N, uint32_t r, uint32_t q) {
        if (N >= n + 32 * T) rows<T, true>(a, c, m, n, part, M, N, r, q);
        else rows<T, false>(a, c, m, n, part, M, N, r, q);
    }
    template <int T, bool INSIDE>
    static __device__ __forceinline__ void rows(const Args &a, const f32x16 (&c)[T][T], uint32_t m, uint32_t n, uint32_t part, uint32_t M, uint32_t N, uint32_t r, uint32_t q) {
        uint32_t left = N > n + 4 * q ? N - n - 4 * q : 0;      // columns from this lane's first one on: a part of none counts for nothing
        // 16 T comparisons with it kept for their next use take two scalar registers each, more than there are
        auto compare_anew = [&] {
            if constexpr (!INSIDE) asm volatile("" : "+v"(left));
        };
#pragma unroll
        for (int i = 0; i < T; ++i) {
            // Read from the matrix unit's registers row by row: the compiler would bring all 16 T^2 at once, 40 of them for T = 4 by way of memory (700 MB with 8192 rows against 128000).
            f32x16 z[T];
#pragma unroll
            for (int k = 0; k < T; ++k) {
                z[k] = c[i][k];
                asm volatile("" : "+a"(z[k]));
            }
            const uint32_t row = m + i * 32 + r;
            const bool there = row < M;
            const int64_t target = there ? a.target[row] : -1;
            float top = -__builtin_inff();
            compare_anew();
#pragma unroll
            for (int k = 0; k < T; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (INSIDE || k * 32 + e / 4 * 8 + e % 4 < left) top = fmaxf(top, z[k][e]);
            top = fmaxf(top, __shfl_xor(top, 32));
            // NaN passes: it is not the largest, but its exponential is NaN.  Where there is none but -infinity their exponentials are 0.
            const float from = top == -__builtin_inff() ? 0.0f : top;
            float sum = 0;
            compare_anew();
#pragma unroll
            for (int k = 0; k < T; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (INSIDE || k * 32 + e / 4 * 8 + e % 4 < left) sum += exp_of(z[k][e] - from);
            sum += __shfl_xor(sum, 32);
            if (there && q == 0) a.parts[(size_t)(a.part0 + part) * M + row] = Part{top, sum};
            const int64_t hit = target < 0 ? -1 : target - a.first - n - 4 * q;
            if (hit >= 0 && hit < 32 * T && hit < left) {
#pragma unroll
                for (int k = 0; k < T; ++k)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if ((uint32_t)hit == k * 32 + e / 4 * 8 + e % 4) a.picked[row] = z[k][e];
            }
        }
    }
};

struct JoinArgs {
    const Part *parts;
    const float *picked;
    const int64_t *target;
    float *loss, *lse;
    uint32_t T, count, rows;       // rows: of a block, a power of two; 256 / rows threads share one
    int64_t V;
};

__device__ __forceinline__ Part joined(Part x, Part y) {
    const float top = fmaxf(x.top, y.top);
    if (top == -__builtin_inff()) return Part{top, x.sum + y.sum};      // 0, or NaN
    return Part{top, x.sum * exp_of(x.top - top) + y.sum * exp_of(y.top - top)};
}

// The parts of a row, in an order that depends on their number and on T alone; eight loads of a thread are on the way together.  us with 16 rows a block / with 64 and a load at a time: 8192 rows of 1000
// parts (66 MB) 15 / 134, 301 of 314 4.6 / 30.6.
__global__ __launch_bounds__(256) void join_stats_kernel(const JoinArgs a) {
    __shared__ Part shared[256];
    const uint32_t in = threadIdx.x & (a.rows - 1), row = blockIdx.x * a.rows + in, slices = 256 / a.rows;
    Part s{-__builtin_inff(), 0.0f};
    if (row < a.T)
        for (uint32_t k = threadIdx.x / a.rows; k < a.count; k += 8 * slices) {
            Part p[8];
            float top = -__builtin_inff();
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x) {
                const uint32_t at = k + x * slices;
                p[x] = at < a.count ? a.parts[(size_t)at * a.T + row] : Part{-__builtin_inff(), 0.0f};
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) top = fmaxf(top, p[x].top);
            float sum = 0;
#pragma unroll
            for (int x = 0; x < 8; ++x) sum += top == -__builtin_inff() ? p[x].sum : p[x].sum * exp_of(p[x].top - top);
            s = joined(s, Part{top, sum});
        }
    shared[threadIdx.x] = s;
    __syncthreads();
    for (uint32_t half = 128; half >= a.rows; half >>= 1) {
        if (threadIdx.x < half) shared[threadIdx.x] = joined(shared[threadIdx.x], shared[threadIdx.x + half]);
        __syncthreads();
    }
    if (threadIdx.x >= a.rows || row >= a.T) return;
    s = shared[threadIdx.x];
    const float log_sum = logf(s.sum);
    const int64_t target = a.target[row];
    a.lse[row] = s.top + log_sum;
    // Not lse - picked: lse is rounded by the logits' size, 6e-5 where they are near 1000, while top - picked is exact wherever they are near each other, and 0 where the target is the
    // likeliest, whose loss is then the logarithm alone.
    a.loss[row] = target < 0 ? 0.0f : target < a.V ? (s.top - a.picked[row]) + log_sum : __builtin_nanf("");
}

// ------------------------------------------------------------ backward ----

// D of a row t is scale x factor_t x (softmax - target).  scale is the largest |dloss| of a row with a target and is multiplied in when the
// gradients are whole: where all rows weigh the same the factors are 1, and the target's entries, softmax - 1, lose next to nothing to
// bf16, where dloss itself would be off by up to 2^-8 in all rows alike.
struct FactorArgs {
    const float *dloss;            // NULL: 1
    const int64_t *target;
    float *factor, *scale;         // factor NULL: not wanted
    int64_t V;
    uint32_t T, padded;
};

constexpr uint32_t kPrepareThreads = 256;

// by one block
__device__ __forceinline__ void write_factors(const FactorArgs &a) {
    __shared__ float tops[kPrepareThreads / 64];
    float top = 0;
    // eight rows' loads on the way together
    auto rows = [&](uint32_t count, auto each) {
        for (uint32_t t0 = threadIdx.x; t0 < count; t0 += 8 * kPrepareThreads) {
            int64_t target[8];
            float w[8];
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x) {
                const uint32_t t = t0 + x * kPrepareThreads;
                target[x] = t < a.T ? a.target[t] : -1;
                w[x] = t < a.T && a.dloss ? a.dloss[t] : 1.0f;
            }
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x)
                if (t0 + x * kPrepareThreads < count) each(t0 + x * kPrepareThreads, target[x], w[x]);
        }
    };
    rows(a.T, [&](uint32_t, int64_t target, float w) { top = fmaxf(top, target < 0 ? 0.0f : fabsf(w)); });      // not of NaN, which its own row's factor keeps
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = 0;
    for (uint32_t k = 0; k < kPrepareThreads / 64; ++k) top = fmaxf(top, tops[k]);
    // 1 where there is nothing to weigh, or an infinity
    const float scale = top > 0.0f && top < __builtin_inff() ? top : 1.0f;
    if (threadIdx.x == 0) *a.scale = scale;
    rows(a.padded, [&](uint32_t t, int64_t target, float w) { a.factor[t] = target < 0 ? 0.0f : target >= a.V ? __builtin_nanf("") : w / scale; });
}

// D, whole eights of columns and rows: zero beyond the vocabulary and in rows without a target
template <bool RAGGED>
struct SoftmaxEnd {
    static constexpr bool kStrips = true, kParts = false, kSymmetric = false, kRagged = RAGGED;
    struct Args {
        const float *lse, *factor;
        const int64_t *target;
        int64_t first;             // token of column 0
        __bf16 *d;
        uint32_t ld, T, vocab;     // vocab: columns there are
    };
    struct Besides {
        float lse, factor;
        int64_t target;
    };
    static __device__ __forceinline__ Besides load(const Args &a, uint32_t, uint32_t row, uint32_t, uint32_t) {
        return row < a.T ? Besides{a.lse[row], a.factor[row], a.target[row]} : Besides{0, 0, -1};
    }
    static __device__ __forceinline__ void finish(const Args &a, const Besides &b, uint32_t, uint32_t col, f32x4 (&v)[2]) {
        const uint64_t behind = (uint64_t)(b.target - a.first - col);
        const uint32_t hit = b.target >= 0 && behind < 8 ? (uint32_t)behind : 8u;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const float p = exp_of(v[x / 4][x % 4] - b.lse);
            v[x / 4][x % 4] = b.factor * (hit == x ? p - 1.0f : p);
        }
        if (b.target < 0 || col + 8 > a.vocab)      // NaN times zero would not be zero
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if (b.target < 0 || col + x >= a.vocab) v[x / 4][x % 4] = 0.0f;
    }
    static __device__ __forceinline__ void put(const Args &a, uint32_t, uint32_t row, uint32_t col, const f32x4 (&v)[2], uint32_t) {
        product::bf16x8 o;
#pragma unroll
        for (int x = 0; x < 8; ++x) o[x] = (__bf16)v[x / 4][x % 4];
        *reinterpret_cast<u32x4 *>(a.d + (size_t)row * a.ld + col) = __builtin_bit_cast(u32x4, o);
    }
};

// A gradient, or with the pieces before it the sum so far
struct GradientEnd {
    static constexpr bool kStrips = true, kParts = true, kSymmetric = false, kRagged = false;
    struct Args {
        const float *scale;
        float *sum;                // rows x N: not wanted where a piece is all there is
        void *out;
        uint64_t ld;
        bool first, last, bf16;
    };
    struct Besides {
        f32x4 v[2];
    };
    static __device__ __forceinline__ Besides load(const Args &a, uint32_t, uint32_t row, uint32_t col, uint32_t N) {
        Besides b = {};
        if (a.first) return b;
        const float *sum = a.sum + (size_t)row * N + col;
        if (N - col >= 8)
#pragma unroll
            for (int h = 0; h < 2; ++h) b.v[h] = *reinterpret_cast<const product::f32x4_any *>(sum + 4 * h);
        else
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x)
                if (col + x < N) b.v[x / 4][x % 4] = sum[x];
        return b;
    }
    static __device__ __forceinline__ void finish(const Args &, const Besides &b, uint32_t, uint32_t, f32x4 (&v)[2]) { v[0] += b.v[0], v[1] += b.v[1]; }
    static __device__ __forceinline__ void put(const Args &a, uint32_t, uint32_t row, uint32_t col, f32x4 (&v)[2], uint32_t N) {
        const uint32_t n = N - col;
        if (!a.last) {
            product::store_eight<float, f32x4>(a.sum + (size_t)row * N + col, v, n);
            return;
        }
        const float scale = *a.scale;
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x / 4][x % 4] *= scale;
        product::store_out(a.out, a.bf16, (size_t)row * a.ld + col, v, n);
    }
};

// ------------------------------------------------------ operands that are copied ----

// rows x cols elements with zeros around them, rows of `ld` (a multiple of 64) elements from 16-byte aligned memory: an operand that the products can load.
// Rows without a target become zero, so that whatever a padded batch holds there meets a zero of D as a zero.
struct Copy {
    const uint16_t *from;
    uint16_t *to;
    const int64_t *target;         // NULL: all rows stay
    uint64_t ld_from;
    uint32_t rows, cols, ld, lines;
    uint32_t blocks;               // 0: nothing to copy
};

__device__ __forceinline__ void copy_rows(const Copy &a, uint32_t block) {
    const uint64_t at = (uint64_t)block * kPrepareThreads + threadIdx.x;
    const uint32_t across = a.ld / 8;
    const uint32_t row = (uint32_t)(at / across), col = (uint32_t)(at - (uint64_t)row * across) * 8;
    if (row >= a.lines) return;
    u32x4 v = {0, 0, 0, 0};
    if (row < a.rows && col < a.cols && (!a.target || a.target[row] >= 0)) {
        const uint16_t *from = a.from + row * a.ld_from + col;
        if (col + 8 <= a.cols) v = *reinterpret_cast<const product::u32x4_16 *>(from);
        else
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x)
                if (col + x < a.cols) v[x / 2] |= (uint32_t)from[x] << (x % 2 * 16);
    }
    *reinterpret_cast<u32x4 *>(a.to + (size_t)row * a.ld + col) = v;
}

// What comes before the products, in one launch: the rows' factors by the first block, then the copies.
struct PrepareArgs {
    FactorArgs factors;
    Copy h, w;
};

__global__ __launch_bounds__(kPrepareThreads) void prepare_kernel(const PrepareArgs a) {
    uint32_t block = blockIdx.x;
    if (a.factors.factor && block-- == 0) write_factors(a.factors);
    else if (block < a.h.blocks) copy_rows(a.h, block);
    else copy_rows(a.w, block - a.h.blocks);
}

// the gradient of no rows at all
struct ZeroArgs {
    void *out;
    uint64_t ld, size;
    uint32_t cols;
    bool bf16;
};

__global__ __launch_bounds__(256) void zero_kernel(const ZeroArgs a) {
    for (uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x; at < a.size; at += (uint64_t)gridDim.x * 256) {
        const uint64_t row = at / a.cols, to = row * a.ld + at - row * a.cols;
        if (a.bf16) static_cast<uint16_t *>(a.out)[to] = 0;
        else static_cast<float *>(a.out)[to] = 0;
    }
}

}  // namespace loss
