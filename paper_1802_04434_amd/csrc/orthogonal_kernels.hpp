// The update of a matrix, orthogonalised: with X = u / |u|_F and a polynomial p(s) = a s + b s^3 + c s^5 that takes (0, 1] to near 1 when
// repeated, `steps` times X <- U p(S) V' for X = U S V', by products alone:
//     A = X X' (X'X for a tall X),  B = b A + c A A,  X <- a X + B X  (a X + X B).
//
// What is held in how many bits.  X is the sum of two fp16, hi + lo, 22 bits; the products take hi, A and B in fp16 (11 bits), all scaled by
// 2^12, since no entry of X passes 1.2 or of B 2.9 and the smallest entries stay normal: 8192 x 8192 equal ones are 2^-13, and in lo 2^-25.  Against the formula in 64 bits, for
// gradients and for normally distributed entries of 20 to 512 rows, five steps are off by 0.6e-3 to 1.7e-3 of the result's norm;
// with X in fp16 alone by up to 6e-3, in bf16 by 1e-2 to 5e-2.  Towards the end, where the singular values are near 1 and B is about -2.4 on them, a X and B X cancel, and the
// rounding of hi weighs three times what is left; so the last B, and the one before it, are computed as B + mu I, of smaller norm, and a X as (a - mu) X.
#pragma once
#include "product_kernels.hpp"

#pragma clang fp contract(off)

namespace orthogonal {

using product::f16x8;
using product::f32x4;
using product::u32x4;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kLast = 2.0f, kBefore = 0.8f;      // mu of the last step and of the one before it
constexpr float kScale = 4096.0f, kUnscale = 1.0f / 4096.0f;

// ------------------------------------------------------------ the update's norm ----

// g, and with momentum m <- beta m + (1 - beta) g, u = m or beta m + (1 - beta) g; else u = g
struct BeginArgs {
    const void *g;
    float *m;                      // (stack, rows, cols), or NULL
    double *sums;                  // of u^2: (stack, block)
    _Float16 *hi, *lo;             // (stack, padded rows, padded cols)
    uint64_t ld, apart;            // of g
    uint32_t rows, cols, rows_padded, cols_padded, blocks;
    float beta;
    bool bf16, ahead, flat;        // flat: g has no gaps, so that a matrix is one long row
};

__device__ __forceinline__ float update_of(const BeginArgs &a, float g, float m) {
    return !a.m ? g : a.ahead ? ss::momentum(a.beta, 1.0f - a.beta, m, g) : m;
}

// n of eight neighbours, zero beyond
__device__ __forceinline__ void load_eight(float (&v)[8], const void *p, bool bf16, size_t at, uint32_t n) {
    if (n >= 8 && bf16) {
        const u32x4 w = *reinterpret_cast<const product::u32x4_16 *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = ss::widen_bf16((uint16_t)(w[x / 2] >> (x % 2 * 16)));
    } else if (n >= 8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 w = *reinterpret_cast<const product::f32x4_any *>(static_cast<const float *>(p) + at + 4 * h);
#pragma unroll
            for (int x = 0; x < 4; ++x) v[4 * h + x] = w[x];
        }
    } else {
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x)
            v[x] = x >= n ? 0.0f : bf16 ? ss::widen_bf16(static_cast<const uint16_t *>(p)[at + x]) : static_cast<const float *>(p)[at + x];
    }
}

// Squares are exact in fp64 and added there.  A wave takes 512 neighbours of a row at a time.  us: 4096 x 4096 bf16 with momentum NORM_STEP, 8192 x 8192 bf16 NORM_LARGE.
__global__ __launch_bounds__(256) void norm_kernel(const BeginArgs a) {
    __shared__ double shared[4];
    const uint32_t stack = blockIdx.y, lane = threadIdx.x & 63u;
    const uint64_t size = (uint64_t)a.rows * a.cols, cols = a.flat ? size : a.cols;
    const uint32_t rows = a.flat ? 1 : a.rows, across = (uint32_t)((cols + 511) / 512);
    const uint64_t units = (uint64_t)rows * across;
    double sum = 0;
    for (uint64_t unit = product::uniform(blockIdx.x * 4 + (threadIdx.x >> 6)); unit < units; unit += (uint64_t)a.blocks * 4) {
        const uint32_t row = (uint32_t)(unit / across);
        const uint64_t col = (unit - (uint64_t)row * across) * 512 + lane * 8;
        if (col >= cols) continue;
        const uint32_t n = cols - col < 8 ? (uint32_t)(cols - col) : 8u;
        float g[8], m[8] = {};
        load_eight(g, a.g, a.bf16, stack * a.apart + row * a.ld + col, n);
        if (a.m) {
            float *to = a.m + stack * size + row * cols + col;
            load_eight(m, to, false, 0, n);
            f32x4 v[2];
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x / 4][x % 4] = m[x] = ss::momentum(a.beta, 1.0f - a.beta, m[x], g[x]);
            product::store_eight<float, f32x4>(to, v, n);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const double u = update_of(a, g[x], m[x]);
            if (x < n) sum += u * u;
        }
    }
    sum = ss::sum_wave(sum);
    if (lane == 63) shared[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[(size_t)stack * a.blocks + blockIdx.x] = shared[0] + shared[1] + shared[2] + shared[3];
}

// 4096 / norm as f x p x p: f in [1, 4) and p a power of two, so that no product with an element of the matrix leaves fp32's range on the way and only
// the last one rounds; all of it zero for a matrix of zeros, NaN where the norm is not finite
struct Scale {
    float f, p;
    __device__ __forceinline__ explicit Scale(double sum) {
        if (sum == 0) f = 0, p = 1;
        else if (!(sum < __builtin_inf())) f = __builtin_nanf(""), p = 1;
        else {
            const double s = (double)kScale / sqrt(sum);        // 2^-130 (many elements near the largest) to 2^161
            const int half = (int)(__builtin_bit_cast(uint64_t, s) >> 52) - 1023 >> 1;
            const double one = __builtin_bit_cast(double, (uint64_t)(1023 + half) << 52);
            p = (float)one;
            f = (float)(s / one / one);
        }
    }
    __device__ __forceinline__ float operator()(float u) const { return u * p * p * f; }
};

// X = u / |u|, scaled, with zeros around it
__global__ __launch_bounds__(256) void scale_kernel(const BeginArgs a) {
    __shared__ double shared[4];
    const uint32_t stack = blockIdx.y;
    const uint32_t across = a.cols_padded / 8, at = blockIdx.x * 256 + threadIdx.x;
    const uint32_t row = at / across, col = (at - row * across) * 8;
    const bool there = row < a.rows && col < a.cols;
    const uint32_t n = there ? (a.cols - col < 8 ? a.cols - col : 8u) : 0u;
    float g[8] = {}, m[8] = {};
    if (there) {
        load_eight(g, a.g, a.bf16, stack * a.apart + row * a.ld + col, n);
        if (a.m) load_eight(m, a.m, false, ((size_t)stack * a.rows + row) * a.cols + col, n);
    }
    double sum = 0;
    for (uint32_t k = threadIdx.x; k < a.blocks; k += 256) sum += a.sums[(size_t)stack * a.blocks + k];
    sum = ss::sum_wave(sum);
    if ((threadIdx.x & 63) == 63) shared[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (row >= a.rows_padded) return;
    const Scale scale(shared[0] + shared[1] + shared[2] + shared[3]);
    f16x8 hi, lo;
#pragma unroll
    for (uint32_t x = 0; x < 8; ++x) {
        const float v = x < n ? scale(update_of(a, g[x], m[x])) : 0.0f;
        hi[x] = (_Float16)v;
        lo[x] = (_Float16)(v - (float)hi[x]);
    }
    const size_t to = ((size_t)stack * a.rows_padded + row) * a.cols_padded + col;
    *reinterpret_cast<u32x4 *>(a.hi + to) = __builtin_bit_cast(u32x4, hi);
    *reinterpret_cast<u32x4 *>(a.lo + to) = __builtin_bit_cast(u32x4, lo);
}

// ------------------------------------------------------------ what becomes of a product ----

// A = X X', from sums that are scaled twice
struct SquareEnd {
    static constexpr bool kStrips = true;
    struct Args {
        _Float16 *out;
        uint64_t apart;
    };
    static __device__ __forceinline__ void store(const Args &a, uint32_t stack, uint32_t row, uint32_t col, const f32x4 (&v)[2], uint32_t N) {
        f16x8 o;
#pragma unroll
        for (int x = 0; x < 8; ++x) o[x] = (_Float16)(v[x / 4][x % 4] * kUnscale);
        *reinterpret_cast<u32x4 *>(a.out + stack * a.apart + (size_t)row * N + col) = __builtin_bit_cast(u32x4, o);
    }
};

// B + mu I = b A + c A A + mu I
struct PolynomialEnd {
    static constexpr bool kStrips = true;
    struct Args {
        const _Float16 *a;
        _Float16 *out;
        uint64_t apart;
        float mu;
    };
    static __device__ __forceinline__ void store(const Args &a, uint32_t stack, uint32_t row, uint32_t col, const f32x4 (&v)[2], uint32_t N) {
        const size_t at = stack * a.apart + (size_t)row * N + col;
        const f16x8 was = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4 *>(a.a + at));
        f16x8 o;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            float s = kB * (float)was[x] + kC * (v[x / 4][x % 4] * kUnscale);
            if (row == col + x) s += a.mu * kScale;
            o[x] = (_Float16)s;
        }
        *reinterpret_cast<u32x4 *>(a.out + at) = __builtin_bit_cast(u32x4, o);
    }
};

// X <- (a - mu) X + (B + mu I) X; the last time into the result, or off the parameters
struct UpdateEnd {
    static constexpr bool kStrips = true;
    struct Args {
        const _Float16 *hi;
        _Float16 *lo, *hi_out;     // lo in place
        void *out;                 // NULL: not the last time
        uint64_t apart, ld, out_apart;
        uint32_t rows, cols;       // of the result
        float factor;              // a - mu
        float delta;               // out <- out - delta X where `step`
        bool step, bf16;
    };
    static __device__ __forceinline__ void store(const Args &a, uint32_t stack, uint32_t row, uint32_t col, f32x4 (&v)[2], uint32_t N) {
        const size_t at = stack * a.apart + (size_t)row * N + col;
        const f16x8 hi = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4 *>(a.hi + at));
        const f16x8 lo = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4 *>(a.lo + at));
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x / 4][x % 4] = a.factor * ((float)hi[x] + (float)lo[x]) + v[x / 4][x % 4] * kUnscale;
        if (!a.out) {
            f16x8 h, l;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                h[x] = (_Float16)v[x / 4][x % 4];
                l[x] = (_Float16)(v[x / 4][x % 4] - (float)h[x]);
            }
            *reinterpret_cast<u32x4 *>(a.hi_out + at) = __builtin_bit_cast(u32x4, h);
            *reinterpret_cast<u32x4 *>(a.lo + at) = __builtin_bit_cast(u32x4, l);
            return;
        }
        if (row >= a.rows || col >= a.cols) return;
        const uint32_t n = a.cols - col;
        const size_t to = stack * a.out_apart + row * a.ld + col;
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x / 4][x % 4] *= kUnscale;
        if (a.step) {
            float *p = static_cast<float *>(a.out) + to;
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x)
                if (x < n) v[x / 4][x % 4] = p[x] - a.delta * v[x / 4][x % 4];
        }
        product::store_out(a.out, a.bf16, to, v, n);
    }
};

}  // namespace orthogonal
