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

__device__ __forceinline__ float element(const void *p, bool bf16, size_t at) {
    return bf16 ? ss::widen_bf16(static_cast<const uint16_t *>(p)[at]) : static_cast<const float *>(p)[at];
}

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
    bool bf16, ahead;
};

__device__ __forceinline__ float update_of(const BeginArgs &a, float g, float m) {
    return !a.m ? g : a.ahead ? ss::momentum(a.beta, 1.0f - a.beta, m, g) : m;
}

__global__ __launch_bounds__(256) void norm_kernel(const BeginArgs a) {
    __shared__ double shared[4];
    const uint32_t stack = blockIdx.y;
    const size_t size = (size_t)a.rows * a.cols;
    double sum = 0;
    for (size_t at = (size_t)blockIdx.x * 256 + threadIdx.x; at < size; at += (size_t)a.blocks * 256) {
        const uint32_t row = (uint32_t)(at / a.cols), col = (uint32_t)(at - (size_t)row * a.cols);
        const float g = element(a.g, a.bf16, stack * a.apart + row * a.ld + col);
        float m = 0;
        if (a.m) {
            float *to = a.m + stack * size + at;
            m = ss::momentum(a.beta, 1.0f - a.beta, *to, g);
            *to = m;
        }
        const double u = update_of(a, g, m);
        sum += u * u;
    }
    sum = ss::sum_wave(sum);
    if ((threadIdx.x & 63) == 63) shared[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[(size_t)stack * a.blocks + blockIdx.x] = shared[0] + shared[1] + shared[2] + shared[3];
}

// X = u / |u|, scaled, with zeros around it; zero if u is, NaN if its norm is not finite
__global__ __launch_bounds__(256) void scale_kernel(const BeginArgs a) {
    __shared__ double shared[4];
    const uint32_t stack = blockIdx.y;
    double sum = 0;
    for (uint32_t k = threadIdx.x; k < a.blocks; k += 256) sum += a.sums[(size_t)stack * a.blocks + k];
    sum = ss::sum_wave(sum);
    if ((threadIdx.x & 63) == 63) shared[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = shared[0] + shared[1] + shared[2] + shared[3];
    const double scale = sum == 0 ? 0 : sum < __builtin_inf() ? kScale / sqrt(sum) : __builtin_nan("");
    const uint32_t across = a.cols_padded / 8;
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t row = (uint32_t)(at / across), col = (uint32_t)(at - (uint64_t)row * across) * 8;
    if (row >= a.rows_padded) return;
    f16x8 hi = {}, lo = {};
    if (row < a.rows)
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x)
            if (col + x < a.cols) {
                const float g = element(a.g, a.bf16, stack * a.apart + row * a.ld + col + x);
                const float m = a.m ? a.m[((size_t)stack * a.rows + row) * a.cols + col + x] : 0;
                const double v = update_of(a, g, m) * scale;
                hi[x] = (_Float16)(float)v;
                lo[x] = (_Float16)(float)(v - (double)(float)hi[x]);
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
