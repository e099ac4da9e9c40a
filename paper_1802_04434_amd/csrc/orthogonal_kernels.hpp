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
using product::f32x16;
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

// Squares are exact in fp64 and added there.  A wave takes 512 neighbours of a row at a time.  us: 4096 x 4096 bf16 with momentum 31, 8192 x 8192 bf16 44 (3 TB/s).
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
            const int half = ((int)(__builtin_bit_cast(uint64_t, s) >> 52) - 1023) >> 1;
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

// eight neighbours as hi, and lo where it is wanted
__device__ __forceinline__ void put_eight(_Float16 *hi, _Float16 *lo, size_t at, const f32x4 (&v)[2]) {
    f16x8 h;
#pragma unroll
    for (int x = 0; x < 8; ++x) h[x] = (_Float16)v[x / 4][x % 4];
    *reinterpret_cast<u32x4 *>(hi + at) = __builtin_bit_cast(u32x4, h);
    if (!lo) return;
    f16x8 l;
#pragma unroll
    for (int x = 0; x < 8; ++x) l[x] = (_Float16)(v[x / 4][x % 4] - (float)h[x]);
    *reinterpret_cast<u32x4 *>(lo + at) = __builtin_bit_cast(u32x4, l);
}
struct Eight {
    u32x4 hi, lo;
};
__device__ __forceinline__ Eight load_halves(const _Float16 *hi, const _Float16 *lo, size_t at) {
    return Eight{*reinterpret_cast<const u32x4 *>(hi + at), lo ? *reinterpret_cast<const u32x4 *>(lo + at) : u32x4{0, 0, 0, 0}};
}
__device__ __forceinline__ void sum_halves(f32x4 (&v)[2], const Eight &e) {
    const f16x8 h = __builtin_bit_cast(f16x8, e.hi), l = __builtin_bit_cast(f16x8, e.lo);
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x / 4][x % 4] = (float)h[x] + (float)l[x];
}

// A = X X', from sums that are scaled twice
struct SquareEnd {
    static constexpr bool kStrips = true, kParts = true, kSymmetric = true, kRagged = false;
    struct Args {
        _Float16 *hi, *lo;
        uint64_t apart;
    };
    typedef product::None Besides;
    static __device__ __forceinline__ Besides load(const Args &, uint32_t, uint32_t, uint32_t, uint32_t) { return {}; }
    static __device__ __forceinline__ void finish(const Args &, const Besides &, uint32_t, uint32_t, f32x4 (&v)[2]) {
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x / 4][x % 4] *= kUnscale;
    }
    static __device__ __forceinline__ void put(const Args &a, uint32_t stack, uint32_t row, uint32_t col, const f32x4 (&v)[2], uint32_t N) {
        put_eight(a.hi, a.lo, stack * a.apart + (size_t)row * N + col, v);
    }
};

// B + mu I = b A + c A A + mu I
struct PolynomialEnd {
    static constexpr bool kStrips = true, kParts = false, kSymmetric = true, kRagged = false;
    struct Args {
        const _Float16 *a_hi, *a_lo;
        _Float16 *hi, *lo;
        uint64_t apart;
        float mu;
    };
    typedef Eight Besides;
    static __device__ __forceinline__ Besides load(const Args &a, uint32_t stack, uint32_t row, uint32_t col, uint32_t N) {
        return load_halves(a.a_hi, a.a_lo, stack * a.apart + (size_t)row * N + col);
    }
    static __device__ __forceinline__ void finish(const Args &a, const Besides &besides, uint32_t row, uint32_t col, f32x4 (&v)[2]) {
        f32x4 was[2];
        sum_halves(was, besides);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            v[x / 4][x % 4] = kB * was[x / 4][x % 4] + kC * (v[x / 4][x % 4] * kUnscale);
            if (row == col + x) v[x / 4][x % 4] += a.mu * kScale;
        }
    }
    static __device__ __forceinline__ void put(const Args &a, uint32_t stack, uint32_t row, uint32_t col, const f32x4 (&v)[2], uint32_t N) {
        put_eight(a.hi, a.lo, stack * a.apart + (size_t)row * N + col, v);
    }
};

// X <- (a - mu) X + (B + mu I) X; the last time into the result, or off the parameters
struct UpdateEnd {
    static constexpr bool kStrips = true, kParts = false, kSymmetric = false, kRagged = false;
    struct Args {
        const _Float16 *hi, *lo;
        _Float16 *hi_out, *lo_out;
        void *out;                 // NULL: not the last time
        uint64_t apart, ld, out_apart;
        uint32_t rows, cols;       // of the result
        float factor;              // a - mu
        float delta;               // out <- out - delta X where `step`
        bool step, bf16;
    };
    typedef Eight Besides;
    static __device__ __forceinline__ Besides load(const Args &a, uint32_t stack, uint32_t row, uint32_t col, uint32_t N) {
        return load_halves(a.hi, a.lo, stack * a.apart + (size_t)row * N + col);
    }
    static __device__ __forceinline__ void finish(const Args &a, const Besides &besides, uint32_t, uint32_t, f32x4 (&v)[2]) {
        f32x4 was[2];
        sum_halves(was, besides);
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x / 4][x % 4] = a.factor * was[x / 4][x % 4] + v[x / 4][x % 4] * kUnscale;
    }
    static __device__ __forceinline__ void put(const Args &a, uint32_t stack, uint32_t row, uint32_t col, f32x4 (&v)[2], uint32_t N) {
        if (!a.out) {
            put_eight(a.hi_out, a.lo_out, stack * a.apart + (size_t)row * N + col, v);
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

// ------------------------------------------------------------ small matrices, whole ----

// A matrix that fits into LDS with A beside it takes one block and one launch: 64 x 64 18 us (60 in the launches of the products above), 128 x 128 50 (85).  X lies as
// `longer` rows of `shorter` entries, whichever way round g does; both X and A are held in 22 bits, as hi + lo, and products are hi hi + hi lo + lo hi, which costs little here: what bounds
// it is the way from one product to the next, through LDS and a barrier.
struct WholeArgs {
    BeginArgs begin;
    void *out;
    uint64_t ld, apart;
    float delta;
    uint32_t steps;
    bool step, bf16;
};

constexpr int kWholeWaves = 16, kWholeTiles = 2;     // tiles of 32 squared that a wave may have to itself
constexpr int kWholeUnits = 4;                       // eights of a row that a thread brings: 32 tiles have no more
constexpr uint32_t kWholeBytes = 160 * 1024 - 256, kWholeHalf = 80 * 1024 - 256;

__host__ __device__ constexpr uint32_t whole_bytes(uint32_t shorter, uint32_t longer) { return 4 * (shorter + longer) * shorter; }

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Rows of S (32, 64, 96 or 128) entries in LDS.  Chunk c (eight entries) of row r lies at place c ^ x(r), so that neither 16 rows' same chunk nor four rows' four
// neighbouring chunks share a bank: the first is what a read along the rows takes at a time, the second one down them.
template <uint32_t S>
__device__ __forceinline__ uint32_t place(uint32_t row, uint32_t col) {
    const uint32_t x = (row >> 2 & 3u) ^ (S == 128 ? (row & 3u) << 2 : S == 64 ? (row & 2u) << 1 : 0u);
    return row * S * 2 + (((col >> 3) ^ x) << 4) + (col & 7u) * 2;
}

// eight neighbouring k of a row
template <uint32_t S>
__device__ __forceinline__ u32x4 along(const char *p, uint32_t row, uint32_t k, uint32_t lane) {
    return *reinterpret_cast<const u32x4 *>(p + place<S>(row + (lane & 31u), k + (lane >> 5) * 8));
}
// the same of a column, for k that lies down
template <uint32_t S>
__device__ __forceinline__ u32x4 down(const char *p, uint32_t col, uint32_t k, uint32_t lane) {
    const uint32_t t = lane & 15u, row = k + (lane >> 5) * 8 + (t >> 2), at = col + (lane >> 4 & 1u) * 16 + (t & 3u) * 4;
    typedef product::u32x2 u32x2;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((product::LdsFour)(p + place<S>(row, at))));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((product::LdsFour)(p + place<S>(row + 4, at))));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
}

// A tile of 32 squared: 32 rows (or columns, DOWN) from m on of one matrix with those from n on of the other, over `depth` (a multiple of 32).  Two sums, so that a
// multiplication seldom waits for the one before it, and the fragments of two steps on the way together.
template <uint32_t S, bool DOWN>
__device__ __forceinline__ f32x16 whole_tile(const char *mh, const char *ml, uint32_t m, const char *nh, const char *nl, uint32_t n, uint32_t depth, uint32_t lane) {
    f32x16 s = {}, t = {};
    auto read = [&](const char *p, uint32_t at, uint32_t k) { return DOWN ? down<S>(p, at, k, lane) : along<S>(p, at, k, lane); };
    auto multiply = [&](uint32_t k) {
        u32x4 f[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) f[h][0] = read(nh, n, k + 16 * h), f[h][1] = read(mh, m, k + 16 * h), f[h][2] = read(ml, m, k + 16 * h), f[h][3] = read(nl, n, k + 16 * h);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s = product::F16::multiply(f[h][0], f[h][1], s);
            t = product::F16::multiply(f[h][0], f[h][2], t);
            t = product::F16::multiply(f[h][3], f[h][1], t);
        }
    };
    if constexpr (DOWN) {
        for (uint32_t k = 0; k < depth; k += 32) multiply(k);
    } else {
#pragma unroll 2
        for (uint32_t k = 0; k < S; k += 32) multiply(k);
    }
    return s + t;
}

// four neighbours as hi + lo
__device__ __forceinline__ void put_four(char *hi, char *lo, size_t at, const f32x4 &v) {
    f16x4 h, l;
#pragma unroll
    for (int x = 0; x < 4; ++x) h[x] = (_Float16)v[x], l[x] = (_Float16)(v[x] - (float)h[x]);
    *reinterpret_cast<f16x4 *>(hi + at) = h;
    *reinterpret_cast<f16x4 *>(lo + at) = l;
}
__device__ __forceinline__ f32x4 get_four(const char *hi, const char *lo, uint32_t at) {
    const f16x4 h = *reinterpret_cast<const f16x4 *>(hi + at), l = *reinterpret_cast<const f16x4 *>(lo + at);
    return f32x4{(float)h[0] + (float)l[0], (float)h[1] + (float)l[1], (float)h[2] + (float)l[2], (float)h[3] + (float)l[3]};
}

template <uint32_t S, uint32_t BYTES>
__global__ __launch_bounds__(64 * kWholeWaves) void whole_kernel(const WholeArgs p) {
    __shared__ __attribute__((aligned(16))) char lds[BYTES];
    __shared__ double shared[kWholeWaves];
    constexpr uint32_t kThreads = 64 * kWholeWaves;
    const BeginArgs &a = p.begin;
    const uint32_t stack = blockIdx.x, lane = threadIdx.x & 63u, wave = product::uniform(threadIdx.x >> 6), r = lane & 31u, q = lane >> 5;
    const bool tall = a.rows > a.cols;
    const uint32_t longer = tall ? a.rows_padded : a.cols_padded;
    char *const xh = lds, *const xl = xh + longer * S * 2, *const ah = xl + longer * S * 2, *const al = ah + S * S * 2;
    // eights of a row, kept in registers: all loads are on the way together
    const uint32_t size = a.rows * a.cols, eights = (a.cols + 7) / 8, units = a.rows * eights;
    float u[kWholeUnits][8];
    double sum = 0;
#pragma unroll
    for (int k = 0; k < kWholeUnits; ++k) {
        const uint32_t unit = threadIdx.x + k * kThreads, row = unit / eights, col = (unit - row * eights) * 8;
        if (unit < units) load_eight(u[k], a.g, a.bf16, stack * a.apart + row * a.ld + col, a.cols - col);
        else
#pragma unroll
            for (int x = 0; x < 8; ++x) u[k][x] = 0;
    }
    if (a.m) {
#pragma unroll
        for (int k = 0; k < kWholeUnits; ++k) {
            const uint32_t unit = threadIdx.x + k * kThreads, row = unit / eights, col = (unit - row * eights) * 8;
            if (unit >= units) break;
            float *to = a.m + (size_t)stack * size + row * a.cols + col;
            float m[8];
            load_eight(m, to, false, 0, a.cols - col);
            f32x4 v[2];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                v[x / 4][x % 4] = m[x] = ss::momentum(a.beta, 1.0f - a.beta, m[x], u[k][x]);
                u[k][x] = update_of(a, u[k][x], m[x]);
            }
            product::store_eight<float, f32x4>(to, v, a.cols - col);
        }
    }
#pragma unroll
    for (int k = 0; k < kWholeUnits; ++k)
#pragma unroll
        for (int x = 0; x < 8; ++x) sum += (double)u[k][x] * (double)u[k][x];     // zero beyond a row
    sum = ss::sum_wave(sum);
    if (lane == 63) shared[wave] = sum;
    for (uint32_t at = threadIdx.x * 16; at < 4 * longer * S; at += kThreads * 16) *reinterpret_cast<u32x4 *>(lds + at) = u32x4{0, 0, 0, 0};
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int k = 0; k < kWholeWaves; ++k) sum += shared[k];
    const Scale scale(sum);
#pragma unroll
    for (int k = 0; k < kWholeUnits; ++k) {
        const uint32_t unit = threadIdx.x + k * kThreads, row = unit / eights, col = (unit - row * eights) * 8;
        if (unit >= units) break;
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x) {
            if (col + x >= a.cols) break;
            const float v = scale(u[k][x]);
            const uint32_t to = tall ? place<S>(row, col + x) : place<S>(col + x, row);
            const _Float16 h = (_Float16)v;
            *reinterpret_cast<_Float16 *>(xh + to) = h;
            *reinterpret_cast<_Float16 *>(xl + to) = (_Float16)(v - (float)h);
        }
    }
    __syncthreads();
    constexpr uint32_t across = S / 32, squares = across * across;
    const uint32_t tiles = longer / 32 * across;
    for (uint32_t step = 0; step < p.steps; ++step) {
        const float mu = step + 1 == p.steps ? kLast : step + 2 == p.steps ? kBefore : 0.0f;
        // A = X'X
        if (wave < squares) {
            const uint32_t m = wave / across * 32, n = wave % across * 32;
            const f32x16 s = whole_tile<S, true>(xh, xl, m, xh, xl, n, longer, lane);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                put_four(ah, al, place<S>(m + r, n + 8 * e + 4 * q), f32x4{s[4 * e], s[4 * e + 1], s[4 * e + 2], s[4 * e + 3]} * kUnscale);
        }
        __syncthreads();
        // B + mu I = b A + c A A + mu I, in A's place, and then X <- (a - mu) X + X (B + mu I)
#pragma unroll 1
        for (int x_too = 0; x_too < 2; ++x_too) {
            char *const ph = x_too ? xh : ah, *const pl = x_too ? xl : al;
            const uint32_t count = x_too ? tiles : squares;
            const float was_by = x_too ? kA - mu : kB, sum_by = x_too ? kUnscale : kC * kUnscale, diagonal = x_too ? 0.0f : mu * kScale;
            f32x16 c[kWholeTiles];
#pragma unroll
            for (int i = 0; i < kWholeTiles; ++i) {
                const uint32_t tile = wave + i * kWholeWaves, m = tile / across * 32, n = tile % across * 32;
                if (tile >= count) break;
                c[i] = whole_tile<S, false>(ph, pl, m, ah, al, n, S, lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 was = get_four(ph, pl, place<S>(m + r, n + 8 * e + 4 * q));
#pragma unroll
                    for (int x = 0; x < 4; ++x) c[i][4 * e + x] = __builtin_fmaf(was_by, was[x], c[i][4 * e + x] * sum_by);
                }
                if (m == n && diagonal != 0.0f)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (r == e / 4 * 8 + 4 * q + e % 4) c[i][e] += diagonal;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWholeTiles; ++i) {
                const uint32_t tile = wave + i * kWholeWaves, m = tile / across * 32, n = tile % across * 32;
                if (tile >= count) break;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    put_four(ph, pl, place<S>(m + r, n + 8 * e + 4 * q), f32x4{c[i][4 * e], c[i][4 * e + 1], c[i][4 * e + 2], c[i][4 * e + 3]});
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int k = 0; k < kWholeUnits; ++k) {
        const uint32_t unit = threadIdx.x + k * kThreads, row = unit / eights, col = (unit - row * eights) * 8, n = a.cols - col;
        if (unit >= units) break;
        f32x4 v[2];
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x) {
            const uint32_t at = x >= n ? 0 : tall ? place<S>(row, col + x) : place<S>(col + x, row);
            v[x / 4][x % 4] = ((float)*reinterpret_cast<const _Float16 *>(xh + at) + (float)*reinterpret_cast<const _Float16 *>(xl + at)) * kUnscale;
        }
        const size_t to = stack * p.apart + row * p.ld + col;
        if (p.step) {
            float was[8];
            load_eight(was, p.out, false, to, n);
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x / 4][x % 4] = was[x] - p.delta * v[x / 4][x % 4];
        }
        product::store_out(p.out, p.bf16, to, v, n);
    }
}

// ------------------------------------------------------------ long matrices with a short side, in slices ----
// With a shorter side of 128 at most, B is so small that every block computes it for itself: a block has a slice of X's longer side in LDS, makes B of A there, its slice of the next X, and that
// slice's part of the next A, so that a step takes two launches instead of three or four: this, and the one that adds the parts.  Both X and A have 22 bits, as above.
// 25 x 7616 takes 48 us in 12 launches (100 with the products above), 1000 x 120 with its momentum 73 (101); most of a launch is the way to it and back.
template <uint32_t S>
constexpr uint32_t kSlice = S <= 64 ? 128 : 64;      // of the longer side: one eight of a row of g, and one tile of 32 squared a wave

struct SliceArgs {
    BeginArgs begin;               // hi, lo: (stack, slices, kSlice, S)
    const _Float16 *a_hi, *a_lo;   // (stack, S, S); NULL the first time, when the slice comes from g
    float *parts;                  // (stack, slices, S, S)
    void *out;                     // NULL: not the last time
    uint64_t ld, apart;
    float delta, mu;
    uint32_t slices;
    bool step, bf16;
};

// rows of S entries between memory and LDS
template <uint32_t S>
__device__ __forceinline__ void bring_rows(char *lds, const _Float16 *from, uint32_t rows) {
    for (uint32_t at = threadIdx.x; at < rows * (S / 8); at += 64 * kWholeWaves)
        *reinterpret_cast<u32x4 *>(lds + place<S>(at / (S / 8), at % (S / 8) * 8)) = *reinterpret_cast<const u32x4 *>(from + at * 8);
}
template <uint32_t S>
__device__ __forceinline__ void take_rows(const char *lds, _Float16 *to, uint32_t rows) {
    for (uint32_t at = threadIdx.x; at < rows * (S / 8); at += 64 * kWholeWaves)
        *reinterpret_cast<u32x4 *>(to + at * 8) = *reinterpret_cast<const u32x4 *>(lds + place<S>(at / (S / 8), at % (S / 8) * 8));
}

template <uint32_t S>
__global__ __launch_bounds__(64 * kWholeWaves) void slice_kernel(const SliceArgs p) {
    constexpr uint32_t W = kSlice<S>, kX = W * S * 2, kSquare = S * S * 2, across = S / 32;
    static_assert(across * across <= kWholeWaves && W / 32 * across <= kWholeWaves && W * S / 8 <= 64 * kWholeWaves, "one tile a wave, one eight a thread");
    __shared__ __attribute__((aligned(16))) char lds[2 * (kX + kSquare)];
    __shared__ double shared[kWholeWaves];
    char *const xh = lds, *const xl = xh + kX, *const ah = xl + kX, *const al = ah + kSquare;
    const BeginArgs &a = p.begin;
    const uint32_t slice = blockIdx.x, stack = blockIdx.y, lane = threadIdx.x & 63u, wave = product::uniform(threadIdx.x >> 6), r = lane & 31u, q = lane >> 5;
    const bool tall = a.rows > a.cols;
    // this thread's eight of g: of a row of the slice, or of a row's part that belongs to it
    const uint32_t eights = tall ? (a.cols + 7) / 8 : W / 8, line = threadIdx.x / eights, first = threadIdx.x % eights * 8;
    const uint32_t row = tall ? slice * W + line : line, col = tall ? first : slice * W + first;
    const bool mine = (tall ? line < W : true) && row < a.rows && col < a.cols;
    const uint32_t n = mine ? a.cols - col : 0;
    auto entry = [&](uint32_t x) { return tall ? place<S>(line, first + x) : place<S>(first + x, line); };
    _Float16 *const hi = a.hi + ((size_t)stack * p.slices + slice) * W * S, *const lo = a.lo + ((size_t)stack * p.slices + slice) * W * S;
    if (!p.a_hi) {
        float g[8] = {}, m[8] = {};
        if (mine) {
            load_eight(g, a.g, a.bf16, stack * a.apart + row * a.ld + col, n);
            if (a.m) load_eight(m, a.m, false, ((size_t)stack * a.rows + row) * a.cols + col, n);
        }
        double sum = 0;
        for (uint32_t k = threadIdx.x; k < a.blocks; k += 64 * kWholeWaves) sum += a.sums[(size_t)stack * a.blocks + k];
        sum = ss::sum_wave(sum);
        if (lane == 63) shared[wave] = sum;
        for (uint32_t at = threadIdx.x * 16; at < 2 * kX; at += 64 * kWholeWaves * 16) *reinterpret_cast<u32x4 *>(lds + at) = u32x4{0, 0, 0, 0};
        __syncthreads();
        sum = 0;
        for (int k = 0; k < kWholeWaves; ++k) sum += shared[k];
        const Scale scale(sum);
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x)
            if (x < n) {
                const float v = scale(update_of(a, g[x], m[x]));
                const _Float16 h = (_Float16)v;
                *reinterpret_cast<_Float16 *>(xh + entry(x)) = h;
                *reinterpret_cast<_Float16 *>(xl + entry(x)) = (_Float16)(v - (float)h);
            }
        __syncthreads();
    } else {
        bring_rows<S>(xh, hi, W);
        bring_rows<S>(xl, lo, W);
        bring_rows<S>(ah, p.a_hi + (size_t)stack * S * S, S);
        bring_rows<S>(al, p.a_lo + (size_t)stack * S * S, S);
        __syncthreads();
        // B + mu I in A's place, then X <- (a - mu) X + X (B + mu I)
#pragma unroll 1
        for (int x_too = 0; x_too < 2; ++x_too) {
            char *const ph = x_too ? xh : ah, *const pl = x_too ? xl : al;
            const float was_by = x_too ? ::orthogonal::kA - p.mu : kB, sum_by = x_too ? kUnscale : kC * kUnscale, diagonal = x_too ? 0.0f : p.mu * kScale;
            const bool busy = wave < (x_too ? W / 32 * across : across * across);
            const uint32_t m = wave / across * 32, n0 = wave % across * 32;
            f32x16 c = {};
            if (busy) {
                c = whole_tile<S, false>(ph, pl, m, ah, al, n0, S, lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 was = get_four(ph, pl, place<S>(m + r, n0 + 8 * e + 4 * q));
#pragma unroll
                    for (int x = 0; x < 4; ++x) c[4 * e + x] = __builtin_fmaf(was_by, was[x], c[4 * e + x] * sum_by);
                }
                if (m == n0 && diagonal != 0.0f)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (r == e / 4 * 8 + 4 * q + e % 4) c[e] += diagonal;
            }
            __syncthreads();
            if (busy)
#pragma unroll
                for (int e = 0; e < 4; ++e) put_four(ph, pl, place<S>(m + r, n0 + 8 * e + 4 * q), f32x4{c[4 * e], c[4 * e + 1], c[4 * e + 2], c[4 * e + 3]});
            __syncthreads();
        }
    }
    if (p.out) {
        if (!mine) return;
        f32x4 v[2];
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x) {
            const uint32_t at = x < n ? entry(x) : 0;
            v[x / 4][x % 4] = ((float)*reinterpret_cast<const _Float16 *>(xh + at) + (float)*reinterpret_cast<const _Float16 *>(xl + at)) * kUnscale;
        }
        const size_t to = stack * p.apart + row * p.ld + col;
        if (p.step) {
            float was[8];
            load_eight(was, p.out, false, to, n);
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x / 4][x % 4] = was[x] - p.delta * v[x / 4][x % 4];
        }
        product::store_out(p.out, p.bf16, to, v, n);
        return;
    }
    take_rows<S>(xh, hi, W);
    take_rows<S>(xl, lo, W);
    if (wave >= across * across) return;
    const uint32_t m = wave / across * 32, n0 = wave % across * 32;
    const f32x16 c = whole_tile<S, true>(xh, xl, m, xh, xl, n0, W, lane);
    float *to = p.parts + ((size_t)stack * p.slices + slice) * S * S + (m + r) * S + n0 + 4 * q;
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<f32x4 *>(to + 8 * e) = f32x4{c[4 * e], c[4 * e + 1], c[4 * e + 2], c[4 * e + 3]};
}

struct SumArgs {
    const float *parts;
    _Float16 *hi, *lo;
    uint32_t size, slices;         // S x S; parts of each
};

// A of its parts: 16 threads share four neighbours' parts, in an order that depends on their number alone
__global__ __launch_bounds__(256) void sum_kernel(const SumArgs p) {
    __shared__ f32x4 shared[16][17];
    const uint32_t four = blockIdx.x * 16 + (threadIdx.x & 15u), share = threadIdx.x >> 4, stack = blockIdx.y;
    const float *from = p.parts + (size_t)stack * p.slices * p.size + four * 4;
    f32x4 s = {0, 0, 0, 0};
#pragma unroll 8
    for (uint32_t k = share; k < p.slices; k += 16) s += *reinterpret_cast<const f32x4 *>(from + (size_t)k * p.size);
    shared[threadIdx.x & 15u][share] = s;
    __syncthreads();
    if (threadIdx.x >= 16) return;
    s = shared[threadIdx.x][0];
    for (int k = 1; k < 16; ++k) s += shared[threadIdx.x][k];
    const size_t at = ((size_t)stack * p.size + four * 4) * sizeof(_Float16);
    put_four(reinterpret_cast<char *>(p.hi), reinterpret_cast<char *>(p.lo), at, s * kUnscale);
}

}  // namespace orthogonal
