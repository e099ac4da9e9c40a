// Matrices in microscaled 4-bit floating point (E2M1 codes, one power of two for 32 of them): quantisation along rows and
// down columns, the values back, the product A B^T, and the product with a few rows that are quantised on the way.
//
// The matrix unit takes the codes and the scales as they are stored: v_mfma_scale_f32_32x32x64_f8f6f4 multiplies 32 x 64 by
// 64 x 32 codes, each lane giving the 32 codes (16 bytes) of one row's block and that block's scale byte, which the
// instruction picks out of a register of four.  Which 32 of the columns a lane's block is makes no difference as long as
// both operands take the same; so a lane takes four blocks that lie side by side, 64 bytes of codes and one
// dword of scales, and the scales are stored as those dwords, a wave's rows after one another.
#pragma once
#include <type_traits>

#include "common.hpp"

#pragma clang fp contract(off)

namespace mx4 {

using ss::f32x4;
using ss::u32x4;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
// plain matrices are aligned to their element alone
typedef u32x4 u32x4_f32 __attribute__((aligned(4)));
typedef u32x4 u32x4_bf16 __attribute__((aligned(2)));

constexpr uint32_t kBlockCols = 32;     // codes that share a scale
constexpr uint32_t kGroupCols = 128;    // columns whose scales are one dword
constexpr uint32_t kGroupBytes = 64;    // and their codes

// a value that all lanes have, for the scalar unit
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// ------------------------------------------------------------ quantise ----

// The scale's byte for a block whose largest magnitude has these bits: floor(log2) - 2, at least 0 (2^-127); 127 for a block of
// zeros; 255 where there is an infinity or a NaN.  The exponent of a subnormal reads as 0, and so does its byte.
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
    const uint32_t e = bits >> 23;
    const uint32_t byte = e > 2u ? e - 2u : 0u;
    return bits == 0u ? 127u : e == 255u ? 255u : byte;
}

// 2^(byte - 127); infinity for 255
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

__device__ __forceinline__ uint32_t dpp_xor1(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1 /* quad_perm [1,0,3,2] */, 0xF, 0xF, false); }
__device__ __forceinline__ uint32_t dpp_xor2(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E /* quad_perm [2,3,0,1] */, 0xF, 0xF, false); }
__device__ __forceinline__ uint32_t dpp_mirror8(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141 /* row_half_mirror */, 0xF, 0xF, false); }

// lane SEL of each four, for each of them; the lane N further on of 16
template <int SEL>
__device__ __forceinline__ uint32_t dpp_quad(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, SEL /* quad_perm */, 0xF, 0xF, false); }
template <int N>
__device__ __forceinline__ uint32_t dpp_turn(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N /* row_ror */, 0xF, 0xF, false); }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t pk_umax16(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// 16 bytes of a row: four fp32 or eight bf16.  Magnitudes are compared as integers, in which infinities and NaN are largest.
struct F32 {
    typedef float elem;
    static constexpr uint32_t kPer = 4, kLanes = 8;            // elements a lane, lanes a block
    template <bool ONCE = false>
    static __device__ __forceinline__ u32x4 load(const void *p) {
        const u32x4_f32 *q = static_cast<const u32x4_f32 *>(p);
        return ONCE ? __builtin_nontemporal_load(q) : *q;
    }
    // without the first s elements, zeros behind
    static __device__ __forceinline__ u32x4 drop(u32x4 v, uint32_t s) {
        if (s & 1u) v = u32x4{v[1], v[2], v[3], 0};
        if (s & 2u) v = u32x4{v[2], v[3], 0, 0};
        return v;
    }
    static __device__ __forceinline__ u32x4 magnitudes(u32x4 v) { return v & 0x7FFFFFFFu; }
    static __device__ __forceinline__ u32x4 larger(u32x4 a, u32x4 b) { return __builtin_elementwise_max(a, b); }
    // bits of the largest of 32, as an fp32, in all of their lanes
    static __device__ __forceinline__ uint32_t row_max(u32x4 m) {
        uint32_t v = umax(umax(m[0], m[1]), umax(m[2], m[3]));
        v = umax(v, dpp_xor1(v));
        v = umax(v, dpp_xor2(v));
        return umax(v, dpp_mirror8(v));
    }
    // bits of element c's magnitude, as an fp32
    static __device__ __forceinline__ uint32_t pick(u32x4 m, int c) { return m[c]; }
    // bits of the largest of 32 in four rows, in all of their lanes
    static __device__ __forceinline__ void four_max(const u32x4 (&v)[4], uint32_t (&bits)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) bits[i] = row_max(magnitudes(v[i]));
    }
    // of lanes k, k + 8, k + 16 and k + 24 the bytes as a dword
    static __device__ __forceinline__ uint32_t gather_four(uint32_t byte, uint32_t lane) {
        uint32_t v = byte << ((lane >> 3 & 3u) * 8);
        v |= dpp_turn<8>(v);
        return v | (uint32_t)__shfl_xor((int)v, 16);
    }
    static __device__ __forceinline__ uint32_t row_codes(u32x4 v, float scale) {
        uint32_t o = 0;
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(v[0]), __uint_as_float(v[1]), scale, 0);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(v[2]), __uint_as_float(v[3]), scale, 1);
    }
    static __device__ __forceinline__ void store_row_codes(uint8_t *p, uint32_t codes) { *reinterpret_cast<uint16_t *>(p) = (uint16_t)codes; }
    // codes of element c in eight rows
    static __device__ __forceinline__ uint32_t column_codes(const u32x4 *v, int c, float scale) {
        uint32_t o = 0;
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(v[0][c]), __uint_as_float(v[1][c]), scale, 0);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(v[2][c]), __uint_as_float(v[3][c]), scale, 1);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(v[4][c]), __uint_as_float(v[5][c]), scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, __uint_as_float(v[6][c]), __uint_as_float(v[7][c]), scale, 3);
    }
};

struct Bf16 {
    typedef uint16_t elem;
    static constexpr uint32_t kPer = 8, kLanes = 4;
    template <bool ONCE = false>
    static __device__ __forceinline__ u32x4 load(const void *p) {
        const u32x4_bf16 *q = static_cast<const u32x4_bf16 *>(p);
        return ONCE ? __builtin_nontemporal_load(q) : *q;
    }
    static __device__ __forceinline__ u32x4 drop(u32x4 v, uint32_t s) {
        if (s & 1u) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
        if (s & 2u) v = u32x4{v[1], v[2], v[3], 0};
        if (s & 4u) v = u32x4{v[2], v[3], 0, 0};
        return v;
    }
    static __device__ __forceinline__ u32x4 magnitudes(u32x4 v) { return v & 0x7FFF7FFFu; }
    static __device__ __forceinline__ u32x4 larger(u32x4 a, u32x4 b) {
        u32x4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = pk_umax16(a[k], b[k]);
        return o;
    }
    static __device__ __forceinline__ uint32_t pick(u32x4 m, int c) { return c & 1 ? m[c >> 1] & 0xFFFF0000u : m[c >> 1] << 16; }
    static __device__ __forceinline__ void four_max(const u32x4 (&v)[4], uint32_t (&bits)[4]) {
        uint32_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4 e = magnitudes(v[i]);
            m[i] = pk_umax16(pk_umax16(e[0], e[1]), pk_umax16(e[2], e[3]));
        }
        // two rows side by side
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            uint32_t two = pk_umax16(__builtin_amdgcn_perm(m[i + 1], m[i], 0x05040100u), __builtin_amdgcn_perm(m[i + 1], m[i], 0x07060302u));
            two = pk_umax16(two, dpp_xor1(two));
            two = pk_umax16(two, dpp_xor2(two));
            bits[i] = two << 16;
            bits[i + 1] = two & 0xFFFF0000u;
        }
    }
    // of lanes k, k + 4, k + 8 and k + 12 the bytes as a dword
    static __device__ __forceinline__ uint32_t gather_four(uint32_t byte, uint32_t lane) {
        uint32_t v = byte << ((lane >> 2 & 3u) * 8);
        v |= dpp_turn<4>(v);
        return v | dpp_turn<8>(v);
    }
    static __device__ __forceinline__ bf16x2 pair(uint32_t v) { return __builtin_bit_cast(bf16x2, v); }
    static __device__ __forceinline__ uint32_t row_codes(u32x4 v, float scale) {
        uint32_t o = 0;
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, pair(v[0]), scale, 0);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, pair(v[1]), scale, 1);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, pair(v[2]), scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, pair(v[3]), scale, 3);
    }
    static __device__ __forceinline__ void store_row_codes(uint8_t *p, uint32_t codes) { *reinterpret_cast<uint32_t *>(p) = codes; }
    static __device__ __forceinline__ uint32_t column_codes(const u32x4 *v, int c, float scale) {
        uint32_t o = 0;
        // the two rows' halves side by side
        auto two = [&](int r) {
            return pair(__builtin_amdgcn_perm(v[r + 1][c >> 1], v[r][c >> 1], c & 1 ? 0x07060302u : 0x05040100u));
        };
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two(0), scale, 0);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two(2), scale, 1);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two(4), scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two(6), scale, 3);
    }
};

struct QuantizeArgs {
    const void *x;
    uint8_t *data;             // NULL: not wanted
    uint32_t *scales;
    uint8_t *data_t;
    uint32_t *scales_t;
    size_t ld;
    uint32_t rows, cols;
    uint32_t chunks;           // of 64 lanes' columns
};

// kPer elements of row `row` from column `col` on, one by one; zeros where the matrix ends
template <typename T>
__device__ __forceinline__ u32x4 load_part(const QuantizeArgs &a, uint32_t row, uint32_t col) {
    u32x4 v = {0, 0, 0, 0};
    if (row >= a.rows) return v;
    const typename T::elem *p = static_cast<const typename T::elem *>(a.x) + (size_t)row * a.ld + col;
    if (col + T::kPer <= a.cols) return T::load(p);
#pragma unroll
    for (uint32_t k = 0; k < T::kPer; ++k)
        if (col + k < a.cols) {
            const uint32_t e = sizeof(p[0]) == 2 ? (uint32_t)reinterpret_cast<const uint16_t *>(p)[k] : reinterpret_cast<const uint32_t *>(p)[k];
            if constexpr (sizeof(p[0]) == 2) v[k >> 1] |= e << (16 * (k & 1));
            else v[k] = e;
        }
    return v;
}

// R rows' parts, out together; INSIDE: nothing ends in them.  But for bf16 down the columns, where half a wave has other rows, they are the same for all lanes, so that their addresses are the
// scalar unit's.  Where the matrix ends a lane loads what ends with it and drops the front, so that no load waits for a test: waited for one by one 16 rows took 8 us.
template <typename T, int R, bool INSIDE, bool ONCE>
__device__ __forceinline__ void load_rows(u32x4 (&v)[R], const QuantizeArgs &a, uint32_t row0, uint32_t col) {
    const typename T::elem *x = static_cast<const typename T::elem *>(a.x);
    if (!INSIDE && a.cols < T::kPer) {
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = load_part<T>(a, row0 + r, col);
        return;
    }
    const uint32_t from = INSIDE || col + T::kPer <= a.cols ? col : a.cols - T::kPer, over = col - from;      // kPer and more: nothing left
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t row = INSIDE || row0 + r < a.rows ? row0 + r : a.rows - 1;
        v[r] = T::template load<ONCE>(x + (size_t)row * a.ld + from);
    }
    if (INSIDE) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (a.cols % T::kPer) v[r] = T::drop(v[r], over);
        const bool none = row0 + r >= a.rows || over >= T::kPer;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[r][k] = none ? 0u : v[r][k];
    }
}

// Four rows' parts, of which a lane of four finds one's scale for all of them: their codes, and in lane k the dword of the scales of row k & 3 and of the lane's group
template <typename T>
__device__ __forceinline__ uint32_t quantize_four(const u32x4 (&v)[4], uint32_t lane, uint32_t (&codes)[4]) {
    uint32_t bits[4];
    T::four_max(v, bits);
    const uint32_t byte = scale_byte(lane & 2u ? (lane & 1u ? bits[3] : bits[2]) : (lane & 1u ? bits[1] : bits[0])), scale = __float_as_uint(scale_of(byte));
    codes[0] = T::row_codes(v[0], __uint_as_float(dpp_quad<0x00>(scale)));
    codes[1] = T::row_codes(v[1], __uint_as_float(dpp_quad<0x55>(scale)));
    codes[2] = T::row_codes(v[2], __uint_as_float(dpp_quad<0xAA>(scale)));
    codes[3] = T::row_codes(v[3], __uint_as_float(dpp_quad<0xFF>(scale)));
    return T::gather_four(byte, lane);
}

// Along the rows alone: a wave takes four rows of 64 lanes' columns, four waves a block one below the other; 2 or 8 rows a wave were 10 % slower.  Memory bounds it: 8192 x 8192
// bf16 28 us (6.0 TB/s, a copy of as many bytes 25), fp32 48 (6.3 TB/s); 257 x 1000 3.4, a launch.
constexpr int kQuantizeRows = 4;
template <typename T, bool ONCE, bool INSIDE>
__device__ __forceinline__ void quantize_rows(const QuantizeArgs &a, uint32_t lane, uint32_t row0, uint32_t col) {
    const uint32_t padded = (a.cols + 127u) & ~127u;
    u32x4 v[kQuantizeRows];
    load_rows<T, kQuantizeRows, INSIDE, ONCE>(v, a, row0, col);
    uint32_t codes[kQuantizeRows];
    const uint32_t scales = quantize_four<T>(v, lane, codes);
#pragma unroll
    for (int r = 0; r < kQuantizeRows; ++r)
        if (INSIDE || (row0 + r < a.rows && col < padded)) T::store_row_codes(a.data + (size_t)(row0 + r) * (padded / 2) + col / 2, codes[r]);
    const uint32_t row = row0 + (lane & 3u);
    if ((lane & (4 * T::kLanes - 1)) < 4 && (INSIDE || (row < a.rows && col < padded))) a.scales[(size_t)(col / kGroupCols) * a.rows + row] = scales;
}

template <typename T, bool ONCE>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantizeArgs a) {
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
    const uint32_t band = uniform(blockIdx.x / a.chunks), chunk = blockIdx.x - band * a.chunks, row0 = (band * 4 + wave) * kQuantizeRows;
    const uint32_t col = (chunk * 64 + lane) * T::kPer;
    if ((chunk + 1) * 64 * T::kPer <= a.cols && row0 + kQuantizeRows <= a.rows) quantize_rows<T, ONCE, true>(a, lane, row0, col);
    else quantize_rows<T, ONCE, false>(a, lane, row0, col);
}

// Down the columns, and along the rows too where wanted, in one pass.  A lane holds 16 rows of 16 bytes in registers, so that half of a column's block is its own; the other half is
// that of another lane, with which it compares its largest magnitudes.  A block takes 128 rows, of which a column's codes are 64 bytes: they go through LDS, so that they leave as
// such (straight from the lanes they would be a few bytes here and there).  kAcross lanes take a row side by side: 32 of bf16, four blocks of which fit a compute unit, where a block of twice
// the width, of which two do, takes 41.7 us for 37.3 at 8192 x 8192; but 64 of fp32, whose rows' codes are half as long (60.3 for 65.2).
// us, 8192 x 8192 along both: bf16 37.3 (5.5 TB/s), fp32 60.3 (5.6 TB/s), where each by itself would take 28 + 35 and 48 + 54; 4099 x 8192 bf16 22.9.  What bounds it is that a block loads,
// computes and stores one after the other: more of them do not fit the registers (80 of them: spills, 45.7).
constexpr int kBothRows = 16;
template <typename T>
constexpr uint32_t kAcross = T::kPer == 8 ? 32 : 64;
template <typename T>
constexpr uint32_t kBothThreads = kAcross<T> * 128 / kBothRows;

template <typename T>
struct BothShared {
    uint8_t codes[kAcross<T> * T::kPer * kGroupBytes];
    u32x4 largest[kAcross<T> == 64 ? kBothThreads<T> : 1];
    uint32_t scales[kAcross<T> * T::kPer];
};

template <typename T, bool ROWS, bool ONCE, bool INSIDE>
__device__ __forceinline__ void quantize_both(const QuantizeArgs &a, BothShared<T> &shared, uint32_t lane, uint32_t share, uint32_t row0, uint32_t col) {
    constexpr int R = kBothRows;
    constexpr uint32_t kPiece = R / 2, kPlaces = kGroupBytes / kPiece;
    const uint32_t padded = (a.cols + 127u) & ~127u;
    u32x4 v[R];
    load_rows<T, R, INSIDE, ONCE>(v, a, row0, col);
    u32x4 m = T::magnitudes(v[0]);
    if constexpr (ROWS) {
        constexpr uint32_t kGroupLanes = 4 * T::kLanes;        // whose blocks share a dword: 32 or 16
        uint32_t kept = 0;
#pragma unroll
        for (int r = 0; r < R; r += 4) {
            const u32x4 part[4] = {v[r], v[r + 1], v[r + 2], v[r + 3]};
#pragma unroll
            for (int i = 0; i < 4; ++i) m = T::larger(m, T::magnitudes(part[i]));
            uint32_t codes[4];
            const uint32_t scales = quantize_four<T>(part, lane, codes);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (INSIDE || (row0 + r + i < a.rows && col < padded)) T::store_row_codes(a.data + (size_t)(row0 + r + i) * (padded / 2) + col / 2, codes[i]);
            // lane k of the group keeps row k's, so that they leave side by side
            if ((lane & (kGroupLanes - 4)) == (uint32_t)r) kept = scales;
        }
        const uint32_t row = row0 + (lane & (kGroupLanes - 1));
        if ((lane & (kGroupLanes - 1)) < R && (INSIDE || (row < a.rows && col < padded))) a.scales[(size_t)(col / kGroupCols) * a.rows + row] = kept;
    } else {
#pragma unroll
        for (int r = 1; r < R; ++r) m = T::larger(m, T::magnitudes(v[r]));
    }
    u32x4 others;
    if constexpr (kAcross<T> == 64) {
        shared.largest[threadIdx.x] = m;
        __syncthreads();
        others = shared.largest[threadIdx.x ^ 64u];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) others[k] = (uint32_t)__shfl_xor((int)m[k], 32);
    }
    m = T::larger(m, others);
#pragma unroll
    for (int c = 0; c < (int)T::kPer; ++c) {
        const uint32_t byte = scale_byte(T::pick(m, c));
        const float scale = scale_of(byte);
        const uint32_t column = (lane & (kAcross<T> - 1)) * T::kPer + c;
        // piece s of a column at place s ^ lane, for the banks' sake
        uint32_t *to = reinterpret_cast<uint32_t *>(shared.codes + column * kGroupBytes + ((share ^ (lane & (kPlaces - 1))) * kPiece));
#pragma unroll
        for (int k = 0; k < R / 8; ++k) to[k] = T::column_codes(v + 8 * k, c, scale);
        if (share % 2 == 0) reinterpret_cast<uint8_t *>(&shared.scales[column])[share / 2] = (uint8_t)byte;
    }
}

template <typename T, bool ROWS, bool ONCE>
__global__ __launch_bounds__(kBothThreads<T>, 4) void quantize_both_kernel(const QuantizeArgs a) {
    constexpr uint32_t kColumns = kAcross<T> * T::kPer, kThreads = kBothThreads<T>, kPiece = kBothRows / 2, kPlaces = kGroupBytes / kPiece;
    __shared__ BothShared<T> shared;
    const uint32_t lane = threadIdx.x & 63u, share = kAcross<T> == 64 ? uniform(threadIdx.x / 64) : threadIdx.x / 32;      // of the rows
    // the band that may be short comes first: 4099 x 8192 in bf16, when its 528 blocks were to share 512 places, 28.9 -> 27.2 us
    const uint32_t from_last = uniform(blockIdx.x / a.chunks), chunk = blockIdx.x - from_last * a.chunks, band = (a.rows + 127) / 128 - 1 - from_last, row0 = band * 128 + share * kBothRows;
    const uint32_t first = chunk * kColumns, col = first + (lane & (kAcross<T> - 1)) * T::kPer;
    if (first + kColumns <= a.cols && band * 128 + 128 <= a.rows) quantize_both<T, ROWS, ONCE, true>(a, shared, lane, share, row0, col);
    else quantize_both<T, ROWS, ONCE, false>(a, shared, lane, share, row0, col);
    __syncthreads();
    const size_t row_bytes = (((size_t)a.rows + 127) & ~(size_t)127) / 2;
#pragma unroll
    for (uint32_t i = threadIdx.x; i < kColumns * 4; i += kThreads) {
        const uint32_t column = i >> 2, part = i & 3u, mixed = column / T::kPer & (kPlaces - 1);
        if (first + column >= a.cols) continue;
        const uint8_t *codes = shared.codes + column * kGroupBytes;
        u32x4 v;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
            v[k] = *reinterpret_cast<const uint32_t *>(codes + (((part * 16 + k * 4) / kPiece) ^ mixed) * kPiece + (k * 4) % kPiece);
        *reinterpret_cast<u32x4 *>(a.data_t + (size_t)(first + column) * row_bytes + band * kGroupBytes + part * 16) = v;
    }
    if (threadIdx.x < kColumns && first + threadIdx.x < a.cols) a.scales_t[(size_t)band * a.cols + first + threadIdx.x] = shared.scales[threadIdx.x];
}

// ---------------------------------------------------------- dequantise ----

struct DequantizeArgs {
    const uint8_t *data;
    const uint8_t *scales;
    void *out;
    size_t ld;
    uint32_t rows, cols;
    uint32_t chunks;           // of 512 columns
};

// A lane takes eight codes, a wave R rows of 512 columns.  Stored with nt: 8192 x 8192 bf16 25.0 us (6.8 TB/s) against 33.4.  To fp32, a lane's 32 bytes in two stores, 116 us (2.6
// TB/s).
template <bool OUT_BF16, int R>
__global__ __launch_bounds__(256) void dequantize_kernel(const DequantizeArgs a) {
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
    const uint32_t band = uniform(blockIdx.x / a.chunks), chunk = blockIdx.x - band * a.chunks, row0 = (band * 4 + wave) * R;
    const uint32_t col = (chunk * 64 + lane) * 8, padded = (a.cols + 127u) & ~127u;
    if (col >= a.cols) return;
    uint32_t codes[R], bytes[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t row = row0 + r;
        codes[r] = bytes[r] = 0;
        if (row < a.rows) {
            codes[r] = *reinterpret_cast<const uint32_t *>(a.data + (size_t)row * (padded / 2) + col / 2);
            bytes[r] = a.scales[((size_t)(col / kGroupCols) * a.rows + row) * 4 + (col / kBlockCols & 3u)];
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t row = row0 + r;
        if (row >= a.rows) continue;
        const float scale = scale_of(bytes[r]);
        const bool nan = bytes[r] == 255u;
        const size_t at = (size_t)row * a.ld + col;
        if constexpr (OUT_BF16) {
            u32x4 o;
            o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], scale, 0));
            o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], scale, 1));
            o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], scale, 2));
            o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], scale, 3));
            if (nan) o = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
            uint16_t *to = static_cast<uint16_t *>(a.out) + at;
            if (col + 8 <= a.cols) __builtin_nontemporal_store(o, reinterpret_cast<u32x4_bf16 *>(to));
            else
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (col + k < a.cols) to[k] = (uint16_t)(o[k >> 1] >> (16 * (k & 1)));
        } else {
            f32x2 p[4];
            p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], scale, 0);
            p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], scale, 1);
            p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], scale, 2);
            p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], scale, 3);
            u32x4 o[2];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k >> 2][k & 3] = nan ? 0x7FC00000u : __float_as_uint(p[k >> 1][k & 1]);
            uint32_t *to = static_cast<uint32_t *>(a.out) + at;
            if (col + 8 <= a.cols) {
                __builtin_nontemporal_store(o[0], reinterpret_cast<u32x4_f32 *>(to));
                __builtin_nontemporal_store(o[1], reinterpret_cast<u32x4_f32 *>(to) + 1);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (col + k < a.cols) to[k] = o[k >> 2][k & 3];
            }
        }
    }
}

// ------------------------------------------------------------- product ----

__device__ __forceinline__ i32x8 widened(u32x4 v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }

template <bool OUT_BF16>
__device__ __forceinline__ void store_out(void *out, size_t at, float v) {
    if constexpr (OUT_BF16) static_cast<__bf16 *>(out)[at] = (__bf16)v;
    else static_cast<float *>(out)[at] = v;
}

// Tiles of 2 x 2 waves, each 32 T rows by 32 T columns of the result.  A step is two groups of 128 columns, multiplied in four quarters of 64; the
// fragments of the next quarter are read while one is multiplied.  Of each of the tile's rows of an operand a step takes 128 bytes of codes, loaded
// straight into LDS, which has room for five operands' steps: both of the one that is read, both of the next one and the first of the one
// after that.  So there is always something to load: the second operand of the next step right after the last one's place is free, when it has
// the rest of the step to arrive, then the first one of the step after it, spread over the multiplications.
//
// The matrix unit bounds it, and that the card's power: multiplying registers of random codes without a load reaches 6.75 PFLOP/s.  8192 x 8192 x 16384 to fp32 458 to 490 us (4.5 to 4.8 PFLOP/s), by card and day, of
// which bringing the operands costs 50, and in each of four rounds nothing is multiplied for 3 at the start and for 14 at the end, while 67 MB of results leave; 4096 cubed to bf16 32 to 36 us (4.0 PFLOP/s).  In 16 x 16 x
// 128 it is no faster (532 us): a scaled multiplication takes two issue slots, and one wave a SIMD has no more of them.  Smaller tiles (T = 2, 1) are for results that do not
// fill the card in large ones; which, the cost model on the host says.
struct TilesArgs {
    const uint8_t *a, *b;
    const uint32_t *sa, *sb;
    void *out;                 // or the partial sums, split after split
    size_t ld;
    uint32_t M, N;             // of this launch, which may be a part of the product
    uint32_t rows_a, rows_b;   // of the operands: from one group's scales to the next one's
    uint32_t groups;           // of 128 columns
    uint32_t tiles_m, tiles_n;
    uint32_t splits;
    bool kept;                 // the result, in the memory-side cache
};

// all but the last N loads of this wave are there (neither a barrier nor a read waits for loads into LDS by itself), and so is what it read from LDS
template <int N>
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

// 16 bytes at any alignment, sent on by the L2 at once: what is left there is sent when the kernel ends, with nothing beside it.  The next instruction may change v only
// when the store has read it.
__device__ __forceinline__ void store_through(void *p, u32x4 v) { asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(p), "v"(v) : "memory"); }

template <int T>
struct Fragments {
    u32x4 a[T], b[T];
};

// part of 2 T of the multiplications of a quarter; BYTE: which one, and of the scales' bytes.  b is the first operand, so that a lane has four
// neighbours of a row of the result.
template <int BYTE, int T>
__device__ __forceinline__ void multiply(f32x16 (&c)[T][T], const Fragments<T> &f, const uint32_t (&s)[2 * T], int part) {
#pragma unroll
    for (int x = part * T / 2; x < (part + 1) * T / 2; ++x)
        c[x / T][x % T] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widened(f.b[x % T]), widened(f.a[x / T]), c[x / T][x % T], 4, 4, BYTE, (int)s[T + x % T],
                                                                          BYTE, (int)s[x / T]);
}

template <bool OUT_BF16, int T>
__global__ __launch_bounds__(256, 1) void matmul_tiles_kernel(const TilesArgs p) {
    constexpr uint32_t B = 64 * T, kRow = 2 * kGroupBytes, kUnit = B * kRow, kRing = 5 * kUnit;
    __shared__ __attribute__((aligned(128))) char lds[kRing];
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
    const uint32_t r = lane & 31u, q = lane >> 5;
    // neighbouring blocks go to the eight dies in turn: each die takes a run of tiles, four tile rows high
    const uint32_t total = gridDim.x, die = blockIdx.x & 7u, share = total >> 3, more = total & 7u;
    uint32_t at = die * share + (die < more ? die : more) + (blockIdx.x >> 3);
    const uint32_t tiles = p.tiles_m * p.tiles_n, split = uniform(at / tiles);
    at -= split * tiles;
    constexpr uint32_t kHigh = 4;
    const uint32_t band = uniform(at / (kHigh * p.tiles_n)), in = at - band * kHigh * p.tiles_n;
    const uint32_t left = p.tiles_m - band * kHigh, high = left < kHigh ? left : kHigh, column = uniform(in / high);
    const uint32_t m0 = (band * kHigh + in - column * high) * B, n0 = column * B;
    const uint32_t steps = (p.groups + 1) / 2, each = uniform(steps / p.splits), over = steps - each * p.splits;
    const uint32_t from = split * each + (split < over ? split : over), to = from + each + (split < over ? 1u : 0u);
    const uint32_t row_bytes = p.groups * kGroupBytes;

    // Where a lane's 16 bytes of eight rows come from: chunk c of row r goes to place c ^ (r / 2 & 7) of its row in LDS, so that the rows
    // that a read takes together lie in different banks.  Rows beyond the matrix are its last one; they are not stored.
    constexpr int L = B / 32;       // loads a wave for one operand's step
    uint32_t from_a[L], from_b[L];
    const uint32_t chunk = ((lane & 7u) ^ ((wave & 1u) * 4 + (lane >> 4))) * 16, last_a = p.M - 1 - m0, last_b = p.N - 1 - n0;
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const uint32_t row = (wave + 4 * i) * 8 + (lane >> 3);
        from_a[i] = (row < last_a ? row : last_a) * row_bytes + chunk;
        from_b[i] = (row < last_b ? row : last_b) * row_bytes + chunk;
    }
    const ss::Window wa = ss::window(p.a, (size_t)m0 * row_bytes, (last_a + 1 < B ? last_a + 1 : B) * row_bytes);
    const ss::Window wb = ss::window(p.b, (size_t)n0 * row_bytes, (last_b + 1 < B ? last_b + 1 : B) * row_bytes);
    typedef __attribute__((address_space(3))) void *Lds;
    // the last steps load the last one again, which nothing reads: a branch would part the loop
    auto column_of = [&](uint32_t step) { return (int)((step < to ? step : to - 1) * kRow); };
    auto fetch_a = [&](int i, uint32_t place, int column) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(wa, (Lds)(lds + place + (wave + 4 * i) * 1024), 16, (int)from_a[i], column, 0, 0);
    };
    auto fetch_b = [&](int i, uint32_t place, int column) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(wb, (Lds)(lds + place + (wave + 4 * i) * 1024), 16, (int)from_b[i], column, 0, 0);
    };
    // scales: a dword a row and group, straight into registers
    const uint32_t ma = (wave & 1u) * T * 32, nb = (wave >> 1) * T * 32;
    uint32_t at_a[T], at_b[T], s[2 * T], next[2 * T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const uint32_t m = ma + i * 32 + r, n = nb + i * 32 + r;
        at_a[i] = ((m < last_a ? m : last_a) + m0 + q * p.rows_a) * 4;
        at_b[i] = ((n < last_b ? n : last_b) + n0 + q * p.rows_b) * 4;
    }
    auto fetch_scales = [&](uint32_t (&to_s)[2 * T], uint32_t step) {
        // Of a last step with one group the other one's scales read as zero on both sides: whatever codes stand in their place (the next row's), their
        // products are below 2^-240 and leave every sum as it is.
        const bool two = p.groups - 2 * step >= 2;
        const ss::Window va = ss::window(p.sa, (size_t)(2 * step) * p.rows_a * 4, uniform((two ? p.rows_a + p.M : p.M) * 4));
        const ss::Window vb = ss::window(p.sb, (size_t)(2 * step) * p.rows_b * 4, uniform((two ? p.rows_b + p.N : p.N) * 4));
#pragma unroll
        for (int i = 0; i < T; ++i) to_s[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(va, (int)at_a[i], 0, 0);
#pragma unroll
        for (int i = 0; i < T; ++i) to_s[T + i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(vb, (int)at_b[i], 0, 0);
    };
    // fragment i of quarter j, in the order in which they are wanted: each lane's block is chunk 4 q + j of its row
    uint32_t of_quarter[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) of_quarter[j] = r * kRow + (((4 * q + j) ^ (r >> 1 & 7u)) * 16);
    auto read = [&](Fragments<T> &f, int i, int j, uint32_t a, uint32_t b) {
        if (i < T) f.b[i] = *reinterpret_cast<const u32x4 *>(lds + b + nb * kRow + of_quarter[j] + i * 32 * kRow);
        else f.a[i - T] = *reinterpret_cast<const u32x4 *>(lds + a + ma * kRow + of_quarter[j] + (i - T) * 32 * kRow);
    };
    f32x16 c[T][T] = {};
    if (from < to) {
        Fragments<T> f0, f1;
        uint32_t a = 0, b = kUnit, a1 = 2 * kUnit, b1 = 3 * kUnit, free = 4 * kUnit;     // places of this step's operands, the next one's, and of what comes next
#pragma unroll
        for (int i = 0; i < L; ++i) fetch_a(i, a, column_of(from)), fetch_b(i, b, column_of(from));
        fetch_scales(s, from);
#pragma unroll
        for (int i = 0; i < L; ++i) fetch_a(i, a1, column_of(from + 1)), fetch_b(i, b1, column_of(from + 1));
        arrived<2 * L>();
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int i = 0; i < 2 * T; ++i) read(f0, i, 0, a, b);
        __builtin_amdgcn_sched_barrier(0);
        for (uint32_t step = from; step < to; ++step) {
            const int column = column_of(step + 2);
            // Part by part, with a read and perhaps a load in each: in one go they would keep the matrix unit waiting while their queues are full
            fetch_scales(next, step + 1 < to ? step + 1 : step);
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f1, part, 1, a, b);
                multiply<0>(c, f0, s, part);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f0, part, 2, a, b);
                if (part % 2 == 0) fetch_a(part / 2, free, column);
                multiply<1>(c, f1, s, part);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f1, part, 3, a, b);
                if (part % 2 == 0) fetch_a(T + part / 2, free, column);
                multiply<2>(c, f0, s, part);
                __builtin_amdgcn_sched_barrier(0);
            }
            // this step's places have been read by all, and the next one's operands are there
            arrived<L>();
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f0, part, 0, a1, b1);
                fetch_b(part, a, column);
                multiply<3>(c, f1, s, part);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < 2 * T; ++i) s[i] = next[i];
            const uint32_t was_a = a, was_b = b;
            a = a1, b = b1, a1 = free, b1 = was_a, free = was_b;
        }
        arrived<0>();       // nothing is on its way into LDS that the next block may have
    }
    // The result leaves through LDS, 32 rows of a wave at a time, so that a store takes 1 KB and whole lines: from where the sums are it would be 16 or 8 bytes a lane of 32
    // rows.  Each wave has a part of the ring to itself.
    typedef typename std::conditional<OUT_BF16, __bf16, float>::type Out;
    typedef typename std::conditional<OUT_BF16, bf16x4, f32x4>::type Four;
    typedef typename std::conditional<OUT_BF16, u32x4_bf16, u32x4_f32>::type Vector;
    constexpr uint32_t kPer = 16 / sizeof(Out), kChunks = 32 * T / kPer, kRows = 64 / kChunks, kStrip = 32 * kChunks * 16;
    const size_t base = (size_t)split * p.M * p.N;      // of partial sums; split is 0 where there are none
    Out *out = static_cast<Out *>(p.out) + base + (size_t)(m0 + ma) * p.ld + n0 + nb;
    char *mine = lds + wave * (kRing / 4);
    __builtin_amdgcn_s_barrier();       // all have read what the ring held
    const uint32_t of = lane / kChunks, chunk_out = lane % kChunks;
    const bool inside = nb + (chunk_out + 1) * kPer <= last_b + 1;
#pragma unroll
    for (int i = 0; i < T; ++i) {
        char *strip = mine + (i & 1) * kStrip;
        // chunk c of row r at place c ^ r, for the banks' sake
#pragma unroll
        for (int k = 0; k < T; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t col = k * 32 + 8 * e + 4 * q, at = (col / kPer) ^ (r & (kChunks - 1));
                Four v;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = (Out)c[i][k][4 * e + x];
                *reinterpret_cast<Four *>(strip + (r * kChunks + at) * 16 + col % kPer * sizeof(Out)) = v;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (uint32_t j = 0; j < 32 / kRows; ++j) {
            const uint32_t row = j * kRows + of;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(strip + (row * kChunks + (chunk_out ^ (row & (kChunks - 1)))) * 16);
            if (ma + i * 32 + row > last_a) continue;
            Out *to = out + (size_t)(i * 32 + row) * p.ld + chunk_out * kPer;
            if (inside && p.kept) store_through(to, v);
            else if (inside) __builtin_nontemporal_store(v, reinterpret_cast<Vector *>(to));
            else
#pragma unroll
                for (uint32_t x = 0; x < kPer; ++x)
                    if (nb + chunk_out * kPer + x <= last_b) to[x] = __builtin_bit_cast(typename std::conditional<OUT_BF16, bf16x8, f32x4>::type, v)[x];
        }
    }
}

struct JoinArgs {
    const float *parts;
    void *out;
    size_t ld;
    uint32_t M, N, splits;
};

// the partial sums, one after the other, four neighbours a lane.  64 x 64 x 16384 in 64 parts takes 7.1 us with the product (14.0 with one part's load at a time).
template <bool OUT_BF16>
__global__ __launch_bounds__(256) void join_kernel(const JoinArgs p) {
    const size_t size = (size_t)p.M * p.N, at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= size) return;
    const uint32_t n = size - at < 4 ? (uint32_t)(size - at) : 4u;
    f32x4 s = {0, 0, 0, 0};
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    // the loads of eight parts go out together
    if (n == 4) {
#pragma unroll 8
        for (uint32_t k = 0; k < p.splits; ++k) s += *reinterpret_cast<const f32x4_any *>(p.parts + k * size + at);
    } else {
        for (uint32_t i = 0; i < n; ++i)
#pragma unroll 8
            for (uint32_t k = 0; k < p.splits; ++k) s[i] += p.parts[k * size + at + i];
    }
    uint32_t row = (uint32_t)(at / p.N), col = (uint32_t)(at - (size_t)row * p.N);
    for (uint32_t i = 0; i < n; ++i) {
        store_out<OUT_BF16>(p.out, (size_t)row * p.ld + col, s[i]);
        if (++col == p.N) col = 0, ++row;
    }
}

// ------------------------------------------------- product of a few rows ----
// Up to 16 rows of x, quantised on the way.  A wave streams 16 rows of w, or SPLIT of a block's waves share them, each with every SPLIT-th step of 512
// columns, and their sums are added through LDS in order.  A block first brings x in MX4 into LDS, or as many steps of it as fit, while its waves' first steps of w are on
// the way.  What has to be read is w, and that is what bounds it: its steps go straight into LDS, each wave's into a ring of its own, so that a load
// takes 256 bytes of a row and many are on the way.  us, 8192 columns and 28672 rows of w (129 MB): one row of x 21.2 (5.9 TB/s), sixteen 27.0 (4.6 TB/s), where each block's
// quantisation of x, about 60 MB of it out of the L2s, is 5; 4096 x 4096, one row 4.0 (a launch is 3.4), sixteen 7.

struct LinearArgs {
    const void *x;             // or x's codes
    const uint32_t *sx;        // their scales
    const uint8_t *w;
    const uint32_t *sw;
    void *out;
    size_t ldx, ldt, ldn;      // of x; of the result from one of x's rows to the next, and from one of w's
    uint32_t T, N, K, groups;
    uint32_t rows_x, rows_w;   // from one group's scales to the next one's
    uint32_t log_split;
};

constexpr int kLinearWaves = 8;
constexpr uint32_t kLinearGroups = 4, kLinearCodeBytes = 16 * kLinearGroups * kGroupBytes, kLinearStepBytes = kLinearCodeBytes + 16 * kLinearGroups * 4;     // a step of 16 rows: codes, scales

// The scales of one step, for the first n of a matrix' rows: where they begin, in bytes, and how many of them can be read.  A large matrix has more than 4 GiB of scales, which 32 bits do not
// address; of a step there are 2 GiB at most.
struct ScaleWindow {
    size_t from;
    uint32_t bytes;
};

constexpr ScaleWindow scale_window(uint32_t groups, uint32_t step, uint32_t rows, uint32_t n) {
    const uint32_t first = step * kLinearGroups, left = groups - first;
    return {(size_t)first * rows * 4, (((left < kLinearGroups ? left : kLinearGroups) - 1) * rows + n) * 4};
}

// STEPS of x in LDS, DEPTH of w for each wave
template <int STEPS, int DEPTH>
struct LinearShared {
    u32x4 codes[STEPS][kLinearGroups * 4][16];
    uint32_t scales[STEPS][64];
    __attribute__((aligned(128))) char w[kLinearWaves][DEPTH][kLinearStepBytes];
};

// Brings rows of x, four parts of 64 lanes' columns at once, the next ones on the way; `then` after the first ones.  Every block does it, so it is kept short:
// a lane of four finds one part's scale for all of them, and the loop is not unrolled, since its first pass waits for the instructions themselves.
template <typename T, int STEPS, int DEPTH, typename F>
__device__ __forceinline__ void bring_x(LinearShared<STEPS, DEPTH> &shared, const LinearArgs &a, uint32_t base, uint32_t steps, uint32_t lane, uint32_t wave, F then) {
    constexpr uint32_t kWidth = 64 * T::kPer, kStep = kLinearGroups * kGroupCols, kParts = kStep / kWidth;
    const uint32_t fours = (steps * kParts + 3) / 4;
    struct Item {
        uint32_t token, four;
    };
    auto load = [&](u32x4 (&v)[4], Item at) {
        const typename T::elem *x = static_cast<const typename T::elem *>(a.x) + (size_t)at.token * a.ldx;
        const uint32_t col = base * kStep + at.four * 4 * kWidth + lane * T::kPer, last = a.K - T::kPer;
        // where x ends a lane loads what ends with it
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = T::load(x + (col + i * kWidth < last ? col + i * kWidth : last));
    };
    auto put = [&](const u32x4 (&v)[4], Item at) {
        uint32_t codes[4];
        const uint32_t dword = quantize_four<T>(v, lane, codes);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t part = at.four * 4 + i, block = (i % kParts) * (kWidth / kBlockCols) + lane / T::kLanes;
            // rows are mixed, so that a row's blocks lie in different banks
            uint8_t *to = reinterpret_cast<uint8_t *>(&shared.codes[part / kParts][block][at.token ^ block]);
            T::store_row_codes(to + (lane & (T::kLanes - 1)) * (T::kPer / 2), codes[i]);
        }
        const uint32_t part = at.four * 4 + (lane & 3u), group = part % kParts * (kWidth / kGroupCols) + lane / (4 * T::kLanes);
        if ((lane & (4 * T::kLanes - 1)) < 4) shared.scales[part / kParts][group * 16 + at.token] = dword;
    };
    const uint32_t more = uniform(kLinearWaves / fours), rest = kLinearWaves - more * fours;
    auto advance = [&](Item &i) {
        i.token += more, i.four += rest;
        if (i.four >= fours) i.four -= fours, ++i.token;
    };
    Item at;
    at.token = uniform(wave / fours);
    at.four = wave - at.token * fours;
    if (a.K < T::kPer) {
        then();
        QuantizeArgs m{};
        m.x = a.x;
        m.ld = a.ldx;
        m.rows = a.T;
        m.cols = a.K;
        for (; at.token < a.T; advance(at)) {
            u32x4 v[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) v[i] = load_part<T>(m, at.token, (at.four * 4 + i) * kWidth + lane * T::kPer);
            put(v, at);
        }
        return;
    }
    u32x4 v[4];
    if (at.token < a.T) load(v, at);
    then();
    while (at.token < a.T) {
        const uint32_t first = base * kStep + at.four * 4 * kWidth;
        if (first + 4 * kWidth > a.K) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t col = first + i * kWidth + lane * T::kPer, over = col + T::kPer <= a.K ? 0 : col - (a.K - T::kPer);
                if (a.K % T::kPer) v[i] = T::drop(v[i], over);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i][k] = over >= T::kPer ? 0u : v[i][k];
            }
        }
        const Item now = at;
        advance(at);
        put(v, now);
        if (at.token < a.T) load(v, at);
    }
}

// x is in MX4 already
struct Codes {};

template <int STEPS, int DEPTH>
__device__ __forceinline__ void bring_codes(LinearShared<STEPS, DEPTH> &shared, const LinearArgs &a, uint32_t base, uint32_t steps) {
    // 16 lanes a step of a row
    constexpr uint32_t kAtOnce = 4, kThreads = 64 * kLinearWaves;
    const uint32_t block = threadIdx.x & 15u, items = a.T * steps, part = 65536 / a.T + 1;
    for (uint32_t first = threadIdx.x / 16; first < items; first += kAtOnce * (kThreads / 16)) {
        u32x4 v[kAtOnce];
        uint32_t s[kAtOnce];
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            const uint32_t wanted = first + k * (kThreads / 16), item = wanted < items ? wanted : items - 1;
            const uint32_t step = item * part >> 16, token = item - step * a.T;       // divided by T: exact for the few items
            const uint32_t group = (base + step) * kLinearGroups + block / 4, of_scale = (base + step) * kLinearGroups + (block & 3u);
            const uint32_t last = a.groups - 1;
            v[k] = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(a.x) + (size_t)token * a.groups * kGroupBytes + (size_t)(group < last ? group : last) * kGroupBytes +
                                                    (block & 3u) * 16);
            s[k] = a.sx[(size_t)(of_scale < last ? of_scale : last) * a.rows_x + token];
            if (group > last) v[k] = u32x4{0, 0, 0, 0};
            if (of_scale > last) s[k] = 0;
        }
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            const uint32_t item = first + k * (kThreads / 16), step = item * part >> 16, token = item - step * a.T;
            if (item >= items) break;
            shared.codes[step][block][token ^ block] = v[k];
            if (block < 4) shared.scales[step][block * 16 + token] = s[k];
        }
    }
}

template <typename T, bool OUT_BF16, bool ONCE, int STEPS, int DEPTH>
__global__ __launch_bounds__(64 * kLinearWaves) void linear_kernel(const LinearArgs a) {
    __shared__ LinearShared<STEPS, DEPTH> shared;
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), r = lane & 15u, q = lane >> 4;
    const uint32_t split = 1u << a.log_split, share = wave & (split - 1);
    const uint32_t n0 = (blockIdx.x * (kLinearWaves >> a.log_split) + (wave >> a.log_split)) * 16;
    const uint32_t steps = (a.groups + kLinearGroups - 1) / kLinearGroups, mine = steps > share ? (steps - share + split - 1) >> a.log_split : 0;
    const uint32_t row_bytes = a.groups * kGroupBytes;
    // Rows beyond w read as zero.  Groups beyond the last are the next row's codes, with scales that read as zero; x's codes are zero there.
    const uint32_t rows = n0 < a.N ? (a.N - n0 < 16 ? a.N - n0 : 16) : 0;
    const ss::Window ww = ss::window(a.w, (size_t)(rows ? n0 : 0) * row_bytes, rows * row_bytes);
    typedef __attribute__((address_space(3))) void *Lds;
    uint32_t from[4];       // 16 lanes take 256 bytes of a row, chunk c of row r to place c ^ r
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) from[i] = (4 * i + q) * row_bytes + ((r ^ (4 * i + q)) * 16);
    const uint32_t from_s = (q * a.rows_w + (n0 + r < a.N ? n0 + r : a.N - 1)) * 4;
    // Rows that begin a power of two apart begin in the same memory channels: each wave begins at another of its steps (8192 columns and 28672 rows 28.5 -> 23.1 us)
    const uint32_t per = STEPS >> a.log_split, pass = per << a.log_split, tile = n0 / 16;       // of a pass' steps so many are this wave's
    const uint32_t tail = uniform(mine % per), turn = uniform(tile % per), turn_tail = tail ? uniform(tile % tail) : 0;
    // step k of this wave, which is in the pass that begins with `begin`, or after it
    auto step_of = [&](uint32_t k, uint32_t begin) {
        if (k >= mine) k = mine - 1;
        while (k >= begin + per) begin += per;
        const uint32_t left = mine - begin < per ? tail : per;
        uint32_t i = k - begin + (mine - begin < per ? turn_tail : turn);
        if (i >= left) i -= left;
        return ((begin + i) << a.log_split) + share;
    };
    auto fetch = [&](uint32_t place, uint32_t k, uint32_t begin) {
        const uint32_t step = mine ? step_of(k, begin) : 0;
        const ScaleWindow s = scale_window(a.groups, step, a.rows_w, a.N);
        const ss::Window ws = ss::window(a.sw, s.from, s.bytes);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ww, (Lds)(shared.w[wave][place] + i * 1024), 16, (int)from[i], (int)(step * (kLinearGroups * kGroupBytes)), 0, ONCE ? 2 : 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ws, (Lds)(shared.w[wave][place] + kLinearCodeBytes), 4, (int)from_s, 0, 0, 0);
    };
    f32x4 c = {0, 0, 0, 0};
    uint32_t k = 0, place = 0;
    for (uint32_t base = 0; base < steps; base += pass) {
        const uint32_t count = steps - base < pass ? steps - base : pass, begin = k;
        if (base) __syncthreads();
        auto start = [&] {
            if (base) return;
#pragma unroll
            for (int i = 0; i < DEPTH; ++i) fetch((uint32_t)i, (uint32_t)i, 0);
        };
        if constexpr (std::is_same<T, Codes>::value) {
            start();
            bring_codes(shared, a, base, count);
        } else {
            bring_x<T>(shared, a, base, count, lane, wave, start);
        }
        __syncthreads();
        const uint32_t end = mine < begin + per ? mine : begin + per;
        for (; k < end; ++k) {
            arrived<5 * (DEPTH - 1)>();
            u32x4 f[4], g[4];
            const uint32_t at = step_of(k, begin) - base;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                g[j] = *reinterpret_cast<const u32x4 *>(shared.w[wave][place] + r * 256 + (((q * 4 + j) ^ r) * 16));
                f[j] = shared.codes[at][q * 4 + j][r ^ (q * 4 + j)];
            }
            const uint32_t sx = shared.scales[at][lane], sn = reinterpret_cast<const uint32_t *>(shared.w[wave][place] + kLinearCodeBytes)[lane];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch(place, k + DEPTH, begin);
            place = place + 1 < DEPTH ? place + 1 : 0;
            c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widened(f[0]), widened(g[0]), c, 4, 4, 0, (int)sx, 0, (int)sn);
            c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widened(f[1]), widened(g[1]), c, 4, 4, 1, (int)sx, 1, (int)sn);
            c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widened(f[2]), widened(g[2]), c, 4, 4, 2, (int)sx, 2, (int)sn);
            c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widened(f[3]), widened(g[3]), c, 4, 4, 3, (int)sx, 3, (int)sn);
        }
    }
    arrived<0>();       // nothing is on its way into LDS that others may have
    if (split > 1) {
        f32x4 *part = reinterpret_cast<f32x4 *>(shared.w[wave][0]);
        part[lane] = c;
        __syncthreads();
        if (share) return;
        for (uint32_t i = 1; i < split; ++i) c += reinterpret_cast<const f32x4 *>(shared.w[wave + i][0])[lane];
    }
    const uint32_t n = n0 + r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t t = 4 * q + i;
        if (t < a.T && n < a.N) store_out<OUT_BF16>(a.out, (size_t)t * a.ldt + n * a.ldn, c[i]);
    }
}

}  // namespace mx4
