// Products of matrices of 16-bit elements with sums in fp32, and what is done with each sum before it leaves: the core of the
// loss over a vocabulary (loss_kernels.hpp) and of orthogonalised updates (orthogonal_kernels.hpp).
//
// The result is C[m][n] = sum over k of A(m, k) B(n, k).  Either operand lies in memory along k (a row for each m, its k side by
// side) or down k (a row for each k, its m side by side), so that neither the operands of a backward pass nor a symmetric
// product need a transposed copy: LDS is read with ds_read_b64_tr_b16 where an operand lies down.
#pragma once
#include <type_traits>

#include "common.hpp"

#pragma clang fp contract(off)

namespace product {

using ss::f32x4;
using ss::u32x4;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// matrices of a caller are aligned to their element alone
typedef u32x4 u32x4_16 __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// a value that all lanes have, for the scalar unit
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// v_mfma_f32_32x32x16: a lane gives eight neighbouring k of row lane % 32; lanes 32 and up have the other eight
struct Bf16 {
    static __device__ __forceinline__ f32x16 multiply(u32x4 b, u32x4 a, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
    }
};
struct F16 {
    static __device__ __forceinline__ f32x16 multiply(u32x4 b, u32x4 a, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
    }
};

constexpr uint32_t kStep = 64;      // k of one step

struct Operand {
    const void *p;
    uint32_t ld;         // elements from one row to the next; rows start at multiples of 4 bytes
    uint32_t rows;       // m there are: those beyond read as the last one, or what lies behind it in its 16 bytes
    uint32_t depth;      // k there are, of an operand that lies down: those beyond read as the last one.  Along k there are whole steps, or what stands in their place is masked (kRagged).
    uint64_t apart;      // elements from one matrix of a stack to the next
    int64_t lo;          // of an operand that is the sum of two: elements from one to the other
    uint64_t bytes;      // a caller's buffer: what lies beyond is not read, and zero.  0: memory of our own, which goes on
};

constexpr uint32_t kHigh = 4;      // tile rows of a band, in which tiles are taken column by column

// tiles of the first `bands` bands of a square of n tiles a side that begin at the diagonal, and the few below it in each band's first columns
__host__ __device__ constexpr uint32_t half_tiles(uint32_t n, uint32_t bands) {
    const uint32_t whole = bands * kHigh <= n ? bands : n / kHigh, rest = n - whole * kHigh;
    return kHigh * (whole * n - kHigh * (whole * (whole - (whole > 0)) / 2)) + (bands > whole ? rest * rest : 0);
}

template <typename EndArgs>
struct TilesArgs {
    Operand a, b;
    uint32_t M, N;                    // of the result
    uint32_t steps;
    uint32_t tail;                    // k of the last step, if it is ragged
    uint32_t once;                    // steps of one product.  Operands that are sums of two take three: first times first, A's second times first, first times B's second.
    uint32_t tiles_m, tiles_n;
    uint32_t splits;                  // of k
    uint32_t bands;                   // of a symmetric result, of which only the tiles on and above the diagonal are computed, each written twice; 0: all of them
    float *parts;                     // the partial sums, if splits > 1: (stack, split, M, N)
    EndArgs end;
};

// all but the last N loads of this wave are there (neither a barrier nor a read waits for loads into LDS by itself), and so is what it read from LDS
template <int N>
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

// 16 bytes a lane straight into LDS, one lane's behind the other's from `to` on.  Not by the builtin: after one the compiler lets no ds_read_b64_tr_b16 go before all loads into LDS are there, whatever
// part of it they go to (8192 x 4096 x 8192 with both operands down k 1,191 us).  What a step reads has been waited for with arrived().  Addresses are multiples of 4 bytes; a dword beyond `end`
// is not read, and zero in LDS.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"      // m0 is reserved, but not in use here: no other instruction of these kernels reads it
__device__ __forceinline__ void load_to_lds(const char *base, size_t behind, uint64_t end, uint32_t offset, uint32_t to) {
    const uint64_t p = reinterpret_cast<uint64_t>(base) + behind, left = end > p ? end - p : 0;
    const u32x4 window = {(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, left < 0xFFFFFFFFu ? (uint32_t)left : 0xFFFFFFFFu, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(window) : "m0");
}
#pragma clang diagnostic pop

typedef __attribute__((address_space(3))) void *Lds;
typedef __attribute__((address_space(3))) i16x4 *LdsFour;

// One operand's way into LDS and out of it, for a tile of 64 T rows, four waves; a step has 8,192 T bytes.
//   along k: a row has 128 bytes; chunk c (16 bytes) of row r lies at place c ^ (r / 2 & 7) of its row, so that the rows that a read
//            takes together lie in different banks
//   down k:  a row (of one k) has 128 T bytes; groups of 64 bytes are exchanged by the row's number modulo 4 (T = 1: by its second bit),
//            for the same reason
template <bool DOWN, int T>
struct Way {
    static constexpr uint32_t kRow = DOWN ? 128 * T : 128, kPerLoad = 1024 / kRow;
    static constexpr int kLoads = 2 * T;     // of a wave, for a step
    const char *base;
    uint64_t end;
    uint32_t ld_bytes, depth;
    uint32_t from[DOWN ? 2 : kLoads];
    uint32_t at[DOWN ? T : 4];

    // rows m0 to m0 + 64 T; the wave multiplies those from `mine` on
    __device__ __forceinline__ Way(const Operand &o, uint32_t stack, uint32_t m0, uint32_t mine, uint32_t lane, uint32_t wave)
        : base(static_cast<const char *>(o.p) + (stack * o.apart + (DOWN ? (size_t)m0 : (size_t)m0 * o.ld)) * 2),
          end(o.bytes ? reinterpret_cast<uint64_t>(o.p) + o.bytes : ~0ull), ld_bytes(o.ld * 2), depth(o.depth) {
        const uint32_t last = o.rows - 1 - m0;
        if constexpr (DOWN) {
            const uint32_t k = wave * kPerLoad + lane / (64 / kPerLoad), place = lane % (64 / kPerLoad);
            const uint32_t chunk = place ^ (T > 1 ? (k & 3u) * 4 : (k >> 1 & 1u) * 4);
            from[0] = k * ld_bytes;
            from[1] = (chunk < last / 8 ? chunk : last / 8) * 16;
            // four k of 16 neighbouring m: a lane gives four m of one k, and is given four k of one m
            const uint32_t t = lane & 15u;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                const uint32_t group = (mine / 32 + i) ^ (T > 1 ? t >> 2 : t >> 3);
                at[i] = ((lane >> 5) * 32 + (t >> 2)) * kRow + group * 64 + (lane >> 4 & 1u) * 32 + (t & 3u) * 8;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t row = (wave + 4 * i) * 8 + (lane >> 3), chunk = (lane & 7u) ^ (row >> 1 & 7u);
                from[i] = (row < last ? row : last) * ld_bytes + chunk * 16;
            }
            const uint32_t r = lane & 31u, q = lane >> 5;
#pragma unroll
            for (int j = 0; j < 4; ++j) at[j] = (mine + r) * kRow + (((4 * q + j) ^ (r >> 1 & 7u)) * 16);
        }
    }
    __device__ __forceinline__ void fetch(char *lds, int i, uint32_t place, uint32_t step, int64_t lo, uint32_t wave) const {
        uint32_t offset;
        size_t behind;
        if constexpr (DOWN) {
            const uint32_t left = depth - 1 - step * kStep, last = (left < kStep - 1 ? left : kStep - 1) * ld_bytes;
            const uint32_t k = from[0] + 4 * i * kPerLoad * ld_bytes;
            offset = (k < last ? k : last) + from[1];
            behind = (size_t)step * kStep * ld_bytes + lo;
        } else {
            offset = from[i];
            behind = (size_t)step * kStep * 2 + lo;
        }
        load_to_lds(base, behind, end, offset, (uint32_t)reinterpret_cast<uintptr_t>((Lds)lds) + place + (wave + 4 * i) * 1024);
    }
    // block i (32 rows) of quarter j (16 of the k): lanes below 32 have k 8 j to 8 j + 7 of the step, the others those 32 further on
    __device__ __forceinline__ u32x4 read(const char *lds, int i, int j, uint32_t place) const {
        if constexpr (DOWN) {
            const char *p = lds + place + at[i] + j * 8 * kRow;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour)p));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour)(p + 4 * kRow)));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else return *reinterpret_cast<const u32x4 *>(lds + place + at[j] + i * 32 * kRow);
    }
};

template <int T>
struct Fragments {
    u32x4 a[T], b[T];
};

// part of 2 T of the multiplications of a quarter.  b is the first operand, so that a lane has four neighbours of a row of the result.
template <typename E, int T>
__device__ __forceinline__ void multiply(f32x16 (&c)[T][T], const Fragments<T> &f, int part) {
#pragma unroll
    for (int x = part * T / 2; x < (part + 1) * T / 2; ++x) c[x / T][x % T] = E::multiply(f.b[x % T], f.a[x / T], c[x / T][x % T]);
}

// eight neighbours of a row, rounded to the nearest, ties to even; `n` of them where the row ends
template <typename E, typename V>
__device__ __forceinline__ void store_eight(E *to, const f32x4 (&v)[2], uint32_t n) {
    if (n >= 8) {
        if constexpr (sizeof(E) == 2) {
            V o;
#pragma unroll
            for (int x = 0; x < 8; ++x) o[x] = (E)v[x / 4][x % 4];
            *reinterpret_cast<u32x4_16 *>(to) = __builtin_bit_cast(u32x4, o);
        } else {
            *reinterpret_cast<f32x4_any *>(to) = v[0];
            *reinterpret_cast<f32x4_any *>(to + 4) = v[1];
        }
    } else {
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x)
            if (x < n) to[x] = (E)v[x / 4][x % 4];
    }
}
__device__ __forceinline__ void store_out(void *to, bool bf16, size_t at, const f32x4 (&v)[2], uint32_t n) {
    if (bf16) store_eight<__bf16, bf16x8>(static_cast<__bf16 *>(to) + at, v, n);
    else store_eight<float, f32x4>(static_cast<float *>(to) + at, v, n);
}

// What becomes of eight neighbouring sums, as an End says it: load() brings what it takes besides (None where that is nothing), finish() computes, put() writes.  kStrips: it is given
// them so, and not a wave's whole tile; kParts: the sum over k may come in parts; kSymmetric: the result may be computed by half; kRagged: b's last step along k is not whole.
struct None {};

// Tiles of 2 x 2 waves, each 32 T rows by 32 T columns of the result.  A step is 64 of k, multiplied in four quarters; the fragments of the
// next quarter are read while one is multiplied.  Operands are loaded straight into LDS, which has room for five operands' steps: both of the one that is
// read, both of the next one and the first of the one after that.  So there is always something to load: the second operand of the next step right after the last one's
// place is free, then the first one of the step after it, spread over the multiplications.
// SHORT, for a few steps: one step is all that LDS holds, so that eight blocks instead of four share a compute unit, and wait for their loads and write their results in turn: that is what bounds such
// products.  us, SHORT / tiles of 64 / of 128: gradients of 19840 x 2258 from 64 rows 25.9 / 43.5 / 41.0, 84096 x 212 from 64 15.2 / 23.5 / 24.2, 32000 x 1024 from 128 23.8 / 38.9 / 32.1, 32000 x 2048 from 256
// 57.3 / 89.3 / 69.7, 32000 x 512 from 512 28.6 / - / 26.5.
template <typename E, bool A_DOWN, bool B_DOWN, int T, typename End, bool SHORT = false>
__global__ __launch_bounds__(256, 1) void tiles_kernel(const TilesArgs<typename End::Args> p) {
    constexpr uint32_t B = 64 * T, kUnit = B * 128, kRing = (SHORT ? 2 : 5) * kUnit;
    static_assert(!SHORT || T == 1, "one strip");
    constexpr int L = 2 * T;
    __shared__ __attribute__((aligned(1024))) char lds[kRing];
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
    const uint32_t r = lane & 31u, q = lane >> 5;
    // neighbouring blocks go to the eight dies in turn: each die takes a run of tiles, four tile rows high
    const uint32_t total = gridDim.x, die = blockIdx.x & 7u, share = total >> 3, more = total & 7u;
    uint32_t at = die * share + (die < more ? die : more) + (blockIdx.x >> 3);
    const uint32_t tiles = p.bands ? half_tiles(p.tiles_m, p.bands) : p.tiles_m * p.tiles_n, whole = uniform(at / tiles), stack = uniform(whole / p.splits), split = whole - stack * p.splits;
    at -= whole * tiles;
    uint32_t band = 0, first = 0, in;         // first: the band's first column
    if (p.bands) {
        while (band + 1 < p.bands && at >= half_tiles(p.tiles_m, band + 1)) ++band;
        first = band * kHigh;
        in = at - half_tiles(p.tiles_m, band);
    } else {
        band = uniform(at / (kHigh * p.tiles_n));
        in = at - band * kHigh * p.tiles_n;
    }
    const uint32_t left = p.tiles_m - band * kHigh, high = left < kHigh ? left : kHigh, column = first + uniform(in / high);
    const uint32_t tile_row = band * kHigh + in - (column - first) * high, m0 = tile_row * B, n0 = column * B;
    if (p.bands && tile_row > column) return;
    const uint32_t each = uniform(p.steps / p.splits), over = p.steps - each * p.splits;
    const uint32_t from = split * each + (split < over ? split : over), to = from + each + (split < over ? 1u : 0u);

    const uint32_t ma = (wave & 1u) * T * 32, nb = (wave >> 1) * T * 32;
    const Way<A_DOWN, T> wa(p.a, stack, m0, ma, lane, wave);
    const Way<B_DOWN, T> wb(p.b, stack, n0, nb, lane, wave);
    // the last steps load the last one again, which nothing reads: a branch would part the loop
    struct At {
        uint32_t step;
        int64_t a, b;
    };
    auto step_of = [&](uint32_t step) {
        step = step < to ? step : to - 1;
        const bool second = step >= p.once, third = step >= 2 * p.once;
        return At{third ? step - 2 * p.once : second ? step - p.once : step, second && !third ? p.a.lo * 2 : 0, third ? p.b.lo * 2 : 0};
    };
    auto read = [&](Fragments<T> &f, int i, int j, uint32_t a, uint32_t b) {
        if (i < T) f.b[i] = wb.read(lds, i, j, b);
        else f.a[i - T] = wa.read(lds, i - T, j, a);
    };
    f32x16 c[T][T] = {};
    // b's k beyond the last one, which a's zeros alone would not undo: they may be NaN
    auto mask_of = [&](int j, int left) {       // left: k that this lane has, of 32
        u32x4 mask;
#pragma unroll
        for (int d = 0; d < 4; ++d) mask[d] = 8 * j + 2 * d + 1 < left ? ~0u : 8 * j + 2 * d < left ? 0xFFFFu : 0u;
        return mask;
    };
    u32x4 kept[4];
    auto keep = [&](Fragments<T> &f, int j) {
        if constexpr (End::kRagged)
#pragma unroll
            for (int i = 0; i < T; ++i) f.b[i] &= kept[j];
    };
    auto mask = [&] {
#pragma unroll
        for (int j = 0; j < 4; ++j) kept[j] = mask_of(j, (int)p.tail - 32 * (int)q);
    };
    if constexpr (End::kRagged)
#pragma unroll
        for (int j = 0; j < 4; ++j) kept[j] = u32x4{~0u, ~0u, ~0u, ~0u};
    if constexpr (SHORT) {
        for (uint32_t step = 0; step < p.steps; ++step) {
            if (step) __builtin_amdgcn_s_barrier();     // all have read the one before it
            const At coming = step_of(step);
#pragma unroll
            for (int i = 0; i < L; ++i) wa.fetch(lds, i, 0, coming.step, coming.a, wave), wb.fetch(lds, i, kUnit, coming.step, coming.b, wave);
            arrived<0>();
            __builtin_amdgcn_s_barrier();
            // Where the last step is not whole, two quarters at a time, with masks that are made right where they are used: all four at once, or masks kept through the steps, take more than 64
            // registers, and four blocks share a compute unit, not eight.  us so / with 116 registers: gradients of 1000 rows against 50000 x 33 90 / 101, 900 against 32000 x 250 95 / 106, 64 against 84096 x 212 52.5 / 53.8.
            constexpr int kAtOnce = End::kRagged ? 2 : 4;
#pragma unroll
            for (int j0 = 0; j0 < 4; j0 += kAtOnce) {
                Fragments<T> f[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                    for (int i = 0; i < 2 * T; ++i) read(f[j], i, j0 + j, 0, kUnit);
                if constexpr (End::kRagged) {
                    if (step + 1 == to) {
                        int left = (int)p.tail - 32 * (int)q;
                        asm volatile("" : "+v"(left));
#pragma unroll
                        for (int j = 0; j < kAtOnce; ++j) f[j].b[0] &= mask_of(j0 + j, left);
                    }
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                    for (int part = 0; part < 2 * T; ++part) multiply<E>(c, f[j], part);
                if constexpr (End::kRagged) __builtin_amdgcn_sched_barrier(0);
            }
            arrived<0>();
        }
        arrived<0>();       // what was read is here before the strips take its place
    } else if (from < to) {
        Fragments<T> f0, f1;
        uint32_t a = 0, b = kUnit, a1 = 2 * kUnit, b1 = 3 * kUnit, free = 4 * kUnit;     // places of this step's operands, the next one's, and of what comes next
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const At coming = step_of(from + k);
#pragma unroll
            for (int i = 0; i < L; ++i) wa.fetch(lds, i, k ? a1 : a, coming.step, coming.a, wave), wb.fetch(lds, i, k ? b1 : b, coming.step, coming.b, wave);
        }
        arrived<2 * L>();
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int i = 0; i < 2 * T; ++i) read(f0, i, 0, a, b);
        __builtin_amdgcn_sched_barrier(0);
        for (uint32_t step = from; step < to; ++step) {
            const At coming = step_of(step + 2);
            if constexpr (End::kRagged) {
                if (step + 1 == to) mask();
            }
            keep(f0, 0);
            // Part by part, with a read and perhaps a load in each: in one go they would keep the matrix unit waiting while their queues are full
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f1, part, 1, a, b);
                multiply<E>(c, f0, part);
                __builtin_amdgcn_sched_barrier(0);
            }
            keep(f1, 1);
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f0, part, 2, a, b);
                if (part % 2 == 0) wa.fetch(lds, part / 2, free, coming.step, coming.a, wave);
                multiply<E>(c, f1, part);
                __builtin_amdgcn_sched_barrier(0);
            }
            keep(f0, 2);
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f1, part, 3, a, b);
                if (part % 2 == 0) wa.fetch(lds, T + part / 2, free, coming.step, coming.a, wave);
                multiply<E>(c, f0, part);
                __builtin_amdgcn_sched_barrier(0);
            }
            // this step's places have been read by all, and the next one's operands are there
            arrived<L>();
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            keep(f1, 3);
#pragma unroll
            for (int part = 0; part < 2 * T; ++part) {
                read(f0, part, 0, a1, b1);
                wb.fetch(lds, part, a, coming.step, coming.b, wave);
                multiply<E>(c, f1, part);
                __builtin_amdgcn_sched_barrier(0);
            }
            const uint32_t was_a = a, was_b = b;
            a = a1, b = b1, a1 = free, b1 = was_a, free = was_b;
        }
        arrived<0>();       // nothing is on its way into LDS that the next block may have
    }
    if constexpr (!End::kStrips) {
        End::finish(p.end, c, m0 + ma, n0 + nb, 2 * column + (wave >> 1), p.M, p.N, r, q);
    } else {
        // The result passes through LDS, 32 rows of a wave at a time, so that a lane has eight neighbours of a row and stores take whole lines.  Each wave has a part of
        // the ring to itself; chunk c (four sums) of row r lies at place c ^ r, for the banks' sake.
        constexpr uint32_t kChunks = 8 * T, kStrip = 32 * kChunks * 16, kAcross = 4 * T, kRows = 64 / kAcross;
        char *mine = lds + wave * (SHORT ? 1 : 2) * kStrip;
        __builtin_amdgcn_s_barrier();       // all have read what the ring held
        const uint32_t of = lane / kAcross, eight = lane % kAcross, col = n0 + nb + eight * 8;
#pragma unroll
        for (int i = 0; i < T; ++i) {
            char *strip = mine + (i & 1) * kStrip;
            // all of a strip's loads are on the way together
            typename End::Besides besides[32 / kRows];
#pragma unroll
            for (uint32_t j = 0; j < 32 / kRows; ++j) {
                const uint32_t m = m0 + ma + i * 32 + j * kRows + of;
                if ((!End::kParts || p.splits == 1) && m < p.M && col < p.N) besides[j] = End::load(p.end, stack, m, col, p.N);
            }
#pragma unroll
            for (int k = 0; k < T; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<f32x4 *>(strip + (r * kChunks + ((k * 8 + 2 * e + q) ^ (r & (kChunks - 1)))) * 16) =
                        f32x4{c[i][k][4 * e], c[i][k][4 * e + 1], c[i][k][4 * e + 2], c[i][k][4 * e + 3]};
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (uint32_t j = 0; j < 32 / kRows; ++j) {
                const uint32_t row = j * kRows + of, m = m0 + ma + i * 32 + row;
                f32x4 v[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) v[h] = *reinterpret_cast<const f32x4 *>(strip + (row * kChunks + ((2 * eight + h) ^ (row & (kChunks - 1)))) * 16);
                if (m >= p.M || col >= p.N) continue;
                if constexpr (End::kParts) {
                    if (p.splits > 1) {
                        store_eight<float, f32x4>(p.parts + ((size_t)whole * p.M + m) * p.N + col, v, p.N - col);
                        continue;
                    }
                }
                End::finish(p.end, besides[j], m, col, v);
                End::put(p.end, stack, m, col, v, p.N);
                if constexpr (End::kSymmetric) {
                    if (p.bands)       // for the columns, below
#pragma unroll
                        for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4 *>(strip + (row * kChunks + ((2 * eight + h) ^ (row & (kChunks - 1)))) * 16) = v[h];
                }
            }
            if constexpr (End::kSymmetric) {
                if (!p.bands || tile_row == column) continue;
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                // the same 32 rows as columns: four lanes have a column's eights, one behind the other
#pragma unroll
                for (uint32_t j = 0; j < 2 * T; ++j) {
                    const uint32_t n = j * 16 + (lane >> 2), row = (lane & 3u) * 8;
                    f32x4 v[2];
#pragma unroll
                    for (uint32_t x = 0; x < 8; ++x)
                        v[x / 4][x % 4] = *reinterpret_cast<const float *>(strip + ((row + x) * kChunks + ((n >> 2) ^ ((row + x) & (kChunks - 1)))) * 16 + (n & 3u) * 4);
                    if (n0 + nb + n < p.N && m0 + ma + i * 32 + row < p.M) End::put(p.end, stack, n0 + nb + n, m0 + ma + i * 32 + row, v, p.N);
                }
            }
        }
    }
}

template <typename EndArgs>
struct JoinArgs {
    const float *parts;
    uint32_t M, N, splits, across;      // across: eights of a row
    uint64_t eights;                    // of all rows of the stack
    uint32_t slices;                    // threads that share an eight's parts: a power of two, 64 at most
    EndArgs end;
};

// The partial sums, eight neighbours a lane; where there are few of them and many parts, several lanes share them: 2 x 212 in 256 parts 5.3 us (one lane for each 23).
template <typename End>
__global__ __launch_bounds__(256) void join_kernel(const JoinArgs<typename End::Args> p) {
    const uint64_t thread = (uint64_t)blockIdx.x * 256 + threadIdx.x, at = thread / p.slices;
    const uint32_t slice = (uint32_t)thread & (p.slices - 1);
    if (at >= p.eights) return;         // whole groups of slices
    const uint64_t line = at / p.across;
    const uint32_t col = (uint32_t)(at - line * p.across) * 8, stack = (uint32_t)(line / p.M), row = (uint32_t)(line - (uint64_t)stack * p.M);
    const size_t size = (size_t)p.M * p.N;
    const float *from = p.parts + (size_t)stack * p.splits * size + (size_t)row * p.N + col;
    f32x4 v[2] = {};
    if (col + 8 <= p.N) {
#pragma unroll 4
        for (uint32_t k = slice; k < p.splits; k += p.slices)
#pragma unroll
            for (int h = 0; h < 2; ++h) v[h] += *reinterpret_cast<const f32x4_any *>(from + k * size + 4 * h);
    } else {
        for (uint32_t k = slice; k < p.splits; k += p.slices)
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if (col + x < p.N) v[x / 4][x % 4] += from[k * size + x];
    }
    for (uint32_t apart = 1; apart < p.slices; apart *= 2)
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x / 4][x % 4] += __shfl_xor(v[x / 4][x % 4], apart);
    if (slice) return;
    End::finish(p.end, End::load(p.end, stack, row, col, p.N), row, col, v);
    End::put(p.end, stack, row, col, v, p.N);
}

}  // namespace product
