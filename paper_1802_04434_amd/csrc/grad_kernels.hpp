// A model's gradients on their way into a step: the norm over many tensors of two types, and clipping to it.
//
//   norm = sqrt( sum_t sum_i g_t[i]^2 )          c = min(1, max_norm / (norm + 1e-6))          out_t = c g_t
//
// Both stream: the norm reads every byte once, clipping reads and writes every element once, nothing is
// computed that memory would wait for.  What is particular is the list.  A launch takes a few hundred tensors in its
// argument block (no table in memory that somebody has to keep, and no copy to the device in front of the call); the
// tensors are cut into units of one size, numbered through, and a block finds the tensor of its unit with one
// parallel comparison of the units' numbers.  Gradients may start at any element of a buffer: units begin at the 16-byte
// boundary at or below a tensor's first element, and what does not fill 16 bytes at the two ends goes
// element by element, a lane each.
#pragma once
#include "common.hpp"

#pragma clang fp contract(off)

namespace grads {

using ss::f32x4;
using ss::u16x4;
using ss::u32x4;
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1), aligned(4))) const f32x4 f32x4_any;      // at any element
typedef __attribute__((address_space(1), aligned(2))) const u16x8 u16x8_any;
typedef __attribute__((address_space(1), aligned(2))) const u16x4 u16x4_any;

// Addresses are numbers in the argument block, from which the compiler cannot tell that they are device memory
template <typename T>
using Global = __attribute__((address_space(1))) T *;
template <typename T>
__device__ __forceinline__ T ld_once(uint64_t at) {
    return __builtin_nontemporal_load((Global<const T>)at);
}
template <typename T>
__device__ __forceinline__ T ld_one(uint64_t at) {
    return *(Global<const T>)at;
}
template <typename T>
__device__ __forceinline__ void st_once(uint64_t at, T v) {
    __builtin_nontemporal_store(v, (Global<T>)at);
}

// Tensors of one launch: the argument blocks stay below 4 KiB
constexpr int kNormTensors = 256, kClipTensors = 176, kClipPlaces = 192;     // a multiple of the lanes

// Which tensor has unit u: the last one that begins at or before it (tensors without units begin where the next does).
// Loads by lane, which wait for nothing, and a count of the lanes that say yes, where a binary search would be eight dependent loads.
template <int TENSORS>
__device__ __forceinline__ uint32_t tensor_of(const uint32_t *first, uint32_t n, uint32_t u) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t at[TENSORS / 64], before = 0;
#pragma unroll
    for (uint32_t k = 0; k < TENSORS / 64; ++k) at[k] = first[lane + 64 * k];
#pragma unroll
    for (uint32_t k = 0; k < TENSORS / 64; ++k) before += (uint32_t)__popcll(__ballot(lane + 64 * k < n && at[k] <= u));
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)before) - 1;
}

// The elements of a tensor that do not fill 16 bytes at its two ends, one a lane: of the `each` lanes from 0 on those of the first 16 bytes, from 8 on
// those of the last.  The tensor is elements [lead, span) from a 16-byte boundary; `each` of them fill 16 bytes.  False: the lane has none.
__device__ __forceinline__ bool edge_element(uint32_t lane, uint32_t lead, size_t span, uint32_t each, bool first, bool last, size_t &e) {
    const size_t whole = span / each * each;
    const bool ahead = lane < each, behind = lane >= 8 && lane < 8 + each;
    e = ahead ? lane : whole + lane - 8;
    // one lot of 16 bytes that both ends are in counts as the first
    return (ahead && first && lead && e >= lead && e < span) || (behind && last && e < span && !(whole == 0 && lead));
}

// ---------------------------------------------------------------- norm ----
// Block b takes units [U b / G, U (b + 1) / G) of U, BATCH of them in flight; the lanes' sums in fp64 go through lane moves and LDS
// into a slot, and the block that takes the last ticket adds the slots in a fixed order and writes the norm.  As in the density few large
// blocks, since tickets on one address take 11 ns each; here they are taken in two levels, 16 groups on lines of their own and one
// above: 48 in a row instead of 512, and 32 instead of 256 from a GiB on.  Of several launches all but the last one add to the slots and take no tickets.
// Measured, us: 1.5 G bf16 436 to 457 (6.6 to 6.9 TB/s), 25.6 M fp32 in 161 tensors 20 (5.2 TB/s), of which ramp and the tail of dependent trips are 5; 272,474 in 65
// tensors 5.4, of which the host's call alone is 5.2.

constexpr int kNormThreads = 512;
constexpr int kNormBlocks = 512;
constexpr int kNormGroups = 16;
constexpr uint32_t kNormUnit = kNormThreads * 16;          // bytes

struct NormScratch {
    struct Ticket {
        unsigned long long n;                              // zero between calls
        unsigned long long pad[7];
    };
    Ticket top, group[kNormGroups];
    double partial[kNormBlocks];
};

struct NormArgs {
    uint64_t at[kNormTensors];         // address; bit 0: bf16
    uint32_t first[kNormTensors + 1];  // first unit; [n]: number of units
    uint16_t rest[kNormTensors];       // bytes in the last unit, less one
    uint32_t n;
    uint32_t opens, closes;            // first, last launch of the call
    uint32_t slots;                    // blocks of the call's largest launch, and of the first
    float *norm;
    NormScratch *scratch;
};

// the square of a 24-bit significand is exact in fp64: one rounding for product and sum
__device__ __forceinline__ void add_square(double &s, float v) {
    const double a = (double)v;
    s = __builtin_fma(a, a, s);
}

template <bool BF16>
__device__ __forceinline__ void add_squares(double &s, u32x4 q) {
    if constexpr (BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            add_square(s, __uint_as_float(q[k] << 16));
            add_square(s, __uint_as_float(q[k] & 0xFFFF0000u));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) add_square(s, __uint_as_float(q[k]));
    }
}

// units [k, end) of the tensor whose elements are bytes [head, span) from `base`
template <bool BF16, int BATCH, bool ONCE>
__device__ __forceinline__ double tensor_squares(uint64_t base, uint32_t head, size_t span, uint32_t k, uint32_t end) {
    constexpr uint32_t kSize = BF16 ? 2 : 4;
    size_t e;
    float edge = 0.0f;
    const uint32_t units = (uint32_t)((span + kNormUnit - 1) / kNormUnit);
    if (edge_element(threadIdx.x, head / kSize, span / kSize, 16 / kSize, k == 0, end == units, e)) {
        if constexpr (BF16) edge = ss::widen_bf16(ld_one<uint16_t>(base + e * kSize));
        else edge = ld_one<float>(base + e * kSize);
    }
    double sum = 0.0;
    // the 16-byte lots that are all the tensor's
    const size_t lo = (head + 15u) / 16, hi = span / 16;
    if (lo < hi)
        for (; k < end; k += BATCH) {
            u32x4 q[BATCH];
            const size_t at = (size_t)k * kNormThreads + threadIdx.x;
            if ((size_t)k * kNormThreads >= lo && (size_t)(k + BATCH) * kNormThreads <= hi && k + BATCH <= end) {
#pragma unroll
                for (int r = 0; r < BATCH; ++r) q[r] = (ONCE ? ld_once<u32x4> : ld_one<u32x4>)(base + (at + (size_t)r * kNormThreads) * 16);
            } else {        // some are not, or another block's: loaded where there are some, and left out
                bool in[BATCH];
#pragma unroll
                for (int r = 0; r < BATCH; ++r) {
                    const size_t i = at + (size_t)r * kNormThreads, from = i < lo ? lo : i < hi ? i : hi - 1;
                    in[r] = i >= lo && i < hi && k + r < end;
                    q[r] = (ONCE ? ld_once<u32x4> : ld_one<u32x4>)(base + from * 16);
                }
#pragma unroll
                for (int r = 0; r < BATCH; ++r)
#pragma unroll
                    for (int x = 0; x < 4; ++x) q[r][x] = in[r] ? q[r][x] : 0u;
            }
            double t = 0.0;
#pragma unroll
            for (int r = 0; r < BATCH; ++r) add_squares<BF16>(t, q[r]);
            sum += t;
        }
    add_square(sum, edge);
    return sum;
}

template <int BATCH, bool ONCE>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(const NormArgs a) {
    constexpr int kWaves = kNormThreads / 64;
    static_assert(kWaves == 8, "sum8 adds the waves' sums");
    __shared__ double part[kWaves];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, b = blockIdx.x, G = gridDim.x;
    const uint64_t units = a.first[a.n];
    uint32_t u = (uint32_t)(units * b / G);
    const uint32_t end = (uint32_t)(units * (b + 1) / G);
    double sum = 0.0;
    if (u < end) {
        for (uint32_t t = tensor_of<kNormTensors>(a.first, a.n, u); u < end; ++t) {
            const uint32_t lo = a.first[t], hi = a.first[t + 1], stop = hi < end ? hi : end;
            if (u >= stop) continue;                       // a tensor without elements
            const uint64_t at = a.at[t];
            const uint64_t base = at & ~(uint64_t)15;
            const uint32_t head = (uint32_t)at & 14u;
            const size_t span = (size_t)(hi - lo - 1) * kNormUnit + a.rest[t] + 1u;
            sum += at & 1u ? tensor_squares<true, BATCH, ONCE>(base, head, span, u - lo, stop - lo)
                           : tensor_squares<false, BATCH, ONCE>(base, head, span, u - lo, stop - lo);
            u = stop;
        }
    }
    sum = ss::sum_wave(sum);
    if (lane == 63) part[tid >> 6] = sum;
    __syncthreads();
    if (tid >= 64) return;
    sum = ss::sum8(part[lane & (kWaves - 1)]);
    if (!a.closes || a.slots > 1) {
        unsigned last = 0;
        if (lane == 0) {
            if (!a.opens) sum += a.scratch->partial[b];    // written by the launch before
            __hip_atomic_store(&a.scratch->partial[b], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (a.closes) {
                // the slot has been performed at device scope before the ticket is taken, as in the density
                const uint32_t group = b % kNormGroups, members = (G - group + kNormGroups - 1) / kNormGroups;
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                last = __hip_atomic_fetch_add(&a.scratch->group[group].n, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == members - 1ull;
                asm volatile("" ::: "memory");
                // every ticket of the group has come back, and so have its slots, before the one above is taken
                if (last) {
                    const uint32_t groups = G < kNormGroups ? G : kNormGroups;
                    __hip_atomic_store(&a.scratch->group[group].n, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    last = __hip_atomic_fetch_add(&a.scratch->top.n, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1ull;
                }
            }
        }
        if (!__builtin_amdgcn_readfirstlane(last)) return;
        asm volatile("" ::: "memory");                     // the loads below stay behind the ticket
        constexpr int kSlots = kNormBlocks / 64;
        double s[kSlots];
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            const uint32_t slot = lane + 64 * k;
            s[k] = slot < a.slots ? __hip_atomic_load(&a.scratch->partial[slot], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        }
#pragma unroll
        for (int k = 1; k < kSlots; ++k) s[0] += s[k];
        sum = ss::sum_wave(s[0]);
        if (lane != 63) return;
        __hip_atomic_store(&a.scratch->top.n, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else if (lane != 63) {
        return;
    }
    *a.norm = (float)__builtin_sqrt(sum);
}

// ---------------------------------------------------------------- clip ----
// A block takes kClipRows rows of 16 bytes a lane, aligned to 16 bytes where they are written; they are read at whatever address that gives.  Many short blocks, since there is nothing
// to add up: us for 25.6 M fp32 in 161 tensors, 1 / 2 / 8 rows 48 / 31 / 42, and runs of units a block 40 to 48.  That is 6.5 TB/s, what a copy takes;
// 138 M of both types into fp32 160 us (5.6 TB/s).  The other forms on 25.6 M: fp32 to bf16 26 us (5.9 TB/s), bf16 to bf16 17.5 (5.8), bf16 to fp32
// 26 (5.9), in place fp32 36 (5.7) and bf16 18 (5.7), and within the bound, where nothing is to do, 5.0 and 3.5.

constexpr int kClipThreads = 256;
template <bool IN_BF16, bool OUT_BF16>
constexpr int kClipRows = IN_BF16 && !OUT_BF16 ? 4 : 2;
template <bool IN_BF16, bool OUT_BF16>
constexpr uint32_t kClipUnit = kClipThreads * kClipRows<IN_BF16, OUT_BF16> * (OUT_BF16 ? 8 : 4);           // elements

struct ClipArgs {
    uint64_t at[kClipTensors];         // addresses; bit 0: bf16
    uint64_t out[kClipTensors];
    uint32_t first[kClipPlaces];       // first unit; [n]: number of units
    uint16_t rest[kClipTensors];       // elements in the last unit, less one
    uint32_t n;
    float max_norm;
    const float *norm;
};

__device__ __forceinline__ float clip_factor(float norm, float max_norm) {
    const float c = max_norm / (norm + 1e-6f);
    return c >= 1.0f ? 1.0f : c;       // NaN stays
}

// unit k of a tensor; its element i is element lead + i of the span
template <bool IN_BF16, bool OUT_BF16>
__device__ __forceinline__ void clip_unit(uint64_t in, uint64_t out, uint32_t lead, size_t span, uint32_t k, float c) {
    constexpr uint32_t kIn = IN_BF16 ? 2 : 4, kOut = OUT_BF16 ? 2 : 4, V = 16 / kOut, kUnit = kClipUnit<IN_BF16, OUT_BF16>;
    constexpr int R = kClipRows<IN_BF16, OUT_BF16>;
    in -= lead * kIn, out -= lead * kOut;
    const size_t unit = (size_t)k * kUnit, at = unit + threadIdx.x * V;
    // the lots of 16 bytes that are all the tensor's
    const size_t lo = (lead + V - 1) / V * V, hi = span / V * V;
    float v[R][V];
    bool has[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const size_t e = at + (size_t)r * kClipThreads * V;
        has[r] = e >= lo && e < hi;
        if (!has[r]) continue;
        const uint64_t from = in + e * kIn;
        if constexpr (IN_BF16 && V == 8) {
            const u16x8 q = *(u16x8_any *)from;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[r][i] = ss::widen_bf16(q[i]);
        } else if constexpr (IN_BF16) {
            const u16x4 q = *(u16x4_any *)from;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[r][i] = ss::widen_bf16(q[i]);
        } else {
#pragma unroll
            for (uint32_t x = 0; x < V; x += 4) {
                const f32x4 q = *(f32x4_any *)(from + x * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[r][x + i] = q[i];
            }
        }
    }
    size_t e;
    float edge = 0.0f;
    const bool at_edge = edge_element(threadIdx.x, lead, span, V, k == 0, unit + kUnit >= span, e);
    if (at_edge) {
        if constexpr (IN_BF16) edge = ss::widen_bf16(ld_one<uint16_t>(in + e * kIn));
        else edge = ld_one<float>(in + e * kIn);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!has[r]) continue;
        const uint64_t to = out + (at + (size_t)r * kClipThreads * V) * kOut;
        if constexpr (OUT_BF16) {
            bf16x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (__bf16)(c * v[r][i]);
            st_once<bf16x8>(to, o);
        } else {
            f32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = c * v[r][i];
            st_once<f32x4>(to, o);
        }
    }
    if (at_edge) {
        if constexpr (OUT_BF16) st_once<__bf16>(out + e * kOut, (__bf16)(c * edge));
        else st_once<float>(out + e * kOut, c * edge);
    }
}

__global__ __launch_bounds__(kClipThreads) void clip_kernel(const ClipArgs a) {
    const uint32_t u = blockIdx.x, t = tensor_of<kClipPlaces>(a.first, a.n, u);
    const float c = clip_factor(*a.norm, a.max_norm);
    const uint64_t in = a.at[t], out = a.out[t];
    if (in == out && c == 1.0f) return;                    // in place, and within the bound
    const uint32_t lo = a.first[t], units = a.first[t + 1] - lo, rest = a.rest[t] + 1u;
    const uint64_t from = in & ~(uint64_t)1, to = out & ~(uint64_t)1;
    const auto span = [&](uint32_t unit) { return (size_t)(units - 1) * unit + rest; };
    if (out & 1u) {
        const uint32_t lead = (uint32_t)(to & 15u) >> 1;
        if (in & 1u) clip_unit<true, true>(from, to, lead, span(kClipUnit<true, true>), u - lo, c);
        else clip_unit<false, true>(from, to, lead, span(kClipUnit<false, true>), u - lo, c);
    } else {
        const uint32_t lead = (uint32_t)(to & 15u) >> 2;
        if (in & 1u) clip_unit<true, false>(from, to, lead, span(kClipUnit<true, false>), u - lo, c);
        else clip_unit<false, false>(from, to, lead, span(kClipUnit<false, false>), u - lo, c);
    }
}

}  // namespace grads
