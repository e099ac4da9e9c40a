// A model's gradients on their way into a step: the norm over many tensors of two types, and clipping to it.
//
//   norm = sqrt( sum_t sum_i g_t[i]^2 )          c = min(1, max_norm / (norm + 1e-6))          out_t = c g_t
//
// Both stream: the norm reads every byte once, clipping reads and writes every element once, nothing is
// computed that memory would wait for.  What is particular is the list.  A launch takes kTensors tensors in its
// argument block (no table in memory that somebody has to keep, and no copy to the device in front of the call); the
// tensors are cut into units of one size, numbered through, and a block finds the tensor of its unit with one
// parallel comparison of the units' numbers.  Gradients may start at any element of a buffer: units begin at the 16-byte
// boundary at or below a tensor's first element, and the lanes at the two ends, whose 16 bytes are
// not all the tensor's, go element by element.
#pragma once
#include "common.hpp"

#pragma clang fp contract(off)

namespace grads {

using ss::f32x4;
using ss::u32x4;
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1), aligned(4))) const f32x4 f32x4_any;      // at any element
typedef __attribute__((address_space(1), aligned(2))) const u16x8 u16x8_any;

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

// of one launch; the argument block stays below 4 KiB with two addresses a tensor
constexpr int kTensors = 176;

// Which tensor has unit u: the last one that begins at or before it (tensors without units begin where the next does).
// Three loads by lane and a count of the lanes that say yes, where a binary search would be eight dependent loads.
__device__ __forceinline__ uint32_t tensor_of(const uint32_t *first, uint32_t n, uint32_t u) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t before = 0;
#pragma unroll
    for (uint32_t k = 0; k < (kTensors + 63) / 64; ++k) {
        const uint32_t t = lane + 64 * k;
        const bool yes = t < n && first[t < n ? t : 0] <= u;
        before += (uint32_t)__popcll(__ballot(yes));
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)before) - 1;
}

// ---------------------------------------------------------------- norm ----
// Block b takes units [U b / G, U (b + 1) / G) of U, kBatch of them in flight; the lanes' sums in fp64 go through lane moves and LDS
// into a slot, and the block that takes the last ticket adds the slots in a fixed order and, in the last of
// several launches, writes the norm.  As in the density few large blocks, since tickets on one address take 11 ns each;
// here they are taken in two levels, 16 groups on lines of their own and one above, 32 in a row instead of 256.

constexpr int kNormThreads = 512;
constexpr int kNormBlocks = 256;
constexpr int kNormGroups = 16;
constexpr uint32_t kNormUnit = kNormThreads * 16;          // bytes
constexpr int kBatch = 8;

struct NormScratch {
    struct Ticket {
        unsigned long long n;                              // zero between calls
        unsigned long long pad[7];
    };
    Ticket top, group[kNormGroups];
    double total;                                          // of the launches before, within a call
    double pad[7];
    double partial[kNormBlocks];
};

struct NormArgs {
    uint64_t at[kTensors];             // address; bit 0: bf16
    uint32_t first[kTensors + 1];      // first unit; [n]: number of units
    uint16_t rest[kTensors];           // bytes in the last unit, less one
    uint32_t n;
    uint32_t opens, closes;            // first, last launch of the call
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
template <bool BF16>
__device__ __forceinline__ double tensor_squares(uint64_t base, uint32_t head, size_t span, uint32_t k, uint32_t end) {
    constexpr uint32_t kSize = BF16 ? 2 : 4;
    const uint32_t at = threadIdx.x * 16;
    double sum = 0.0;
    // the ends: a unit that is not all the tensor's
    auto ragged = [&](uint32_t unit) {
        const size_t o = (size_t)unit * kNormUnit + at;
        if (o >= head && o + 16 <= span) add_squares<BF16>(sum, ld_once<u32x4>(base + o));
        else
            for (size_t p = o; p < o + 16; p += kSize)
                if (p >= head && p < span) {
                    if constexpr (BF16) add_square(sum, ss::widen_bf16(ld_one<uint16_t>(base + p)));
                    else add_square(sum, ld_one<float>(base + p));
                }
    };
    if (k < end && k == 0 && head) ragged(k++);
    const uint32_t whole = (uint32_t)(span / kNormUnit);
    const bool tail = end > whole && k < end;
    if (tail) --end;
    uint64_t p = base + (size_t)k * kNormUnit + at;
    for (; k + kBatch <= end; k += kBatch, p += (size_t)kBatch * kNormUnit) {
        u32x4 q[kBatch];
#pragma unroll
        for (int r = 0; r < kBatch; ++r) q[r] = ld_once<u32x4>(p + (size_t)r * kNormUnit);
        double t = 0.0;
#pragma unroll
        for (int r = 0; r < kBatch; ++r) add_squares<BF16>(t, q[r]);
        sum += t;
    }
    if (k < end) {          // fewer than kBatch, out together
        u32x4 q[kBatch - 1];
#pragma unroll
        for (int r = 0; r < kBatch - 1; ++r) {
            q[r] = u32x4{0, 0, 0, 0};
            if (k + r < end) q[r] = ld_once<u32x4>(p + (size_t)r * kNormUnit);
        }
        double t = 0.0;
#pragma unroll
        for (int r = 0; r < kBatch - 1; ++r) add_squares<BF16>(t, q[r]);
        sum += t;
    }
    if (tail) ragged(whole);
    return sum;
}

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
        for (uint32_t t = tensor_of(a.first, a.n, u); u < end; ++t) {
            const uint32_t lo = a.first[t], hi = a.first[t + 1], stop = hi < end ? hi : end;
            if (u >= stop) continue;                       // a tensor without elements
            const uint64_t at = a.at[t];
            const uint64_t base = at & ~(uint64_t)15;
            const uint32_t head = (uint32_t)at & 14u;
            const size_t span = (size_t)(hi - lo - 1) * kNormUnit + a.rest[t] + 1u;
            sum += at & 1u ? tensor_squares<true>(base, head, span, u - lo, stop - lo)
                           : tensor_squares<false>(base, head, span, u - lo, stop - lo);
            u = stop;
        }
    }
    sum = ss::sum_wave(sum);
    if (lane == 63) part[tid >> 6] = sum;
    __syncthreads();
    if (tid >= 64) return;
    sum = ss::sum8(part[lane & (kWaves - 1)]);
    if (G > 1) {
        unsigned last = 0;
        if (lane == 0) {
            // the slot has been performed at device scope before the ticket is taken, as in the density
            const uint32_t group = b % kNormGroups, members = (G - group + kNormGroups - 1) / kNormGroups;
            __hip_atomic_store(&a.scratch->partial[b], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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
        if (!__builtin_amdgcn_readfirstlane(last)) return;
        asm volatile("" ::: "memory");                     // the loads below stay behind the ticket
        constexpr int kSlots = kNormBlocks / 64;
        double s[kSlots];
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            const uint32_t slot = lane + 64 * k;
            s[k] = slot < G ? __hip_atomic_load(&a.scratch->partial[slot], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        }
        sum = ss::sum_wave((s[0] + s[1]) + (s[2] + s[3]));
        if (lane != 63) return;
        __hip_atomic_store(&a.scratch->top.n, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else if (lane != 63) {
        return;
    }
    if (!a.opens) sum += a.scratch->total;                 // written by the launch before
    if (a.closes) *a.norm = (float)__builtin_sqrt(sum);
    else a.scratch->total = sum;
}

// ---------------------------------------------------------------- clip ----
// A lane takes eight elements, aligned to 16 bytes where they are written; they are read at whatever address that gives.

constexpr int kClipThreads = 256;
constexpr uint32_t kClipUnit = kClipThreads * 8;           // elements

struct ClipArgs {
    uint64_t at[kTensors];             // addresses; bit 0: bf16
    uint64_t out[kTensors];
    uint32_t first[kTensors + 1];
    uint16_t rest[kTensors];           // elements in the last unit, less one
    uint32_t n;
    float max_norm;
    const float *norm;
};

__device__ __forceinline__ float clip_factor(float norm, float max_norm) {
    const float c = max_norm / (norm + 1e-6f);
    return c >= 1.0f ? 1.0f : c;       // NaN stays
}

template <bool IN_BF16, bool OUT_BF16>
__device__ __forceinline__ void clip_unit(uint64_t in, uint64_t out, uint32_t lead, size_t span, uint32_t k, float c) {
    constexpr uint32_t kIn = IN_BF16 ? 2 : 4, kOut = OUT_BF16 ? 2 : 4;
    // element e of the span is element e - lead of the tensor
    const size_t e = (size_t)k * kClipUnit + threadIdx.x * 8;
    const uint64_t from = in + (e - lead) * kIn, to = out + (e - lead) * kOut;
    if (e >= lead && e + 8 <= span) {
        float v[8];
        if constexpr (IN_BF16) {
            const u16x8 q = __builtin_nontemporal_load((u16x8_any *)from);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = ss::widen_bf16(q[i]);
        } else {
            const f32x4 q0 = __builtin_nontemporal_load((f32x4_any *)from);
            const f32x4 q1 = __builtin_nontemporal_load((f32x4_any *)(from + 16));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = q0[i], v[4 + i] = q1[i];
        }
        if constexpr (OUT_BF16) {
            bf16x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (__bf16)(c * v[i]);
            st_once<bf16x8>(to, o);
        } else {
            f32x4 o0, o1;
#pragma unroll
            for (int i = 0; i < 4; ++i) o0[i] = c * v[i], o1[i] = c * v[4 + i];
            st_once<f32x4>(to, o0);
            st_once<f32x4>(to + 16, o1);
        }
        return;
    }
    for (int i = 0; i < 8; ++i) {
        if (e + i < lead || e + i >= span) continue;
        float v;
        if constexpr (IN_BF16) v = ss::widen_bf16(ld_one<uint16_t>(from + i * kIn));
        else v = ld_one<float>(from + i * kIn);
        if constexpr (OUT_BF16) st_once<__bf16>(to + i * kOut, (__bf16)(c * v));
        else st_once<float>(to + i * kOut, c * v);
    }
}

__global__ __launch_bounds__(kClipThreads) void clip_kernel(const ClipArgs a) {
    const uint32_t u = blockIdx.x, t = tensor_of(a.first, a.n, u);
    const float c = clip_factor(*a.norm, a.max_norm);
    const uint64_t in = a.at[t], out = a.out[t];
    if (in == out && c == 1.0f) return;                    // in place, and within the bound
    const uint32_t lo = a.first[t], units = a.first[t + 1] - lo;
    const size_t span = (size_t)(units - 1) * kClipUnit + a.rest[t] + 1u;
    const uint64_t from = in & ~(uint64_t)1, to = out & ~(uint64_t)1;
    if (out & 1u) {
        const uint32_t lead = (uint32_t)(to & 15u) >> 1;
        if (in & 1u) clip_unit<true, true>(from, to, lead, span, u - lo, c);
        else clip_unit<false, true>(from, to, lead, span, u - lo, c);
    } else {
        const uint32_t lead = (uint32_t)(to & 15u) >> 2;
        if (in & 1u) clip_unit<true, false>(from, to, lead, span, u - lo, c);
        else clip_unit<false, false>(from, to, lead, span, u - lo, c);
    }
}

}  // namespace grads
