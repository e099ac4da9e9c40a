// C ABI of orthogonalised updates (see include/signsgd.h): validation and launches.
#include <algorithm>
#include <cmath>

#include "api_common.hpp"
#include "orthogonal_kernels.hpp"
#include "product_launch.hpp"

namespace {

using namespace host;
using product::Layout;
using product::Operand;
using product::Plan;
using product::rounded;

struct Stack {
    size_t count, rows, cols;
    bool empty() const { return count == 0 || rows == 0 || cols == 0; }
    bool bad() const {
        return count > SS_ORTHOGONAL_MAX_COUNT || rows > SS_ORTHOGONAL_MAX_DIM || cols > SS_ORTHOGONAL_MAX_DIM || std::min(rows, cols) > SS_ORTHOGONAL_MAX_SHORT ||
               (!empty() && rounded(rows, 64) * rounded(cols, 64) > SS_ORTHOGONAL_MAX_ELEMENTS / count);
    }
    // matrices in rows `ld` apart, `apart` elements from one to the next; together 2^41 elements, which no card holds, so that no span of theirs passes 64 bits
    bool bad(size_t ld, size_t apart) const {
        constexpr size_t kMost = (size_t)1 << 40;
        return ld < cols || (rows > 1 && ld > kMost / (rows - 1)) || (count > 1 && (apart < (rows - 1) * ld + cols || apart > kMost / (count - 1)));
    }
    Span of(const void *p, size_t ld, size_t apart, ss_dtype dt, bool written) const { return span(p, ((count - 1) * apart + (rows - 1) * ld + cols) * grad_bytes(dt), written); }
};

inline bool element_aligned(const void *p, ss_dtype dt) { return reinterpret_cast<uintptr_t>(p) % grad_bytes(dt) == 0; }

// blocks that add up a matrix's squares
inline size_t norm_blocks(const Stack &s) { return std::min(std::max((s.rows * s.cols + 2047) / 2048, (size_t)1), std::max((size_t)1024 / s.count, (size_t)1)); }

// How many of the last steps multiply operands of 22 bits, in three products of 11: where the result is fp32, and the matrix so short that its roundings do not average out.  Off
// by, of the result's norm, without / with: 40 x 40 1.1e-3 / 1e-4, 120 x 1000 7.9e-4 / 1e-4, 512 squared 6.1e-4 / 3.9e-4, 1024 x 2048 4.2e-4.
inline int twofold_steps(size_t shorter, bool fp32) { return !fp32 || shorter >= 1024 ? 0 : shorter >= 512 ? 1 : shorter >= 256 ? 2 : 3; }

// A shorter side of 128 at most, and slices of the longer one.  A block of 96 and 128 has a compute unit to itself and makes B as every other one does: many of them take longer than the
// products in tiles.  us, in slices / in tiles to bf16 / to fp32: 25 x 7616 48 / 90 / 100, 64 x 64000 115 / 128 / 151, 1000 x 120 73 / 89 / 100, 128 x 8128 102 / 100 / 120, 128 x 16000 122 / 114 /
// 135, 128 x 60000 304 / 170 / 213; 25 of 1000 x 120 167 / 121 / 148.
struct Slices {
    size_t shorter, slice, count;      // count 0: another way is taken
    explicit Slices(const Stack &s) : shorter(rounded(std::min(s.rows, s.cols), 32)), slice(shorter <= 64 ? 128 : 64), count((std::max(s.rows, s.cols) + slice - 1) / slice) {
        if (shorter > 128 || count > 1024 || (shorter > 64 && s.count * count * shorter * shorter > (size_t)1 << 21)) count = 0;
    }
};

struct SlicePlace {
    size_t sums, hi, lo, a_hi, a_lo, parts, bytes;
    SlicePlace(const Stack &s, const Slices &t) {
        Layout l;
        sums = l.take(s.count * norm_blocks(s) * sizeof(double));
        hi = l.take(s.count * t.count * t.slice * t.shorter * 2);
        lo = l.take(s.count * t.count * t.slice * t.shorter * 2);
        a_hi = l.take(s.count * t.shorter * t.shorter * 2);
        a_lo = l.take(s.count * t.shorter * t.shorter * 2);
        parts = l.take(s.count * t.count * t.shorter * t.shorter * sizeof(float));
        bytes = l.bytes;
    }
};

struct Plans {
    Plan square, polynomial, update;
};

struct Place {
    size_t rows, cols, shorter, longer;       // whole steps
    Plans once, twofold;
    size_t sums, hi[2], lo[2], a[2], b[2], parts, bytes;

    Place(const Stack &s) {
        rows = rounded(s.rows, 64), cols = rounded(s.cols, 64);
        shorter = std::min(rows, cols), longer = std::max(rows, cols);
        const bool some = twofold_steps(shorter, true) > 0;
        Layout l;
        sums = l.take(s.count * norm_blocks(s) * sizeof(double));
        for (int k = 0; k < 2; ++k) {
            hi[k] = l.take(s.count * rows * cols * 2);
            lo[k] = k == 0 || some ? l.take(s.count * rows * cols * 2) : lo[0];      // in place where no product reads it
            a[k] = k == 0 || some ? l.take(s.count * shorter * shorter * 2) : 0;
            b[k] = k == 0 || some ? l.take(s.count * shorter * shorter * 2) : 0;
        }
        size_t most = 0;
        for (Plans *p : {&once, &twofold}) {
            const size_t times = p == &twofold ? 3 : 1;
            p->square = product::plan_of(shorter, shorter, times * longer, s.count, true, true);
            p->polynomial = product::plan_of(shorter, shorter, times * shorter, s.count, false, true);
            p->update = product::plan_of(rows, cols, times * shorter, s.count, false);
            if (p == &once || some)
                most = std::max(most, parts_bytes(p->square, s.count, shorter, shorter));
        }
        parts = l.take(most);
        bytes = l.bytes;
    }
};

inline size_t scratch_of(const Stack &s) {
    const Slices slices(s);
    return slices.count ? SlicePlace(s, slices).bytes : Place(s).bytes;
}

// a gradient on its way into an update, and where the update goes
struct Ends {
    const void *g;
    ss_dtype gdt;
    size_t ld, apart;
    float *m;
    float beta;
    bool ahead;
    void *out;
    ss_dtype odt;
    size_t ldo, aparto;
    float delta;
    bool step;
};

// Whether a matrix is worked on whole, by one block.  It has to fit into LDS, and one block sums over the longer side alone.  us, whole / in slices, any type: 64 x 64 18 / 49, 64 x 300
// 46 / 50, 64 x 480 65 / 50, 32 x 300 29 / 41, 32 x 900 65 / 43, 128 x 128 50 / 71; 48 of 64 x 300 47 / 63.
inline bool fits(const Stack &s) {
    const size_t shorter = rounded(std::min(s.rows, s.cols), 32), longer = rounded(std::max(s.rows, s.cols), 32);
    constexpr size_t kTiles = orthogonal::kWholeWaves * orthogonal::kWholeTiles;
    return shorter <= 128 && longer <= 320 && longer / 32 * (shorter / 32) <= kTiles && orthogonal::whole_bytes((uint32_t)shorter, (uint32_t)longer) <= orthogonal::kWholeBytes;
}

inline float mu_of(int step, int steps) { return step + 1 == steps ? orthogonal::kLast : step + 2 == steps ? orthogonal::kBefore : 0.0f; }

// two blocks on a compute unit where its LDS has room for them
inline auto whole(uint32_t shorter, bool half) {
    using namespace orthogonal;
    switch (shorter) {
        case 32: return whole_kernel<32, kWholeHalf>;
        case 64: return half ? whole_kernel<64, kWholeHalf> : whole_kernel<64, kWholeBytes>;
        case 96: return half ? whole_kernel<96, kWholeHalf> : whole_kernel<96, kWholeBytes>;
        default: return whole_kernel<128, kWholeBytes>;      // A alone has 64 KB, X as much
    }
}

int orthogonalized(const Stack &s, const Ends &e, int steps, char *scratch, hipStream_t stream) {
    using namespace orthogonal;
    if (fits(s)) {
        const uint32_t rows = (uint32_t)rounded(s.rows, 32), cols = (uint32_t)rounded(s.cols, 32), bytes = whole_bytes(std::min(rows, cols), std::max(rows, cols));
        const WholeArgs a{{e.g, e.m, nullptr, nullptr, nullptr, e.ld, e.apart, (uint32_t)s.rows, (uint32_t)s.cols, rows, cols, 0, e.beta, e.gdt == SS_BF16, e.ahead, false},
                          e.out, e.ldo, e.aparto, e.delta, (uint32_t)steps, e.step, e.odt == SS_BF16};
        const auto kernel = whole(std::min(rows, cols), bytes <= kWholeHalf);
        return launch(kernel, s.count, 0, stream, a, 64 * kWholeWaves);
    }
    const size_t blocks = norm_blocks(s);
    if (const Slices slices(s); slices.count) {
        const SlicePlace place(s, slices);
        auto half = [&](size_t at) { return reinterpret_cast<_Float16 *>(scratch + at); };
        float *parts = reinterpret_cast<float *>(scratch + place.parts);
        const BeginArgs begin{e.g, e.m, reinterpret_cast<double *>(scratch + place.sums), half(place.hi), half(place.lo), e.ld, e.apart, (uint32_t)s.rows, (uint32_t)s.cols, 0, 0,
                              (uint32_t)blocks, e.beta, e.gdt == SS_BF16, e.ahead, e.ld == s.cols || s.rows == 1};
        int rc = launch(norm_kernel, blocks, 0, stream, begin, 256, (int)s.count);
        const uint32_t size = (uint32_t)(slices.shorter * slices.shorter);
        const auto kernel = slices.shorter == 32 ? slice_kernel<32> : slices.shorter == 64 ? slice_kernel<64> : slices.shorter == 96 ? slice_kernel<96> : slice_kernel<128>;
        for (int k = -1; rc == SS_OK && k < steps; ++k) {
            const SliceArgs a{begin, k < 0 ? nullptr : half(place.a_hi), half(place.a_lo), parts, k + 1 == steps ? e.out : nullptr, e.ldo, e.aparto, e.delta, mu_of(k, steps), (uint32_t)slices.count,
                              e.step, e.odt == SS_BF16};
            rc = launch(kernel, slices.count, 0, stream, a, 64 * kWholeWaves, (int)s.count);
            if (rc == SS_OK && k + 1 < steps)
                rc = launch(sum_kernel, size / 64, 0, stream, SumArgs{parts, half(place.a_hi), half(place.a_lo), size, (uint32_t)slices.count}, 256, (int)s.count);
        }
        return rc;
    }
    const Place place(s);
    auto half = [&](size_t at) { return reinterpret_cast<_Float16 *>(scratch + at); };
    _Float16 *hi[2] = {half(place.hi[0]), half(place.hi[1])}, *lo[2] = {half(place.lo[0]), half(place.lo[1])}, *a[2] = {half(place.a[0]), half(place.a[1])}, *b[2] = {half(place.b[0]), half(place.b[1])};
    float *parts = reinterpret_cast<float *>(scratch + place.parts);
    const BeginArgs begin{e.g, e.m, reinterpret_cast<double *>(scratch + place.sums), hi[0], lo[0], e.ld, e.apart, (uint32_t)s.rows, (uint32_t)s.cols, (uint32_t)place.rows,
                          (uint32_t)place.cols, (uint32_t)blocks, e.beta, e.gdt == SS_BF16, e.ahead, e.ld == s.cols || s.rows == 1};
    int rc = launch(norm_kernel, blocks, 0, stream, begin, 256, (int)s.count);
    if (rc != SS_OK) return rc;
    rc = launch(scale_kernel, (place.rows * place.cols / 8 + 255) / 256, 0, stream, begin, 256, (int)s.count);
    if (rc != SS_OK) return rc;
    const bool tall = place.rows > place.cols;
    const uint32_t R = (uint32_t)place.rows, C = (uint32_t)place.cols, S = (uint32_t)place.shorter;
    const uint64_t whole = (uint64_t)R * C, square = (uint64_t)S * S;
    const int precise = twofold_steps(place.shorter, e.odt == SS_F32);
    for (int k = 0; k < steps; ++k) {
        const bool last = k + 1 == steps, twofold = k + precise >= steps;
        const float mu = mu_of(k, steps);
        const int at = k & 1, next = ~k & 1;
        const Plans &plans = twofold ? place.twofold : place.once;
        const Operand x{hi[at], C, R, R, whole, lo[at] - hi[at], 0}, down{hi[at], C, C, R, whole, lo[at] - hi[at], 0}, as{a[0], S, S, S, square, a[1] - a[0], 0}, bs{b[0], S, S, S, square, b[1] - b[0], 0};
        _Float16 *const a_lo = twofold ? a[1] : nullptr, *const b_lo = twofold ? b[1] : nullptr;
        const SquareEnd::Args square_end{a[0], a_lo, square};
        if (tall) rc = product::run<product::F16, true, true, SquareEnd>(plans.square, {down, down, s.count, S, S, R / product::kStep, parts, twofold}, square_end, stream);
        else rc = product::run<product::F16, false, false, SquareEnd>(plans.square, {x, x, s.count, S, S, C / product::kStep, parts, twofold}, square_end, stream);
        if (rc != SS_OK) return rc;
        rc = product::run<product::F16, false, false, PolynomialEnd>(plans.polynomial, {as, as, s.count, S, S, S / product::kStep, parts, twofold}, {a[0], a_lo, b[0], b_lo, square, mu}, stream);
        if (rc != SS_OK) return rc;
        const UpdateEnd::Args end{hi[at], lo[at], hi[next], lo[next], last ? e.out : nullptr, whole, e.ldo, e.aparto, (uint32_t)s.rows, (uint32_t)s.cols, kA - mu, e.delta, e.step, e.odt == SS_BF16};
        if (tall) rc = product::run<product::F16, false, false, UpdateEnd>(plans.update, {x, bs, s.count, R, C, S / product::kStep, parts, twofold}, end, stream);
        else rc = product::run<product::F16, false, true, UpdateEnd>(plans.update, {bs, down, s.count, R, C, S / product::kStep, parts, twofold}, end, stream);
        if (rc != SS_OK) return rc;
    }
    return SS_OK;
}

}  // namespace

extern "C" {

size_t ss_orthogonalize_scratch_bytes(size_t count, size_t rows, size_t cols) {
    const Stack s{count, rows, cols};
    return s.empty() || s.bad() ? 0 : scratch_of(s);
}

int ss_orthogonalize(const void *g, ss_dtype gdt, size_t count, size_t rows, size_t cols, size_t ld, size_t apart, int steps, void *out, ss_dtype odt, size_t ldo,
                     size_t aparto, void *scratch, size_t scratch_bytes, void *hip_stream) {
    if ((gdt != SS_F32 && gdt != SS_BF16) || (odt != SS_F32 && odt != SS_BF16)) return SS_ERR_DTYPE;
    const Stack s{count, rows, cols};
    if (s.bad() || steps < 1 || steps > SS_ORTHOGONAL_MAX_STEPS) return SS_ERR_ARG;
    if (s.empty()) return SS_OK;
    if (s.bad(ld, apart) || s.bad(ldo, aparto)) return SS_ERR_ARG;
    if (!g || !out || !scratch) return SS_ERR_NULL;
    if (!element_aligned(g, gdt) || !element_aligned(out, odt) || !aligned16(scratch)) return SS_ERR_ALIGN;
    Span spans[3] = {s.of(g, ld, apart, gdt, false), s.of(out, ldo, aparto, odt, true), span(scratch, scratch_bytes, true)};
    if (written_spans_overlap(spans, 3) || scratch_bytes < scratch_of(s)) return SS_ERR_ARG;
    return orthogonalized(s, {g, gdt, ld, apart, nullptr, 0, false, out, odt, ldo, aparto, 0, false}, steps, static_cast<char *>(scratch), static_cast<hipStream_t>(hip_stream));
}

int ss_orthogonal_step(const void *g, ss_dtype gdt, size_t count, size_t rows, size_t cols, size_t ld, size_t apart, float *m, float beta, int ahead, int steps, float delta,
                       float *x, void *scratch, size_t scratch_bytes, void *hip_stream) {
    if (gdt != SS_F32 && gdt != SS_BF16) return SS_ERR_DTYPE;
    const Stack s{count, rows, cols};
    if (s.bad() || steps < 1 || steps > SS_ORTHOGONAL_MAX_STEPS || !std::isfinite(beta) || !std::isfinite(delta) || (ahead != 0 && ahead != 1)) return SS_ERR_ARG;
    if (s.empty()) return SS_OK;
    if (s.bad(ld, apart)) return SS_ERR_ARG;
    if (!g || !m || !x || !scratch) return SS_ERR_NULL;
    if (!element_aligned(g, gdt) || !element_aligned(m, SS_F32) || !element_aligned(x, SS_F32) || !aligned16(scratch)) return SS_ERR_ALIGN;
    Span spans[4] = {s.of(g, ld, apart, gdt, false), s.of(m, cols, rows * cols, SS_F32, true), s.of(x, cols, rows * cols, SS_F32, true), span(scratch, scratch_bytes, true)};
    if (written_spans_overlap(spans, 4) || scratch_bytes < scratch_of(s)) return SS_ERR_ARG;
    return orthogonalized(s, {g, gdt, ld, apart, m, beta, ahead == 1, x, SS_F32, cols, rows * cols, delta, true}, steps, static_cast<char *>(scratch),
                          static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
