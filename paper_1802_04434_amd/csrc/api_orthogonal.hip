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
    // matrices in rows `ld` apart, `apart` elements from one to the next
    bool bad(size_t ld, size_t apart) const { return ld < cols || ld > ((size_t)1 << 40) || (count > 1 && apart < (rows - 1) * ld + cols) || apart > ((size_t)1 << 48); }
    Span of(const void *p, size_t ld, size_t apart, ss_dtype dt, bool written) const { return span(p, ((count - 1) * apart + (rows - 1) * ld + cols) * grad_bytes(dt), written); }
};

inline bool element_aligned(const void *p, ss_dtype dt) { return reinterpret_cast<uintptr_t>(p) % grad_bytes(dt) == 0; }

// blocks that add up a matrix's squares
inline size_t norm_blocks(const Stack &s) { return std::min(std::max((s.rows * s.cols + 2047) / 2048, (size_t)1), std::max((size_t)1024 / s.count, (size_t)1)); }

struct Place {
    size_t rows, cols, shorter, longer;       // whole steps
    Plan square, polynomial, update;
    size_t sums, hi[2], lo, a, b, parts, bytes;

    Place(const Stack &s) {
        rows = rounded(s.rows, 64), cols = rounded(s.cols, 64);
        shorter = std::min(rows, cols), longer = std::max(rows, cols);
        square = product::plan_of(shorter, shorter, longer, s.count, true);
        polynomial = product::plan_of(shorter, shorter, shorter, s.count, true);
        update = product::plan_of(rows, cols, shorter, s.count, true);
        Layout l;
        sums = l.take(s.count * norm_blocks(s) * sizeof(double));
        for (size_t &h : hi) h = l.take(s.count * rows * cols * 2);
        lo = l.take(s.count * rows * cols * 2);
        a = l.take(s.count * shorter * shorter * 2);
        b = l.take(s.count * shorter * shorter * 2);
        parts = l.take(std::max({parts_bytes(square, s.count, shorter, shorter), parts_bytes(polynomial, s.count, shorter, shorter), parts_bytes(update, s.count, rows, cols)}));
        bytes = l.bytes;
    }
};

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

int orthogonalized(const Stack &s, const Ends &e, int steps, char *scratch, hipStream_t stream) {
    using namespace orthogonal;
    const Place place(s);
    const size_t blocks = norm_blocks(s);
    _Float16 *hi[2] = {reinterpret_cast<_Float16 *>(scratch + place.hi[0]), reinterpret_cast<_Float16 *>(scratch + place.hi[1])};
    _Float16 *lo = reinterpret_cast<_Float16 *>(scratch + place.lo), *a = reinterpret_cast<_Float16 *>(scratch + place.a), *b = reinterpret_cast<_Float16 *>(scratch + place.b);
    float *parts = reinterpret_cast<float *>(scratch + place.parts);
    const BeginArgs begin{e.g, e.m, reinterpret_cast<double *>(scratch + place.sums), hi[0], lo, e.ld, e.apart, (uint32_t)s.rows, (uint32_t)s.cols, (uint32_t)place.rows,
                          (uint32_t)place.cols, (uint32_t)blocks, e.beta, e.gdt == SS_BF16, e.ahead, e.ld == s.cols || s.rows == 1};
    int rc = launch(norm_kernel, blocks, 0, stream, begin, 256, (int)s.count);
    if (rc != SS_OK) return rc;
    rc = launch(scale_kernel, (place.rows * place.cols / 8 + 255) / 256, 0, stream, begin, 256, (int)s.count);
    if (rc != SS_OK) return rc;
    const bool tall = place.rows > place.cols;
    const uint32_t R = (uint32_t)place.rows, C = (uint32_t)place.cols, S = (uint32_t)place.shorter;
    const uint64_t whole = (uint64_t)R * C, square = (uint64_t)S * S;
    for (int k = 0; k < steps; ++k) {
        const bool last = k + 1 == steps;
        const float mu = last ? kLast : k + 2 == steps ? kBefore : 0.0f;
        const Operand x{hi[k & 1], C, R, R, whole}, as{a, S, S, S, square}, bs{b, S, S, S, square};
        if (tall) {
            const Operand down{hi[k & 1], C, C, R, whole};
            rc = product::run<product::F16, true, true, SquareEnd>(place.square, {down, down, s.count, S, S, R / product::kStep, parts}, {a, square}, stream);
        } else {
            rc = product::run<product::F16, false, false, SquareEnd>(place.square, {x, x, s.count, S, S, C / product::kStep, parts}, {a, square}, stream);
        }
        if (rc != SS_OK) return rc;
        rc = product::run<product::F16, false, false, PolynomialEnd>(place.polynomial, {as, as, s.count, S, S, S / product::kStep, parts}, {a, b, square, mu}, stream);
        if (rc != SS_OK) return rc;
        const UpdateEnd::Args end{hi[k & 1], lo, hi[~k & 1], last ? e.out : nullptr, whole, e.ldo, e.aparto, (uint32_t)s.rows, (uint32_t)s.cols, kA - mu, e.delta, e.step, e.odt == SS_BF16};
        if (tall) rc = product::run<product::F16, false, false, UpdateEnd>(place.update, {x, bs, s.count, R, C, S / product::kStep, parts}, end, stream);
        else {
            const Operand down{hi[k & 1], C, C, R, whole};
            rc = product::run<product::F16, false, true, UpdateEnd>(place.update, {bs, down, s.count, R, C, S / product::kStep, parts}, end, stream);
        }
        if (rc != SS_OK) return rc;
    }
    return SS_OK;
}

}  // namespace

extern "C" {

size_t ss_orthogonalize_scratch_bytes(size_t count, size_t rows, size_t cols) {
    const Stack s{count, rows, cols};
    return s.empty() || s.bad() ? 0 : Place(s).bytes;
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
    if (written_spans_overlap(spans, 3) || scratch_bytes < Place(s).bytes) return SS_ERR_ARG;
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
    if (written_spans_overlap(spans, 4) || scratch_bytes < Place(s).bytes) return SS_ERR_ARG;
    return orthogonalized(s, {g, gdt, ld, apart, m, beta, ahead == 1, x, SS_F32, cols, rows * cols, delta, true}, steps, static_cast<char *>(scratch),
                          static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
