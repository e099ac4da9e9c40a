// C ABI of the loss over a vocabulary and its gradient (see include/signsgd.h): validation, pieces and launches.
#include <algorithm>

#include "api_common.hpp"
#include "loss_kernels.hpp"
#include "product_launch.hpp"

namespace {

using namespace host;
using product::Layout;
using product::Operand;
using product::Plan;
using product::Product;
using product::rounded;
using product::tiles_of;

inline bool element_aligned(const void *p, ss_dtype dt) { return reinterpret_cast<uintptr_t>(p) % grad_bytes(dt) == 0; }

inline Span matrix(const void *p, size_t rows, size_t cols, size_t ld, ss_dtype dt, bool written) {
    return span(p, rows && cols ? ((rows - 1) * ld + cols) * grad_bytes(dt) : 0, written);
}

inline bool bad_sizes(size_t T, size_t V, size_t K) {
    return T > SS_LOSS_MAX_ROWS || V > SS_LOSS_MAX_VOCAB || K == 0 || K > SS_LOSS_MAX_WIDTH || V == 0 || rounded(T, 64) * rounded(K, 64) > SS_LOSS_MAX_ELEMENTS;
}
// rows that are read, in place by offsets of 32 bits; and rows that are written, 2^40 elements of them, which no card holds
inline bool bad_ld(size_t ld, size_t cols) { return ld < cols || ld > SS_LOSS_MAX_STRIDE; }
inline bool bad_ld_out(size_t ld, size_t rows, size_t cols) { return ld < cols || (rows > 1 && ld > ((size_t)1 << 40) / (rows - 1)); }

// Whether the products load the caller's matrix as it lies.  Rows at multiples of 16 bytes are; a load of 16 bytes also goes to multiples of 4, but takes longer, which many rows of h
// repeat and a copy does not.  us, w as it lies / copied: a training pass of 2 rows against 19840 x 2258 134 / 171, of 1284 against 3350 x 1118 120 / 115.
inline bool loadable(const void *p, size_t ld, size_t T) {
    if (ld % 8 == 0 && aligned16(p)) return true;
    return T < 1024 && ld % 2 == 0 && reinterpret_cast<uintptr_t>(p) % 4 == 0;
}
inline bool whole(size_t K) { return K % product::kStep == 0; }

// a caller's rows as an operand
inline Operand rows_of(const void *p, size_t rows, size_t cols, size_t ld, size_t m, size_t depth) {
    return {p, (uint32_t)ld, (uint32_t)m, (uint32_t)depth, 0, 0, rounded(((rows - 1) * ld + cols) * 2, 4)};
}

// a product with the weights along their columns
template <template <bool> class End>
int along_weights(const Plan &plan, Product p, size_t K, bool copy, const typename End<false>::Args &end, hipStream_t stream) {
    p.tail = copy || whole(K) ? product::kStep : K % product::kStep;
    if (p.tail == product::kStep) return product::run<product::Bf16, false, false, End<false>>(plan, p, end, stream);
    static_assert(sizeof(typename End<true>::Args) == sizeof end, "the same fields");
    return product::run<product::Bf16, false, false, End<true>>(plan, p, __builtin_bit_cast(typename End<true>::Args, end), stream);
}

// What is computed at a time is a piece of the vocabulary.  Forward 2^36 entries of z, of which none is kept, or as many copied weights as there is room for.  Backward there is room for half of the
// logits in 16 bits, but for kLeastRoom entries at least and kMostRoom at most, which D shares with the copied weights; those have half of it at most.  Fewer entries cost more launches that do not
// fill the card, and dh's fp32 sum is read and written for each piece.  us of the gradients with room for 2^26 / 2^27 / 2^28 entries: 4096 rows against 32000 x 2048 1,449 / 1,401 / 1,402, 2048 against
// 50000 x 1024 792 / 734 / 735, 8192 against 32000 x 1024 1,704 / 1,572 / 1,532, 8192 against 128000 x 4096 20,350 / 20,241 / 19,983, with copied weights 23,480 / 21,650 / 20,930.
constexpr size_t kForwardEntries = (size_t)1 << 36, kLeastRoom = (size_t)1 << 27, kMostRoom = (size_t)1 << 28, kEdge = 256;

struct Sizes {
    size_t T, V, K, T64, K64, room;
    Sizes(size_t t, size_t v, size_t k) : T(t), V(v), K(k), T64(rounded(t, 64)), K64(rounded(k, 64)), room(std::min(std::max(T64 * V / 2, kLeastRoom), kMostRoom)) {}
    // tokens of a piece, where each takes `each` entries: all alike but for the last, which is hardly shorter.  us of the gradients so / as many as there is room for, and the rest: 4096 rows
    // against 32000 x 2048 with copied weights 1,488 / 1,580, 8192 against 128000 x 512 3,760 / 4,010, but 8192 against 128000 x 4096 19,980 / 19,830.
    size_t piece(size_t entries, size_t each) const {
        const size_t most = std::max(entries / each / kEdge * kEdge, 4 * kEdge), pieces = (V + most - 1) / most;
        return std::min(rounded((V + pieces - 1) / pieces, kEdge), V);
    }
    size_t forward(bool copy) const { return std::min(piece(kForwardEntries, T64), copy ? piece(room, 2 * K64) : V); }
    size_t backward(bool copy) const { return piece(room, copy ? std::max(T64 + K64, 2 * K64) : T64); }
    size_t last(size_t piece) const { return V - (V - 1) / piece * piece; }
};

struct ForwardPlace {
    size_t parts, picked, h, w, bytes;
    ForwardPlace(const Sizes &s, bool copy) {
        const size_t piece = s.forward(copy), last = s.last(piece);
        auto parts_of = [&](size_t n) { return 2 * tiles_of(n, product::plan_of(s.T, n, s.K64, 1, false, false, false).tile); };
        Layout l;
        parts = l.take(((s.V - last) / piece * parts_of(piece) + parts_of(last)) * s.T * sizeof(loss::Part));
        picked = l.take(s.T * sizeof(float));
        h = l.take(s.T64 * s.K64 * 2);
        w = l.take(copy ? piece * s.K64 * 2 : 0);
        bytes = l.bytes;
    }
};

struct BackwardPlace {
    size_t factor, scale, h, d, w, sum, parts, bytes;
    BackwardPlace(const Sizes &s, bool copy) {
        const size_t piece = s.backward(copy);
        Layout l;
        factor = l.take(s.T64 * sizeof(float));
        scale = l.take(sizeof(float));
        h = l.take(s.T64 * s.K64 * 2);
        d = l.take(s.T64 * rounded(piece, 64) * 2);
        w = l.take(copy ? piece * s.K64 * 2 : 0);
        sum = l.take(piece < s.V ? s.T * s.K * sizeof(float) : 0);
        size_t of_parts = 0;
        for (const size_t n : {piece, s.last(piece)}) {
            of_parts = std::max(of_parts, parts_bytes(product::plan_of(s.T, s.K, rounded(n, 64), 1, true), 1, s.T, s.K));
            of_parts = std::max(of_parts, parts_bytes(product::plan_of(n, s.K, s.T64, 1, true), 1, n, s.K));
        }
        parts = l.take(of_parts);
        bytes = l.bytes;
    }
};

loss::Copy copy_of(const void *from, size_t ld_from, void *to, size_t rows, size_t cols, size_t ld, size_t lines, const int64_t *target) {
    return {static_cast<const uint16_t *>(from), static_cast<uint16_t *>(to), target, ld_from, (uint32_t)rows, (uint32_t)cols, (uint32_t)ld, (uint32_t)lines,
            (uint32_t)((lines * (ld / 8) + loss::kPrepareThreads - 1) / loss::kPrepareThreads)};
}

int prepare(const loss::PrepareArgs &a, hipStream_t stream) {
    const size_t blocks = (a.factors.factor ? 1 : 0) + (size_t)a.h.blocks + a.w.blocks;
    return blocks ? launch(loss::prepare_kernel, blocks, 0, stream, a, loss::kPrepareThreads) : SS_OK;
}

int check(const void *h, ss_dtype dt, size_t T, size_t ldh, const void *w, size_t V, size_t K, size_t ldw, const int64_t *target) {
    if (dt != SS_BF16) return SS_ERR_DTYPE;
    if (bad_sizes(T, V, K) || bad_ld(ldh, K) || bad_ld(ldw, K)) return SS_ERR_ARG;
    if (T == 0) return SS_OK;
    if (!h || !w || !target) return SS_ERR_NULL;
    if (!element_aligned(h, dt) || !element_aligned(w, dt) || reinterpret_cast<uintptr_t>(target) % 8) return SS_ERR_ALIGN;
    return SS_OK;
}

}  // namespace

extern "C" {

size_t ss_cross_entropy_scratch_bytes(size_t T, size_t V, size_t K) {
    if (bad_sizes(T, V, K) || T == 0) return 0;
    const Sizes s(T, V, K);
    size_t bytes = 0;
    for (const bool copy : {false, true}) bytes = std::max({bytes, ForwardPlace(s, copy).bytes, BackwardPlace(s, copy).bytes});
    return bytes;
}

int ss_cross_entropy(const void *h, ss_dtype dt, size_t T, size_t ldh, const void *w, size_t V, size_t K, size_t ldw, const int64_t *target,
                     float *loss, float *lse, void *scratch, size_t scratch_bytes, void *hip_stream) {
    int rc = check(h, dt, T, ldh, w, V, K, ldw, target);
    if (rc != SS_OK || T == 0) return rc;
    if (!loss || !lse || !scratch) return SS_ERR_NULL;
    if (!element_aligned(loss, SS_F32) || !element_aligned(lse, SS_F32) || !aligned16(scratch)) return SS_ERR_ALIGN;
    Span spans[6] = {matrix(h, T, K, ldh, dt, false), matrix(w, V, K, ldw, dt, false), span(target, T * 8, false), span(loss, T * 4, true), span(lse, T * 4, true),
                     span(scratch, scratch_bytes, true)};
    if (written_spans_overlap(spans, 6)) return SS_ERR_ARG;
    const Sizes s(T, V, K);
    const bool copy = !loadable(w, ldw, T);
    const ForwardPlace place(s, copy);
    if (scratch_bytes < ss_cross_entropy_scratch_bytes(T, V, K)) return SS_ERR_ARG;
    char *base = static_cast<char *>(scratch);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    loss::PrepareArgs before = {};
    if (!loadable(h, ldh, T) || !whole(K)) {
        before.h = copy_of(h, ldh, base + place.h, T, K, s.K64, T, nullptr);
        h = base + place.h, ldh = s.K64;
    }
    const size_t piece = s.forward(copy);
    loss::Part *parts = reinterpret_cast<loss::Part *>(base + place.parts);
    float *picked = reinterpret_cast<float *>(base + place.picked);
    size_t count = 0;
    for (size_t v = 0; v < V; v += piece) {
        const size_t n = std::min(piece, V - v);
        const void *from = static_cast<const char *>(w) + v * ldw * 2;
        if (copy) before.w = copy_of(from, ldw, base + place.w, n, K, s.K64, n, nullptr), from = base + place.w;
        rc = prepare(before, stream);
        if (rc != SS_OK) return rc;
        before = {};
        const Plan plan = product::plan_of(T, n, s.K64, 1, false, false, false);
        const Operand ws = copy ? rows_of(from, n, s.K64, s.K64, n, 0) : rows_of(from, n, K, ldw, n, 0);
        rc = along_weights<loss::StatsEnd>(plan, {rows_of(h, T, s.K64, ldh, T, 0), ws, 1, T, n, s.K64 / product::kStep, nullptr}, K, copy,
                                           {parts, picked, target, (int64_t)v, (uint32_t)count}, stream);
        if (rc != SS_OK) return rc;
        count += 2 * tiles_of(n, plan.tile);
    }
    uint32_t rows = 1;
    while (rows < 16 && rows < T) rows *= 2;
    const loss::JoinArgs join{parts, picked, target, loss, lse, (uint32_t)T, (uint32_t)count, rows, (int64_t)V};
    return launch(loss::join_stats_kernel, (T + rows - 1) / rows, 0, stream, join, 256);
}

int ss_cross_entropy_grad(const void *h, ss_dtype dt, size_t T, size_t ldh, const void *w, size_t V, size_t K, size_t ldw, const int64_t *target,
                          const float *lse, const float *dloss, void *dh, ss_dtype dhdt, size_t lddh, void *dw, ss_dtype dwdt, size_t lddw, void *scratch,
                          size_t scratch_bytes, void *hip_stream) {
    int rc = check(h, dt, T, ldh, w, V, K, ldw, target);
    if (rc != SS_OK) return rc;
    if ((dhdt != SS_F32 && dhdt != SS_BF16) || (dwdt != SS_F32 && dwdt != SS_BF16)) return SS_ERR_DTYPE;
    if ((dh && bad_ld_out(lddh, T, K)) || (dw && bad_ld_out(lddw, V, K))) return SS_ERR_ARG;
    if (T == 0 && !dw) return SS_OK;
    if (T && (!lse || !scratch || (!dh && !dw))) return SS_ERR_NULL;
    if (!element_aligned(lse, SS_F32) || !element_aligned(dloss, SS_F32) || !element_aligned(dh, dhdt) || !element_aligned(dw, dwdt) || !aligned16(scratch)) return SS_ERR_ALIGN;
    Span spans[8] = {matrix(h, T, K, ldh, dt, false), matrix(w, V, K, ldw, dt, false), span(target, T * 8, false), span(lse, T * 4, false), span(dloss, T * 4, false),
                     matrix(dh, T, K, lddh, dhdt, true), matrix(dw, V, K, lddw, dwdt, true), span(scratch, scratch_bytes, true)};
    if (written_spans_overlap(spans, 8)) return SS_ERR_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (T == 0) {
        const loss::ZeroArgs a{dw, lddw, (uint64_t)V * K, (uint32_t)K, dwdt == SS_BF16};
        return launch(loss::zero_kernel, std::min((a.size + 255) / 256, (uint64_t)1 << 16), 0, stream, a, 256);
    }
    const Sizes s(T, V, K);
    const bool copy = !loadable(w, ldw, T);
    const BackwardPlace place(s, copy);
    if (scratch_bytes < ss_cross_entropy_scratch_bytes(T, V, K)) return SS_ERR_ARG;
    char *base = static_cast<char *>(scratch);
    float *factor = reinterpret_cast<float *>(base + place.factor), *scale = reinterpret_cast<float *>(base + place.scale);
    float *sum = reinterpret_cast<float *>(base + place.sum), *parts = reinterpret_cast<float *>(base + place.parts);
    __bf16 *d = reinterpret_cast<__bf16 *>(base + place.d);
    loss::PrepareArgs before = {{dloss, target, factor, scale, (int64_t)V, (uint32_t)T, (uint32_t)s.T64}, copy_of(h, ldh, base + place.h, T, K, s.K64, s.T64, target), {}};
    const size_t piece = s.backward(copy);
    const uint32_t K64 = (uint32_t)s.K64, T64 = (uint32_t)s.T64;
    for (size_t v = 0; v < V; v += piece) {
        const size_t n = std::min(piece, V - v), n64 = rounded(n, 64);
        const void *from = static_cast<const char *>(w) + v * ldw * 2;
        if (copy) before.w = copy_of(from, ldw, base + place.w, n, K, s.K64, n, nullptr), from = base + place.w;
        rc = prepare(before, stream);
        if (rc != SS_OK) return rc;
        before = {};
        const Operand hs{base + place.h, K64, T64, T64, 0, 0, 0}, ds{d, (uint32_t)n64, T64, 0, 0, 0, 0}, ws = copy ? rows_of(from, n, s.K64, s.K64, n, 0) : rows_of(from, n, K, ldw, n, 0);
        rc = along_weights<loss::SoftmaxEnd>(product::plan_of(T64, n64, K64, 1, false), {hs, ws, 1, T64, n64, K64 / product::kStep, nullptr}, K, copy,
                                             {lse, factor, target, (int64_t)v, d, (uint32_t)n64, (uint32_t)T, (uint32_t)n}, stream);
        if (rc != SS_OK) return rc;
        if (dh) {
            // the weights lie down their tokens
            const Operand down = copy ? rows_of(from, n, s.K64, s.K64, K, n) : rows_of(from, n, K, ldw, K, n);
            rc = product::run<product::Bf16, false, true, loss::GradientEnd>(product::plan_of(T, K, n64, 1, true), {ds, down, 1, T, K, n64 / product::kStep, parts},
                                                                             {scale, sum, dh, lddh, v == 0, v + piece >= V, dhdt == SS_BF16}, stream);
            if (rc != SS_OK) return rc;
        }
        if (dw) {
            const Operand d_down{d, (uint32_t)n64, (uint32_t)n64, T64, 0, 0, 0}, h_down{base + place.h, K64, (uint32_t)K, T64, 0, 0, 0};
            rc = product::run<product::Bf16, true, true, loss::GradientEnd>(
                product::plan_of(n, K, s.T64, 1, true), {d_down, h_down, 1, n, K, s.T64 / product::kStep, parts},
                {scale, nullptr, static_cast<char *>(dw) + v * lddw * grad_bytes(dwdt), lddw, true, true, dwdt == SS_BF16}, stream);
            if (rc != SS_OK) return rc;
        }
    }
    return SS_OK;
}

}  // extern "C"
