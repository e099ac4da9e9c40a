// C ABI of the matrices in microscaled 4-bit floating point (see include/signsgd.h): validation, kernel selection and launch.
#include <algorithm>
#include <cmath>

#include "api_common.hpp"
#include "mx4_kernels.hpp"

namespace {

using namespace host;

constexpr size_t kMaxThreads = 0xFFFFFFFFull;      // of a launch

inline size_t groups_of(size_t cols) { return (cols + mx4::kGroupCols - 1) / mx4::kGroupCols; }

inline bool element_aligned(const void *p, ss_dtype dt) { return reinterpret_cast<uintptr_t>(p) % grad_bytes(dt) == 0; }

// from the first to behind the last element of a plain matrix
inline Span matrix(const void *p, size_t rows, size_t cols, size_t ld, ss_dtype dt, bool written) {
    return span(p, rows && cols ? ((rows - 1) * ld + cols) * grad_bytes(dt) : 0, written);
}

inline bool bad_matrix(size_t rows, size_t cols, size_t ld) {
    return rows > SS_MX4_MAX_DIM || cols > SS_MX4_MAX_DIM || ld < cols || ld > ((size_t)1 << 40) || rows * cols > SS_MX4_MAX_ELEMENTS;
}

// From here on a matrix is read with nt: it is not in the memory-side cache.  us along the rows, the columns and both, without / with, three matrices in turn: 8192 x 8192 fp32 (268 MB) 51.8 /
// 48.0, 59.7 / 54.8, 65.4 / 60.5; in bf16 (134 MB), where it makes little difference, 28.2 / 28.8, 34.5 / 35.5, 37.8 / 37.8; 4096 x 8192 bf16 (67 MB), found there, 13.2 / 14.8, 14.9 / 17.3, 17.7 / 21.5.
constexpr size_t kQuantizeOnce = (size_t)1 << 27;

template <typename T>
auto both_kernel(bool rows, bool once) {
    if (rows) return once ? mx4::quantize_both_kernel<T, true, true> : mx4::quantize_both_kernel<T, true, false>;
    return once ? mx4::quantize_both_kernel<T, false, true> : mx4::quantize_both_kernel<T, false, false>;
}

// Weights of 64 MB and more are read with nt, which leaves the caches to others: 21.4 instead of 23.1 us at 28672 by 8192.  Smaller ones may still be there from the
// token before: 10.4 instead of 11.3 us at 16384 by 4096.
constexpr size_t kLinearBlocks = 256, kLinearOnce = (size_t)1 << 26;

// x in LDS: 4,096 columns at a time with three steps of w on the way for each wave, or 10,240 with two, as many as there is room for
template <typename T, bool OUT_BF16>
auto linear_kernel(size_t steps, bool once) {
    if (steps <= 8) return once ? mx4::linear_kernel<T, OUT_BF16, true, 8, 3> : mx4::linear_kernel<T, OUT_BF16, false, 8, 3>;
    return once ? mx4::linear_kernel<T, OUT_BF16, true, 20, 2> : mx4::linear_kernel<T, OUT_BF16, false, 20, 2>;
}

template <typename T>
auto linear_kernel(ss_dtype odt, size_t steps, bool once) { return odt == SS_BF16 ? linear_kernel<T, true>(steps, once) : linear_kernel<T, false>(steps, once); }

inline int few_rows(decltype(linear_kernel<mx4::F32>) *kernels, ss_dtype odt, mx4::LinearArgs a, hipStream_t stream) {
    const size_t tiles = ((size_t)a.N + 15) / 16, steps = ((size_t)a.groups + mx4::kLinearGroups - 1) / mx4::kLinearGroups;
    // as many waves to the same rows as a block on each compute unit gives (one is all that LDS has room for).  us, 1 and 16 rows, 4096 to 5000 columns, in 157 blocks / 313: 4.6 and 7.5 /
    // 7.0 and 12.4
    while (2u << a.log_split <= mx4::kLinearWaves && (tiles << a.log_split) * 2 <= kLinearBlocks * mx4::kLinearWaves && (size_t)1 << a.log_split < steps) ++a.log_split;
    const auto kernel = kernels(odt, steps, (size_t)a.N * a.groups * mx4::kGroupBytes >= kLinearOnce);
    constexpr int kThreads = 64 * mx4::kLinearWaves;
    static_assert(SS_MX4_MAX_DIM / 16 / mx4::kLinearWaves * kThreads <= kMaxThreads, "one launch takes all rows");      // 16 a wave where there are many
    const size_t rows = 16 * (mx4::kLinearWaves >> a.log_split);
    return launch(kernel, ((size_t)a.N + rows - 1) / rows, 0, stream, a, kThreads);
}

// How a product, or a part of one, is cut: tiles of 64 times `tile` squared (0: a few rows or columns of the result, by the kernel for them), and the sum over the
// columns into `splits` parts
struct Plan {
    int tile;
    size_t splits;
    double us;
};

inline size_t tiles_of(size_t n, int tile) { return (n + 64 * (size_t)tile - 1) / (64 * (size_t)tile); }

// What a launch takes by its shape, from products of 64 x 4096 x 4096 to 8192 x 8192 x 16384: us a step of 256 columns with one block on a compute unit
// (large tiles: few on the card) and with as many as fit, and us a block besides, of which the second part is for writing the result.  Two launches cost 3 us more,
// and the partial sums their bytes, written, read and joined at 2.5 TB/s.
inline Plan plan_of(size_t M, size_t N, size_t K, bool may_split) {
    const size_t steps = (groups_of(K) + 1) / 2;
    constexpr struct {
        int tile;
        double fit, alone, full, starts, ends;
    } kShapes[] = {{4, 1, 1.15, 1.65, 3.0, 7.0}, {2, 2, 0.58, 1.06, 2.0, 3.5}, {1, 4, 0.40, 0.87, 1.5, 1.0}};
    Plan best{1, 1, 1e300};
    for (const auto &s : kShapes) {
        const size_t tiles = tiles_of(M, s.tile) * tiles_of(N, s.tile);
        // no more parts than fill the card once
        for (size_t splits = 1; splits == 1 || (may_split && splits * 2 <= steps && tiles * splits <= (size_t)(256 * s.fit)); splits *= 2) {
            const double blocks = (double)(tiles * splits), each = (double)((steps + splits - 1) / splits);
            auto round = [&](double load) {       // blocks a compute unit
                const double crowd = s.fit == 1 ? load : load > 1 ? (load - 1) / (s.fit - 1) : 0;
                return each * (s.alone + (s.full - s.alone) * crowd) + s.starts + s.ends * load / s.fit;
            };
            const double rounds = std::floor(blocks / (256 * s.fit)), rest = blocks / 256 - rounds * s.fit;
            double us = rounds * round(s.fit) + (rest > 0 ? round(rest) : 0);
            if (splits > 1) us += 3.0 + (double)(splits * M * N) * 4 / 2.5e6;
            if (us < best.us) best = Plan{s.tile, splits, us};
        }
    }
    // The few rows' kernel: w's bytes, and what it costs to bring each 10,240 columns of x; tiles have to read w too.  us, few rows / tiles: 1 x 4096 x 4096 4.0 / 8.2, 16 x 8192 x
    // 4096 6.2 / 9.6, 16 x 16384 x 16384 28.2 / 31.7, but 16 x 16 x 32768, of which tiles can split the sum, 12.0 / 7.9
    if (std::min(M, N) <= SS_MX4_LINEAR_MAX_ROWS) {
        const double bytes = (double)std::max(M, N) * groups_of(K) * 68, us = 2.0 + bytes / 6.5e6 + 2.6 * (double)((groups_of(K) - 1) / 80);
        if (us < std::max(best.us, 3.0 + bytes / 4.6e6)) best = Plan{0, 1, us};
    }
    return best;
}

// A result that the memory-side cache can hold stays there.  us, left to the L2 / sent on / with nt: 4096 x 4096 x 4096 in bf16 (33 MB) 37.2 / 35.7 / 36.0, in fp32 41.7 / 40.1 /
// 41.1, 4096 x 8192 x 2048 in bf16 (67 MB) 50.0 / 45.8 / 47.5, in fp32 68.0 / 69.5 / 65.1, 8192 x 12288 x 1024 in fp32 (403 MB) 158 / 134 / 111.
constexpr size_t kProductKeeps = (size_t)1 << 27;

// A part of the result with a plan of its own
struct Part {
    size_t m, n, M, N;
    Plan plan;
};

// A tile that hangs over the edge costs as much as a whole one: where the rows or columns beyond the last whole large tile are few, smaller ones take them.
inline int parts_of(Part (&parts)[3], size_t M, size_t N, size_t K, bool may_split) {
    parts[0] = Part{0, 0, M, N, plan_of(M, N, K, may_split)};
    double least = parts[0].plan.us;
    int count = 1;
    for (const size_t edge : {(size_t)256, (size_t)128}) {
        for (int which = 1; which < 4; ++which) {
            const size_t over_m = M % edge, over_n = N % edge;
            if ((which & 1 && (M < edge || over_m == 0 || over_m > edge / 2)) || (which & 2 && (N < edge || over_n == 0 || over_n > edge / 2))) continue;
            const size_t m = which & 1 ? M - over_m : M, n = which & 2 ? N - over_n : N;
            Part tried[3] = {{0, 0, m, n, plan_of(m, n, K, may_split)}};
            int c = 1;
            if (m < M) tried[c] = Part{m, 0, M - m, N, plan_of(M - m, N, K, may_split)}, ++c;
            if (n < N) tried[c] = Part{0, n, m, N - n, plan_of(m, N - n, K, may_split)}, ++c;
            double us = 1.5 * (c - 1);
            for (int k = 0; k < c; ++k) us += tried[k].plan.us;
            if (us < least) {
                least = us;
                count = c;
                std::copy(tried, tried + c, parts);
            }
        }
    }
    return count;
}

// bytes of partial sums; the parts are computed one after the other
inline size_t scratch_of(const Part *parts, int count) {
    size_t bytes = 0;
    for (int k = 0; k < count; ++k)
        if (parts[k].plan.splits > 1) bytes = std::max(bytes, parts[k].plan.splits * parts[k].M * parts[k].N * sizeof(float));
    return bytes;
}

}  // namespace

extern "C" {

size_t ss_mx4_padded(size_t cols) { return groups_of(cols) * mx4::kGroupCols; }
size_t ss_mx4_data_bytes(size_t rows, size_t cols) { return rows * groups_of(cols) * mx4::kGroupBytes; }
size_t ss_mx4_scale_bytes(size_t rows, size_t cols) { return rows * groups_of(cols) * 4; }

int ss_mx4_quantize(const void *x, ss_dtype xdt, size_t rows, size_t cols, size_t ld, uint8_t *data, uint8_t *scales,
                    uint8_t *data_t, uint8_t *scales_t, void *hip_stream) {
    if (xdt != SS_F32 && xdt != SS_BF16) return SS_ERR_DTYPE;
    if (bad_matrix(rows, cols, ld)) return SS_ERR_ARG;
    if (rows == 0 || cols == 0) return SS_OK;
    if (!x || (!data && !data_t) || !data != !scales || !data_t != !scales_t) return SS_ERR_NULL;
    if (!element_aligned(x, xdt) || !aligned16(data) || !aligned16(scales) || !aligned16(data_t) || !aligned16(scales_t)) return SS_ERR_ALIGN;
    Span spans[5] = {matrix(x, rows, cols, ld, xdt, false), span(data, ss_mx4_data_bytes(rows, cols), true),
                     span(scales, ss_mx4_scale_bytes(rows, cols), true), span(data_t, ss_mx4_data_bytes(cols, rows), true),
                     span(scales_t, ss_mx4_scale_bytes(cols, rows), true)};
    if (written_spans_overlap(spans, 5)) return SS_ERR_ARG;
    mx4::QuantizeArgs a{x, data, reinterpret_cast<uint32_t *>(scales), data_t, reinterpret_cast<uint32_t *>(scales_t), ld,
                        (uint32_t)rows, (uint32_t)cols, 0};
    // columns of a block
    const size_t per = xdt == SS_BF16 ? (data_t ? mx4::kAcross<mx4::Bf16> : 64) * mx4::Bf16::kPer : (data_t ? mx4::kAcross<mx4::F32> : 64) * mx4::F32::kPer;
    a.chunks = (uint32_t)((ss_mx4_padded(cols) + per - 1) / per);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const bool once = rows * cols * grad_bytes(xdt) >= kQuantizeOnce;
    if (data_t) {
        const int threads = xdt == SS_BF16 ? mx4::kBothThreads<mx4::Bf16> : mx4::kBothThreads<mx4::F32>;
        const size_t grid = a.chunks * groups_of(rows);
        if (grid > kMaxThreads / threads) return SS_ERR_ARG;
        const auto kernel = xdt == SS_BF16 ? both_kernel<mx4::Bf16>(data != nullptr, once) : both_kernel<mx4::F32>(data != nullptr, once);
        return launch(kernel, grid, 0, stream, a, threads);
    }
    constexpr size_t kRows = 4 * mx4::kQuantizeRows;       // of a block
    const size_t grid = a.chunks * ((rows + kRows - 1) / kRows);
    if (grid > kMaxThreads / 256) return SS_ERR_ARG;
    const auto kernel = xdt == SS_BF16 ? (once ? mx4::quantize_rows_kernel<mx4::Bf16, true> : mx4::quantize_rows_kernel<mx4::Bf16, false>)
                                       : (once ? mx4::quantize_rows_kernel<mx4::F32, true> : mx4::quantize_rows_kernel<mx4::F32, false>);
    return launch(kernel, grid, 0, stream, a, 256);
}

int ss_mx4_dequantize(const uint8_t *data, const uint8_t *scales, size_t rows, size_t cols, void *out, ss_dtype odt, size_t ld,
                      void *hip_stream) {
    if (odt != SS_F32 && odt != SS_BF16) return SS_ERR_DTYPE;
    if (bad_matrix(rows, cols, ld)) return SS_ERR_ARG;
    if (rows == 0 || cols == 0) return SS_OK;
    if (!data || !scales || !out) return SS_ERR_NULL;
    if (!aligned16(data) || !aligned16(scales) || !element_aligned(out, odt)) return SS_ERR_ALIGN;
    Span spans[3] = {span(data, ss_mx4_data_bytes(rows, cols), false), span(scales, ss_mx4_scale_bytes(rows, cols), false),
                     matrix(out, rows, cols, ld, odt, true)};
    if (written_spans_overlap(spans, 3)) return SS_ERR_ARG;
    constexpr int kRows = 4;
    mx4::DequantizeArgs a{data, scales, out, ld, (uint32_t)rows, (uint32_t)cols, (uint32_t)((cols + 511) / 512)};
    const size_t grid = a.chunks * ((rows + 4 * kRows - 1) / (4 * kRows));
    if (grid > kMaxThreads / 256) return SS_ERR_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return odt == SS_BF16 ? launch(mx4::dequantize_kernel<true, kRows>, grid, 0, stream, a, 256)
                          : launch(mx4::dequantize_kernel<false, kRows>, grid, 0, stream, a, 256);
}

size_t ss_mx4_matmul_scratch_bytes(size_t M, size_t N, size_t K) {
    if (M == 0 || N == 0 || bad_matrix(M, N, N) || K > SS_MX4_MAX_SUM) return 0;
    Part parts[3];
    return scratch_of(parts, parts_of(parts, M, N, K, true));
}

int ss_mx4_matmul(const uint8_t *a_data, const uint8_t *a_scales, const uint8_t *b_data, const uint8_t *b_scales, size_t M, size_t N,
                  size_t K, void *out, ss_dtype odt, size_t ld, void *scratch, size_t scratch_bytes, void *hip_stream) {
    if (odt != SS_F32 && odt != SS_BF16) return SS_ERR_DTYPE;
    if (bad_matrix(M, N, ld) || K > SS_MX4_MAX_SUM) return SS_ERR_ARG;
    if (M == 0 || N == 0) return SS_OK;
    if (!out || (K && (!a_data || !a_scales || !b_data || !b_scales))) return SS_ERR_NULL;
    if (!aligned16(a_data) || !aligned16(a_scales) || !aligned16(b_data) || !aligned16(b_scales) || !aligned16(scratch) ||
        !element_aligned(out, odt))
        return SS_ERR_ALIGN;
    Span spans[6] = {span(a_data, ss_mx4_data_bytes(M, K), false), span(a_scales, ss_mx4_scale_bytes(M, K), false),
                     span(b_data, ss_mx4_data_bytes(N, K), false), span(b_scales, ss_mx4_scale_bytes(N, K), false),
                     matrix(out, M, N, ld, odt, true), span(scratch, scratch_bytes, true)};
    if (written_spans_overlap(spans, 6)) return SS_ERR_ARG;
    Part parts[3];
    int count = parts_of(parts, M, N, K, scratch != nullptr);
    if (scratch && scratch_of(parts, count) > scratch_bytes) count = parts_of(parts, M, N, K, false);
    const size_t groups = groups_of(K);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    for (int k = 0; k < count; ++k) {
        const Part &part = parts[k];
        const int tile = part.plan.tile;
        const bool join = part.plan.splits > 1, bf16 = odt == SS_BF16 && !join;
        void *to = static_cast<char *>(out) + (part.m * ld + part.n) * grad_bytes(odt);
        if (tile == 0) {
            const bool wide = part.M <= part.N;       // a's rows are the few, or b's
            const uint8_t *data[2] = {a_data + part.m * groups * mx4::kGroupBytes, b_data + part.n * groups * mx4::kGroupBytes};
            const uint32_t *scales[2] = {reinterpret_cast<const uint32_t *>(a_scales) + part.m, reinterpret_cast<const uint32_t *>(b_scales) + part.n};
            const uint32_t rows[2] = {(uint32_t)M, (uint32_t)N};
            const int rc = few_rows(linear_kernel<mx4::Codes>, odt,
                                    {data[!wide], scales[!wide], data[wide], scales[wide], to, 0, wide ? ld : 1, wide ? 1 : ld, (uint32_t)std::min(part.M, part.N),
                                     (uint32_t)std::max(part.M, part.N), (uint32_t)K, (uint32_t)groups, rows[!wide], rows[wide], 0},
                                    stream);
            if (rc != SS_OK) return rc;
            continue;
        }
        mx4::TilesArgs a{a_data + part.m * groups * mx4::kGroupBytes, b_data + part.n * groups * mx4::kGroupBytes,
                         reinterpret_cast<const uint32_t *>(a_scales) + part.m, reinterpret_cast<const uint32_t *>(b_scales) + part.n,
                         join ? scratch : to, join ? part.N : ld, (uint32_t)part.M, (uint32_t)part.N, (uint32_t)M, (uint32_t)N, (uint32_t)groups,
                         (uint32_t)tiles_of(part.M, tile), (uint32_t)tiles_of(part.N, tile), (uint32_t)part.plan.splits,
                         join || M * N * grad_bytes(odt) < kProductKeeps};
        const auto kernel = tile == 4 ? (bf16 ? mx4::matmul_tiles_kernel<true, 4> : mx4::matmul_tiles_kernel<false, 4>)
                            : tile == 2 ? (bf16 ? mx4::matmul_tiles_kernel<true, 2> : mx4::matmul_tiles_kernel<false, 2>)
                                        : (bf16 ? mx4::matmul_tiles_kernel<true, 1> : mx4::matmul_tiles_kernel<false, 1>);
        int rc = launch(kernel, (size_t)a.tiles_m * a.tiles_n * a.splits, 0, stream, a, 256);
        if (rc != SS_OK) return rc;
        if (!join) continue;
        const mx4::JoinArgs j{static_cast<const float *>(scratch), to, ld, a.M, a.N, a.splits};
        const size_t blocks = (part.M * part.N + 1023) / 1024;
        rc = odt == SS_BF16 ? launch(mx4::join_kernel<true>, blocks, 0, stream, j, 256) : launch(mx4::join_kernel<false>, blocks, 0, stream, j, 256);
        if (rc != SS_OK) return rc;
    }
    return SS_OK;
}

int ss_mx4_linear(const void *x, ss_dtype xdt, size_t T, size_t ldx, const uint8_t *w_data, const uint8_t *w_scales, size_t N, size_t K,
                  void *out, ss_dtype odt, size_t ldo, void *hip_stream) {
    if ((xdt != SS_F32 && xdt != SS_BF16) || (odt != SS_F32 && odt != SS_BF16)) return SS_ERR_DTYPE;
    if (T > SS_MX4_LINEAR_MAX_ROWS || bad_matrix(T, K, ldx) || bad_matrix(T, N, ldo)) return SS_ERR_ARG;
    if (T == 0 || N == 0) return SS_OK;
    if (!out || (K && (!x || !w_data || !w_scales))) return SS_ERR_NULL;
    if (!element_aligned(x, xdt) || !aligned16(w_data) || !aligned16(w_scales) || !element_aligned(out, odt)) return SS_ERR_ALIGN;
    Span spans[4] = {matrix(x, T, K, ldx, xdt, false), span(w_data, ss_mx4_data_bytes(N, K), false),
                     span(w_scales, ss_mx4_scale_bytes(N, K), false), matrix(out, T, N, ldo, odt, true)};
    if (written_spans_overlap(spans, 4)) return SS_ERR_ARG;
    return few_rows(xdt == SS_BF16 ? linear_kernel<mx4::Bf16> : linear_kernel<mx4::F32>, odt,
                    {x, nullptr, w_data, reinterpret_cast<const uint32_t *>(w_scales), out, ldx, ldo, 1, (uint32_t)T, (uint32_t)N, (uint32_t)K, (uint32_t)groups_of(K), 0,
                     (uint32_t)N, 0},
                    static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
