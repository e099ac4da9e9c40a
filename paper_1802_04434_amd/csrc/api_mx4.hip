// C ABI of the matrices in microscaled 4-bit floating point (see include/signsgd.h): validation, kernel selection and launch.
#include "api_common.hpp"
#include "mx4_kernels.hpp"

namespace {

using namespace host;

inline size_t groups_of(size_t cols) { return (cols + mx4::kGroupCols - 1) / mx4::kGroupCols; }

inline bool element_aligned(const void *p, ss_dtype dt) { return reinterpret_cast<uintptr_t>(p) % grad_bytes(dt) == 0; }

// from the first to behind the last element of a plain matrix
inline Span matrix(const void *p, size_t rows, size_t cols, size_t ld, ss_dtype dt, bool written) {
    return span(p, rows && cols ? ((rows - 1) * ld + cols) * grad_bytes(dt) : 0, written);
}

inline bool bad_matrix(size_t rows, size_t cols, size_t ld) {
    return rows > SS_MX4_MAX_DIM || cols > SS_MX4_MAX_DIM || ld < cols || ld > ((size_t)1 << 40) || rows * cols > SS_MX4_MAX_ELEMENTS;
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
    const size_t per = 64 * (xdt == SS_BF16 ? mx4::Bf16::kPer : mx4::F32::kPer);
    a.chunks = (uint32_t)((ss_mx4_padded(cols) + per - 1) / per);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    constexpr size_t kGrid = ((size_t)1 << 24) - 1;         // 2^32 threads
    if (data_t) {
        const size_t grid = a.chunks * groups_of(rows);
        if (grid > kGrid) return SS_ERR_ARG;
        if (xdt == SS_BF16)
            return data ? launch(mx4::quantize_both_kernel<mx4::Bf16, true>, grid, 0, stream, a, 256)
                        : launch(mx4::quantize_both_kernel<mx4::Bf16, false>, grid, 0, stream, a, 256);
        return data ? launch(mx4::quantize_both_kernel<mx4::F32, true>, grid, 0, stream, a, 256)
                    : launch(mx4::quantize_both_kernel<mx4::F32, false>, grid, 0, stream, a, 256);
    }
    constexpr int kRows = 4;
    const size_t grid = a.chunks * ((rows + 4 * kRows - 1) / (4 * kRows));
    if (grid > kGrid) return SS_ERR_ARG;
    return xdt == SS_BF16 ? launch(mx4::quantize_rows_kernel<mx4::Bf16, kRows>, grid, 0, stream, a, 256)
                          : launch(mx4::quantize_rows_kernel<mx4::F32, kRows>, grid, 0, stream, a, 256);
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
    if (grid > ((size_t)1 << 24) - 1) return SS_ERR_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return odt == SS_BF16 ? launch(mx4::dequantize_kernel<true, kRows>, grid, 0, stream, a, 256)
                          : launch(mx4::dequantize_kernel<false, kRows>, grid, 0, stream, a, 256);
}

size_t ss_mx4_matmul_scratch_bytes(size_t, size_t, size_t) { return 0; }

int ss_mx4_matmul(const uint8_t *a_data, const uint8_t *a_scales, const uint8_t *b_data, const uint8_t *b_scales, size_t M, size_t N,
                  size_t K, void *out, ss_dtype odt, size_t ld, void *scratch, size_t scratch_bytes, void *hip_stream) {
    if (odt != SS_F32 && odt != SS_BF16) return SS_ERR_DTYPE;
    if (bad_matrix(M, N, ld) || K > SS_MX4_MAX_DIM) return SS_ERR_ARG;
    if (M == 0 || N == 0) return SS_OK;
    if (!out || (K && (!a_data || !a_scales || !b_data || !b_scales))) return SS_ERR_NULL;
    if (!aligned16(a_data) || !aligned16(a_scales) || !aligned16(b_data) || !aligned16(b_scales) || !aligned16(scratch) ||
        !element_aligned(out, odt))
        return SS_ERR_ALIGN;
    Span spans[6] = {span(a_data, ss_mx4_data_bytes(M, K), false), span(a_scales, ss_mx4_scale_bytes(M, K), false),
                     span(b_data, ss_mx4_data_bytes(N, K), false), span(b_scales, ss_mx4_scale_bytes(N, K), false),
                     matrix(out, M, N, ld, odt, true), span(scratch, scratch_bytes, true)};
    if (written_spans_overlap(spans, 6)) return SS_ERR_ARG;
    mx4::MatmulArgs a{a_data, b_data, reinterpret_cast<const uint32_t *>(a_scales), reinterpret_cast<const uint32_t *>(b_scales), out, ld,
                      (uint32_t)M, (uint32_t)N, (uint32_t)groups_of(K), (uint32_t)((N + 31) / 32)};
    const size_t grid = (M + 31) / 32 * a.tiles_n;
    if (grid > ((size_t)1 << 26) - 1) return SS_ERR_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return odt == SS_BF16 ? launch(mx4::matmul_kernel<true>, grid, 0, stream, a, 64) : launch(mx4::matmul_kernel<false>, grid, 0, stream, a, 64);
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
    mx4::LinearArgs a{x, w_data, reinterpret_cast<const uint32_t *>(w_scales), out, ldx, ldo, (uint32_t)T, (uint32_t)N, (uint32_t)K,
                      (uint32_t)groups_of(K), 0};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    constexpr int kThreads = 64 * mx4::kLinearWaves;
    constexpr size_t kGrid = ((size_t)1 << 32) / kThreads - 1;
    for (size_t first = 0; first < N; first += kGrid * 16) {
        a.first = (uint32_t)first;
        const size_t grid = std::min((N - first + 15) / 16, kGrid);
        int rc;
        if (xdt == SS_BF16)
            rc = odt == SS_BF16 ? launch(mx4::linear_kernel<mx4::Bf16, true>, grid, 0, stream, a, kThreads)
                                : launch(mx4::linear_kernel<mx4::Bf16, false>, grid, 0, stream, a, kThreads);
        else
            rc = odt == SS_BF16 ? launch(mx4::linear_kernel<mx4::F32, true>, grid, 0, stream, a, kThreads)
                                : launch(mx4::linear_kernel<mx4::F32, false>, grid, 0, stream, a, kThreads);
        if (rc != SS_OK) return rc;
    }
    return SS_OK;
}

}  // extern "C"
