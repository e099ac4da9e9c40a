// C ABI of the operators on lists of gradients (see include/signsgd.h): validation and launch.
#include <new>
#include <type_traits>

#include "api_common.hpp"
#include "grad_kernels.hpp"

namespace {

using namespace host;

static_assert(grads::kNormTensors == SS_GRAD_NORM_PER_LAUNCH && grads::kClipTensors == SS_GRAD_CLIP_PER_LAUNCH, "the header says how many");
static_assert(sizeof(grads::ClipArgs) <= 4096 && sizeof(grads::NormArgs) <= 4096, "argument block");

// elements of one tensor, and bytes of all: no card holds more, and units stay below 2^32
constexpr size_t kMaxLen = (size_t)1 << 40;
constexpr size_t kMaxBytes = (size_t)1 << 42;

// units of one launch of the clip: 2^32 - 1 threads at most
constexpr size_t kClipGrid = ((size_t)1 << 32) / grads::kClipThreads - 1;

inline size_t clip_unit(ss_dtype in, ss_dtype out) {
    if (out == SS_BF16) return in == SS_BF16 ? grads::kClipUnit<true, true> : grads::kClipUnit<false, true>;
    return in == SS_BF16 ? grads::kClipUnit<true, false> : grads::kClipUnit<false, false>;
}

int check_list(const void *const *g, const ss_dtype *gdt, const size_t *len, size_t n) {
    if (n == 0) return SS_OK;
    if (!g || !gdt || !len) return SS_ERR_NULL;
    size_t bytes = 0;
    for (size_t t = 0; t < n; ++t) {
        if (gdt[t] != SS_F32 && gdt[t] != SS_BF16) return SS_ERR_DTYPE;
        if (len[t] == 0) continue;
        if (!g[t]) return SS_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(g[t]) % grad_bytes(gdt[t])) return SS_ERR_ALIGN;
        if (len[t] > kMaxLen) return SS_ERR_ARG;
        bytes += len[t] * grad_bytes(gdt[t]);
        if (bytes > kMaxBytes) return SS_ERR_ARG;
    }
    return SS_OK;
}

inline uint64_t address(const void *p, ss_dtype dt) { return reinterpret_cast<uint64_t>(p) | (dt == SS_BF16 ? 1u : 0u); }

inline bool share(const Span &a, const Span &b) { return a.lo < b.hi && b.lo < a.hi && a.lo < a.hi && b.lo < b.hi; }

// Tensors that are written, in order of their addresses
struct Written {
    Span *s = nullptr;
    size_t n = 0;

    ~Written() { delete[] s; }
    // false: they overlap one another (or there is no memory to find out: *failed)
    bool take(void *const *out, const ss_dtype *odt, const size_t *len, size_t count, bool *failed) {
        s = new (std::nothrow) Span[count ? count : 1];
        *failed = !s;
        if (!s) return false;
        bool ascending = true;
        for (size_t t = 0; t < count; ++t) {
            if (len[t] == 0) continue;
            s[n] = span(out[t], len[t] * grad_bytes(odt[t]), true);
            if (n && s[n].lo < s[n - 1].hi) ascending = false;
            ++n;
        }
        if (ascending) return true;     // parts of one vector, as they come
        std::sort(s, s + n, [](const Span &a, const Span &b) { return a.lo < b.lo; });
        for (size_t k = 1; k < n; ++k)
            if (s[k].lo < s[k - 1].hi) return false;
        return true;
    }
    bool meets(const Span &b) const {
        if (n == 0 || b.lo >= s[n - 1].hi || b.hi <= s[0].lo) return false;
        const Span *k = std::upper_bound(s, s + n, b.lo, [](uintptr_t lo, const Span &x) { return lo < x.hi; });
        return k != s + n && share(*k, b);
    }
};

// Up to here the norm leaves the gradients in the memory-side cache, for the clip that reads them next.  us, norm and both, not kept / kept: 25.6 M fp32
// 20.6 and 57.9 / 21.4 and 53.4, 50 M bf16 in 150 tensors 23.9 and 64.6 / 24.1 and 59.7; 1.5 G bf16 438 / 488.
constexpr size_t kNormKeeps = (size_t)1 << 28;
// From here on 256 blocks with eight units in flight, below 512 with four: us, 256 / 512: 1.5 G bf16 438 / 448; 138 M mixed 67.2 / 64.1, 25.6 M fp32 in 161 tensors 23.2 / 22.5,
// 5 M in 900 36.6 / 29.9, 272,474 in 65 6.5 / 6.2.
constexpr size_t kNormLarge = (size_t)1 << 30;

}  // namespace

extern "C" {

size_t ss_grad_norm_workspace_bytes(void) { return sizeof(grads::NormScratch); }

int ss_grad_norm(const void *const *g, const ss_dtype *gdt, const size_t *len, size_t n, float *norm, void *workspace,
                 void *hip_stream) {
    if (!norm || !workspace) return SS_ERR_NULL;
    const int rc = check_list(g, gdt, len, n);
    if (rc != SS_OK) return rc;
    if (!aligned16(norm) || !aligned16(workspace)) return SS_ERR_ALIGN;
    const Span out = span(norm, sizeof(float), true), ws = span(workspace, sizeof(grads::NormScratch), true);
    if (share(out, ws)) return SS_ERR_ARG;
    for (size_t t = 0; t < n; ++t) {
        const Span s = span(g[t], len[t] * grad_bytes(gdt[t]), false);
        if (share(s, out) || share(s, ws)) return SS_ERR_ARG;
    }
    const auto take = [&](grads::NormArgs &a, size_t t) {      // the tensors of a launch that begins with t; where the next one does
        uint32_t units = 0;
        for (a.n = 0; t < n && a.n < (uint32_t)grads::kNormTensors; ++t) {
            if (len[t] == 0) continue;
            const uint64_t at = address(g[t], gdt[t]);
            const size_t bytes = (size_t)(at & 14u) + len[t] * grad_bytes(gdt[t]);
            a.at[a.n] = at;
            a.first[a.n] = units;
            a.rest[a.n] = (uint16_t)((bytes - 1) % grads::kNormUnit);
            units += (uint32_t)((bytes + grads::kNormUnit - 1) / grads::kNormUnit);
            ++a.n;
        }
        a.first[a.n] = units;
        while (t < n && len[t] == 0) ++t;
        return t;
    };
    size_t bytes = 0;
    for (size_t t = 0; t < n; ++t) bytes += len[t] * grad_bytes(gdt[t]);
    const bool once = bytes > kNormKeeps, large = bytes >= kNormLarge;
    const uint32_t most = large ? grads::kNormBlocks / 2 : grads::kNormBlocks;
    const auto kernel = large ? grads::norm_kernel<8, true> : once ? grads::norm_kernel<4, true> : grads::norm_kernel<4, false>;
    const auto blocks = [&](const grads::NormArgs &a) { return std::min(std::max<uint32_t>(a.first[a.n], 1), most); };
    grads::NormArgs a;
    a.norm = norm;
    a.scratch = static_cast<grads::NormScratch *>(workspace);
    size_t next = take(a, 0);
    // of several launches the first one opens as many slots as the largest can need
    a.slots = next < n ? most : blocks(a);
    for (a.opens = 1;; a.opens = 0) {
        a.closes = next == n;
        const int launched = launch(kernel, a.opens ? a.slots : blocks(a), 0, static_cast<hipStream_t>(hip_stream), a, grads::kNormThreads);
        if (launched != SS_OK || a.closes) return launched;
        next = take(a, next);
    }
}

int ss_grad_clip(const void *const *g, const ss_dtype *gdt, const size_t *len, size_t n, const float *norm, float max_norm,
                 void *const *out, const ss_dtype *odt, void *hip_stream) {
    if (!(max_norm >= 0.0f) || max_norm > __FLT_MAX__) return SS_ERR_ARG;
    if (!norm) return SS_ERR_NULL;
    if (n == 0) return SS_OK;
    int rc = check_list(g, gdt, len, n);
    if (rc == SS_OK) rc = check_list(out, odt, len, n);
    if (rc != SS_OK) return rc;
    if (!aligned16(norm)) return SS_ERR_ALIGN;
    Written written;
    bool failed = false;
    if (!written.take(out, odt, len, n, &failed)) return failed ? SS_ERR_RANGE : SS_ERR_ARG;
    if (written.meets(span(norm, sizeof(float), false))) return SS_ERR_ARG;
    for (size_t t = 0; t < n; ++t)
        if (len[t] && !(g[t] == out[t] && gdt[t] == odt[t]) && written.meets(span(g[t], len[t] * grad_bytes(gdt[t]), false)))
            return SS_ERR_ARG;
    grads::ClipArgs a;
    a.norm = norm;
    a.max_norm = max_norm;
    // a launch's units are its blocks: a tensor that has more than a grid takes is cut
    size_t t = 0, from = 0;
    while (t < n) {
        size_t units = 0;
        for (a.n = 0; t < n && a.n < (uint32_t)grads::kClipTensors && units < kClipGrid;) {
            const size_t size = grad_bytes(gdt[t]), osize = grad_bytes(odt[t]), left = len[t] - from;
            if (left == 0) {
                ++t;
                from = 0;
                continue;
            }
            const size_t unit = clip_unit(gdt[t], odt[t]);
            const uint64_t in = reinterpret_cast<uint64_t>(g[t]) + from * size, to = reinterpret_cast<uint64_t>(out[t]) + from * osize;
            const size_t lead = (to & 15u) / osize, elements = std::min(lead + left, (kClipGrid - units) * unit);
            a.at[a.n] = in | (gdt[t] == SS_BF16 ? 1u : 0u);
            a.out[a.n] = to | (odt[t] == SS_BF16 ? 1u : 0u);
            a.first[a.n] = (uint32_t)units;
            a.rest[a.n] = (uint16_t)((elements - 1) % unit);
            units += (elements + unit - 1) / unit;
            from += elements - lead;
            ++a.n;
        }
        if (a.n == 0) break;
        a.first[a.n] = (uint32_t)units;
        rc = launch(grads::clip_kernel, units, 0, static_cast<hipStream_t>(hip_stream), a, grads::kClipThreads);
        if (rc != SS_OK) return rc;
    }
    return SS_OK;
}

}  // extern "C"
