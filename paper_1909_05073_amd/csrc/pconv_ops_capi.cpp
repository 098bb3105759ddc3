// extern "C" boundary of the 8-bit layers and the gradients (see include/pconv.h for the contract).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "pconv_internal.h"
#include "pconv_ops.h"

using namespace pconv;

namespace {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1, kMaxSide = int64_t(1) << 30, kMaxK = 131071;
constexpr int64_t kMaxTensors = 1 << 24, kMaxElements = int64_t(1) << 45;    // fewer than 2^32 chunks together

int invalid(const char *who, const char *what)
{
    set_error(std::string(who) + ": " + what);
    return PCONV_INVALID_ARG;
}

bool is_dtype(int t) { return t == PCONV_F32 || t == PCONV_BF16; }
int64_t round16(int64_t v) { return (v + 15) / 16 * 16; }

// rows of `len` elements that lie `stride` apart: within the range of a byte offset in 64 bits
bool stride_fits(int64_t rows, int64_t len, int64_t stride) { return stride >= len && stride <= (int64_t(1) << 58) / (rows > 0 ? rows : 1); }

bool sizes_fit(int64_t m, int64_t n, int64_t k) { return m > 0 && n > 0 && k >= 0 && m <= kMaxSide && n <= kMaxSide && k <= kMaxK; }

int check_work(const char *who, const void *work, int64_t have, int64_t need)
{
    if (need > 0 && (!work || have < need)) return invalid(who, "the work space is too small");
    if (need > 0 && reinterpret_cast<uintptr_t>(work) % 16 != 0) return invalid(who, "the work space must be aligned to 16 bytes");
    return PCONV_OK;
}

// What both products check of their weights and outputs, and the product itself but for its activations.
int check_product(const char *who, const int8_t *b, int64_t ldb, const float *sb, const float *bias, void *y, int64_t ldy, int y_dtype,
                  int64_t m, int64_t n, int64_t k, int relu, I8Product &p)
{
    if (m < 0 || n < 0 || k < 0 || m > kMaxSide || n > kMaxSide) return invalid(who, "m and n must be 0 .. 2^30");
    if (k > kMaxK) return invalid(who, "k must be 0 .. 131071");
    if (!is_dtype(y_dtype)) return invalid(who, "unknown dtype of y");
    if (m == 0 || n == 0) return PCONV_OK;
    if (!sb || !y || (k && !b)) return invalid(who, "null pointer argument");
    if (!stride_fits(n, k, ldb) || !stride_fits(m, n, ldy)) return invalid(who, "rows must lie at least their length apart");
    p = I8Product{nullptr, b, nullptr, sb, bias, y, 0, ldb, ldy, int(m), int(n), int(k), relu ? 1 : 0, y_dtype == PCONV_BF16};
    return PCONV_OK;
}

// The tensors that are clipped together, and how they are cut up.
struct Grads {
    const void *const *in;
    void *const *out;
    const int64_t *counts;
    const int32_t *types, *out_types;
    int64_t num;
    int log2;              // elements of a chunk
    int64_t chunks;        // all of them
    int64_t kept;          // bytes of the last gradients that are left in the caches; less than 0: of all

    int64_t tables() const { return (num + kGradTensors - 1) / kGradTensors; }
};

constexpr int64_t kKeptBytes = int64_t(192) << 20, kCachedBytes = int64_t(128) << 20;

Grads grads_of(const void *const *in, void *const *out, const int64_t *counts, const int32_t *types, const int32_t *out_types, int64_t num)
{
    Grads g{in, out, counts, types, out_types, num, 0, 0, -1};
    int64_t elements = 0, bytes = 0, ones = 0, few = 0, many = 0;
    for (int64_t i = 0; i < num; ++i) {
        const int64_t n = counts[i];
        elements += n;
        bytes += n * ((types[i] == PCONV_BF16 ? 2 : 4) + (!out || out[i] == in[i] ? 0 : out_types[i] == PCONV_BF16 ? 2 : 4));
        ones += (n + (1 << kGradLog2One) - 1) >> kGradLog2One;
        few += (n + (1 << kGradLog2Few) - 1) >> kGradLog2Few;
        many += (n + (1 << kGradLog2) - 1) >> kGradLog2;
    }
    // One workgroup for up to two chunks a wave (a launch less on the host: 2.4 us); chunks of 4096 elements while
    // those of 16384 would not be one for each compute unit (where they are, finding a chunk's tensor costs more than
    // it gives).
    if (out && num <= kGradTensors && ones <= 32) { g.log2 = kGradLog2One; g.chunks = ones; }
    else if (elements < int64_t(256) << kGradLog2) { g.log2 = kGradLog2Few; g.chunks = few; }
    else { g.log2 = kGradLog2; g.chunks = many; }
    if (out && bytes > kCachedBytes) g.kept = kKeptBytes;
    return g;
}

// The table of tensors [kGradTensors * i, ..); false where they are all empty.  `behind`: bytes of the gradients behind them.
bool table_of(const Grads &g, int64_t i, int64_t behind, GradTable &t)
{
    const int64_t begin = i * kGradTensors, end = std::min<int64_t>(begin + kGradTensors, g.num);
    t.count = 0; t.chunks = 0; t.passing = 0; t.log2 = g.log2;
    for (int64_t at = begin; at < end; ++at) {
        const int64_t n = g.counts[at];
        if (n == 0) continue;
        const int k = t.count++;
        t.in[k] = g.in[at];
        t.out[k] = g.out ? g.out[at] : nullptr;
        t.start[k] = t.chunks;
        t.last[k] = uint16_t((n - 1) & ((int64_t(1) << g.log2) - 1));
        t.types[k] = uint16_t((g.types[at] == PCONV_BF16 ? 1 : 0) | (g.out && g.out_types[at] == PCONV_BF16 ? 2 : 0));
        t.chunks += uint32_t((n + (int64_t(1) << g.log2) - 1) >> g.log2);
    }
    if (g.kept < 0 || t.count == 0) return t.count > 0;
    t.passing = t.chunks;
    for (int k = t.count - 1; k >= 0 && behind < g.kept; --k) {          // from the last: the chunks that are kept
        const int64_t each = int64_t(t.types[k] & 1 ? 2 : 4) << g.log2, have = (k + 1 < t.count ? t.start[k + 1] : t.chunks) - t.start[k];
        const int64_t keep = std::min(have, (g.kept - behind + each - 1) / each);
        t.passing -= uint32_t(keep);
        behind += keep * each;
    }
    return true;
}

int64_t table_bytes(const Grads &g, int64_t i)
{
    int64_t b = 0;
    for (int64_t at = i * kGradTensors; at < std::min<int64_t>((i + 1) * kGradTensors, g.num); ++at) b += g.counts[at] * (g.types[at] == PCONV_BF16 ? 2 : 4);
    return b;
}

int check_grads(const char *who, const void *const *in, const int64_t *counts, const int32_t *types, int64_t num, float *norm,
                void *work, int64_t work_bytes)
{
    if (num < 0 || num > kMaxTensors) return invalid(who, "num must be 0 .. 2^24");
    if (!norm || !work || (num && (!in || !counts || !types))) return invalid(who, "null pointer argument");
    if (reinterpret_cast<uintptr_t>(work) % 16 != 0) return invalid(who, "the work space must be aligned to 16 bytes");
    if (work_bytes < pconv_grad_workspace(num)) return invalid(who, "the work space is too small");
    int64_t total = 0;
    for (int64_t i = 0; i < num; ++i) {
        if (counts[i] < 0 || counts[i] > kMaxElements || (total += counts[i]) > kMaxElements) return invalid(who, "counts must be 0 .. 2^45, and so their sum");
        if (counts[i] && !in[i]) return invalid(who, "null pointer of a tensor");
        if (!is_dtype(types[i])) return invalid(who, "unknown dtype of a tensor");
        if (counts[i] && reinterpret_cast<uintptr_t>(in[i]) % (types[i] == PCONV_BF16 ? 2 : 4) != 0) return invalid(who, "a tensor must be aligned to its type");
    }
    return PCONV_OK;
}

// The sums of squares of all tables, to work[1 ..]; how many there are.
int sum_squares(const Grads &g, double *work, void *stream, unsigned &sums)
{
    const unsigned cap = unsigned(std::max<int64_t>(64, kGradBlocks / std::max<int64_t>(1, g.tables())));
    int64_t behind = 0;
    if (g.kept >= 0)
        for (int64_t i = 1; i < g.tables(); ++i) behind += table_bytes(g, i);
    sums = 0;
    for (int64_t i = 0; i < g.tables(); ++i) {
        GradTable t;
        if (table_of(g, i, behind, t)) {
            const unsigned blocks = std::min(t.chunks, cap);
            if (const int rc = launch_grad_norm(t, blocks, work + 1 + sums, stream)) return rc;
            sums += blocks;
        }
        if (g.kept >= 0 && i + 1 < g.tables()) behind -= table_bytes(g, i + 1);
    }
    return PCONV_OK;
}

}  // namespace

extern "C" {

int pconv_quantize_rows(const void *x_dev, int64_t x_stride, pconv_dtype x_dtype, int64_t rows, int64_t cols,
                        int8_t *q_dev, int64_t q_stride, float *scale_dev, void *hip_stream)
{
    const char *who = "pconv_quantize_rows";
    if (rows < 0 || cols < 0 || rows > kMaxRows || cols > kMaxRows) return invalid(who, "rows and cols must be 0 .. 2^31 - 1");
    if (!is_dtype(int(x_dtype))) return invalid(who, "unknown dtype");
    if (rows == 0) return PCONV_OK;
    if (!scale_dev || (cols && (!x_dev || !q_dev))) return invalid(who, "null pointer argument");
    if (!stride_fits(rows, cols, x_stride) || !stride_fits(rows, cols, q_stride)) return invalid(who, "rows must lie at least their length apart");
    return launch_quantize_rows(x_dev, x_stride, x_dtype == PCONV_BF16, rows, cols, q_dev, q_stride, cols, scale_dev, hip_stream);
}

int64_t pconv_matmul_i8_workspace(int64_t m, int64_t n, int64_t k, int rows_at_16)
{
    return sizes_fit(m, n, k) ? matmul_i8_work_bytes(m, n, k, rows_at_16 != 0, rows_at_16 != 0) : 0;
}

int pconv_matmul_i8(const int8_t *a_dev, int64_t a_stride, const float *a_scale, const int8_t *b_dev, int64_t b_stride,
                    const float *b_scale, const float *bias_dev, void *y_dev, int64_t y_stride, pconv_dtype y_dtype,
                    int64_t m, int64_t n, int64_t k, int fuse_relu, void *work, int64_t work_bytes, void *hip_stream)
{
    const char *who = "pconv_matmul_i8";
    I8Product p;
    if (const int rc = check_product(who, b_dev, b_stride, b_scale, bias_dev, y_dev, y_stride, int(y_dtype), m, n, k, fuse_relu, p)) return rc;
    if (m == 0 || n == 0) return PCONV_OK;
    if (!a_scale || (k && !a_dev)) return invalid(who, "null pointer argument");
    if (!stride_fits(m, k, a_stride)) return invalid(who, "rows must lie at least their length apart");
    if (const int rc = check_work(who, work, work_bytes, matmul_i8_work_bytes(m, n, k, rows_at_16(a_dev, a_stride), rows_at_16(b_dev, b_stride)))) return rc;
    p.a = a_dev; p.lda = a_stride; p.sa = a_scale;
    return launch_matmul_i8(p, work, hip_stream);
}

int64_t pconv_linear_i8_workspace(int64_t m, int64_t n, int64_t k, int rows_at_16)
{
    return sizes_fit(m, n, k) && !linear_i8_fused(m, n, k, rows_at_16 != 0) ? round16(4 * m) + m * round16(k) + matmul_i8_work_bytes(m, n, k, true, rows_at_16 != 0) : 0;
}

int pconv_linear_i8(const void *x_dev, int64_t x_stride, pconv_dtype x_dtype, const int8_t *w_dev, int64_t w_stride,
                    const float *w_scale, const float *bias_dev, void *y_dev, int64_t y_stride, pconv_dtype y_dtype,
                    int64_t m, int64_t n, int64_t k, int fuse_relu, void *work, int64_t work_bytes, void *hip_stream)
{
    const char *who = "pconv_linear_i8";
    if (!is_dtype(int(x_dtype))) return invalid(who, "unknown dtype of x");
    I8Product p;
    if (const int rc = check_product(who, w_dev, w_stride, w_scale, bias_dev, y_dev, y_stride, int(y_dtype), m, n, k, fuse_relu, p)) return rc;
    if (m == 0 || n == 0) return PCONV_OK;
    if (k && !x_dev) return invalid(who, "null pointer argument");
    if (!stride_fits(m, k, x_stride)) return invalid(who, "rows must lie at least their length apart");
    if (const int rc = check_work(who, work, work_bytes, pconv_linear_i8_workspace(m, n, k, rows_at_16(w_dev, w_stride)))) return rc;
    if (linear_i8_fused(m, n, k, rows_at_16(w_dev, w_stride))) return launch_linear_i8_fused(p, x_dev, x_stride, x_dtype == PCONV_BF16, hip_stream);
    if (const int rc = check_linear_i8_apart(m, n, k)) return rc;
    float *const scale = static_cast<float *>(work);
    int8_t *const q = static_cast<int8_t *>(work) + round16(4 * m);
    const int64_t ldq = round16(k);
    int8_t *rest = q + m * ldq;
    const bool align = !rows_at_16(w_dev, w_stride) && matmul_i8_aligns(m, k);
    const Realign weights = align ? realigned(w_dev, w_stride, p.n, p.k, rest) : Realign{};
    if (const int rc = launch_quantize_rows(x_dev, x_stride, x_dtype == PCONV_BF16, m, k, q, ldq, ldq, scale, hip_stream, align ? &weights : nullptr)) return rc;
    p.a = q; p.lda = ldq; p.sa = scale;
    if (align) { p.b = rest; p.ldb = ldq; p.k = int(ldq); rest += n * ldq; }          // (zeros behind the ends of both)
    return launch_matmul_i8(p, rest, hip_stream);
}

int pconv_debug_i8_plan(int64_t m, int64_t n, int64_t k, pconv_i8_plan *out)
{
    if (!out) return invalid("pconv_debug_i8_plan", "null pointer argument");
    if (!sizes_fit(m, n, k)) return invalid("pconv_debug_i8_plan", "m and n must be 1 .. 2^30, k 0 .. 131071");
    *out = matmul_i8_plan(m, n, k);
    return PCONV_OK;
}

int64_t pconv_grad_workspace(int64_t num)
{
    // one sum for the total, and those of the launches: of kGradBlocks workgroups together, at least 64 each
    const int64_t tables = (std::max<int64_t>(num, 0) + kGradTensors - 1) / kGradTensors;
    return 16 + 8 * std::max<int64_t>(kGradBlocks, 64 * (2 * tables + 1));
}

int pconv_grad_norm(const void *const *grads, const int64_t *counts, const int32_t *dtypes, int64_t num,
                    float *norm_dev, void *work, int64_t work_bytes, void *hip_stream)
{
    if (const int rc = check_grads("pconv_grad_norm", grads, counts, dtypes, num, norm_dev, work, work_bytes)) return rc;
    double *const sums = static_cast<double *>(work);
    unsigned count;
    if (const int rc = sum_squares(grads_of(grads, nullptr, counts, dtypes, nullptr, num), sums, hip_stream, count)) return rc;
    return launch_grad_total(sums + 1, count, sums, norm_dev, hip_stream);
}

int pconv_clip_grads(const void *const *grads, void *const *outs, const int64_t *counts, const int32_t *dtypes,
                     const int32_t *out_dtypes, int64_t num, float max_norm, float eps, float *norm_dev,
                     void *work, int64_t work_bytes, void *hip_stream)
{
    const char *who = "pconv_clip_grads";
    if (const int rc = check_grads(who, grads, counts, dtypes, num, norm_dev, work, work_bytes)) return rc;
    if (num && (!outs || !out_dtypes)) return invalid(who, "null pointer argument");
    if (!(max_norm >= 0.0f)) return invalid(who, "max_norm must be at least 0");
    if (!(eps >= 0.0f) || std::isinf(eps)) return invalid(who, "eps must be a number of at least 0");
    for (int64_t i = 0; i < num; ++i) {
        if (counts[i] && !outs[i]) return invalid(who, "null pointer of an output");
        if (!is_dtype(out_dtypes[i])) return invalid(who, "unknown dtype of an output");
        if (counts[i] && reinterpret_cast<uintptr_t>(outs[i]) % (out_dtypes[i] == PCONV_BF16 ? 2 : 4) != 0) return invalid(who, "an output must be aligned to its type");
        if (counts[i] && outs[i] == grads[i] && out_dtypes[i] != dtypes[i]) return invalid(who, "an output in its gradient's place must have its type");
    }
    const Grads g = grads_of(grads, outs, counts, dtypes, out_dtypes, num);
    GradTable t;
    if (g.log2 == kGradLog2One && g.chunks > 0) {
        (void)table_of(g, 0, 0, t);
        return launch_grad_clip_one(t, max_norm, eps, norm_dev, hip_stream);
    }
    double *const sums = static_cast<double *>(work);
    unsigned count;
    if (const int rc = sum_squares(g, sums, hip_stream, count)) return rc;
    // Every workgroup of the second pass adds the partial sums by itself; with several tables or many workgroups one
    // launch for it takes less.  (Also for nothing at all: the norm is 0.)
    const bool total = g.tables() != 1 || count == 0 || g.chunks > 2 * kGradBlocks;
    if (total)
        if (const int rc = launch_grad_total(sums + 1, count, sums, norm_dev, hip_stream)) return rc;
    int64_t behind = 0;
    for (int64_t i = g.tables() - 1; i >= 0; --i) {
        if (table_of(g, i, behind, t))
            if (const int rc = launch_grad_scale(t, total ? sums : sums + 1, total ? 1 : count, g.kept >= 0, max_norm, eps, total ? nullptr : norm_dev, hip_stream)) return rc;
        if (g.kept >= 0) behind += table_bytes(g, i);
    }
    return PCONV_OK;
}

}  // extern "C"
