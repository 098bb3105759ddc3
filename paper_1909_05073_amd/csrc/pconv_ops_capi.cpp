// extern "C" boundary of the 8-bit and 4-bit layers, the norm, the distillation and the gradients (see include/pconv.h for the contract).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <limits>

#include "pconv_internal.h"
#include "pconv_ops.h"

using namespace pconv;

namespace {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1, kMaxSide = int64_t(1) << 30, kMaxK = 131071;
constexpr int64_t kMaxTop = 1024;                                        // entries of a row of the distillation
constexpr int64_t kMaxBlocks = 1 << 19, kMaxRowBytes = 1 << 23;      // of the 4-bit layers
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

// Rows of 4-bit blocks and their scales: within 32 bits where a tile is read.
int check_blocks(const char *who, const uint8_t *q, int64_t stride, const uint8_t *scale, int64_t slab, int64_t rows, int64_t blocks)
{
    if (!q || !scale) return invalid(who, "null pointer argument");
    if (reinterpret_cast<uintptr_t>(q) % 16 != 0 || stride % 16 != 0) return invalid(who, "rows of 4-bit values must begin at multiples of 16 bytes");
    if (stride < blocks * 16 || stride > kMaxRowBytes) return invalid(who, "rows of 4-bit values must lie at least their length and at most 8 MiB apart");
    if (reinterpret_cast<uintptr_t>(scale) % 8 != 0 || slab % 8 != 0) return invalid(who, "slabs of scales must begin at multiples of 8 bytes");
    if (!stride_fits((blocks + 7) / 8, rows * 8, slab)) return invalid(who, "slabs of scales must lie at least 8 bytes a row apart");
    return PCONV_OK;
}

bool mx4_sizes_fit(int64_t m, int64_t n, int64_t blocks) { return m > 0 && n > 0 && blocks >= 0 && m <= kMaxSide && n <= kMaxSide && blocks <= kMaxBlocks; }

// What both products check of their weights and outputs, and the product itself but for its activations.
int check_product_mx4(const char *who, const uint8_t *b, int64_t ldb, const uint8_t *sb, int64_t slab_b, const float *bias, void *y,
                      int64_t ldy, int y_dtype, int64_t m, int64_t n, int64_t blocks, int relu, Mx4Product &p)
{
    if (m < 0 || n < 0 || m > kMaxSide || n > kMaxSide) return invalid(who, "m and n must be 0 .. 2^30");
    if (!is_dtype(y_dtype)) return invalid(who, "unknown dtype of y");
    if (m == 0 || n == 0) return PCONV_OK;
    if (!y) return invalid(who, "null pointer argument");
    if (!stride_fits(m, n, ldy)) return invalid(who, "rows must lie at least their length apart");
    if (blocks)
        if (const int rc = check_blocks(who, b, ldb, sb, slab_b, n, blocks)) return rc;
    p = Mx4Product{nullptr, b, nullptr, sb, bias, y, 0, ldb, 0, slab_b, ldy, int(m), int(n), int(blocks), relu ? 1 : 0, y_dtype == PCONV_BF16};
    return PCONV_OK;
}

bool at_type(const void *p, int64_t size) { return reinterpret_cast<uintptr_t>(p) % uint64_t(size) == 0; }

// What the calls of the distillation check alike, and what they compute but for their outputs.
int check_distill(const char *who, const void *z, int64_t ldz, int z_type, const void *t, int64_t ldt, int t_type, const void *c, int64_t ldc,
                  int class_bytes, int64_t rows, int64_t v, int64_t top, float temperature, int mean, DistillRows &p)
{
    if (rows < 0 || rows > kMaxRows || v < 0 || v > kMaxSide) return invalid(who, "rows must be 0 .. 2^31 - 1, v 0 .. 2^30");
    if (top < 0 || top > kMaxTop) return invalid(who, "top must be 0 .. 1024");
    if (!is_dtype(z_type) || !is_dtype(t_type)) return invalid(who, "unknown dtype");
    if (class_bytes != 4 && class_bytes != 8) return invalid(who, "classes must have 4 or 8 bytes");
    if (!(temperature > 0.0f) || std::isinf(temperature) || std::isinf(1.0f / temperature) || std::isinf(temperature * temperature))
        return invalid(who, "the temperature must be a number above 0 whose square and reciprocal are numbers");
    if (rows == 0) return PCONV_OK;
    if ((v && !z) || (top && (!t || !c))) return invalid(who, "null pointer argument");
    if (!stride_fits(rows, v, ldz) || !stride_fits(rows, top, ldt) || !stride_fits(rows, top, ldc)) return invalid(who, "rows must lie at least their length apart");
    if (!at_type(z, z_type == PCONV_BF16 ? 2 : 4) || !at_type(t, t_type == PCONV_BF16 ? 2 : 4) || !at_type(c, class_bytes)) return invalid(who, "rows must be aligned to their type");
    const double log2e_t = std::min(1.4426950408889634 / double(temperature), double(std::numeric_limits<float>::max()));
    p = DistillRows{z, t, c, nullptr, nullptr, nullptr, nullptr, ldz, ldt, ldc, 0, rows, 0, int(v), int(top), 1.0f / temperature, float(log2e_t),
                    temperature * temperature, float(double(temperature) / (mean ? double(rows) : 1.0)), z_type == PCONV_BF16,
                    t_type == PCONV_BF16, class_bytes == 8};
    return PCONV_OK;
}

int check_grad_rows(const char *who, void *grad, int64_t ldg, int type, int64_t rows, int64_t v)
{
    if (v && !grad) return invalid(who, "null pointer argument");
    if (!stride_fits(rows, v, ldg)) return invalid(who, "rows must lie at least their length apart");
    return at_type(grad, type == PCONV_BF16 ? 2 : 4) ? PCONV_OK : invalid(who, "rows must be aligned to their type");
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

int pconv_quantize_mx4(const void *x_dev, int64_t x_stride, pconv_dtype x_dtype, int64_t rows, int64_t cols,
                       uint8_t *q_dev, int64_t q_stride, uint8_t *scale_dev, int64_t slab_stride, void *hip_stream)
{
    const char *who = "pconv_quantize_mx4";
    if (rows < 0 || cols < 0 || rows > kMaxSide || cols > kMaxBlocks * 32) return invalid(who, "rows must be 0 .. 2^30, cols 0 .. 2^24");
    if (!is_dtype(int(x_dtype))) return invalid(who, "unknown dtype");
    if (rows == 0 || cols == 0) return PCONV_OK;
    if (!x_dev) return invalid(who, "null pointer argument");
    if (!stride_fits(rows, cols, x_stride)) return invalid(who, "rows must lie at least their length apart");
    if (const int rc = check_blocks(who, q_dev, q_stride, scale_dev, slab_stride, rows, (cols + 31) / 32)) return rc;
    return launch_quantize_mx4(x_dev, x_stride, x_dtype == PCONV_BF16, rows, cols, q_dev, q_stride, scale_dev, slab_stride, hip_stream);
}

int64_t pconv_matmul_mx4_workspace(int64_t m, int64_t n, int64_t blocks) { return mx4_sizes_fit(m, n, blocks) ? matmul_mx4_work_bytes(m, n, blocks) : 0; }

int pconv_matmul_mx4(const uint8_t *a_dev, int64_t a_stride, const uint8_t *a_scale, int64_t a_slab, const uint8_t *b_dev,
                     int64_t b_stride, const uint8_t *b_scale, int64_t b_slab, const float *bias_dev, void *y_dev,
                     int64_t y_stride, pconv_dtype y_dtype, int64_t m, int64_t n, int64_t blocks, int fuse_relu, void *work,
                     int64_t work_bytes, void *hip_stream)
{
    const char *who = "pconv_matmul_mx4";
    if (blocks < 0 || blocks > kMaxBlocks) return invalid(who, "blocks must be 0 .. 2^19");
    Mx4Product p;
    if (const int rc = check_product_mx4(who, b_dev, b_stride, b_scale, b_slab, bias_dev, y_dev, y_stride, int(y_dtype), m, n, blocks, fuse_relu, p)) return rc;
    if (m == 0 || n == 0) return PCONV_OK;
    if (blocks)
        if (const int rc = check_blocks(who, a_dev, a_stride, a_scale, a_slab, m, blocks)) return rc;
    if (const int rc = check_work(who, work, work_bytes, matmul_mx4_work_bytes(m, n, blocks))) return rc;
    p.a = a_dev; p.lda = a_stride; p.sa = a_scale; p.slab_a = a_slab;
    return launch_matmul_mx4(p, work, hip_stream);
}

// Bytes from row to row of activations in the work space: long rows begin where lines of the caches do, or every piece of 128
// bytes that a tile stages is two of them (1908x10592 -> 2440: the product 52 us without, 41).
static int64_t mx4_step(int64_t blocks) { return blocks < 64 ? blocks * 16 : (blocks + 7) / 8 * 128; }

int64_t pconv_linear_mx4_workspace(int64_t m, int64_t n, int64_t k)
{
    if (k < 0 || k > kMaxBlocks * 32 || !mx4_sizes_fit(m, n, (k + 31) / 32)) return 0;
    const int64_t blocks = (k + 31) / 32;
    if (linear_mx4_fused(m, n, blocks)) return 0;
    return m * mx4_step(blocks) + round16((blocks + 7) / 8 * m * 8) + matmul_mx4_work_bytes(m, n, blocks);
}

int pconv_linear_mx4(const void *x_dev, int64_t x_stride, pconv_dtype x_dtype, const uint8_t *w_dev, int64_t w_stride,
                     const uint8_t *w_scale, int64_t w_slab, const float *bias_dev, void *y_dev, int64_t y_stride,
                     pconv_dtype y_dtype, int64_t m, int64_t n, int64_t k, int fuse_relu, void *work, int64_t work_bytes,
                     void *hip_stream)
{
    const char *who = "pconv_linear_mx4";
    if (!is_dtype(int(x_dtype))) return invalid(who, "unknown dtype of x");
    if (k < 0 || k > kMaxBlocks * 32) return invalid(who, "k must be 0 .. 2^24");
    const int64_t blocks = (k + 31) / 32;
    Mx4Product p;
    if (const int rc = check_product_mx4(who, w_dev, w_stride, w_scale, w_slab, bias_dev, y_dev, y_stride, int(y_dtype), m, n, blocks, fuse_relu, p)) return rc;
    if (m == 0 || n == 0) return PCONV_OK;
    if (k && !x_dev) return invalid(who, "null pointer argument");
    if (!stride_fits(m, k, x_stride)) return invalid(who, "rows must lie at least their length apart");
    if (const int rc = check_work(who, work, work_bytes, pconv_linear_mx4_workspace(m, n, k))) return rc;
    if (const int rc = check_matmul_mx4(m, n, blocks)) return rc;
    if (linear_mx4_fused(m, n, blocks)) return launch_linear_mx4_fused(p, x_dev, x_stride, x_dtype == PCONV_BF16, k, hip_stream);
    uint8_t *const q = static_cast<uint8_t *>(work), *const scale = q + m * mx4_step(blocks);
    if (k)
        if (const int rc = launch_quantize_mx4(x_dev, x_stride, x_dtype == PCONV_BF16, m, k, q, mx4_step(blocks), scale, m * 8, hip_stream)) return rc;
    p.a = q; p.lda = mx4_step(blocks); p.sa = scale; p.slab_a = m * 8;
    return launch_matmul_mx4(p, scale + round16((blocks + 7) / 8 * m * 8), hip_stream);
}

int pconv_debug_mx4_plan(int64_t m, int64_t n, int64_t blocks, pconv_mx4_plan *out)
{
    if (!out) return invalid("pconv_debug_mx4_plan", "null pointer argument");
    if (!mx4_sizes_fit(m, n, blocks)) return invalid("pconv_debug_mx4_plan", "m and n must be 1 .. 2^30, blocks 0 .. 2^19");
    *out = matmul_mx4_plan(m, n, blocks);
    return PCONV_OK;
}

int pconv_add_rms_norm_i8(const void *x_dev, int64_t x_stride, const void *residual_dev, int64_t residual_stride, void *sum_dev,
                          int64_t sum_stride, pconv_dtype dtype, const float *weight_dev, float eps, int64_t rows, int64_t cols,
                          int8_t *q_dev, int64_t q_stride, float *scale_dev, void *hip_stream)
{
    const char *who = "pconv_add_rms_norm_i8";
    if (rows < 0 || cols < 0 || rows > kMaxRows || cols > kMaxRows) return invalid(who, "rows and cols must be 0 .. 2^31 - 1");
    if (!is_dtype(int(dtype))) return invalid(who, "unknown dtype");
    if (!(eps > 0.0f) || std::isinf(eps)) return invalid(who, "eps must be a number above 0");
    if (sum_dev && !residual_dev) return invalid(who, "sums are of two operands: there is no residual");
    if (rows == 0) return PCONV_OK;
    if (!scale_dev || (cols && (!x_dev || !q_dev))) return invalid(who, "null pointer argument");
    if (!stride_fits(rows, cols, x_stride) || !stride_fits(rows, cols, q_stride) || (residual_dev && !stride_fits(rows, cols, residual_stride)) ||
        (sum_dev && !stride_fits(rows, cols, sum_stride)))
        return invalid(who, "rows must lie at least their length apart");
    if (sum_dev && rows > 1 && ((sum_dev == x_dev && sum_stride != x_stride) || (sum_dev == residual_dev && sum_stride != residual_stride)))
        return invalid(who, "sums in an operand's place must have its stride");
    const int size = dtype == PCONV_BF16 ? 2 : 4;
    if (!at_type(x_dev, size) || !at_type(residual_dev, size) || !at_type(sum_dev, size) || !at_type(weight_dev, 4)) return invalid(who, "rows must be aligned to their type");
    return launch_add_rms_norm_i8(NormRows{x_dev, residual_dev, sum_dev, weight_dev, q_dev, scale_dev, x_stride, residual_stride, sum_stride, q_stride,
                                           rows, cols, eps}, dtype == PCONV_BF16, hip_stream);
}

int pconv_distill_loss(const void *z_dev, int64_t z_stride, pconv_dtype z_dtype, const void *teacher_dev, int64_t teacher_stride,
                       pconv_dtype teacher_dtype, const void *classes_dev, int64_t classes_stride, int class_bytes, int64_t rows,
                       int64_t v, int64_t top, float temperature, int mean, float *loss_dev, float *total_dev, float *lse_dev,
                       void *hip_stream)
{
    const char *who = "pconv_distill_loss";
    DistillRows p;
    if (const int rc = check_distill(who, z_dev, z_stride, int(z_dtype), teacher_dev, teacher_stride, int(teacher_dtype), classes_dev, classes_stride,
                                     class_bytes, rows, v, top, temperature, mean, p)) return rc;
    if (rows > 0) {
        if (!loss_dev) return invalid(who, "null pointer argument");
        p.loss = loss_dev; p.lse = lse_dev;
        if (const int rc = launch_distill(p, true, false, hip_stream)) return rc;
    }
    return total_dev ? launch_distill_total(loss_dev, rows, mean && rows ? 1.0 / double(rows) : 1.0, total_dev, hip_stream) : PCONV_OK;
}

int pconv_distill_grad(const void *z_dev, int64_t z_stride, pconv_dtype z_dtype, const void *teacher_dev, int64_t teacher_stride,
                       pconv_dtype teacher_dtype, const void *classes_dev, int64_t classes_stride, int class_bytes, int64_t rows,
                       int64_t v, int64_t top, float temperature, int mean, const float *lse_dev, const float *up_dev,
                       int64_t up_step, void *grad_dev, int64_t grad_stride, void *hip_stream)
{
    const char *who = "pconv_distill_grad";
    DistillRows p;
    if (const int rc = check_distill(who, z_dev, z_stride, int(z_dtype), teacher_dev, teacher_stride, int(teacher_dtype), classes_dev, classes_stride,
                                     class_bytes, rows, v, top, temperature, mean, p)) return rc;
    if (up_step != 0 && up_step != 1) return invalid(who, "up_step must be 0 or 1");
    if (rows == 0) return PCONV_OK;
    if (!lse_dev) return invalid(who, "null pointer argument");
    if (const int rc = check_grad_rows(who, grad_dev, grad_stride, int(z_dtype), rows, v)) return rc;
    if (v == 0) return PCONV_OK;
    p.lse = const_cast<float *>(lse_dev); p.up = up_dev; p.up_step = up_step; p.grad = grad_dev; p.ldg = grad_stride;
    return launch_distill(p, false, true, hip_stream);
}

int pconv_distill_loss_grad(const void *z_dev, int64_t z_stride, pconv_dtype z_dtype, const void *teacher_dev, int64_t teacher_stride,
                            pconv_dtype teacher_dtype, const void *classes_dev, int64_t classes_stride, int class_bytes,
                            int64_t rows, int64_t v, int64_t top, float temperature, int mean, float *loss_dev, float *total_dev,
                            void *grad_dev, int64_t grad_stride, void *hip_stream)
{
    const char *who = "pconv_distill_loss_grad";
    DistillRows p;
    if (const int rc = check_distill(who, z_dev, z_stride, int(z_dtype), teacher_dev, teacher_stride, int(teacher_dtype), classes_dev, classes_stride,
                                     class_bytes, rows, v, top, temperature, mean, p)) return rc;
    if (rows > 0) {
        if (!loss_dev) return invalid(who, "null pointer argument");
        if (const int rc = check_grad_rows(who, grad_dev, grad_stride, int(z_dtype), rows, v)) return rc;
        p.loss = loss_dev; p.grad = grad_dev; p.ldg = grad_stride;
        if (const int rc = launch_distill(p, true, true, hip_stream)) return rc;
    }
    return total_dev ? launch_distill_total(loss_dev, rows, mean && rows ? 1.0 / double(rows) : 1.0, total_dev, hip_stream) : PCONV_OK;
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
