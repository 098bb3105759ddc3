// What pconv_ops_capi.cpp and the kernels of the 8-bit layers and the gradients share.
#ifndef PCONV_OPS_H
#define PCONV_OPS_H

#include <cstdint>

#include "pconv.h"

namespace pconv {

// y [m][n] = act((a [m][k] . b [n][k]) * (sa[m] * sb[n]) + bias[n]); strides in elements (those of a and b in bytes too).
struct I8Product {
    const int8_t *a, *b;
    const float *sa, *sb, *bias;
    void *y;
    int64_t lda, ldb, ldy;
    int m, n, k;
    int relu, y_bf16;
};

// Rows that begin anywhere, and where they go: rows of `pieces` times 16 bytes, one behind the other.
struct Realign {
    const int8_t *from;
    int8_t *to;
    int64_t ld;
    int rows, k, pieces;
};

// Launchers: arguments checked, sizes not 0.  They return a pconv_status.  `weights` are brought to multiples of 16
// bytes by the same launch.
int launch_quantize_rows(const void *x, int64_t ldx, int bf16, int64_t rows, int64_t cols, int8_t *q, int64_t ldq,
                         int64_t q_cols, float *scale, void *stream, const Realign *weights = nullptr);
// Whether rows begin at multiples of 16 bytes (and a tile's lie within 32 bits); the work space of a product (copies of
// operands whose rows do not, sums of parts of k), and the product.
bool rows_at_16(const int8_t *at, int64_t ld);
int64_t matmul_i8_work_bytes(int64_t m, int64_t n, int64_t k, bool a_at_16, bool b_at_16);
bool matmul_i8_aligns(int64_t m, int64_t k);             // whether the product of those sizes reads such rows only
Realign realigned(const int8_t *from, int64_t ld, int rows, int k, int8_t *to);
pconv_i8_plan matmul_i8_plan(int64_t m, int64_t n, int64_t k);
int launch_matmul_i8(const I8Product &p, void *work, void *stream);
// Whether rows are so few or so short that they are quantised within the product, and that product (p.a, lda, sa unused).
bool linear_i8_fused(int64_t m, int64_t n, int64_t k, bool b_at_16);
// Whether the product of rows that are quantised by a launch of their own can be launched: asked before that one.
int check_linear_i8_apart(int64_t m, int64_t n, int64_t k);
int launch_linear_i8_fused(const I8Product &p, const void *x, int64_t ldx, int bf16, void *stream);

// Up to kGradTensors tensors travel in the arguments of one launch (4 KiB), cut into chunks of 1 << `log2` elements.
constexpr int kGradTensors = 160, kGradBlocks = 2048;
constexpr int kGradLog2 = 14, kGradLog2Few = 12, kGradLog2One = 10;          // many elements, few, a launch of one workgroup
struct GradTable {
    const void *in[kGradTensors];
    void *out[kGradTensors];
    uint32_t start[kGradTensors];      // first chunk of the tensor (ascending)
    uint16_t last[kGradTensors];       // elements of its last chunk, less one
    uint16_t types[kGradTensors];      // bit 0: input bf16, bit 1: output bf16
    int32_t count, log2;
    uint32_t chunks;
    uint32_t passing;                  // the first pass reads the chunks below this one past the caches
};
int launch_grad_norm(const GradTable &t, unsigned blocks, double *partials, void *stream);
int launch_grad_total(const double *partials, unsigned count, double *total, float *norm, void *stream);
int launch_grad_scale(const GradTable &t, const double *partials, unsigned count, bool passing, float max_norm, float eps, float *norm,
                      void *stream);
// few elements: all of it by one workgroup
int launch_grad_clip_one(const GradTable &t, float max_norm, float eps, float *norm, void *stream);

}  // namespace pconv

#endif
