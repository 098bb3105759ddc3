// What pconv_ops_capi.cpp and the kernels of the 8-bit and 4-bit layers, the norm, the distillation and
// the gradients share.
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

// y [m][n] = act(sum over blocks of 32 of 2^(sa + sb - 254) (a [m][k] . b [n][k]) + bias[n]); rows of 16 bytes a block, scales in
// slabs of 8 blocks, [slab][row][8]; strides in bytes, that of y in elements.
struct Mx4Product {
    const uint8_t *a, *b, *sa, *sb;
    const float *bias;
    void *y;
    int64_t lda, ldb, slab_a, slab_b, ldy;
    int m, n, blocks;
    int relu, y_bf16;
};

int launch_quantize_mx4(const void *x, int64_t ldx, int bf16, int64_t rows, int64_t cols, uint8_t *q, int64_t ldq, uint8_t *scale,
                        int64_t slab_stride, void *stream);
int64_t matmul_mx4_work_bytes(int64_t m, int64_t n, int64_t blocks);
int check_matmul_mx4(int64_t m, int64_t n, int64_t blocks);              // whether the product can be launched
pconv_mx4_plan matmul_mx4_plan(int64_t m, int64_t n, int64_t blocks);
int launch_matmul_mx4(const Mx4Product &p, void *work, void *stream);
// Whether rows are so few that they are quantised within the product, and that product (p.a, lda, sa, slab_a unused).
bool linear_mx4_fused(int64_t m, int64_t n, int64_t blocks);
int launch_linear_mx4_fused(const Mx4Product &p, const void *x, int64_t ldx, int bf16, int64_t k, void *stream);

// s = x + r (r: or null), h = s / sqrt(mean s^2 + eps) * weight (or null), q and scale of h; sum: where s goes (or null).
struct NormRows {
    const void *x, *r;
    void *sum;
    const float *weight;
    int8_t *q;
    float *scale;
    int64_t ldx, ldr, ldsum, ldq, rows, cols;
    float eps;
};
int launch_add_rms_norm_i8(const NormRows &p, int bf16, void *stream);

// Distillation: student's logits z [rows][v], teacher's t [rows][top] at the classes c.
struct DistillRows {
    const void *z, *t, *c;
    float *loss, *lse;                 // [rows]; lse may be null where the loss is computed
    const float *up;                   // the gradient that comes in, up_step from row to row; null: 1
    void *grad;
    int64_t ldz, ldt, ldc, ldg, rows, up_step;
    int v, top;
    float inv_t, log2e_t, t2, factor;  // 1 / T, log2(e) / T, T^2, T and what the rows are divided by
    int z_bf16, t_bf16, c_wide;
};
int launch_distill(const DistillRows &p, bool loss, bool grad, void *stream);
int launch_distill_total(const float *loss, int64_t rows, double scale, float *total, void *stream);

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
