// Products of 8-bit integers with one scale for each row of the activations and one for each output channel, and the
// quantising of rows.
//
//   y[m][n] = act((sum_k a[m][k] b[n][k]) * (sa[m] * sb[n]) + bias[n])
//
// Both operands lie row by row along k, which is what a lane of the matrix instruction wants: 16 consecutive bytes of
// one row.  The weights are the instruction's first operand and the activations its second, so that a lane ends up with
// four neighbouring channels of one row of y.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pconv_internal.h"
#include "pconv_ops.h"

namespace pconv {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

int check_launch(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return PCONV_OK;
    set_error(std::string(what) + ": launch failed: " + hipGetErrorName(e));
    return PCONV_HIP_ERROR;
}

// ---- quantising rows ---------------------------------------------------------------------------------------------------

// The largest magnitude travels as the bits of |x|: ordered like the values, infinity above all numbers and NaN above it.
struct RowScale {
    float scale, inv;
    int mode;                                            // 0: by the reciprocal, 1: tiny scales, by division, 2: all zeros
};

__device__ __forceinline__ RowScale row_scale(uint32_t most)
{
    RowScale r;
    const float amax = __uint_as_float(most);
    if (most >= 0x7F800000u) {
        r.scale = __uint_as_float(0x7FC00000u); r.inv = 0.0f; r.mode = 2;
        return r;
    }
    r.scale = amax / 127.0f;
    r.mode = r.scale >= 0x1p-100f ? 0 : r.scale > 0.0f ? 1 : 2;
    r.inv = r.mode == 0 ? 1.0f / r.scale : 0.0f;
    return r;
}

// The nearest whole number of the nearest fp32 number of x / scale, in the low byte.  The correctly rounded quotient comes
// from the correctly rounded reciprocal by two corrections with the exact remainder (Markstein, 1990): five
// operations for a division's eleven.  That needs remainders that are no denormals, hence the lower limit of mode 0;
// quotients so small that theirs are denormal all round to 0.  Adding 1.5 * 2^23 rounds to a whole number in
// the low bits, ties to even.
__device__ __forceinline__ uint32_t quantize(float x, const RowScale &r)
{
    float t = x * r.inv;
    t = __builtin_fmaf(__builtin_fmaf(-t, r.scale, x), r.inv, t);
    t = __builtin_fmaf(__builtin_fmaf(-t, r.scale, x), r.inv, t);
    return __float_as_uint(t + 12582912.0f);
}

// The rare rows: a scale so small that it is itself rounded to few bits, so that quotients may pass 127.
__device__ __forceinline__ uint32_t quantize_rare(float x, const RowScale &r)
{
    const float t = r.mode == 1 ? fminf(fmaxf(x / r.scale, -127.0f), 127.0f) : 0.0f;
    return __float_as_uint(t + 12582912.0f);
}

__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0C0C0400u), cd = __builtin_amdgcn_perm(d, c, 0x04000C0Cu);
    return ab | cd;
}

// 16 bytes of a row of activations as floats
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    f4 v;
    __device__ __forceinline__ void load(const float *p) { __builtin_memcpy(&v, p, 16); }
    __device__ __forceinline__ float at(int i) const { return v[i]; }
    __device__ __forceinline__ void zero() { v = f4{0, 0, 0, 0}; }
    __device__ __forceinline__ void put(int i, float x) { v[i] = x; }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
};
template <> struct Vec<__bf16> {
    static constexpr int N = 8;
    b8 v;
    __device__ __forceinline__ void load(const __bf16 *p) { __builtin_memcpy(&v, p, 16); }
    __device__ __forceinline__ float at(int i) const { return float(v[i]); }
    __device__ __forceinline__ void zero() { v = b8{}; }
    __device__ __forceinline__ void put(int i, float x) { v[i] = __bf16(x); }
    static __device__ __forceinline__ float one(const __bf16 *p) { return float(*p); }
};

template <typename T>
__device__ __forceinline__ uint32_t most_of(const Vec<T> &v, uint32_t most)
{
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) most = max(most, __float_as_uint(v.at(i)) & 0x7FFFFFFFu);
    return most;
}

// Elements [at, at + N) of a row of `cols`: the last ones one by one, beyond the end zero.
template <typename T>
__device__ __forceinline__ Vec<T> load_part(const T *row, int64_t at, int64_t cols)
{
    Vec<T> v;
    if (at + Vec<T>::N <= cols) {
        v.load(row + at);
    } else {
        v.zero();
        for (int i = 0; i < Vec<T>::N; ++i)
            if (at + i < cols) v.put(i, Vec<T>::one(row + at + i));
    }
    return v;
}

// The same elements quantised, to q; [cols, q_cols) is filled with zeros.
template <typename T>
__device__ __forceinline__ void store_part(const Vec<T> &v, const RowScale &r, int8_t *row, int64_t at, int64_t q_cols)
{
    constexpr int N = Vec<T>::N;
    uint32_t w[N / 4];
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        if (r.mode == 0)
            w[j] = pack4(quantize(v.at(4 * j), r), quantize(v.at(4 * j + 1), r), quantize(v.at(4 * j + 2), r), quantize(v.at(4 * j + 3), r));
        else
            w[j] = pack4(quantize_rare(v.at(4 * j), r), quantize_rare(v.at(4 * j + 1), r), quantize_rare(v.at(4 * j + 2), r),
                         quantize_rare(v.at(4 * j + 3), r));
    }
    if (at + N <= q_cols) {
        __builtin_memcpy(row + at, w, N);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + i < q_cols) row[at + i] = int8_t(w[i / 4] >> (8 * (i & 3)));
    }
}

// TPR threads of a workgroup share a row; each keeps its first KEEP vectors of 16 bytes in registers between finding the
// row's scale and quantising, and reads what lies beyond (from a cache) twice.
template <typename T, int TPR, int THREADS>
__global__ void __launch_bounds__(THREADS)
quantize_rows_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int64_t cols, int8_t *__restrict__ q, int64_t ldq,
                     int64_t q_cols, float *__restrict__ scale)
{
    constexpr int N = Vec<T>::N, KEEP = 4, RPW = THREADS / TPR;
    __shared__ uint32_t lds[THREADS / 64];
    const int sub = int(threadIdx.x) % TPR;
    const int64_t groups = (rows + RPW - 1) / RPW;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t r = g * RPW + int(threadIdx.x) / TPR;
        const bool live = r < rows;
        const T *row = x + (live ? r : rows - 1) * ldx;
        Vec<T> v[KEEP];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) v[i] = load_part(row, (int64_t(i) * TPR + sub) * N, cols);
#pragma unroll
        for (int i = 0; i < KEEP; ++i) most = most_of(v[i], most);
#pragma unroll 4
        for (int64_t at = (int64_t(KEEP) * TPR + sub) * N; at < cols; at += TPR * N) most = most_of(load_part(row, at, cols), most);
#pragma unroll
        for (int d = (TPR < 64 ? TPR : 64) / 2; d; d >>= 1) most = max(most, uint32_t(__shfl_xor(int(most), d)));
        if (TPR > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = most;
            __syncthreads();
            most = 0;
#pragma unroll
            for (int i = 0; i < THREADS / 64; ++i) most = max(most, lds[i]);
        }
        const RowScale s = row_scale(most);
        if (!live) continue;
        int8_t *qrow = q + r * ldq;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) store_part(v[i], s, qrow, (int64_t(i) * TPR + sub) * N, q_cols);
        for (int64_t at = (int64_t(KEEP) * TPR + sub) * N; at < q_cols; at += TPR * N)
            store_part(load_part(row, at, cols), s, qrow, at, q_cols);
        if (sub == 0) scale[r] = s.scale;
    }
}

// ---- the product --------------------------------------------------------------------------------------------------------

// 16 bytes of a row that has `len` bytes, from `at` on; beyond its end zero.
__device__ __forceinline__ v4i load16(const int8_t *row, int at, int len)
{
    v4i v = {0, 0, 0, 0};
    if (at + 16 <= len) {
        __builtin_memcpy(&v, row + at, 16);
    } else if (at < len) {
        uint32_t w[4] = {0, 0, 0, 0};
        for (int i = 0; i < 15; ++i)
            if (at + i < len) w[i >> 2] |= uint32_t(uint8_t(row[at + i])) << (8 * (i & 3));
        v = v4i{int(w[0]), int(w[1]), int(w[2]), int(w[3])};
    }
    return v;
}

// Four neighbouring channels of one row of y.  ReLU keeps NaN.
__device__ __forceinline__ void finish(const I8Product &p, int m, int n, v4i acc, bool wide)
{
    if (m >= p.m || n >= p.n) return;
    const float sa = p.sa[m];
    f4 v;
    const int have = min(4, p.n - n);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = min(n + i, p.n - 1);
        v[i] = float(acc[i]) * (sa * p.sb[at]) + (p.bias ? p.bias[at] : 0.0f);
        if (p.relu) v[i] = v[i] < 0.0f ? 0.0f : v[i];
    }
    const int64_t to = int64_t(m) * p.ldy + n;
    if (p.y_bf16) {
        __bf16 *y = static_cast<__bf16 *>(p.y) + to;
        const b4 w = __builtin_convertvector(v, b4);
        if (have == 4) __builtin_memcpy(y, &w, 8);
        else for (int i = 0; i < have; ++i) y[i] = w[i];
    } else {
        float *y = static_cast<float *>(p.y) + to;
        if (have == 4) __builtin_memcpy(y, &v, 16);
        else for (int i = 0; i < have; ++i) y[i] = v[i];
    }
}

// Tiles of BM rows of y and BN channels, WM x WN waves; stages of BK bytes of k pass through LDS, two at a time.  A
// row of a stage is eight pieces of 16 bytes, stored in an order that depends on the row so that the eight rows that
// are read at once lie in different banks.
template <int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM * WN * 64)
matmul_i8_kernel(const I8Product p)
{
    constexpr int BK = 128, THREADS = WM * WN * 64, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    constexpr int PA = BM * 8 / THREADS, PB = BN * 8 / THREADS;
    __shared__ v4i lds[2][(BM + BN) * 8];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
    const int tiles_n = (p.n + BN - 1) / BN;
    const int m0 = int(blockIdx.x / unsigned(tiles_n)) * BM, n0 = int(blockIdx.x % unsigned(tiles_n)) * BN;
    const int wm = (wave / WN) * TM, wn = (wave % WN) * TN;

    v4i ra[PA], rb[PB];
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int at = i * THREADS + tid, row = min(m0 + at / 8, p.m - 1);
            ra[i] = load16(p.a + int64_t(row) * p.lda, k0 + (at & 7) * 16, p.k);
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int at = i * THREADS + tid, row = min(n0 + at / 8, p.n - 1);
            rb[i] = load16(p.b + int64_t(row) * p.ldb, k0 + (at & 7) * 16, p.k);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int at = i * THREADS + tid, row = at / 8;
            lds[buf][row * 8 + ((at & 7) ^ (row & 7))] = ra[i];
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int at = i * THREADS + tid, row = at / 8;
            lds[buf][BM * 8 + row * 8 + ((at & 7) ^ (row & 7))] = rb[i];
        }
    };
    v4i acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4i{0, 0, 0, 0};
    fetch(0);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int k0 = 0; k0 < p.k; k0 += BK, buf ^= 1) {
        const bool more = k0 + BK < p.k;
        if (more) fetch(k0 + BK);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            v4i a[MT], b[NT];
            const int piece = kk * 4 + (lane >> 4);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int row = wm + i * 16 + (lane & 15);
                a[i] = lds[buf][row * 8 + (piece ^ (row & 7))];
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int row = wn + j * 16 + (lane & 15);
                b[j] = lds[buf][BM * 8 + row * 8 + (piece ^ (row & 7))];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[j], a[i], acc[i][j], 0, 0, 0);
        }
        if (more) store(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            finish(p, m0 + wm + i * 16 + (lane & 15), n0 + wn + j * 16 + (lane >> 4) * 4, acc[i][j], true);
}

// Few rows: 16 channels a workgroup, whose waves share the length of k in steps of 256 bytes and add their sums in LDS.
template <int MT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64)
matmul_i8_rows_kernel(const I8Product p)
{
    __shared__ v4i lds[WAVES][MT][64];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int n0 = int(blockIdx.x) * 16;
    const int8_t *b = p.b + int64_t(min(n0 + (lane & 15), p.n - 1)) * p.ldb;
    const int8_t *a[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = p.a + int64_t(min(i * 16 + (lane & 15), p.m - 1)) * p.lda;
    v4i acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4i{0, 0, 0, 0};
    for (int k0 = wave * 256; k0 < p.k; k0 += WAVES * 256) {
        v4i vb[4], va[4][MT];
        const int at = k0 + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            vb[s] = load16(b, at + s * 64, p.k);
#pragma unroll
            for (int i = 0; i < MT; ++i) va[s][i] = load16(a[i], at + s * 64, p.k);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[s], va[s][i], acc[i], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) lds[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MT; i += WAVES) {
        v4i s = lds[0][i][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += lds[w][i][lane];
        finish(p, i * 16 + (lane & 15), n0 + (lane >> 4) * 4, s, true);
    }
}

}  // namespace

int launch_quantize_rows(const void *x, int64_t ldx, int bf16, int64_t rows, int64_t cols, int8_t *q, int64_t ldq,
                         int64_t q_cols, float *scale, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t vecs = (q_cols + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4);
#define PCONV_LAUNCH(TPR, THREADS)                                                                                             \
    do {                                                                                                                       \
        const unsigned grid = unsigned(std::min<int64_t>((rows + (THREADS / TPR) - 1) / (THREADS / TPR), 1 << 20));            \
        if (bf16) hipLaunchKernelGGL((quantize_rows_kernel<__bf16, TPR, THREADS>), dim3(grid), dim3(THREADS), 0, st,           \
                                     static_cast<const __bf16 *>(x), ldx, rows, cols, q, ldq, q_cols, scale);                  \
        else hipLaunchKernelGGL((quantize_rows_kernel<float, TPR, THREADS>), dim3(grid), dim3(THREADS), 0, st,                 \
                                static_cast<const float *>(x), ldx, rows, cols, q, ldq, q_cols, scale);                        \
    } while (0)
    if (vecs <= 8) PCONV_LAUNCH(8, 256);
    else if (vecs <= 64) PCONV_LAUNCH(16, 256);
    else if (vecs <= 256) PCONV_LAUNCH(64, 256);
    else if (vecs <= 2048) PCONV_LAUNCH(256, 256);
    else PCONV_LAUNCH(1024, 1024);
#undef PCONV_LAUNCH
    return check_launch("pconv_quantize_rows");
}

int launch_matmul_i8(const I8Product &p, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (p.m <= 64) {
        const unsigned grid = unsigned((p.n + 15) / 16);
        if (p.m <= 16) hipLaunchKernelGGL((matmul_i8_rows_kernel<1, 8>), dim3(grid), dim3(512), 0, st, p);
        else if (p.m <= 32) hipLaunchKernelGGL((matmul_i8_rows_kernel<2, 8>), dim3(grid), dim3(512), 0, st, p);
        else hipLaunchKernelGGL((matmul_i8_rows_kernel<4, 8>), dim3(grid), dim3(512), 0, st, p);
        return check_launch("pconv_matmul_i8 (few rows)");
    }
    const int64_t tiles = ((int64_t(p.m) + 127) / 128) * ((int64_t(p.n) + 127) / 128);
    if (tiles >= int64_t(1) << 24) { set_error("pconv_matmul_i8: too many workgroups"); return PCONV_UNSUPPORTED; }
    hipLaunchKernelGGL((matmul_i8_kernel<128, 128, 2, 2>), dim3(unsigned(tiles)), dim3(256), 0, st, p);
    return check_launch("pconv_matmul_i8");
}

}  // namespace pconv
