// Rows of a residual stream: addition, root-mean-square norm, and quantising to 8-bit integers with a scale for each row.
//
//   s[k] = x[k] + r[k]      h[k] = s[k] / sqrt(mean_k s[k]^2 + eps) * weight[k]
//   scale = max_k |h[k]| / 127      q[k] = h[k] / scale, rounded
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pconv_internal.h"
#include "pconv_ops.h"
#include "pconv_rows.h"

namespace pconv {

namespace {

// N values of a row in 32 bits.
template <int N> struct Values { float v[N]; };

template <typename T>
__device__ __forceinline__ Values<Vec<T>::N> sums_of(const Vec<T> &x, const Vec<T> &r, bool add)
{
    Values<Vec<T>::N> s;
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) s.v[i] = add ? x.at(i) + r.at(i) : x.at(i);
    return s;
}

template <typename T>
__device__ __forceinline__ void store_sums(const Values<Vec<T>::N> &s, T *row, int64_t at, int64_t cols)
{
    constexpr int N = Vec<T>::N;
    T w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = T(s.v[i]);
    if (__builtin_expect(at + N <= cols, 1)) {
        __builtin_memcpy(row + at, w, sizeof(w));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + i < cols) row[at + i] = w[i];
    }
}

// The row's factor 1 / sqrt(mean + eps), taken in two parts where the values are so large that it would be a denormal number.
struct Factor { float lift, inv; };

__device__ __forceinline__ Factor factor_of(double squares, int64_t cols, float eps)
{
    const double mean = squares / double(max(cols, int64_t(1))) + double(eps);
    Factor f;
    f.lift = mean > 0x1p200 ? 0x1p-64f : 1.0f;
    f.inv = float(1.0 / (sqrt(mean) * double(f.lift)));
    return f;
}

// s becomes h.
template <int N>
__device__ __forceinline__ void normalise(Values<N> &s, const Factor &f, const float *__restrict__ weight, int64_t at, int64_t cols)
{
    float w[N];
    if (!weight) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 1.0f;
    } else if (__builtin_expect(at + N <= cols, 1)) {
        __builtin_memcpy(w, weight + at, sizeof(w));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = at + i < cols ? weight[at + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) s.v[i] = s.v[i] * f.lift * f.inv * w[i];
}

template <int N>
__device__ __forceinline__ uint32_t most_of_values(const Values<N> &s, uint32_t most)
{
#pragma unroll
    for (int i = 0; i < N; ++i) most = max(most, __float_as_uint(s.v[i]) & 0x7FFFFFFFu);
    return most;
}

template <int N>
__device__ __forceinline__ void store_quantized(const Values<N> &s, const RowScale &r, int8_t *row, int64_t at, int64_t q_cols)
{
    uint32_t w[N / 4];
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = __builtin_expect(r.lifts, 0) ? quantize<true>(s.v[4 * j + i], r) : quantize<false>(s.v[4 * j + i], r);
        w[j] = (__builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u) | __builtin_amdgcn_perm(q[3], q[2], 0x04000C0Cu)) & r.mask;
    }
    if (__builtin_expect(at + N <= q_cols, 1)) {
        __builtin_memcpy(row + at, w, N);
    } else if (__builtin_expect(at < q_cols, 0)) {
        uint64_t all = w[0];
        if (N == 8) all |= uint64_t(w[N / 4 - 1]) << 32;
#pragma unroll 1
        for (int64_t i = at; i < q_cols; ++i, all >>= 8) row[i] = int8_t(all);
    }
}

// The sum over the LANES (up to 64) neighbouring lanes that share a row, in an order that depends on nothing.
template <int LANES>
__device__ __forceinline__ double sum_of_lanes(double v)
{
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// TPR threads of a workgroup share a row; each keeps its first KEEP vectors of 16 bytes in registers as they are normalised and
// quantised, and reads what lies beyond three times (from a cache).  Squares are summed in 64 bits, which no row of fp32
// numbers leaves.  `sum` may be x or r: a thread has read what it overwrites.
template <typename T, int TPR, int KEEP, int THREADS>
__global__ void __launch_bounds__(THREADS)
add_rms_norm_i8_kernel(const NormRows p, const T *x, const T *r, T *sum)
{
    constexpr int N = Vec<T>::N, RPW = THREADS / TPR, WAVES = THREADS / 64;
    __shared__ double squares_of[WAVES];
    __shared__ uint32_t most_of_wave[WAVES];
    const int sub = int(threadIdx.x) % TPR;
    const bool add = r != nullptr;
    const int64_t groups = (p.rows + RPW - 1) / RPW;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t row = g * RPW + int(threadIdx.x) / TPR;
        const bool live = row < p.rows;
        const int64_t at_row = live ? row : p.rows - 1;
        const T *xr = x + at_row * p.ldx, *rr = add ? r + at_row * p.ldr : xr;
        T *sr = sum ? sum + at_row * p.ldsum : nullptr;
        Values<N> s[KEEP];
        double squares = 0;
        auto add_squares = [&](const Values<N> &v) {
#pragma unroll
            for (int i = 0; i < N; ++i) squares = __builtin_fma(double(v.v[i]), double(v.v[i]), squares);
        };
        {
            Vec<T> vx[KEEP], vr[KEEP];
            load_row<T, TPR, KEEP>(xr, sub, p.cols, vx);
            if (add) load_row<T, TPR, KEEP>(rr, sub, p.cols, vr);
#pragma unroll
            for (int i = 0; i < KEEP; ++i) s[i] = sums_of(vx[i], vr[i], add);
        }
        const auto sums_at = [&](int64_t at) {
            const Vec<T> vx = load_vec(xr, at, p.cols);
            return sums_of(vx, add ? load_vec(rr, at, p.cols) : vx, add);
        };
        constexpr int64_t BEYOND = int64_t(KEEP) * TPR * N;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) add_squares(s[i]);
        for (int64_t at = BEYOND + sub * N; at < p.cols; at += TPR * N) add_squares(sums_at(at));
        squares = sum_of_lanes<(TPR < 64 ? TPR : 64)>(squares);
        if (TPR > 64) {
            __syncthreads();                             // (those of the row before are read)
            if ((threadIdx.x & 63) == 0) squares_of[threadIdx.x >> 6] = squares;
            __syncthreads();
            squares = 0;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) squares += squares_of[i];
        }
        if (sum && live) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i) store_sums(s[i], sr, (int64_t(i) * TPR + sub) * N, p.cols);
        }
        const Factor f = factor_of(squares, p.cols, p.eps);
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            normalise(s[i], f, p.weight, (int64_t(i) * TPR + sub) * N, p.cols);
            most = most_of_values(s[i], most);
        }
        for (int64_t at = BEYOND + sub * N; at < p.cols; at += TPR * N) {
            Values<N> v = sums_at(at);
            normalise(v, f, p.weight, at, p.cols);
            most = most_of_values(v, most);
        }
        most = most_of_lanes<(TPR < 64 ? TPR : 64)>(most);
        if (TPR > 64) {
            if ((threadIdx.x & 63) == 0) most_of_wave[threadIdx.x >> 6] = most;
            __syncthreads();
            most = 0;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) most = max(most, most_of_wave[i]);
        }
        const RowScale scale = row_scale(most);
        if (!live) continue;
        int8_t *const q = p.q + row * p.ldq;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) store_quantized(s[i], scale, q, (int64_t(i) * TPR + sub) * N, p.cols);
        for (int64_t at = BEYOND + sub * N; at < p.cols; at += TPR * N) {
            Values<N> v = sums_at(at);
            if (sum) store_sums(v, sr, at, p.cols);
            normalise(v, f, p.weight, at, p.cols);
            store_quantized(v, scale, q, at, p.cols);
        }
        if (sub == 0) p.scale[row] = scale.scale;
    }
}

template <typename T>
void launch_norm(const NormRows &p, hipStream_t st)
{
    const int64_t vecs = (p.cols + Vec<T>::N - 1) / Vec<T>::N;
#define PCONV_LAUNCH(TPR, KEEP, THREADS)                                                                                       \
    hipLaunchKernelGGL((add_rms_norm_i8_kernel<T, TPR, KEEP, THREADS>),                                                        \
                       dim3(unsigned(std::min<int64_t>((p.rows + (THREADS / TPR) - 1) / (THREADS / TPR), 1 << 20))), dim3(THREADS), 0, st, p,  \
                       static_cast<const T *>(p.x), static_cast<const T *>(p.r), static_cast<T *>(p.sum))
    if (vecs <= 8) PCONV_LAUNCH(8, 1, 256);
    else if (vecs <= 16) PCONV_LAUNCH(16, 1, 256);
    else if (vecs <= 32) PCONV_LAUNCH(16, 2, 256);
    else if (vecs <= 64) PCONV_LAUNCH(32, 2, 256);
    else if (vecs <= 128) PCONV_LAUNCH(64, 2, 256);
    else if (vecs <= 256) PCONV_LAUNCH(64, 4, 256);
    else if (vecs <= 512) PCONV_LAUNCH(256, 2, 256);
    else if (vecs <= 1024) PCONV_LAUNCH(256, 4, 256);
    else if (vecs <= 2048) PCONV_LAUNCH(512, 4, 512);
    else PCONV_LAUNCH(1024, 4, 1024);
#undef PCONV_LAUNCH
}

}  // namespace

int launch_add_rms_norm_i8(const NormRows &p, int bf16, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (bf16) launch_norm<__bf16>(p, st);
    else launch_norm<float>(p, st);
    return check_launch("pconv_add_rms_norm_i8");
}

}  // namespace pconv
