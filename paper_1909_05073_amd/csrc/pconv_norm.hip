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

template <typename T, bool PASSING>
__device__ __forceinline__ Vec<T> load_vector(const T *row, int k)
{
    v4i w;
    if constexpr (PASSING) w = load_passing<v4i>(row + int64_t(k) * Vec<T>::N);
    else __builtin_memcpy(&w, row + int64_t(k) * Vec<T>::N, 16);
    Vec<T> v;
    __builtin_memcpy(&v, &w, 16);
    return v;
}

template <typename T>
__device__ __forceinline__ Values<Vec<T>::N> sums_of(const Vec<T> &x, const Vec<T> &r, bool add)
{
    Values<Vec<T>::N> s;
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) s.v[i] = add ? x.at(i) + r.at(i) : x.at(i);
    return s;
}

// The vector k of a row of sums (r: or null).
template <typename T, bool PASSING = false>
__device__ __forceinline__ Values<Vec<T>::N> load_sums(const T *x, const T *r, int k)
{
    const Vec<T> a = load_vector<T, PASSING>(x, k);
    return sums_of(a, r ? load_vector<T, PASSING>(r, k) : a, r != nullptr);
}

template <typename T>
__device__ __forceinline__ void store_sums(const Values<Vec<T>::N> &s, T *row, int k)
{
    constexpr int N = Vec<T>::N;
    T w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = T(s.v[i]);
    __builtin_memcpy(row + int64_t(k) * N, w, sizeof(w));
}

// The row's factor 1 / sqrt(mean + eps), taken in two parts where the values are so large that it would be a denormal number.
struct Factor { float lift, inv; };

__device__ __forceinline__ Factor factor_of(double squares, double count, float eps)
{
    const double mean = squares / count + double(eps);
    Factor f;
    f.lift = mean > 0x1p200 ? 0x1p-64f : 1.0f;
    f.inv = float(1.0 / (sqrt(mean) * double(f.lift)));
    return f;
}

// s becomes h.
template <int N>
__device__ __forceinline__ void normalise(Values<N> &s, const Factor &f, const float *__restrict__ weight, int k)
{
    if (weight) {
        float w[N];
        __builtin_memcpy(w, weight + int64_t(k) * N, sizeof(w));
#pragma unroll
        for (int i = 0; i < N; ++i) s.v[i] = s.v[i] * f.lift * f.inv * w[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s.v[i] = s.v[i] * f.lift * f.inv;
    }
}

template <int N>
__device__ __forceinline__ uint32_t most_of_values(const Values<N> &s, uint32_t most)
{
#pragma unroll
    for (int i = 0; i < N; ++i) most = max(most, __float_as_uint(s.v[i]) & 0x7FFFFFFFu);
    return most;
}

template <bool LIFT, int N>
__device__ __forceinline__ void quantize_values(const Values<N> &s, const RowScale &r, uint32_t (&w)[N / 4])
{
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = quantize<LIFT>(s.v[4 * j + i], r);
        w[j] = (__builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u) | __builtin_amdgcn_perm(q[3], q[2], 0x04000C0Cu)) & r.mask;
    }
}

template <int N>
__device__ __forceinline__ void store_quantized(const Values<N> &s, const RowScale &r, int8_t *row, int k)
{
    uint32_t w[N / 4];
    if (__builtin_expect(r.lifts, 0)) quantize_values<true>(s, r, w);
    else quantize_values<false>(s, r, w);
    __builtin_memcpy(row + int64_t(k) * N, w, N);
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
// quantised, and reads what lies beyond three times (from a cache).  The elements behind the last whole vector go to a
// thread each (one that has up to a vector of them, and loops, takes 2111x4099 fp32 from 13 to 41 us).  Squares are summed
// in 64 bits, which no row of fp32 numbers leaves.  `sum` may be x or r: a thread has read what it overwrites.  Bound by
// memory: 100352x256 bf16 with sums 34.5 us, 5.2 TB/s.
template <typename T, int TPR, int KEEP, int THREADS, bool PASSING>
__global__ void __launch_bounds__(THREADS)
add_rms_norm_i8_kernel(const NormRows p, const T *x, const T *r, T *sum)
{
    constexpr int N = Vec<T>::N, RPW = THREADS / TPR, WAVES = THREADS / 64;
    __shared__ double squares_of[WAVES];
    __shared__ uint32_t most_of_wave[WAVES];
    const int sub = int(threadIdx.x) % TPR;
    const int whole = int(p.cols / N), rest = int(p.cols % N);
    const bool tail = sub < rest;
    // (of rows without a whole vector no weight is read but their elements'; elsewhere threads beyond a row's vectors, whose values
    // are zeros, read its last one)
    const float *const weight = whole > 0 ? p.weight : nullptr;
    const int64_t at_tail = int64_t(whole) * N + sub, groups = (p.rows + RPW - 1) / RPW;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t row = g * RPW + int(threadIdx.x) / TPR;
        const bool live = row < p.rows;
        const int64_t at_row = live ? row : p.rows - 1;
        const T *const xr = x + at_row * p.ldx, *const rr = r ? r + at_row * p.ldr : nullptr;
        T *const sr = sum + (sum ? at_row * p.ldsum : 0);
        Values<N> s[KEEP];
        double squares = 0;
        const auto add_squares = [&](const Values<N> &v) {
#pragma unroll
            for (int i = 0; i < N; ++i) squares = __builtin_fma(double(v.v[i]), double(v.v[i]), squares);
        };
        if constexpr (THREADS < 1024) {
            // (all loads first: with the sums between them they are waited for one by one, 100352x256 bf16 42.2 us for 34.5; 1024
            // threads have no registers for that, 1000x25088 fp32 79 us for 120)
            const v4i none = {0, 0, 0, 0};
            Vec<T> vx[KEEP], vr[KEEP];
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                __builtin_memcpy(&vx[i], &none, 16);
                if (i * TPR + sub < whole) vx[i] = load_vector<T, PASSING>(xr, i * TPR + sub);
            }
            if (rr) {
#pragma unroll
                for (int i = 0; i < KEEP; ++i) {
                    __builtin_memcpy(&vr[i], &none, 16);
                    if (i * TPR + sub < whole) vr[i] = load_vector<T, PASSING>(rr, i * TPR + sub);
                }
            }
#pragma unroll
            for (int i = 0; i < KEEP; ++i) s[i] = sums_of(vx[i], vr[i], rr != nullptr);
        } else {
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                if (i * TPR + sub < whole) {
                    s[i] = load_sums<T, PASSING>(xr, rr, i * TPR + sub);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) s[i].v[e] = 0.0f;
                }
            }
        }
        float last = 0.0f;
        if (tail) last = float(xr[at_tail]) + (rr ? float(rr[at_tail]) : 0.0f);
#pragma unroll
        for (int i = 0; i < KEEP; ++i) add_squares(s[i]);
        for (int k = KEEP * TPR + sub; k < whole; k += TPR) add_squares(load_sums(xr, rr, k));
        squares = __builtin_fma(double(last), double(last), squares);
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
            for (int i = 0; i < KEEP; ++i)
                if (i * TPR + sub < whole) store_sums(s[i], sr, i * TPR + sub);
            if (tail) sr[at_tail] = T(last);
        }
        const Factor f = factor_of(squares, double(max(p.cols, int64_t(1))), p.eps);
        last = last * f.lift * f.inv * (tail && p.weight ? p.weight[at_tail] : 1.0f);
        uint32_t most = __float_as_uint(last) & 0x7FFFFFFFu;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            normalise(s[i], f, weight, min(i * TPR + sub, max(whole - 1, 0)));
            most = most_of_values(s[i], most);
        }
        for (int k = KEEP * TPR + sub; k < whole; k += TPR) {
            Values<N> v = load_sums(xr, rr, k);
            normalise(v, f, weight, k);
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
        for (int i = 0; i < KEEP; ++i)
            if (i * TPR + sub < whole) store_quantized(s[i], scale, q, i * TPR + sub);
        for (int k = KEEP * TPR + sub; k < whole; k += TPR) {
            Values<N> v = load_sums(xr, rr, k);
            if (sum) store_sums(v, sr, k);
            normalise(v, f, weight, k);
            store_quantized(v, scale, q, k);
        }
        if (tail) q[at_tail] = int8_t((scale.lifts ? quantize<true>(last, scale) : quantize<false>(last, scale)) & scale.mask);
        if (sub == 0) p.scale[row] = scale.scale;
    }
}

template <typename T>
void launch_norm(const NormRows &p, hipStream_t st)
{
    const int64_t vecs = p.cols / Vec<T>::N;
#define PCONV_LAUNCH_AS(TPR, KEEP, THREADS, PASSING)                                                                           \
    hipLaunchKernelGGL((add_rms_norm_i8_kernel<T, TPR, KEEP, THREADS, PASSING>),                                               \
                       dim3(unsigned(std::min<int64_t>((p.rows + (THREADS / TPR) - 1) / (THREADS / TPR), 1 << 20))), dim3(THREADS), 0, st, p,  \
                       static_cast<const T *>(p.x), static_cast<const T *>(p.r), static_cast<T *>(p.sum))
#define PCONV_LAUNCH(TPR, KEEP, THREADS)                                                                                       \
    do {                                                                                                                       \
        if (passing && vecs <= TPR * KEEP) PCONV_LAUNCH_AS(TPR, KEEP, THREADS, true); else PCONV_LAUNCH_AS(TPR, KEEP, THREADS, false); \
    } while (0)
    // What is read once and is most of the memory-side cache is read past it (100352x256 fp32, 196 MB: 65.6 us without, 59.0;
    // bf16, 98 MB, of which the cache still holds a part: 38.2 and 42.4).
    const bool passing = p.rows * p.cols * int64_t(sizeof(T)) * (p.r ? 2 : 1) > int64_t(160) << 20;
    if (vecs <= 8) PCONV_LAUNCH(8, 1, 256);
    else if (vecs <= 16) PCONV_LAUNCH(16, 1, 256);
    else if (vecs <= 32) PCONV_LAUNCH(16, 2, 256);
    else if (vecs <= 64) PCONV_LAUNCH(32, 2, 256);
    else if (vecs <= 128) PCONV_LAUNCH(64, 2, 256);
    else if (vecs <= 256) PCONV_LAUNCH(64, 4, 256);
    else if (vecs <= 512) PCONV_LAUNCH(256, 2, 256);
    else if (vecs <= 1024) PCONV_LAUNCH(256, 4, 256);                    // (4000x4096 fp32 and a layer behind it 32.6 us; by 128 threads 35.8, by 512 39.0)
    else if (vecs <= 2048) PCONV_LAUNCH(512, 4, 512);
    else if (vecs <= 4096) PCONV_LAUNCH(512, 8, 512);                    // (by 1024 threads, four vectors each: 2000x25088 bf16 90 us for 82)
    else PCONV_LAUNCH(1024, 32 / Vec<T>::N, 1024);
#undef PCONV_LAUNCH
#undef PCONV_LAUNCH_AS
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
