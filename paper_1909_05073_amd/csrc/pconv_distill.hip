// Distillation from a teacher's largest logits: the loss of each row, and its gradient.
//
//   p[j]  = softmax over the row's entries of teacher[j] / T          lse = log sum_v exp(student[v] / T)
//   loss  = T^2 sum_j p[j] (log p[j] - (student[c[j]] / T - lse))
//   grad[v] = f T (exp(student[v] / T - lse) - sum_(j: c[j] = v) p[j])
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pconv_internal.h"
#include "pconv_ops.h"
#include "pconv_rows.h"

// (loss and gradient have the same bits whichever call gives them: nothing is contracted but what is written as a fused product)
#pragma clang fp contract(off)

namespace pconv {

namespace {

constexpr float kLog2E = 1.44269504088896340736f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// A running maximum and the sum of the exponentials of what is below it; nothing yet: -infinity and 0.
struct Running {
    float most, sum;

    // (values of -infinity add nothing, also where there is nothing else)
    __device__ __forceinline__ float base() const { return most == -INFINITY ? 0.0f : most; }
    __device__ __forceinline__ void join(const Running &o)
    {
        // (a maximum takes a NaN for nothing; the sums hand it on)
        const float m = fmaxf(most, o.most), b = m == -INFINITY ? 0.0f : m;
        sum = sum * exp_of(most - b) + o.sum * exp_of(o.most - b);
        most = m;
    }
};

// TPR threads that share a row: a wave, or all of a workgroup, which meets at barriers.
template <int TPR> struct Group {
    static constexpr int WAVES = TPR / 64;
    static __device__ __forceinline__ void meet()
    {
        if (TPR > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
    // (`room`: WAVES of them in LDS; nobody reads it any more when the next call begins if a meet() lies between)
    static __device__ __forceinline__ Running join(Running v, Running *room)
    {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) v.join(Running{__shfl_xor(v.most, d), __shfl_xor(v.sum, d)});
        if (TPR == 64) return v;
        if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
        __syncthreads();
        v = room[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v.join(room[i]);
        return v;
    }
    static __device__ __forceinline__ float add(float v, float *room)
    {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
        if (TPR == 64) return v;
        if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
        __syncthreads();
        v = room[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += room[i];
        return v;
    }
};

// What a row's entries leave in LDS, `top` of each.
struct Entries {
    float *p, *at;                                       // the teacher's logit over T; the student's at its class
    int *c;                                              // its class; -1: no entry
};

__device__ __forceinline__ float teacher_at(const DistillRows &p, int64_t row, int j)
{
    const int64_t at = row * p.ldt + j;
    return p.t_bf16 ? float(static_cast<const __bf16 *>(p.t)[at]) : static_cast<const float *>(p.t)[at];
}

__device__ __forceinline__ int class_at(const DistillRows &p, int64_t row, int j)
{
    const int64_t at = row * p.ldc + j;
    const int64_t c = p.c_wide ? static_cast<const int64_t *>(p.c)[at] : static_cast<const int32_t *>(p.c)[at];
    return c >= 0 && c < p.v ? int(c) : -1;
}

// The entries of a row; log of the sum that their shares were divided by goes to `log_sum` (with the maximum).  Returns whether
// the row has an entry that counts.
template <typename T, int TPR>
__device__ __forceinline__ bool read_entries(const DistillRows &p, const T *z, int64_t row, int sub, Entries e, Running *room, float &log_sum)
{
    Running r{-INFINITY, 0.0f};
    for (int j = sub; j < p.top; j += TPR) {
        const int c = class_at(p, row, j);
        const float t = c < 0 ? -INFINITY : teacher_at(p, row, j) * p.inv_t;
        e.c[j] = c;
        e.p[j] = t;
        e.at[j] = c < 0 ? 0.0f : float(z[c]);
        r.join(Running{t, t == -INFINITY ? 0.0f : 1.0f});
    }
    r = Group<TPR>::join(r, room);
    log_sum = r.base() + __logf(r.sum);
    const bool some = !(r.most == -INFINITY && r.sum == 0.0f);
    Group<TPR>::meet();
    return some;
}

template <typename T>
__device__ __forceinline__ void store_grads(const float (&g)[Vec<T>::N], T *row, int64_t at, int64_t cols)
{
    constexpr int N = Vec<T>::N;
    T w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = T(g[i]);
    if (__builtin_expect(at + N <= cols, 1)) {
        __builtin_memcpy(row + at, w, sizeof(w));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + i < cols) row[at + i] = w[i];
    }
}

// LOSS: the loss and lse of each row; GRAD: its gradient, from lse where LOSS is false.  TPR threads share a row, which is
// read again for the gradient; then the classes of the entries are written once more with their shares taken off, each by
// the first entry that names it.
template <typename T, int TPR, bool LOSS, bool GRAD>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR)
distill_kernel(const DistillRows p)
{
    constexpr int N = Vec<T>::N, THREADS = TPR < 256 ? 256 : TPR, RPW = THREADS / TPR;
    extern __shared__ float entries[];
    __shared__ Running room_r[2][THREADS / 64];
    __shared__ float room_f[THREADS / 64];
    const int sub = int(threadIdx.x) % TPR, of = int(threadIdx.x) / TPR;
    Entries e;
    e.p = entries + of * 3 * p.top;
    e.at = e.p + p.top;
    e.c = reinterpret_cast<int *>(e.at + p.top);
    for (int64_t row = int64_t(blockIdx.x) * RPW + of; row < p.rows; row += int64_t(gridDim.x) * RPW) {
        const T *const z = static_cast<const T *>(p.z) + row * p.ldz;
        float log_sum;
        const bool some = read_entries<T, TPR>(p, z, row, sub, e, room_r[0], log_sum);
        float lse;
        if constexpr (LOSS) {
            Running r{-INFINITY, 0.0f};
            for (int64_t at = int64_t(sub) * N; at < p.v; at += TPR * N) {
                const Vec<T> v = load_vec(z, at, p.v);
                float x[N], m = -INFINITY;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    x[i] = at + i < p.v ? v.at(i) * p.inv_t : -INFINITY;
                    m = fmaxf(m, x[i]);
                }
                const float b = fmaxf(m, r.most) == -INFINITY ? 0.0f : fmaxf(m, r.most);
                r.sum *= exp_of(r.most - b);
#pragma unroll
                for (int i = 0; i < N; ++i) r.sum += exp_of(x[i] - b);
                r.most = fmaxf(m, r.most);
            }
            r = Group<TPR>::join(r, room_r[1]);
            lse = r.base() + __logf(r.sum);
            float loss = 0;
            for (int j = sub; j < p.top; j += TPR) {
                const float lp = e.p[j] - log_sum;
                if (e.c[j] >= 0 && lp != -INFINITY) loss += exp_of(lp) * (lp - __builtin_fmaf(e.at[j], p.inv_t, -lse));
            }
            loss = Group<TPR>::add(loss, room_f);
            if (sub == 0) {
                p.loss[row] = some ? loss * p.t2 : 0.0f;
                if (p.lse) p.lse[row] = lse;
            }
        } else {
            lse = p.lse[row];
        }
        if constexpr (GRAD) {
            T *const out = static_cast<T *>(p.grad) + row * p.ldg;
            const float f = some ? p.factor * (p.up ? p.up[row * p.up_step] : 1.0f) : 0.0f;
            for (int64_t at = int64_t(sub) * N; at < p.v; at += TPR * N) {
                const Vec<T> v = load_vec(z, at, p.v);
                float g[N];
#pragma unroll
                for (int i = 0; i < N; ++i) g[i] = some ? f * exp_of(__builtin_fmaf(v.at(i), p.inv_t, -lse)) : 0.0f;
                store_grads<T>(g, out, at, p.v);
            }
            __threadfence_block();                       // (the stores of the row are done before some of it is written again)
            Group<TPR>::meet();
            for (int j = sub; j < p.top && some; j += TPR) {
                const int c = e.c[j];
                if (c < 0) continue;
                bool first = true;
                float share = 0;
                for (int i = 0; i < p.top; ++i)
                    if (e.c[i] == c) {
                        first = first && i >= j;
                        share += exp_of(e.p[i] - log_sum);
                    }
                if (first) out[c] = T(f * (exp_of(__builtin_fmaf(e.at[j], p.inv_t, -lse)) - share));
            }
        }
        Group<TPR>::meet();                              // (the entries are read)
    }
}

// The rows' losses together, in 64 bits and a fixed order.
__global__ void __launch_bounds__(1024)
distill_total_kernel(const float *__restrict__ loss, int64_t rows, double scale, float *total)
{
    __shared__ double room[16];
    double s = 0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) s += double(loss[i]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x) return;
    s = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += room[i];
    *total = float(s * scale);
}

template <typename T, bool LOSS, bool GRAD>
void launch_rows(const DistillRows &p, hipStream_t st)
{
    const size_t lds = size_t(p.top) * 12;
    const unsigned most = 1 << 20;
    if (p.v <= 4096) hipLaunchKernelGGL((distill_kernel<T, 64, LOSS, GRAD>), dim3(unsigned(std::min<int64_t>((p.rows + 3) / 4, most))), dim3(256), 4 * lds, st, p);
    else if (p.v <= 16384) hipLaunchKernelGGL((distill_kernel<T, 256, LOSS, GRAD>), dim3(unsigned(std::min<int64_t>(p.rows, most))), dim3(256), lds, st, p);
    else hipLaunchKernelGGL((distill_kernel<T, 1024, LOSS, GRAD>), dim3(unsigned(std::min<int64_t>(p.rows, most))), dim3(1024), lds, st, p);
}

}  // namespace

int launch_distill(const DistillRows &p, bool loss, bool grad, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
#define PCONV_LAUNCH(T)                                                                                                        \
    do {                                                                                                                       \
        if (loss && grad) launch_rows<T, true, true>(p, st);                                                                   \
        else if (loss) launch_rows<T, true, false>(p, st);                                                                     \
        else launch_rows<T, false, true>(p, st);                                                                               \
    } while (0)
    if (p.z_bf16) PCONV_LAUNCH(__bf16); else PCONV_LAUNCH(float);
#undef PCONV_LAUNCH
    return check_launch("pconv_distill");
}

int launch_distill_total(const float *loss, int64_t rows, double scale, float *total, void *stream)
{
    hipLaunchKernelGGL(distill_total_kernel, dim3(1), dim3(1024), 0, static_cast<hipStream_t>(stream), loss, rows, scale, total);
    return check_launch("pconv_distill (the rows' losses together)");
}

}  // namespace pconv
