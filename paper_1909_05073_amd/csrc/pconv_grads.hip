// The norm of the gradients of many tensors together, and their scaling where it passes a limit.
//
// norm = sqrt(sum g^2), out = g * min(1, max_norm / (norm + eps)).  Two passes, because no element can be scaled
// before the last one is summed; both are bound by memory (three operations an element).  A launch takes the tensors'
// addresses in its arguments, so a step needs no table in device memory.  The tensors are cut into chunks; the
// workgroups of the first pass take every gridDim-th chunk, those of the second one chunk each.
//
// Up to 128 MB of elements and outputs are left in the caches (87 MB 25.9 us, 28 with stores past them; 216 MB 73 and
// 60).  Of more, the first pass reads past the caches all but the last 192 MB, which the second pass, from the last
// chunk to the first, finds in the 256 MB memory-side cache; its stores pass the caches too.  138 million fp32
// elements: first pass 86 us (6.4 TB/s; 129 where the caches were left full of outputs), second 190 us (206 with
// nothing kept).
#include <hip/hip_runtime.h>

#include "pconv_internal.h"
#include "pconv_ops.h"

namespace pconv {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;

struct Chunk { const void *in; void *out; uint32_t n; int types; bool passing; };

// Which tensor a chunk belongs to: every lane compares the starts of three, which costs one access instead of a search's eight.
__device__ __forceinline__ Chunk find_chunk(const GradTable &t, uint32_t c)
{
    const int lane = int(threadIdx.x) & 63;
    int at = -1;
    for (int i = 0; i < t.count; i += 64)
        at += __popcll(__ballot(i + lane < t.count && t.start[min(i + lane, t.count - 1)] <= c));
    at = __builtin_amdgcn_readfirstlane(at);
    const uint32_t next = at + 1 < t.count ? t.start[at + 1] : t.chunks;
    const int types = t.types[at];
    const int64_t off = int64_t(c - t.start[at]) << t.log2;
    Chunk r;
    r.in = static_cast<const char *>(t.in[at]) + off * (types & 1 ? 2 : 4);
    r.out = t.out[at] ? static_cast<char *>(t.out[at]) + off * (types & 2 ? 2 : 4) : nullptr;
    r.n = c + 1 == next ? uint32_t(t.last[at]) + 1u : 1u << t.log2;
    r.types = types;
    r.passing = c < t.passing;
    return r;
}

// Sum over the workgroup in a fixed order; every thread gets it.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double *lds)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if (THREADS == 64) return v;
    __syncthreads();                                     // (lds may still be read from the sum before)
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
    return s;
}

// Vectors that are aligned to their elements only.  PASSING: they leave no trace in the caches.
template <bool PASSING, typename V, typename E>
__device__ __forceinline__ V load_at(const E *p)
{
    typedef V Fit __attribute__((aligned(sizeof(E))));
    if constexpr (PASSING) {
        return __builtin_nontemporal_load(reinterpret_cast<const Fit *>(p));
    } else {
        V v;
        __builtin_memcpy(&v, p, sizeof(V));
        return v;
    }
}

template <bool PASSING, typename V, typename E>
__device__ __forceinline__ void store_at(E *p, V v)
{
    typedef V Fit __attribute__((aligned(sizeof(E))));
    if constexpr (PASSING) __builtin_nontemporal_store(v, reinterpret_cast<Fit *>(p));
    else __builtin_memcpy(p, &v, sizeof(V));
}

// Squares are formed and summed in fp64: exact up to the sum's rounding, and no fp32 gradient overflows it.  AT_ONCE
// vectors of 16 bytes are under way together.
template <int THREADS, typename V, typename E, bool PASSING>
__device__ __forceinline__ double sum_squares(const E *p, uint32_t n, uint32_t tid)
{
    constexpr int N = 16 / sizeof(E), AT_ONCE = 8;
    double s0 = 0, s1 = 0;
    const uint32_t full = n / N;
    uint32_t i = tid;
    for (; i + (AT_ONCE - 1) * THREADS < full; i += AT_ONCE * THREADS) {
        V v[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) v[u] = load_at<PASSING, V>(p + size_t(i + u * THREADS) * N);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const double x = double(float(v[u][j])), y = double(float(v[u][j + 1]));
                s0 += x * x; s1 += y * y;
            }
    }
#pragma unroll 4
    for (; i < full; i += THREADS) {
        const V v = load_at<PASSING, V>(p + size_t(i) * N);
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            const double x = double(float(v[j])), y = double(float(v[j + 1]));
            s0 += x * x; s1 += y * y;
        }
    }
    for (uint32_t k = full * N + tid; k < n; k += THREADS) { const double x = double(float(p[k])); s0 += x * x; }
    return s0 + s1;
}

template <int THREADS>
__device__ __forceinline__ double chunk_squares(const Chunk &c, uint32_t tid)
{
    if (c.types & 1) {
        const __bf16 *p = static_cast<const __bf16 *>(c.in);
        return c.passing ? sum_squares<THREADS, b8, __bf16, true>(p, c.n, tid) : sum_squares<THREADS, b8, __bf16, false>(p, c.n, tid);
    }
    const float *p = static_cast<const float *>(c.in);
    return c.passing ? sum_squares<THREADS, f4, float, true>(p, c.n, tid) : sum_squares<THREADS, f4, float, false>(p, c.n, tid);
}

// The factor is first * then.  A norm near or beyond the largest fp32 number makes a factor that fp32 holds in few bits or not
// at all; 2^-64 of it is taken first then (exactly, unless the result is as good as 0).
struct Factor { float first, then; };

__device__ __forceinline__ Factor factor_of(double total, float max_norm, float eps)
{
    const double least = sqrt(total) + double(eps);
    // (also for an infinite norm and limit and for 0 and 0, whose quotients are no numbers; a norm that is NaN goes on)
    if (double(max_norm) >= least) return Factor{1.0f, 1.0f};
    const double f = double(max_norm) / least;
    if (f < 0x1p-100) return Factor{0x1p-64f, float(f * 0x1p64)};
    return Factor{1.0f, float(f)};
}

// 16 bytes of the wider type at a time: a wave's stores are whole lines.
template <int THREADS, typename E, typename O, bool PASSING>
__device__ __forceinline__ void scale(const E *p, O *q, uint32_t n, Factor f, uint32_t tid)
{
    constexpr int N = 16 / (sizeof(E) > sizeof(O) ? sizeof(E) : sizeof(O)), AT_ONCE = 8;
    typedef E VE __attribute__((ext_vector_type(N)));
    typedef O VO __attribute__((ext_vector_type(N)));
    typedef float VF __attribute__((ext_vector_type(N)));
    const uint32_t full = n / N;
    uint32_t i = tid;
    for (; i + (AT_ONCE - 1) * THREADS < full; i += AT_ONCE * THREADS) {
        VE v[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) v[u] = load_at<PASSING, VE>(p + size_t(i + u * THREADS) * N);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const VF w = __builtin_convertvector(v[u], VF) * f.first * f.then;
            store_at<PASSING>(q + size_t(i + u * THREADS) * N, __builtin_convertvector(w, VO));
        }
    }
#pragma unroll 2
    for (; i < full; i += THREADS) {
        const VF w = __builtin_convertvector(load_at<PASSING, VE>(p + size_t(i) * N), VF) * f.first * f.then;
        store_at<PASSING>(q + size_t(i) * N, __builtin_convertvector(w, VO));
    }
    for (uint32_t k = full * N + tid; k < n; k += THREADS) q[k] = O(float(p[k]) * f.first * f.then);
}

// out = in * factor.  Gradients scaled in place by exactly 1 stay as they are.
template <int THREADS, bool PASSING>
__device__ __forceinline__ void chunk_scale(const Chunk &c, Factor f, uint32_t tid)
{
    if (c.in == c.out && f.then == 1.0f && f.first == 1.0f) return;
    const __bf16 *pb = static_cast<const __bf16 *>(c.in); const float *pf = static_cast<const float *>(c.in);
    __bf16 *qb = static_cast<__bf16 *>(c.out); float *qf = static_cast<float *>(c.out);
    if (c.types == 0) scale<THREADS, float, float, PASSING>(pf, qf, c.n, f, tid);
    else if (c.types == 1) scale<THREADS, __bf16, float, PASSING>(pb, qf, c.n, f, tid);
    else if (c.types == 2) scale<THREADS, float, __bf16, PASSING>(pf, qb, c.n, f, tid);
    else scale<THREADS, __bf16, __bf16, PASSING>(pb, qb, c.n, f, tid);
}

__global__ void __launch_bounds__(kThreads)
grad_norm_kernel(const GradTable t, double *__restrict__ partials)
{
    __shared__ double lds[kThreads / 64];
    double s = 0;
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) s += chunk_squares<kThreads>(find_chunk(t, c), threadIdx.x);
    s = block_sum<kThreads>(s, lds);
    if (threadIdx.x == 0) partials[blockIdx.x] = s;
}

template <int THREADS>
__device__ __forceinline__ double total_of(const double *partials, uint32_t count, double *lds)
{
    double s = 0;
    for (uint32_t i = threadIdx.x; i < count; i += THREADS) s += partials[i];
    return block_sum<THREADS>(s, lds);
}

// One workgroup: the sum of all partial sums, and the norm.
__global__ void __launch_bounds__(kThreads)
grad_total_kernel(const double *__restrict__ partials, uint32_t count, double *total, float *norm)
{
    __shared__ double lds[kThreads / 64];
    const double s = total_of<kThreads>(partials, count, lds);
    if (threadIdx.x == 0) {
        total[0] = s;
        if (norm) norm[0] = float(sqrt(s));
    }
}

// The chunks from the last to the first: what the first pass read last is what the caches still hold.
template <bool PASSING>
__global__ void __launch_bounds__(kThreads)
grad_scale_kernel(const GradTable t, const double *__restrict__ partials, uint32_t count, float max_norm, float eps,
                  float *norm)
{
    __shared__ double lds[kThreads / 64];
    const double s = count > 1 ? total_of<kThreads>(partials, count, lds) : partials[0];
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = float(sqrt(s));
    const Factor f = factor_of(s, max_norm, eps);
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x)
        chunk_scale<kThreads, PASSING>(find_chunk(t, t.chunks - 1 - c), f, threadIdx.x);
}

// Few elements: one workgroup, whose waves take the chunks in turn, does both passes (2320 elements 4.7 us, two
// kernels 3.1 and 3.8).
__global__ void __launch_bounds__(1024)
grad_clip_one_kernel(const GradTable t, float max_norm, float eps, float *norm)
{
    __shared__ double lds[16];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double s = 0;
    for (uint32_t c = wave; c < t.chunks; c += 16) s += chunk_squares<64>(find_chunk(t, c), lane);
    s = block_sum<1024>(s, lds);
    if (threadIdx.x == 0) norm[0] = float(sqrt(s));
    const Factor f = factor_of(s, max_norm, eps);
    for (uint32_t c = wave; c < t.chunks; c += 16) chunk_scale<64, false>(find_chunk(t, c), f, lane);
}

int check_launch(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return PCONV_OK;
    set_error(std::string(what) + ": launch failed: " + hipGetErrorName(e));
    return PCONV_HIP_ERROR;
}

}  // namespace

int launch_grad_norm(const GradTable &t, unsigned blocks, double *partials, void *stream)
{
    hipLaunchKernelGGL(grad_norm_kernel, dim3(blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream), t, partials);
    return check_launch("gradients (sum of squares)");
}

int launch_grad_total(const double *partials, unsigned count, double *total, float *norm, void *stream)
{
    hipLaunchKernelGGL(grad_total_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), partials, count, total, norm);
    return check_launch("gradients (total)");
}

int launch_grad_scale(const GradTable &t, const double *partials, unsigned count, bool passing, float max_norm, float eps, float *norm,
                      void *stream)
{
    const dim3 grid(t.chunks < (1u << 20) ? t.chunks : 1u << 20);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (passing) hipLaunchKernelGGL(grad_scale_kernel<true>, grid, dim3(kThreads), 0, st, t, partials, count, max_norm, eps, norm);
    else hipLaunchKernelGGL(grad_scale_kernel<false>, grid, dim3(kThreads), 0, st, t, partials, count, max_norm, eps, norm);
    return check_launch("gradients (scaling)");
}

int launch_grad_clip_one(const GradTable &t, float max_norm, float eps, float *norm, void *stream)
{
    hipLaunchKernelGGL(grad_clip_one_kernel, dim3(1), dim3(1024), 0, static_cast<hipStream_t>(stream), t, max_norm, eps, norm);
    return check_launch("gradients (one workgroup)");
}

}  // namespace pconv
