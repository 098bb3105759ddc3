// The norm of the gradients of many tensors together, and their scaling where it passes a limit.
//
// norm = sqrt(sum g^2), out = g * min(1, max_norm / (norm + eps)).  Two passes, because no element can be scaled
// before the last one is summed; both are bound by memory (three operations an element).  A launch takes the
// tensors' addresses in its arguments, so a step needs no table in device memory.  The tensors are cut into chunks
// of kGradChunk elements (64 KiB in fp32) and a workgroup takes every gridDim-th chunk.
#include <hip/hip_runtime.h>

#include "pconv_internal.h"
#include "pconv_ops.h"

namespace pconv {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;

struct Chunk { const void *in; void *out; uint32_t n; int types; };

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
    const int64_t off = int64_t(c - t.start[at]) * kGradChunk;
    Chunk r;
    r.in = static_cast<const char *>(t.in[at]) + off * (types & 1 ? 2 : 4);
    r.out = t.out[at] ? static_cast<char *>(t.out[at]) + off * (types & 2 ? 2 : 4) : nullptr;
    r.n = c + 1 == next ? uint32_t(t.last[at]) + 1u : uint32_t(kGradChunk);
    r.types = types;
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

// Squares are formed and summed in fp64: exact up to the sum's rounding, and no fp32 gradient overflows it.
template <int THREADS>
__device__ __forceinline__ double chunk_squares(const Chunk &c)
{
    double s0 = 0, s1 = 0;
    if (c.types & 1) {
        const __bf16 *p = static_cast<const __bf16 *>(c.in);
        const uint32_t full = c.n / 8;
#pragma unroll 4
        for (uint32_t i = threadIdx.x; i < full; i += THREADS) {
            b8 v;
            __builtin_memcpy(&v, p + size_t(i) * 8, 16);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const double x = double(float(v[j])), y = double(float(v[j + 1]));
                s0 += x * x; s1 += y * y;
            }
        }
        for (uint32_t i = full * 8 + threadIdx.x; i < c.n; i += THREADS) { const double x = double(float(p[i])); s0 += x * x; }
    } else {
        const float *p = static_cast<const float *>(c.in);
        const uint32_t full = c.n / 4;
#pragma unroll 8
        for (uint32_t i = threadIdx.x; i < full; i += THREADS) {
            f4 v;
            __builtin_memcpy(&v, p + size_t(i) * 4, 16);
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const double x = double(v[j]), y = double(v[j + 1]);
                s0 += x * x; s1 += y * y;
            }
        }
        for (uint32_t i = full * 4 + threadIdx.x; i < c.n; i += THREADS) { const double x = double(p[i]); s0 += x * x; }
    }
    return s0 + s1;
}

// The factor is first * then.  A norm near or beyond the largest fp32 number makes a factor that fp32 holds in few bits or not
// at all; 2^-64 of it is taken first then (exactly, unless the result is as good as 0).
struct Factor { float first, then; };

__device__ __forceinline__ Factor factor_of(double total, float max_norm, float eps)
{
    const double f = double(max_norm) / (sqrt(total) + double(eps));
    // (0 / 0, a limit of zero and gradients of zero, is NaN as well: eps keeps it away)
    if (f >= 1.0) return Factor{1.0f, 1.0f};
    if (f < 0x1p-100) return Factor{0x1p-64f, float(f * 0x1p64)};
    return Factor{1.0f, float(f)};
}

// out = in * factor.  Gradients scaled in place by exactly 1 stay as they are.
template <int THREADS>
__device__ __forceinline__ void chunk_scale(const Chunk &c, Factor f)
{
    if (c.in == c.out && f.then == 1.0f && f.first == 1.0f) return;
    const uint32_t full = c.n / 4;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < full; i += THREADS) {
        f4 v;
        if (c.types & 1) {
            b4 w;
            __builtin_memcpy(&w, static_cast<const __bf16 *>(c.in) + size_t(i) * 4, 8);
            v = __builtin_convertvector(w, f4);
        } else {
            __builtin_memcpy(&v, static_cast<const float *>(c.in) + size_t(i) * 4, 16);
        }
        v = v * f.first * f.then;
        if (c.types & 2) {
            const b4 w = __builtin_convertvector(v, b4);
            __builtin_memcpy(static_cast<__bf16 *>(c.out) + size_t(i) * 4, &w, 8);
        } else {
            __builtin_memcpy(static_cast<float *>(c.out) + size_t(i) * 4, &v, 16);
        }
    }
    for (uint32_t i = full * 4 + threadIdx.x; i < c.n; i += THREADS) {
        const float v = (c.types & 1 ? float(static_cast<const __bf16 *>(c.in)[i]) : static_cast<const float *>(c.in)[i]) * f.first * f.then;
        if (c.types & 2) static_cast<__bf16 *>(c.out)[i] = __bf16(v);
        else static_cast<float *>(c.out)[i] = v;
    }
}

__global__ void __launch_bounds__(kThreads)
grad_norm_kernel(const GradTable t, double *__restrict__ partials)
{
    __shared__ double lds[kThreads / 64];
    double s = 0;
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) s += chunk_squares<kThreads>(find_chunk(t, c));
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

// One workgroup: the sum of all partial sums to total[0] (in its place, or behind the partials) and the norm.
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

// The chunks are walked from the last to the first: what the first pass read last is what the caches still hold.
__global__ void __launch_bounds__(kThreads)
grad_scale_kernel(const GradTable t, const double *__restrict__ partials, uint32_t count, float max_norm, float eps,
                  float *norm)
{
    __shared__ double lds[kThreads / 64];
    const double s = total_of<kThreads>(partials, count, lds);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = float(sqrt(s));
    const Factor f = factor_of(s, max_norm, eps);
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) chunk_scale<kThreads>(find_chunk(t, t.chunks - 1 - c), f);
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

int launch_grad_scale(const GradTable &t, unsigned blocks, const double *partials, unsigned count, float max_norm, float eps,
                      float *norm, void *stream)
{
    hipLaunchKernelGGL(grad_scale_kernel, dim3(blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream), t, partials, count,
                       max_norm, eps, norm);
    return check_launch("gradients (scaling)");
}

}  // namespace pconv
