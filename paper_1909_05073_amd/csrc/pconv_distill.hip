// Distillation from a teacher's largest logits: the loss of each row, and its gradient.
//
//   p[j]  = softmax over the row's entries of teacher[j] / T          lse = log sum_v exp(student[v] / T)
//   loss  = T^2 sum_j p[j] (log p[j] - (student[c[j]] / T - lse))
//   grad[v] = f T (exp(student[v] / T - lse) - sum_(j: c[j] = v) p[j])
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "pconv_internal.h"
#include "pconv_ops.h"
#include "pconv_rows.h"

// (loss and gradient have the same bits whichever call gives them: nothing is contracted but what is written as a fused product)
#pragma clang fp contract(off)

namespace pconv {

namespace {

constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float quick_exp(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// e^x: the exponent's rounding is taken back, which would be |x| / 2 steps of the result.
__device__ __forceinline__ float exp_of(float x)
{
    const float t = x * kLog2E, e = __builtin_amdgcn_exp2f(t), r = __builtin_fmaf(x, kLog2E, -t) * kLn2;
    return e > 0.0f ? __builtin_fmaf(e, r, e) : e;       // (0 of -infinity; a NaN)
}

// A logarithm b as an exponent of 2, and the power of two by which that exponent was rounded: e^(x - b) is scale 2^(x log2 e - hi).
struct Base {
    float hi, scale;
    __device__ __forceinline__ explicit Base(float b) : hi(b * kLog2E), scale(__builtin_amdgcn_exp2f(-__builtin_fmaf(b, kLog2E, -hi))) {}
};

// What all 64 lanes of a wave have together, in an order that depends on nothing; ADD: the sum, else the maximum.
template <bool ADD>
__device__ __forceinline__ float of_wave(float v)
{
    const auto join = [](float a, float b) { return ADD ? a + b : fmaxf(a, b); };
#define PCONV_OTHER(CTRL) __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(0, int(__float_as_uint(v)), CTRL, 0xF, 0xF, true)))
    v = join(v, PCONV_OTHER(0xB1));                      // the other of a pair
    v = join(v, PCONV_OTHER(0x4E));                      // the other pair of four
    v = join(v, PCONV_OTHER(0x141));                     // the other four of eight
    v = join(v, PCONV_OTHER(0x140));                     // the other eight of sixteen
#undef PCONV_OTHER
    v = join(v, __shfl_xor(v, 16));
    return join(v, __shfl_xor(v, 32));
}

// A running maximum and the sum of the exponentials of what is below it; nothing yet: -infinity and 0.
struct Running {
    float most, sum;

    // (values of -infinity add nothing, also where there is nothing else)
    __device__ __forceinline__ float base() const { return most == -INFINITY ? 0.0f : most; }
    __device__ __forceinline__ void join(const Running &o)
    {
        // (a maximum takes a NaN for nothing; the sums hand it on)
        const float m = fmaxf(most, o.most), b = m == -INFINITY ? 0.0f : m;
        sum = sum * quick_exp(most - b) + o.sum * quick_exp(o.most - b);
        most = m;
    }
    // (the maximum first: one exponential a lane instead of two at each step; 8192x1001 bf16 17.0 us -> 15.6)
    __device__ __forceinline__ void join_lanes()
    {
        const float mine = most;
        most = of_wave<false>(most);
        sum = of_wave<true>(sum * quick_exp(mine - base()));
    }
};

// What the TPR threads of a row, a wave or all of a workgroup, find together; their order depends on nothing.  `room`: a place
// for each wave, not read any more by a call before.
template <int TPR>
__device__ __forceinline__ void join_threads(Running &z, Running &t, Running (*room)[2])
{
    z.join_lanes();
    t.join_lanes();
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) {
            room[threadIdx.x >> 6][0] = z;
            room[threadIdx.x >> 6][1] = t;
        }
        __syncthreads();
        // (all maxima first: one exponential a wave, which do not wait for each other)
        const auto all = [&](int which) {
            Running r{room[0][which].most, 0.0f};
#pragma unroll
            for (int i = 1; i < TPR / 64; ++i) r.most = fmaxf(r.most, room[i][which].most);
            const float b = r.base();
#pragma unroll
            for (int i = 0; i < TPR / 64; ++i) r.sum += room[i][which].sum * quick_exp(room[i][which].most - b);
            return r;
        };
        z = all(0);
        t = all(1);
    }
}

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

// Vectors first, first + TPR, .. below `whole`, U of them; -infinity in the place of those that are not there.
template <typename T, int TPR, int U>
__device__ __forceinline__ void load_vectors(const T *z, int first, int whole, Vec<T> (&v)[U])
{
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int k = first + i * TPR;
        if (k < whole) {
            __builtin_memcpy(&v[i].v, z + int64_t(k) * Vec<T>::N, 16);
        } else {
#pragma unroll
            for (int e = 0; e < Vec<T>::N; ++e) v[i].v[e] = T(-INFINITY);
        }
    }
}

// Values stay as they came between their uses: without this bf16 ones are kept as floats too, and 32768 of a workgroup take 221
// registers.
template <typename T, int U>
__device__ __forceinline__ void keep_packed(Vec<T> (&v)[U])
{
#pragma unroll
    for (int i = 0; i < U; ++i) asm volatile("" : "+v"(v[i].v));
}

// e^(z / T - b) for a maximum or a sum b of such quotients; the caller multiplies by the scale of b's Base.  One fused product and one
// power of two: the exponent is rounded once, by what its difference from b is worth.  Where b is large (FAR) the quotient is rounded as
// b was: with a fused product what b came from differs from it by up to half a step, whose exponential is infinite from logits of
// 10^10 on, the type's lowest value among them, unless T is a power of two.  (Rounded always: 2000x50000 bf16 95.8 -> 101.2 us.)
struct Quotients {
    float inv_t, log2e_t;                                // 1 / T and log2(e) / T
    template <bool FAR>
    __device__ __forceinline__ float exp_less(float z, float b, const Base &base) const
    {
        return FAR ? __builtin_amdgcn_exp2f((z * inv_t - b) * kLog2E) : __builtin_amdgcn_exp2f(__builtin_fmaf(z, log2e_t, -base.hi));
    }
};

// Whether b is so in some thread of the wave (half a step of 2^20 is 2^-4).
__device__ __forceinline__ bool is_far(float b) { return __builtin_amdgcn_ballot_w64(fabsf(b) >= 0x1p20f) != 0; }

// The values of vectors, over T, join what a thread has found.
template <typename T, int U>
__device__ __forceinline__ void join_vectors(Running &r, Vec<T> (&v)[U], const Quotients &q)
{
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < Vec<T>::N; ++e) m = fmaxf(m, v[i].at(e));
    m = fmaxf(r.most, m * q.inv_t);
    const float b = m == -INFINITY ? 0.0f : m;
    r.sum *= quick_exp(r.most - b);
    keep_packed(v);
    const Base base(b);
    const auto sum_of = [&](auto far) {
        float sum = 0;
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int e = 0; e < Vec<T>::N; ++e) sum += q.exp_less<decltype(far)::value>(v[i].at(e), b, base);
        return sum;
    };
    if (__builtin_expect(is_far(b), 0)) r.sum += sum_of(std::true_type());
    else r.sum += sum_of(std::false_type()) * base.scale;
    r.most = m;
}

// LOSS: the loss and lse of each row; GRAD: its gradient, from lse where LOSS is false.  TPR threads share a row, which they
// read U vectors of 16 bytes a thread at a time; where both are computed the first U of each stay in registers from the
// sums to the gradient, and what lies beyond is read twice.  Bound by memory where rows are long and many: both of 4096x32768 bf16
// 117 us, 4.6 TB/s.  The entries' shares and classes lie in LDS.  The gradient is written as if there were no entries; behind a barrier the first
// entry that names a class writes it again with the shares of all that name it taken off.
template <typename T, int TPR, int U, bool LOSS, bool GRAD>
__global__ void __launch_bounds__(TPR == 64 ? 256 : TPR)
distill_kernel(const DistillRows p)
{
    // (four rows a workgroup where each has a wave; where there are barriers all threads share one)
    constexpr int N = Vec<T>::N, THREADS = TPR == 64 ? 256 : TPR, RPW = THREADS / TPR, WAVES = TPR / 64, E = TPR == 64 ? 2 : 1;
    extern __shared__ float entries[];
    __shared__ Running room[THREADS / 64][2];
    __shared__ float losses[THREADS / 64];
    const int sub = int(threadIdx.x) % TPR, of = int(threadIdx.x) / TPR;
    const int whole = p.v / N, rest = p.v % N;           // whole vectors of a row; the elements behind them go to a thread each
    const int fours = (p.top + 3) / 4;
    float *const share = entries + of * 12 * fours, *const at_class = share + 4 * fours;
    int *const cls = reinterpret_cast<int *>(at_class + 4 * fours);
    const Quotients quot{p.inv_t, p.log2e_t};
    const auto meet = [] {
        if constexpr (TPR > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        }
    };
    for (int64_t row = int64_t(blockIdx.x) * RPW + of; row < p.rows; row += int64_t(gridDim.x) * RPW) {
        const T *const z = static_cast<const T *>(p.z) + row * p.ldz;
        // Each thread's first entries are asked for all at once (rows of a wave with 78 entries 18.9 -> 11.6 us for 73x3341), and before the
        // row where one wave reads it (8192x4000 bf16 35.5 -> 33.8; behind it where there are more: 4096x32768 bf16 128.9 -> 127.6).
        Vec<T> v[U];
        if constexpr (TPR > 64) load_vectors<T, TPR, U>(z, sub, whole, v);
        int own[E];
        float asked[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int j = sub + e * TPR;
            own[e] = j < p.top ? class_at(p, row, j) : -1;
            asked[e] = j < p.top ? teacher_at(p, row, j) : -INFINITY;
        }
        if constexpr (TPR == 64) load_vectors<T, TPR, U>(z, sub, whole, v);
        const float last = sub < rest ? float(z[int64_t(whole) * N + sub]) : -INFINITY;
        Running t{-INFINITY, 0.0f}, r{-INFINITY, 0.0f};
        const auto enter = [&](int j, int c, float of_teacher) {
            const float x = c < 0 ? -INFINITY : of_teacher * p.inv_t;
            cls[j] = c;
            share[j] = x;
            if (c >= 0) at_class[j] = float(z[c]);
            t.join(Running{x, x == -INFINITY ? 0.0f : 1.0f});
        };
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (sub + e * TPR < 4 * fours) enter(sub + e * TPR, own[e], asked[e]);
        for (int j = sub + E * TPR; j < 4 * fours; j += TPR) {
            const int c = j < p.top ? class_at(p, row, j) : -1;
            enter(j, c, c < 0 ? 0.0f : teacher_at(p, row, j));
        }
        if constexpr (LOSS) {
            join_vectors<T, U>(r, v, quot);
            for (int k = U * TPR + sub; k < whole; k += U * TPR) {
                Vec<T> w[U];
                load_vectors<T, TPR, U>(z, k, whole, w);
                join_vectors<T, U>(r, w, quot);
            }
            if (sub < rest) r.join(Running{last * p.inv_t, last == -INFINITY ? 0.0f : 1.0f});
        }
        join_threads<TPR>(r, t, room + of * WAVES);
        const bool some = !(t.most == -INFINITY && t.sum == 0.0f);
        // (maxima and logarithms of sums stay apart where they can: together they are rounded to a step of the maximum)
        const float z_base = r.base(), z_log = LOSS ? __logf(r.sum) : 0.0f, lse = LOSS ? z_base + z_log : p.lse[row];
        const float t_base = t.base(), t_log = LOSS ? __logf(t.sum) : 0.0f, t_inv = some ? 1.0f / t.sum : 0.0f;
        float loss = 0;
        for (int j = sub; j < 4 * fours; j += TPR) {
            const float below = share[j] - t_base, part = cls[j] >= 0 ? exp_of(below) * t_inv : 0.0f;
            // (a share that is 0, or too small for fp32, counts nothing, also where the student rules its class out)
            if (LOSS && part != 0.0f) loss += part * ((below - t_log) - ((at_class[j] * p.inv_t - z_base) - z_log));
            share[j] = part;
        }
        T *const out = static_cast<T *>(p.grad) + row * p.ldg;
        const float f = GRAD && some ? p.factor * (p.up ? p.up[row * p.up_step] : 1.0f) : 0.0f;
        const Base base(lse);
        if constexpr (GRAD) {
            const auto write_all = [&](auto far) {
                const float scaled = decltype(far)::value ? f : f * base.scale;
                const auto grad_of = [&](float x) { return some ? scaled * quot.exp_less<decltype(far)::value>(x, lse, base) : 0.0f; };
                const auto write = [&](const Vec<T> &x, int k) {
                    T w[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) w[i] = T(grad_of(x.at(i)));
                    if (k < whole) __builtin_memcpy(out + int64_t(k) * N, w, 16);
                };
                keep_packed(v);
#pragma unroll
                for (int i = 0; i < U; ++i) write(v[i], sub + i * TPR);
                for (int k = U * TPR + sub; k < whole; k += U * TPR) {
                    Vec<T> w[U];
                    load_vectors<T, TPR, U>(z, k, whole, w);
#pragma unroll
                    for (int i = 0; i < U; ++i) write(w[i], k + i * TPR);
                }
                if (sub < rest) out[int64_t(whole) * N + sub] = T(grad_of(last));
            };
            if (__builtin_expect(is_far(lse), 0)) write_all(std::true_type());
            else write_all(std::false_type());
        }
        if constexpr (LOSS) {
            loss = of_wave<true>(loss);
            if (TPR > 64 && (threadIdx.x & 63) == 0) losses[threadIdx.x >> 6] = loss;
        }
        // (the stores of the row are done before some of it is written again: a barrier alone waits for LDS only)
        if (GRAD) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        meet();
        if (LOSS && sub == 0) {
            if constexpr (TPR > 64) {
                loss = losses[0];
#pragma unroll
                for (int i = 1; i < WAVES; ++i) loss += losses[i];
            }
            p.loss[row] = some ? loss * p.t2 : 0.0f;
            if (p.lse) p.lse[row] = lse;
        }
        if constexpr (GRAD) {
            for (int j = sub; j < p.top && some; j += TPR) {
                const int c = cls[j];
                if (c < 0) continue;
                // (lists seldom name a class twice: how often is counted first, which takes half of the reads; 8192x300 with 128 entries
                // 40.9 -> 22.3 us together with the loads above)
                int named = 0;
#pragma unroll 4
                for (int i = 0; i < fours; ++i) {
                    const v4i others = reinterpret_cast<const v4i *>(cls)[i];
#pragma unroll
                    for (int q = 0; q < 4; ++q) named += others[q] == c ? 1 : 0;
                }
                bool first = true;
                float off = share[j];
                if (named > 1) {
                    off = 0;
                    for (int i = 0; i < fours; ++i) {
                        const v4i others = reinterpret_cast<const v4i *>(cls)[i];
                        const f4 shares = reinterpret_cast<const f4 *>(share)[i];
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (others[q] == c) {
                                first = first && 4 * i + q >= j;
                                off += shares[q];
                            }
                    }
                }
                if (first) out[c] = T(f * (exp_of(at_class[j] * p.inv_t - lse) - off));
            }
        }
        if (row + int64_t(gridDim.x) * RPW < p.rows) meet();             // (the entries are read)
    }
}

// The rows' losses together, in 64 bits and a fixed order.
__global__ void __launch_bounds__(1024)
distill_total_kernel(const float *__restrict__ loss, int64_t rows, double scale, float *total)
{
    __shared__ double room[16];
    double s = 0;
#pragma unroll 8
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
    const size_t lds = size_t((p.top + 3) / 4) * 48;
    const int64_t vecs = (int64_t(p.v) + Vec<T>::N - 1) / Vec<T>::N;
#define PCONV_LAUNCH(TPR, U)                                                                                                   \
    do {                                                                                                                       \
        constexpr int RPW = TPR == 64 ? 4 : 1;                                                                                 \
        hipLaunchKernelGGL((distill_kernel<T, TPR, U, LOSS, GRAD>), dim3(unsigned(std::min<int64_t>((p.rows + RPW - 1) / RPW, 1 << 20))),  \
                           dim3(RPW * TPR), RPW * lds, st, p);                                                                 \
    } while (0)
    // Loss and gradient have the same bits together and apart: the same threads a row for all, which decide in what order the entries'
    // shares and the logits are added.  More threads a row meet more
    // often than what they do in between is worth (8192x4000 bf16 38.4 us by 256, 34.7 by 64; 1999x10007 fp32 through autograd 59.8
    // by 512, 54.2 by 256; 4096x32768 bf16 171 by 1024, 116 by 512; 4x41829 16.2 by 1024, 14.6), fewer read more of a row
    // twice (4096x32768 133 by 256).  Eight vectors a thread keep longer rows, but take as long where the last are missing
    // (4096 vectors a row 125 us by four, 116 by eight; 3750 of them 106.1 by four, 107.5 by eight).
    if constexpr (LOSS) {
        if (vecs <= 64 * 2) PCONV_LAUNCH(64, 2);
        else if (vecs <= 64 * 4) PCONV_LAUNCH(64, 4);
        else if (vecs <= 64 * 8) PCONV_LAUNCH(64, 8);
        else if (vecs <= 256 * 4) PCONV_LAUNCH(256, 4);
        else if (vecs <= 256 * 10) PCONV_LAUNCH(256, 8);
        else if (vecs <= 512 * 15 / 2) PCONV_LAUNCH(512, 4);
        else PCONV_LAUNCH(512, 8);
    } else {
        if (vecs <= 64 * 8) PCONV_LAUNCH(64, 4);
        else if (vecs <= 256 * 10) PCONV_LAUNCH(256, 4);
        else PCONV_LAUNCH(512, 4);
    }
#undef PCONV_LAUNCH
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
