// What the kernels over rows share: loads of rows that begin and end anywhere, the quantising of values to 8-bit integers, the
// staging of tiles, launches.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "pconv_internal.h"

namespace pconv {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint16_t u2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

// Workgroups of up to 512 threads that one dimension of a launch may have: fewer than 2^32 threads.
constexpr int64_t kMaxGroups = (int64_t(1) << 23) - 1;

inline int check_launch(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return PCONV_OK;
    set_error(std::string(what) + ": launch failed: " + hipGetErrorName(e));
    return PCONV_HIP_ERROR;
}

// ---- quantising rows ---------------------------------------------------------------------------------------------------

// The largest magnitude travels as the bits of |x|: ordered like the values, infinity above all numbers and NaN above it.
struct RowScale {
    float scale;                                         // what is handed out: NaN where the row holds an infinity or a NaN
    float step, inv, lift;                               // scale * lift, its reciprocal, and a power of two
    uint32_t mask;                                       // 0: all of the row is 0
    bool lifts;                                          // a row of the wave is lifted
};

__device__ __forceinline__ RowScale row_scale(uint32_t most)
{
    RowScale r;
    const bool bad = most >= 0x7F800000u;
    const float s = bad ? 0.0f : __uint_as_float(most) / 127.0f;
    r.scale = bad ? __uint_as_float(0x7FC00000u) : s;
    r.lift = s < 0x1p-60f ? 0x1p64f : 1.0f;
    r.step = s * r.lift;
    r.inv = s > 0.0f ? 1.0f / r.step : 0.0f;
    r.mask = s > 0.0f ? 0xFFFFFFFFu : 0u;
    r.lifts = __builtin_amdgcn_ballot_w64(s > 0.0f && s < 0x1p-60f) != 0;
    return r;
}

// The nearest whole number of the nearest fp32 number of x / scale, in the low byte.  The correctly rounded quotient comes
// from the correctly rounded reciprocal by two corrections with the exact remainder (Markstein, 1990): five operations for a
// division's eleven.  Adding 1.5 * 2^23 rounds to a whole number in the low bits, ties to even.
//
// LIFT, for waves that hold a row of small values: those rows are lifted by a power of two first, so that a remainder that
// decides is no denormal; a scale that is itself a denormal is rounded to few bits, and quotients that pass 127 are cut.
template <bool LIFT>
__device__ __forceinline__ uint32_t quantize(float x, const RowScale &r)
{
    if (LIFT) x *= r.lift;
    float t = x * r.inv;
    t = __builtin_fmaf(__builtin_fmaf(-t, r.step, x), r.inv, t);
    t = __builtin_fmaf(__builtin_fmaf(-t, r.step, x), r.inv, t);
    if (LIFT) t = __builtin_amdgcn_fmed3f(t, -127.0f, 127.0f);
    return __float_as_uint(t + 12582912.0f);
}

// 16 bytes of a row of activations
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    f4 v;
    __device__ __forceinline__ float at(int i) const { return v[i]; }
};
template <> struct Vec<__bf16> {
    static constexpr int N = 8;
    b8 v;
    __device__ __forceinline__ float at(int i) const { return float(v[i]); }
};

// (The bits of |x| as a float's; bf16 values two at a time.)
__device__ __forceinline__ uint32_t most_of(const Vec<float> &v, uint32_t most)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, __float_as_uint(v.v[i]) & 0x7FFFFFFFu);
    return most;
}

__device__ __forceinline__ uint32_t most_of(const Vec<__bf16> &v, uint32_t most)
{
    v4u w;
    __builtin_memcpy(&w, &v.v, 16);
    u2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u2, uint32_t(w[i] & 0x7FFF7FFFu)));
    return max(most, uint32_t(max(m.x, m.y)) << 16);
}

// The `size` (< 16) bytes that a row of `len` bytes has from `at` on, the rest zero: cut out of the row's last 16 bytes.
__device__ __forceinline__ v4i load_end(const void *row, int64_t at, int64_t len)
{
    uint64_t lo = 0, hi = 0;
    const uint8_t *p = static_cast<const uint8_t *>(row);
    if (len >= 16) {
        uint64_t w[2];
        __builtin_memcpy(w, p + len - 16, 16);
        const int bits = 8 * int(at + 16 - len);         // 8 .. 120
        lo = bits < 64 ? (w[0] >> bits) | (w[1] << (64 - bits)) : w[1] >> (bits - 64);
        hi = bits < 64 ? w[1] >> bits : 0;
    } else {
#pragma unroll 1
        for (int i = 0; i < int(len); ++i) {             // (at is 0)
            const uint64_t v = uint64_t(p[i]) << (8 * (i & 7));
            if (i < 8) lo |= v; else hi |= v;
        }
    }
    return v4i{int(lo), int(lo >> 32), int(hi), int(hi >> 32)};
}

// Elements [at, at + N) of a row of `cols`; beyond its end zero.
template <typename T>
__device__ __forceinline__ Vec<T> load_vec(const T *row, int64_t at, int64_t cols)
{
    v4i w = {0, 0, 0, 0};
    if (__builtin_expect(at + Vec<T>::N <= cols, 1)) __builtin_memcpy(&w, row + at, 16);
    else if (__builtin_expect(at < cols, 0)) w = load_end(row, at * int(sizeof(T)), cols * int(sizeof(T)));
    Vec<T> v;
    __builtin_memcpy(&v, &w, 16);
    return v;
}

// (A load that leaves no trace in the caches.)
template <typename V, typename E>
__device__ __forceinline__ V load_passing(const E *p)
{
    typedef V Fit __attribute__((aligned(sizeof(E))));
    return __builtin_nontemporal_load(reinterpret_cast<const Fit *>(p));
}

// The vectors sub, sub + LANES, .. of a row: KEEP of them.  (One piece of code for the row's end, not KEEP.)
template <typename T, int LANES, int KEEP, bool EXACT = false, bool PASSING = false>
__device__ __forceinline__ void load_row(const T *row, int sub, int64_t cols, Vec<T> (&v)[KEEP])
{
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t at = (int64_t(i) * LANES + sub) * N;
        v4i w = {0, 0, 0, 0};
        if (at + N <= cols) {
            if constexpr (PASSING) w = load_passing<v4i>(row + at);
            else __builtin_memcpy(&w, row + at, 16);
        }
        __builtin_memcpy(&v[i], &w, 16);
    }
    const int64_t last = cols / N;
    if (!EXACT && __builtin_expect(cols % N != 0, 0) && last < KEEP * LANES) {
        const v4i w = load_end(row, last * 16, cols * int(sizeof(T)));
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (i * LANES + sub == last) __builtin_memcpy(&v[i], &w, 16);
    }
}

template <bool LIFT, typename T>
__device__ __forceinline__ void quantize_as(const Vec<T> &v, const RowScale &r, uint32_t (&w)[Vec<T>::N / 4])
{
#pragma unroll
    for (int j = 0; j < Vec<T>::N / 4; ++j) {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = quantize<LIFT>(v.at(4 * j + i), r);
        w[j] = (__builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u) | __builtin_amdgcn_perm(q[3], q[2], 0x04000C0Cu)) & r.mask;
    }
}

template <typename T>
__device__ __forceinline__ void quantize_vec(const Vec<T> &v, const RowScale &r, uint32_t (&w)[Vec<T>::N / 4])
{
    if (__builtin_expect(r.lifts, 0)) quantize_as<true>(v, r, w);
    else quantize_as<false>(v, r, w);
}

// The same elements quantised, to a row of q_cols bytes.
template <typename T>
__device__ __forceinline__ void store_vec(const Vec<T> &v, const RowScale &r, int8_t *row, int64_t at, int64_t q_cols)
{
    constexpr int N = Vec<T>::N;
    uint32_t w[N / 4];
    quantize_vec(v, r, w);
    if (__builtin_expect(at + N <= q_cols, 1)) {
        __builtin_memcpy(row + at, w, N);
    } else if (__builtin_expect(at < q_cols, 0)) {
        uint64_t all = w[0];
        if (N == 8) all |= uint64_t(w[N / 4 - 1]) << 32;
#pragma unroll 1
        for (int64_t i = at; i < q_cols; ++i, all >>= 8) row[i] = int8_t(all);
    }
}

// The largest value over the 8 or 16 neighbouring lanes that share a row.
template <int LANES>
__device__ __forceinline__ uint32_t most_of_lanes(uint32_t v)
{
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xF, 0xF, true)));       // the other of a pair
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x4E, 0xF, 0xF, true)));       // the other pair of four
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x141, 0xF, 0xF, true)));      // the other four of eight
    if (LANES >= 16) v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x140, 0xF, 0xF, true)));
    if (LANES >= 32) v = max(v, uint32_t(__shfl_xor(int(v), 16)));
    if (LANES >= 64) v = max(v, uint32_t(__shfl_xor(int(v), 32)));
    return v;
}

// ---- tiles -----------------------------------------------------------------------------------------------------------

// How a wave's channels are dealt to the first operand's rows, so that 16 bytes are stored at once and four lanes store
// 64: a lane gets four of each matrix instruction's sixteen, which are 16 bytes of fp32; of bf16 the fours of two
// instructions are neighbours.  row(j, r): channel of row r of instruction j; first(j, g): first of the four that lanes
// 16 g .. hold.
template <typename Y> struct Deal;
template <> struct Deal<float> {
    static constexpr int SH = 2;                         // (bits 0, 1 and SH of a row tell eight rows r apart)
    static __device__ __forceinline__ int row(int j, int r) { return j * 16 + r; }
    static __device__ __forceinline__ int first(int j, int g) { return j * 16 + g * 4; }
};
template <> struct Deal<__bf16> {
    static constexpr int SH = 3;
    static __device__ __forceinline__ int row(int j, int r) { return (j >> 1) * 32 + (r >> 2) * 8 + (j & 1) * 4 + (r & 3); }
    static __device__ __forceinline__ int first(int j, int g) { return (j >> 1) * 32 + g * 8 + (j & 1) * 4; }
};

__device__ __forceinline__ v4u buffer_at(const int8_t *p)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    v4u r;
    r.x = __builtin_amdgcn_readfirstlane(uint32_t(at));
    r.y = __builtin_amdgcn_readfirstlane(uint32_t(at >> 32) & 0xFFFFu);
    r.z = 0x90000000u;                                   // (a tile's rows are within 2^31 bytes and a row's length)
    r.w = 0x00020000u;
    return r;
}
constexpr uint32_t kNowhere = 0xC0000000u;               // beyond the buffer, whatever is added: nothing is read, LDS gets zeros

// Which tile a workgroup computes.  Workgroups go round the 8 XCDs, each of which has a level-2 cache of its own: an
// XCD gets a run of tiles, and a run goes down GROUP tiles of rows before it goes on to the next tile of channels, so
// that the tiles that run at one time on an XCD share rows of both operands.
__device__ __forceinline__ void tile_at(unsigned id, unsigned tiles_m, unsigned tiles_n, unsigned &tm, unsigned &tn)
{
    constexpr unsigned XCDS = 8, GROUP = 8;
    const unsigned all = tiles_m * tiles_n, x = id % XCDS, per = all / XCDS, more = all % XCDS;
    const unsigned t = x * per + min(x, more) + id / XCDS;
    const unsigned g = t / (GROUP * tiles_n), in = t % (GROUP * tiles_n), rows = min(GROUP, tiles_m - g * GROUP);
    tm = g * GROUP + in % rows;
    tn = in / rows;
}

// Waits until at most `behind` (0 .. MOST) stages of L loads each of this wave are under way and its reads of LDS are
// done, and for the other waves of the workgroup to get there.
template <int MOST, int L>
__device__ __forceinline__ void wait_for_stages(int behind)
{
    if constexpr (MOST > 0) {
        if (behind == MOST) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n s_barrier" ::"n"(MOST * L) : "memory");
        else wait_for_stages<MOST - 1, L>(behind);
    } else {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n s_barrier" ::: "memory");
    }
}

// Waits until at most `behind` (0 .. MOST) groups of L loads each of this wave are under way.
template <int MOST, int L>
__device__ __forceinline__ void wait_for_loads(int behind)
{
    if constexpr (MOST > 0) {
        if (behind >= MOST) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(MOST * L) : "memory");
        else wait_for_loads<MOST - 1, L>(behind);
    } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
}

}  // namespace pconv
