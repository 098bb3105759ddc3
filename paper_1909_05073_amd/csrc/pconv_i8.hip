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
#include <type_traits>

#include "pconv_internal.h"
#include "pconv_ops.h"

namespace pconv {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
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

template <typename T>
__device__ __forceinline__ void quantize_part(const Vec<T> &v, const RowScale &r, uint32_t (&w)[Vec<T>::N / 4])
{
#pragma unroll
    for (int j = 0; j < Vec<T>::N / 4; ++j) {
        if (r.mode == 0)
            w[j] = pack4(quantize(v.at(4 * j), r), quantize(v.at(4 * j + 1), r), quantize(v.at(4 * j + 2), r), quantize(v.at(4 * j + 3), r));
        else
            w[j] = pack4(quantize_rare(v.at(4 * j), r), quantize_rare(v.at(4 * j + 1), r), quantize_rare(v.at(4 * j + 2), r),
                         quantize_rare(v.at(4 * j + 3), r));
    }
}

// The same elements quantised, to q; [cols, q_cols) is filled with zeros.
template <typename T>
__device__ __forceinline__ void store_part(const Vec<T> &v, const RowScale &r, int8_t *row, int64_t at, int64_t q_cols)
{
    constexpr int N = Vec<T>::N;
    uint32_t w[N / 4];
    quantize_part(v, r, w);
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

// Four neighbouring channels of one row of y, from n on.  ReLU keeps NaN.
struct Channels { f4 scale, bias; };

__device__ __forceinline__ Channels channels_at(const I8Product &p, int n)
{
    Channels c;
    if (n + 4 <= p.n) {
        __builtin_memcpy(&c.scale, p.sb + n, 16);
        if (p.bias) __builtin_memcpy(&c.bias, p.bias + n, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = min(n + i, p.n - 1);          // (what lies beyond the last channel is not stored)
            c.scale[i] = p.sb[at];
            if (p.bias) c.bias[i] = p.bias[at];
        }
    }
    if (!p.bias) c.bias = f4{0, 0, 0, 0};
    return c;
}

__device__ __forceinline__ f4 values_of(const I8Product &p, v4i acc, float sa, const Channels &c)
{
    f4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = float(acc[i]) * (sa * c.scale[i]) + c.bias[i];
        if (p.relu) v[i] = v[i] < 0.0f ? 0.0f : v[i];
    }
    return v;
}

template <typename Y, int N, typename V>
__device__ __forceinline__ void store_channels(const I8Product &p, int m, int n, V v)
{
    Y *y = static_cast<Y *>(p.y) + (int64_t(m) * p.ldy + n);
    if (n + N <= p.n) {
        __builtin_memcpy(y, &v, N * sizeof(Y));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (n + i < p.n) y[i] = v[i];
    }
}

// How a wave's channels are dealt to the first operand's rows: a lane gets four of each matrix instruction's sixteen, and Deal::G
// instructions' fours are neighbours, so that 16 bytes are stored at once and four lanes store 64 (fp32: 4 channels,
// bf16: 8).  row(j, r): channel of row r of instruction j; first(j, g): first of the four that lanes 16 g .. hold.
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

// Rows m + 16 i of y, the NT * 16 channels from n0 on; the lane has `lane & 15` in m and its group in `g`.
template <typename Y, int MT, int NT>
__device__ __forceinline__ void store_tile(const I8Product &p, int m, int n0, int g, const v4i (&acc)[MT][NT], const float (&sa)[MT])
{
    static_assert(NT % 2 == 0, "");
#pragma unroll
    for (int j = 0; j < NT; j += 2) {
        const int n = n0 + Deal<Y>::first(j, g), n2 = n0 + Deal<Y>::first(j + 1, g);
        if (n >= p.n) continue;
        const Channels c = channels_at(p, n), c2 = channels_at(p, n2);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (m + 16 * i >= p.m) continue;
            const f4 v = values_of(p, acc[i][j], sa[i], c), w = values_of(p, acc[i][j + 1], sa[i], c2);
            if (sizeof(Y) == 4) {
                store_channels<float, 4>(p, m + 16 * i, n, v);
                if (n2 < p.n) store_channels<float, 4>(p, m + 16 * i, n2, w);
            } else {
                const b8 o = __builtin_convertvector(__builtin_shufflevector(v, w, 0, 1, 2, 3, 4, 5, 6, 7), b8);
                store_channels<__bf16, 8>(p, m + 16 * i, n, o);
            }
        }
    }
}

__device__ __forceinline__ v4u buffer_at(const int8_t *p)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    v4u r;
    r.x = __builtin_amdgcn_readfirstlane(uint32_t(at));
    r.y = __builtin_amdgcn_readfirstlane(uint32_t(at >> 32) & 0xFFFFu);
    r.z = 0xFFFFFFFFu;
    r.w = 0x00020000u;
    return r;
}

// Which tile a workgroup computes.  Workgroups go round the 8 XCDs, each of which has a level-2 cache of its own: an XCD gets
// a run of tiles, and a run goes down GROUP tiles of rows before it goes on to the next tile of channels, so that the tiles that
// run at one time on an XCD share rows of both operands.
__device__ __forceinline__ void tile_at(unsigned id, unsigned tiles_m, unsigned tiles_n, unsigned &tm, unsigned &tn)
{
    constexpr unsigned XCDS = 8, GROUP = 8;
    const unsigned all = tiles_m * tiles_n, x = id % XCDS, per = all / XCDS, more = all % XCDS;
    const unsigned t = x * per + min(x, more) + id / XCDS;
    const unsigned g = t / (GROUP * tiles_n), in = t % (GROUP * tiles_n), rows = min(GROUP, tiles_m - g * GROUP);
    tm = g * GROUP + in % rows;
    tn = in / rows;
}

// Tiles of BM rows of y and BN channels, WM x WN waves.  128 bytes of k of all the tile's rows are a stage; S stages lie in
// LDS.  A row of a stage is eight pieces of 16 bytes, stored in an order that depends on the row so that the eight rows that are
// read at once lie in different banks.
//
// DMA: stages go from memory to LDS past the registers, S - 1 of them ahead of the one that is multiplied; a wave waits for its own
// loads of the next stage, and the barrier then tells it that everybody's are there and that the stage before is read.  What
// is left of k behind the last whole stage goes through registers, and so does everything where rows do not begin at
// multiples of 16 bytes (DMA = false; one stage ahead).
//
// `splits` workgroups share a tile, each with its part of k; their sums go to `part` [splits][m][n4], n4 = n rounded up to four.
template <typename Y, int BM, int BN, int WM, int WN, int S, bool DMA>
__global__ void __launch_bounds__(WM * WN * 64)
matmul_i8_kernel(const I8Product p, int splits, int *part)
{
    constexpr int BK = 128, NW = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    constexpr int PA = BM / 8 / NW, PB = BN / 8 / NW;    // blocks of eight rows that a wave stages
    static_assert(PA * NW * 8 == BM && PB * NW * 8 == BN, "");
    __shared__ v4i lds[S * (BM + BN) * 8];
    constexpr int STAGE = (BM + BN) * 8;
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned tiles_n = unsigned(p.n + BN - 1) / BN, tiles_m = unsigned(p.m + BM - 1) / BM;
    unsigned tm, tn;
    tile_at(blockIdx.x / unsigned(splits), tiles_m, tiles_n, tm, tn);
    const int split = int(blockIdx.x % unsigned(splits));
    const int m0 = int(tm) * BM, n0 = int(tn) * BN;
    const int wm = (wave / WN) * TM, wn = (wave % WN) * TN;
    // this workgroup's part of k: whole stages but for the last one's end
    const int stages = (p.k + BK - 1) / BK;
    const int s_begin = int(int64_t(stages) * split / splits), s_end = int(int64_t(stages) * (split + 1) / splits);
    const int k_begin = s_begin * BK, k_end = min(s_end * BK, p.k);

    // order of the pieces of a row of weights: the rows that are read at once differ in three of their bits
    auto key_b = [](int row) { return (row & 3) | (((row >> Deal<Y>::SH) & 1) << 2); };

    v4i acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4i{0, 0, 0, 0};

    auto multiply = [&](const v4i *st) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            v4i a[MT], b[NT];
            const int piece = kk * 4 + (lane >> 4), r = lane & 15;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int row = wm + i * 16 + r;
                a[i] = st[row * 8 + (piece ^ (row & 7))];
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int row = wn + Deal<Y>::row(j, r);
                b[j] = st[BM * 8 + row * 8 + (piece ^ key_b(row))];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[j], a[i], acc[i][j], 0, 0, 0);
        }
    };

    // through registers: a thread fetches the pieces at its place in every block of eight rows
    v4i ra[PA], rb[PB];
    auto fetch = [&](int k0) {
        const int at = k0 + (lane & 7) * 16;
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int row = min(m0 + (i * NW + wave) * 8 + (lane >> 3), p.m - 1);
            ra[i] = load16(p.a + int64_t(row) * p.lda, at, k_end);
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int row = min(n0 + (i * NW + wave) * 8 + (lane >> 3), p.n - 1);
            rb[i] = load16(p.b + int64_t(row) * p.ldb, at, k_end);
        }
    };
    auto store = [&](v4i *st) {
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int row = (i * NW + wave) * 8 + (lane >> 3);
            st[row * 8 + ((lane & 7) ^ (row & 7))] = ra[i];
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int row = (i * NW + wave) * 8 + (lane >> 3);
            st[BM * 8 + row * 8 + ((lane & 7) ^ key_b(row))] = rb[i];
        }
    };

    if (DMA) {
        const v4u at_a = buffer_at(p.a + int64_t(m0) * p.lda + k_begin), at_b = buffer_at(p.b + int64_t(n0) * p.ldb + k_begin);
        uint32_t off_a[PA], off_b[PB];
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int row = (i * NW + wave) * 8 + (lane >> 3);
            off_a[i] = uint32_t(min(row, p.m - 1 - m0)) * uint32_t(p.lda) + uint32_t(((lane & 7) ^ (row & 7)) * 16);
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int row = (i * NW + wave) * 8 + (lane >> 3);
            off_b[i] = uint32_t(min(row, p.n - 1 - n0)) * uint32_t(p.ldb) + uint32_t(((lane & 7) ^ key_b(row)) * 16);
        }
        const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)) + uint32_t(wave) * 1024u;
        // (written as assembly so that the compiler does not wait for these loads before every read of LDS)
        auto stage = [&](int s) {
            const uint32_t to = base + uint32_t(s % S) * uint32_t(STAGE * 16), k0 = uint32_t(s) * BK;
#pragma unroll
            for (int i = 0; i < PA; ++i)
                asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                             ::"v"(off_a[i]), "s"(to + uint32_t(i * NW * 1024)), "s"(at_a), "s"(k0) : "memory");
#pragma unroll
            for (int i = 0; i < PB; ++i)
                asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                             ::"v"(off_b[i]), "s"(to + uint32_t(BM * 128 + i * NW * 1024)), "s"(at_b), "s"(k0) : "memory");
        };
        constexpr int L = PA + PB;
        static_assert((S - 2) * L <= 63, "");
        const int whole = (k_end - k_begin) / BK;
#pragma unroll
        for (int s = 0; s < S - 1; ++s)
            if (s < whole) stage(s);
        for (int s = 0; s < whole; ++s) {
            // the loads of stage s are done when at most those of the stages behind it are under way
            const int behind = min(S - 2, whole - 1 - s);
            if (behind == S - 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n s_barrier" ::"n"((S - 2) * L) : "memory");
            else if (S > 3 && behind == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n s_barrier" ::"n"(L) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n s_barrier" ::: "memory");
            if (s + S - 1 < whole) stage(s + S - 1);
            multiply(lds + (s % S) * STAGE);
        }
        if (k_begin + whole * BK < k_end) {
            fetch(k_begin + whole * BK);
            __syncthreads();
            store(lds);
            __syncthreads();
            multiply(lds);
        }
    } else {
        if (k_begin < k_end) {
            fetch(k_begin);
            store(lds);
        }
        __syncthreads();
        int buf = 0;
        for (int k0 = k_begin; k0 < k_end; k0 += BK, buf ^= 1) {
            const bool more = k0 + BK < k_end;
            if (more) fetch(k0 + BK);
            multiply(lds + buf * STAGE);
            if (more) store(lds + (buf ^ 1) * STAGE);
            __syncthreads();
        }
    }

    const int m = m0 + wm + (lane & 15), g = lane >> 4;
    if (splits > 1) {
        const int64_t n4 = (int64_t(p.n) + 3) / 4 * 4;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = n0 + wn + Deal<Y>::first(j, g);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (m + 16 * i < p.m && n < p.n) __builtin_memcpy(part + (int64_t(split) * p.m + m + 16 * i) * n4 + n, &acc[i][j], 16);
        }
        return;
    }
    float sa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) sa[i] = p.sa[min(m + 16 * i, p.m - 1)];
    store_tile<Y, MT, NT>(p, m, n0 + wn, g, acc, sa);
}

// y of the sums of `splits` parts of k; a thread has four channels.
__global__ void __launch_bounds__(256)
matmul_i8_join_kernel(const I8Product p, int splits, const int *__restrict__ part)
{
    const int64_t quads = (int64_t(p.n) + 3) / 4, all = quads * p.m;
    for (int64_t t = int64_t(blockIdx.x) * 256 + threadIdx.x; t < all; t += int64_t(gridDim.x) * 256) {
        const int m = int(t / quads), n = int(t % quads) * 4;
        v4i s = {0, 0, 0, 0};
#pragma unroll 4
        for (int i = 0; i < splits; ++i) {
            v4i v;
            __builtin_memcpy(&v, part + (int64_t(i) * all + t) * 4, 16);
            s += v;
        }
        const f4 v = values_of(p, s, p.sa[m], channels_at(p, n));
        if (p.y_bf16) store_channels<__bf16, 4>(p, m, n, __builtin_convertvector(v, b4));
        else store_channels<float, 4>(p, m, n, v);
    }
}

// The largest value over the 8 or 16 neighbouring lanes that share a row.
template <int LANES>
__device__ __forceinline__ uint32_t most_of_lanes(uint32_t v)
{
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xF, 0xF, true)));       // the other of a pair
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x4E, 0xF, 0xF, true)));       // the other pair of four
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x141, 0xF, 0xF, true)));      // the other four of eight
    if (LANES == 16) v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x140, 0xF, 0xF, true)));
    return v;
}

// Short rows (k up to kThinK): all of k of 16 * MT rows of activations lies in LDS, so that there is no loop of stages and one read of
// the activations; where they come as floats (T) they are quantised on their way there and never leave the chip.
// The weights, which every workgroup reads and the level-2 caches hold, go to the registers directly.  Four waves share
// the rows and take groups of 64 channels in turn.  blockIdx.y: a part of the channels, a multiple of 64 (`part_n`).
//
// LANES lanes quantise a row, KEEP vectors of 16 bytes each.
constexpr int kThinK = 512;

template <typename T, typename Y, int MT, int LANES, int KEEP>
__global__ void __launch_bounds__(256)
linear_i8_thin_kernel(const I8Product p, const T *__restrict__ x, int64_t ldx, int part_n)
{
    constexpr int BM = 16 * MT, NT = 4;
    extern __shared__ v4i thin_lds[];                    // BM rows of `pieces` times 16 bytes, and the scales of the rows
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int m0 = int(blockIdx.x) * BM, pieces = (p.k + 127) / 128 * 8;
    float *const scales = reinterpret_cast<float *>(thin_lds + BM * pieces);
    if (sizeof(T) == 1) {
        for (int at = int(threadIdx.x); at < BM * pieces; at += 256) {
            const int row = at / pieces, c = at - row * pieces;
            thin_lds[row * pieces + (c ^ (row & 7))] =
                load16(reinterpret_cast<const int8_t *>(x) + int64_t(min(m0 + row, p.m - 1)) * ldx, c * 16, p.k);
        }
        for (int row = int(threadIdx.x); row < BM; row += 256) scales[row] = p.sa[min(m0 + row, p.m - 1)];
    } else {
        using V = Vec<std::conditional_t<sizeof(T) == 1, float, T>>;
        using E = std::conditional_t<sizeof(T) == 1, float, T>;
        constexpr int N = V::N, AT_ONCE = 64 / LANES, PASSES = BM / 4 / AT_ONCE;
        const int sub = lane % LANES;
        V v[PASSES][KEEP];
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int row = wave * (BM / 4) + i * AT_ONCE + lane / LANES;
            const E *from = reinterpret_cast<const E *>(x) + int64_t(min(m0 + row, p.m - 1)) * ldx;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) v[i][q] = load_part(from, (q * LANES + sub) * N, p.k);
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int row = wave * (BM / 4) + i * AT_ONCE + lane / LANES;
            uint32_t most = 0;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) most = most_of(v[i][q], most);
            const RowScale s = row_scale(most_of_lanes<LANES>(most));
            if (sub == 0) scales[row] = s.scale;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                const int byte = (q * LANES + sub) * N, c = byte / 16;
                uint32_t w[N / 4];
                quantize_part(v[i][q], s, w);
                if (c < pieces) __builtin_memcpy(reinterpret_cast<int8_t *>(thin_lds + row * pieces + (c ^ (row & 7))) + byte % 16, w, N);
            }
        }
    }
    __syncthreads();

    const int r = lane & 15, g = lane >> 4, n_end = min(p.n, int(blockIdx.y + 1) * part_n);
    for (int n0 = int(blockIdx.y) * part_n + wave * 64; n0 < n_end; n0 += 256) {
        const int8_t *b[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = p.b + int64_t(min(n0 + Deal<Y>::row(j, r), p.n - 1)) * p.ldb;
        v4i acc[MT][NT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = v4i{0, 0, 0, 0};
        auto step = [&](const v4i (&vb)[NT], int k0) {
            v4i va[MT];
            const int c = k0 / 16 + g;
#pragma unroll
            for (int i = 0; i < MT; ++i) va[i] = thin_lds[(i * 16 + r) * pieces + (c ^ (r & 7))];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[j], va[i], acc[i][j], 0, 0, 0);
        };
        auto fetch = [&](v4i (&vb)[NT], int k0) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (k0 + 64 <= p.k) __builtin_memcpy(&vb[j], b[j] + k0 + g * 16, 16);
                else vb[j] = load16(b[j], k0 + g * 16, p.k);
            }
        };
        v4i now[NT], next[NT];
        if (p.k > 0) fetch(now, 0);
        for (int k0 = 0; k0 < p.k; k0 += 64) {
            if (k0 + 64 < p.k) fetch(next, k0 + 64);
            step(now, k0);
#pragma unroll
            for (int j = 0; j < NT; ++j) now[j] = next[j];
        }
        float sa[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = scales[i * 16 + r];
        store_tile<Y, MT, NT>(p, m0 + r, n0, g, acc, sa);
    }
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
        const int m = i * 16 + (lane & 15), n = n0 + (lane >> 4) * 4;
        if (m >= p.m || n >= p.n) continue;
        const f4 v = values_of(p, s, p.sa[m], channels_at(p, n));
        if (p.y_bf16) store_channels<__bf16, 4>(p, m, n, __builtin_convertvector(v, b4));
        else store_channels<float, 4>(p, m, n, v);
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

namespace {

// How a product of more rows than matmul_i8_rows_kernel serves is cut up: the tile (an index into launch_tiles) and over how
// many workgroups the length of k is split.
struct Cut { int tile, splits; };

constexpr int kTileM[] = {32, 64, 128, 256}, kTileN[] = {128, 128, 128, 256};

Cut cut_of(int64_t m, int64_t n, int64_t k)
{
    const auto tiles = [&](int t) { return ((m + kTileM[t] - 1) / kTileM[t]) * ((n + kTileN[t] - 1) / kTileN[t]); };
    Cut c{m <= 32 ? 0 : m <= 64 ? 1 : 2, 1};
    if (tiles(3) >= 256) c.tile = 3;
    else if (c.tile == 2 && tiles(2) < 256 && tiles(1) >= 2 * tiles(2) && tiles(1) <= 512) c.tile = 1;
    const int64_t stages = (k + 127) / 128;
    if (tiles(c.tile) <= 128 && stages >= 8)
        c.splits = int(std::min<int64_t>(std::min<int64_t>(256 / tiles(c.tile), stages / 4), 32));
    return c;
}

template <int BM, int BN, int WM, int WN, int S>
void launch_tiles(const I8Product &p, int splits, int *part, bool dma, hipStream_t st)
{
    const unsigned grid = unsigned(((int64_t(p.m) + BM - 1) / BM) * ((int64_t(p.n) + BN - 1) / BN) * splits);
#define PCONV_LAUNCH(Y, STAGES, DMA) \
    hipLaunchKernelGGL((matmul_i8_kernel<Y, BM, BN, WM, WN, STAGES, DMA>), dim3(grid), dim3(WM * WN * 64), 0, st, p, splits, part)
    if (p.y_bf16) { if (dma) PCONV_LAUNCH(__bf16, S, true); else PCONV_LAUNCH(__bf16, 2, false); }
    else { if (dma) PCONV_LAUNCH(float, S, true); else PCONV_LAUNCH(float, 2, false); }
#undef PCONV_LAUNCH
}

constexpr int64_t kRowsM = 16;                           // matmul_i8_rows_kernel serves up to so many rows

// Rows of T (int8_t: quantised already, with their scales in p) times weights, k up to kThinK.
template <typename T, int LANES, int KEEP>
int launch_thin(const I8Product &p, const T *x, int64_t ldx, hipStream_t st)
{
    const int64_t big = (int64_t(p.m) + 63) / 64, groups = (int64_t(p.n) + 255) / 256;
    const int mt = big * groups >= 512 ? 4 : 2;
    const int64_t tiles = (int64_t(p.m) + 16 * mt - 1) / (16 * mt);
    const int64_t parts = std::min<int64_t>(groups, std::max<int64_t>(1, 1024 / tiles));
    const int part_n = int((groups + parts - 1) / parts * 256);
    if (tiles >= int64_t(1) << 24) { set_error("pconv_matmul_i8: too many workgroups"); return PCONV_UNSUPPORTED; }
    const dim3 grid(unsigned(tiles), unsigned((int64_t(p.n) + part_n - 1) / part_n));
    const size_t lds = size_t(16 * mt) * ((p.k + 127) / 128 * 128 + 4);
#define PCONV_LAUNCH(Y, MT) hipLaunchKernelGGL((linear_i8_thin_kernel<T, Y, MT, LANES, KEEP>), grid, dim3(256), lds, st, p, x, ldx, part_n)
    if (p.y_bf16) { if (mt == 4) PCONV_LAUNCH(__bf16, 4); else PCONV_LAUNCH(__bf16, 2); }
    else { if (mt == 4) PCONV_LAUNCH(float, 4); else PCONV_LAUNCH(float, 2); }
#undef PCONV_LAUNCH
    return check_launch("pconv_linear_i8 (short rows)");
}

}  // namespace

bool linear_i8_thin(int64_t m, int64_t n, int64_t k) { return m > kRowsM && k <= kThinK; }

int launch_linear_i8_thin(const I8Product &p, const void *x, int64_t ldx, int bf16, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (bf16) {
        const __bf16 *const at = static_cast<const __bf16 *>(x);
        if (p.k <= 64) return launch_thin<__bf16, 8, 1>(p, at, ldx, st);
        if (p.k <= 128) return launch_thin<__bf16, 16, 1>(p, at, ldx, st);
        if (p.k <= 256) return launch_thin<__bf16, 16, 2>(p, at, ldx, st);
        return launch_thin<__bf16, 16, 4>(p, at, ldx, st);
    }
    const float *const at = static_cast<const float *>(x);
    if (p.k <= 64) return launch_thin<float, 16, 1>(p, at, ldx, st);
    if (p.k <= 128) return launch_thin<float, 16, 2>(p, at, ldx, st);
    if (p.k <= 256) return launch_thin<float, 16, 4>(p, at, ldx, st);
    return launch_thin<float, 16, 8>(p, at, ldx, st);
}

int64_t matmul_i8_part_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m <= kRowsM || linear_i8_thin(m, n, k)) return 0;
    const Cut c = cut_of(m, n, k);
    return c.splits > 1 ? c.splits * m * ((n + 3) / 4 * 4) * 4 : 0;
}

int launch_matmul_i8(const I8Product &p, void *part, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (p.m <= kRowsM) {
        hipLaunchKernelGGL((matmul_i8_rows_kernel<1, 8>), dim3(unsigned((p.n + 15) / 16)), dim3(512), 0, st, p);
        return check_launch("pconv_matmul_i8 (few rows)");
    }
    if (linear_i8_thin(p.m, p.n, p.k)) return launch_thin<int8_t, 8, 1>(p, p.a, p.lda, st);
    const Cut c = cut_of(p.m, p.n, p.k);
    const int64_t tiles = ((int64_t(p.m) + kTileM[c.tile] - 1) / kTileM[c.tile]) * ((int64_t(p.n) + kTileN[c.tile] - 1) / kTileN[c.tile]);
    if (tiles * c.splits >= int64_t(1) << 23) { set_error("pconv_matmul_i8: too many workgroups"); return PCONV_UNSUPPORTED; }
    // rows at multiples of 16 bytes, a tile's rows within 32 bits
    const auto fits = [](const int8_t *at, int64_t ld) { return reinterpret_cast<uintptr_t>(at) % 16 == 0 && ld % 16 == 0 && ld <= 1 << 23; };
    const bool dma = fits(p.a, p.lda) && fits(p.b, p.ldb);
    int *const sums = static_cast<int *>(part);
    if (c.tile == 0) launch_tiles<32, 128, 1, 4, 4>(p, c.splits, sums, dma, st);
    else if (c.tile == 1) launch_tiles<64, 128, 2, 2, 3>(p, c.splits, sums, dma, st);
    else if (c.tile == 2) launch_tiles<128, 128, 2, 2, 2>(p, c.splits, sums, dma, st);
    else launch_tiles<256, 256, 2, 4, 2>(p, c.splits, sums, dma, st);
    if (const int rc = check_launch("pconv_matmul_i8")) return rc;
    if (c.splits == 1) return PCONV_OK;
    const int64_t quads = (int64_t(p.n) + 3) / 4 * p.m;
    hipLaunchKernelGGL(matmul_i8_join_kernel, dim3(unsigned(std::min<int64_t>((quads + 255) / 256, 1 << 16))), dim3(256), 0, st, p, c.splits, sums);
    return check_launch("pconv_matmul_i8 (joining the parts of k)");
}

}  // namespace pconv
