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
#include "pconv_rows.h"

namespace pconv {

bool rows_at_16(const int8_t *at, int64_t ld) { return reinterpret_cast<uintptr_t>(at) % 16 == 0 && ld % 16 == 0 && ld <= 1 << 23; }

namespace {

int too_many_groups()
{
    set_error("8-bit layers: too many workgroups for one launch");
    return PCONV_UNSUPPORTED;
}

// ---- quantising rows ---------------------------------------------------------------------------------------------------

// 16 bytes of a row that has `len` bytes, from `at` on; beyond its end zero.
template <bool EXACT = false>
__device__ __forceinline__ v4i load16(const int8_t *row, int at, int len)
{
    v4i v = {0, 0, 0, 0};
    if (__builtin_expect(at + 16 <= len, 1)) __builtin_memcpy(&v, row + at, 16);
    else if (!EXACT && __builtin_expect(at < len, 0)) v = load_end(row, at, len);
    return v;
}

// 16 bytes at an address of any alignment, as the five words that hold them.  (A load of 16 bytes that is not aligned
// to a word takes 2.6 times one that is: 6x17360 -> 562 31 us and 16.)  No word is read that holds none of the bytes.
__device__ __forceinline__ v4i load16_loose(const int8_t *p)
{
    const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p)) & 3u;
    const int8_t *const q = p - off;
    typedef v4i Words __attribute__((aligned(4)));
    const v4i w = *reinterpret_cast<const Words *>(q);
    const uint32_t last = *reinterpret_cast<const uint32_t *>(q + (off ? 16 : 12));
    v4i v;
    v[0] = int(__builtin_amdgcn_alignbyte(uint32_t(w[1]), uint32_t(w[0]), off));
    v[1] = int(__builtin_amdgcn_alignbyte(uint32_t(w[2]), uint32_t(w[1]), off));
    v[2] = int(__builtin_amdgcn_alignbyte(uint32_t(w[3]), uint32_t(w[2]), off));
    v[3] = int(__builtin_amdgcn_alignbyte(last, uint32_t(w[3]), off));
    return v;
}

// Rows to multiples of 16 bytes, zeros behind their ends, by `threads` threads.
__device__ __forceinline__ void realign(const Realign &a, int64_t thread, int64_t threads)
{
    const int64_t all = int64_t(a.rows) * a.pieces;
#pragma unroll 1
    for (int64_t t = thread; t < all; t += threads) {
        const int64_t row = t / a.pieces;
        const int at = int(t - row * a.pieces) * 16;
        const int8_t *from = a.from + row * a.ld;
        const v4i v = at + 16 <= a.k ? load16_loose(from + at) : load16(from, at, a.k);
        __builtin_memcpy(a.to + t * 16, &v, 16);
    }
}

// TPR threads of a workgroup share a row; each keeps its first KEEP vectors of 16 bytes in registers between finding
// the row's scale and quantising, and reads what lies beyond (from a cache) twice.  [cols, q_cols) is filled with
// zeros.  The workgroups from `blocks` on bring the rows of a product's weights to multiples of 16 bytes meanwhile (a
// launch less).  Code that runs is kept short: a launch of one wave's work a SIMD spends its time on fetching
// instructions.  Bound by memory: 8192x4096 bf16 20 us, 5.0 TB/s.
template <typename T, int TPR, int KEEP, int THREADS, bool PASSING>
__global__ void __launch_bounds__(THREADS)
quantize_rows_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int64_t cols, int8_t *__restrict__ q, int64_t ldq,
                     int64_t q_cols, float *__restrict__ scale, unsigned blocks, const Realign weights)
{
    constexpr int N = Vec<T>::N, RPW = THREADS / TPR;
    __shared__ uint32_t lds[THREADS / 64];
    if (__builtin_expect(blockIdx.x >= blocks, 0)) {
        realign(weights, int64_t(blockIdx.x - blocks) * THREADS + threadIdx.x, int64_t(gridDim.x - blocks) * THREADS);
        return;
    }
    const int sub = int(threadIdx.x) % TPR;
    const int64_t groups = (rows + RPW - 1) / RPW;
    for (int64_t g = blockIdx.x; g < groups; g += blocks) {
        const int64_t r = g * RPW + int(threadIdx.x) / TPR;
        const bool live = r < rows;
        const T *row = x + (live ? r : rows - 1) * ldx;
        Vec<T> v[KEEP];
        uint32_t most = 0;
        load_row<T, TPR, KEEP, false, PASSING>(row, sub, cols, v);
#pragma unroll
        for (int i = 0; i < KEEP; ++i) most = most_of(v[i], most);
        for (int64_t at = (int64_t(KEEP) * TPR + sub) * N; at < cols; at += TPR * N) most = most_of(load_vec(row, at, cols), most);
        most = most_of_lanes<(TPR < 64 ? TPR : 64)>(most);
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
        for (int i = 0; i < KEEP; ++i) store_vec(v[i], s, qrow, (int64_t(i) * TPR + sub) * N, q_cols);
        for (int64_t at = (int64_t(KEEP) * TPR + sub) * N; at < q_cols; at += TPR * N)
            store_vec(load_vec(row, at, cols), s, qrow, at, q_cols);
        if (sub == 0) scale[r] = s.scale;
    }
}

// ---- the product --------------------------------------------------------------------------------------------------------

// Four neighbouring channels of one row of y, from n on.  ReLU keeps NaN.
struct Channels { f4 scale, bias; };

__device__ __forceinline__ bool rows_at_words(const int8_t *p, int64_t ld) { return ((reinterpret_cast<uintptr_t>(p) | uint64_t(ld)) & 3u) == 0; }

// EXACT (here and below): sizes are such that nothing ends inside what a lane reads or writes at once.
template <bool EXACT = false>
__device__ __forceinline__ Channels channels_at(const I8Product &p, int n)
{
    Channels c;
    if (EXACT || __builtin_expect(n + 4 <= p.n, 1)) {
        if (EXACT) n = min(n, p.n - 4);
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

template <typename Y, int N, bool EXACT = false, typename V>
__device__ __forceinline__ void store_channels(const I8Product &p, int m, int n, V v)
{
    Y *y = static_cast<Y *>(p.y) + (int64_t(m) * p.ldy + n);
    if (EXACT || __builtin_expect(n + N <= p.n, 1)) {
        __builtin_memcpy(y, &v, N * sizeof(Y));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (n + i < p.n) y[i] = v[i];
    }
}

// Rows m + 16 i of y, the NT * 16 channels from n0 on; the lane has `lane & 15` in m and its group in `g`.  Scales
// and biases are read before anything is stored: behind a store they would be waited for one by one.
template <typename Y, int NT, bool EXACT = false>
__device__ __forceinline__ void load_channels(const I8Product &p, int n0, int g, Channels (&c)[NT])
{
#pragma unroll
    for (int j = 0; j < NT; ++j) c[j] = channels_at<EXACT>(p, n0 + Deal<Y>::first(j, g));
}

template <typename Y, int MT, int NT, bool EXACT = false>
__device__ __forceinline__ void store_tile(const I8Product &p, int m, int n0, int g, const v4i (&acc)[MT][NT], const float (&sa)[MT],
                                           const Channels (&c)[NT])
{
    static_assert(NT % 2 == 0, "");
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if (m + 16 * i >= p.m) continue;
#pragma unroll
        for (int j = 0; j < NT; j += 2) {
            const int n = n0 + Deal<Y>::first(j, g), n2 = n0 + Deal<Y>::first(j + 1, g);
            if (n >= p.n) continue;
            const f4 v = values_of(p, acc[i][j], sa[i], c[j]), w = values_of(p, acc[i][j + 1], sa[i], c[j + 1]);
            if (sizeof(Y) == 4) {
                store_channels<float, 4, EXACT>(p, m + 16 * i, n, v);
                if (n2 < p.n) store_channels<float, 4, EXACT>(p, m + 16 * i, n2, w);
            } else {
                const b8 o = __builtin_convertvector(__builtin_shufflevector(v, w, 0, 1, 2, 3, 4, 5, 6, 7), b8);
                store_channels<__bf16, 8, EXACT>(p, m + 16 * i, n, o);
            }
        }
    }
}

// Tiles of BM rows of y and BN channels, WM x WN waves, and KG such sets of waves that take the stages in turn (a
// stage takes a wave 0.4 us of waiting for one thing after the other, however far ahead it is loaded).  128 bytes of
// k of all the tile's rows are a stage; S stages lie in LDS.  A row of a stage is eight pieces of 16 bytes, stored in
// an order that depends on the row so that the eight rows that are read at once lie in different banks.
//
// Stages go from memory to LDS past the registers, S - 1 of them ahead of the one that is multiplied; a wave waits
// for its own loads of the next stage, and the barrier then tells it that everybody's are there and that the stage
// before is read.  In the last stage the pieces behind the end of k are zeros.  Where k ends inside a piece the piece
// is loaded whole (what lies behind it is still before the next row, so the last rows of all go through registers),
// and the activations' part behind k is cleared in LDS.  Rows begin at multiples of 16 bytes (realign_kernel sees to
// it).
//
// `splits` workgroups share a tile, each with its part of k; their sums go to `part` [splits][m][n4], n4 = n rounded
// up to four.
//
// Bound by the matrix units, which are busy for half of the cycles, and the clock that the card allows them (8192x4096
// -> 4096: 123 us, 2.2 POP/s, in runs of 117 to 143; zeros 110 us), with few rows by memory (32x25088 -> 4096: 22 us,
// 4.7 TB/s), with few tiles by a stage's latencies (777x1155 -> 1001: 8.6 us).
template <typename Y, int BM, int BN, int WM, int WN, int S, int KG>
__global__ void __launch_bounds__(KG * WM * WN * 64)
matmul_i8_kernel(const I8Product p, int splits, int *part)
{
    constexpr int BK = 128, NW = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    constexpr int PA = BM / 8 / NW, PB = BN / 8 / NW;    // blocks of eight rows that a wave stages
    static_assert(PA * NW * 8 == BM && PB * NW * 8 == BN, "");
    constexpr int STAGE = (BM + BN) * 8, SUMS = NW * MT * NT * 64;       // (of one set of waves)
    __shared__ v4i lds[S * KG * STAGE];
    static_assert(KG == 1 || (KG - 1) * SUMS <= S * KG * STAGE, "");
    const int lane = int(threadIdx.x) & 63, set = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / (NW * 64));
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6) % NW;
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

    const v4u at_a = buffer_at(p.a + int64_t(m0) * p.lda + k_begin), at_b = buffer_at(p.b + int64_t(n0) * p.ldb + k_begin);
    uint32_t off_a[PA], off_b[PB];
    int end_a[PA], end_b[PB];                            // (a lane's piece is loaded if k reaches behind this byte of the stage)
#pragma unroll
    for (int i = 0; i < PA; ++i) {
        const int row = (i * NW + wave) * 8 + (lane >> 3);
        const int col = ((lane & 7) ^ (row & 7)) * 16;
        end_a[i] = col + (m0 + row < p.m - 1 ? 0 : 15);
        off_a[i] = uint32_t(min(row, p.m - 1 - m0)) * uint32_t(p.lda) + uint32_t(col);
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
        const int row = (i * NW + wave) * 8 + (lane >> 3);
        const int col = ((lane & 7) ^ key_b(row)) * 16;
        end_b[i] = col + (n0 + row < p.n - 1 ? 0 : 15);
        off_b[i] = uint32_t(min(row, p.n - 1 - n0)) * uint32_t(p.ldb) + uint32_t(col);
    }
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)) + uint32_t(set) * uint32_t(STAGE * 16) + uint32_t(wave) * 1024u;
    // (written as assembly so that the compiler does not wait for these loads before every read of LDS)
    const int length = k_end - k_begin, whole = length / BK, rest = length % BK;
    const int count = whole + (rest > 0 ? 1 : 0);
    // stage `turn` of this set is stage turn * KG + set of all
    auto stage = [&](int turn) {
        const int s = turn * KG + set;
        const uint32_t to = base + uint32_t(turn % S) * uint32_t(KG * STAGE * 16), k0 = uint32_t(s) * BK;
        const int have = s < whole ? BK : rest;
#pragma unroll
        for (int i = 0; i < PA; ++i)
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                         ::"v"(end_a[i] < have ? off_a[i] : kNowhere), "s"(to + uint32_t(i * NW * 1024)), "s"(at_a), "s"(k0) : "memory");
#pragma unroll
        for (int i = 0; i < PB; ++i)
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                         ::"v"(end_b[i] < have ? off_b[i] : kNowhere), "s"(to + uint32_t(BM * 128 + i * NW * 1024)), "s"(at_b), "s"(k0) : "memory");
    };
    constexpr int L = PA + PB;
    static_assert((S - 2) * L <= 63, "");
    const int mine = (count - set + KG - 1) / KG;        // stages of this set (count >= 0, so at least 0)
    const bool ragged = rest % 16 != 0;                  // k ends inside a piece
    const int turns = (count + KG - 1) / KG;
#pragma unroll
    for (int t = 0; t < S - 1; ++t)
        if (t < mine) stage(t);
#pragma unroll 1
    for (int t = 0; t < turns; ++t) {
        // the loads of this turn are done when at most those of the turns behind it are under way
        wait_for_stages<S - 2, L>(min(S - 2, max(0, mine - 1 - t)));
        if (t + S - 1 < mine) stage(t + S - 1);
        v4i *const st = lds + ((t % S) * KG + set) * STAGE;
        if (ragged && t == whole / KG) {
            if (set == whole % KG) {
                const int piece = rest / 16, at = k_begin + whole * BK + piece * 16;
                for (int row = wave * 64 + lane; row < BM; row += NW * 64) {
                    v4i v = st[row * 8 + (piece ^ (row & 7))];
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int bits = max(0, min(32, (rest % 16 - 4 * w) * 8));
                        v[w] &= int(uint32_t((uint64_t(1) << bits) - 1));
                    }
                    if (m0 + row >= p.m - 1) v = load16(p.a + int64_t(p.m - 1) * p.lda, at, k_end);
                    st[row * 8 + (piece ^ (row & 7))] = v;
                }
                for (int row = wave * 64 + lane; row < BN; row += NW * 64)
                    if (n0 + row >= p.n - 1) st[BM * 8 + row * 8 + (piece ^ key_b(row))] = load16(p.b + int64_t(p.n - 1) * p.ldb, at, k_end);
            }
            __syncthreads();
        }
        if (KG == 1 || t * KG + set < count) multiply(st);
    }
    if constexpr (KG > 1) {                              // the sets' sums come together
        __syncthreads();
        v4i *const to = lds + wave * (MT * NT * 64) + lane;
        if (set > 0) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) to[(set - 1) * SUMS + (i * NT + j) * 64] = acc[i][j];
        }
        __syncthreads();
        if (set > 0) return;
#pragma unroll
        for (int q = 0; q < KG - 1; ++q)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] += to[q * SUMS + (i * NT + j) * 64];
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
    Channels c[NT];
    load_channels<Y, NT>(p, n0 + wn, g, c);
    store_tile<Y, MT, NT>(p, m, n0 + wn, g, acc, sa, c);
}

// Rows of one or two matrices to multiples of 16 bytes (blockIdx.y: which).  1001x1155: 3.8 us.
__global__ void __launch_bounds__(256)
realign_kernel(const Realign a0, const Realign a1)
{
    realign(blockIdx.y ? a1 : a0, int64_t(blockIdx.x) * 256 + threadIdx.x, int64_t(gridDim.x) * 256);
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

// Short rows (k up to kThinK): all of k of BM rows of activations lies in LDS, so that there is no loop of stages and
// one read of the activations; where they come as floats they are quantised on their way there and never leave the
// chip.
constexpr int kThinK = 512, kThinLongK = 2048;           // (quantised within the product, and where thin_long() says so)
constexpr int thin_rows(int ks) { return ks <= 16 ? 64 : 32; }           // rows of a workgroup in whole pieces

// LDS holds rows of PIECES times 16 bytes, whose order makes the 16 lanes that are read at once differ in their
// places modulo 256 bytes.
template <int KS> struct ThinLds {
    static constexpr int PIECES = KS < 2 ? 8 : KS * 4, KEY = PIECES < 16 ? 7 : 15;
    static __device__ __forceinline__ int at(int row, int piece) { return row * PIECES + (piece ^ (row & KEY)); }
};

// Quantising BM rows of up to KS * 64 elements by W waves: LANES lanes a row, KEEP vectors of 16 bytes each.
template <typename T, int KS, int W, int BM> struct ThinRows {
    static constexpr int N = Vec<T>::N, VECS = KS * 64 / N, LANES = VECS < 16 ? VECS : 16, KEEP = VECS / LANES;
    static constexpr int AT_ONCE = 64 / LANES, PASSES = BM / W / AT_ONCE;
    static_assert(PASSES * AT_ONCE * W == BM, "");

    template <bool EXACT>
    static __device__ __forceinline__ void load(const T *x, int64_t ldx, int m0, int m, int k, int wave, int lane, Vec<T> (&v)[PASSES][KEEP])
    {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int row = wave * (BM / W) + i * AT_ONCE + lane / LANES;
            load_row<T, LANES, KEEP, EXACT>(x + int64_t(min(m0 + row, m - 1)) * ldx, lane % LANES, k, v[i]);
        }
    }

    static __device__ __forceinline__ void store(const Vec<T> (&v)[PASSES][KEEP], int k, int wave, int lane, v4i *lds, float *scales)
    {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int row = wave * (BM / W) + i * AT_ONCE + lane / LANES;
            uint32_t most = 0;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) most = most_of(v[i][q], most);
            const RowScale s = row_scale(most_of_lanes<LANES>(most));
            if (lane % LANES == 0) scales[row] = s.scale;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                if (KS > 8 && q * LANES * N >= (k + 127) / 128 * 128) continue;            // (behind the last step)
                const int byte = (q * LANES + lane % LANES) * N;
                uint32_t w[N / 4];
                quantize_vec(v[i][q], s, w);
                __builtin_memcpy(reinterpret_cast<int8_t *>(lds + ThinLds<KS>::at(row, byte / 16)) + byte % 16, w, N);
            }
        }
    }
};

// Short rows in whole pieces: k a multiple of 16, n of 8, the rows of the weights at multiples of 16 bytes.  Eight
// waves share 64 rows (32 where k passes 1024), MH sets of them a part of the rows each, and take groups of 32
// channels in turn; blockIdx.y: a part of the channels (`part_n`).  The weights, which every workgroup reads and the
// level-2 caches hold, come in steps of 128 bytes of k of a group's channels (k up to 64: one step, to the
// registers), past the registers to a ring of D steps in LDS that is the wave's own: no barrier, and eight lanes read
// 128 bytes of a row together (read as the matrix instruction wants them, no two lanes do, and a quarter of the
// cache's rate is all there is).  Bound by memory and a workgroup's start and end: 100352x64 -> 256 bf16 15.6 us, 4.1
// TB/s.
template <typename T, typename Y, int KS, int MH>
__global__ void __launch_bounds__(512, KS <= 4 ? 4 : 2)
linear_i8_thin_kernel(const I8Product p, const T *__restrict__ x, int64_t ldx, int part_n)
{
    constexpr int W = 8, BM = thin_rows(KS), MT = BM / 16 / MH, NT = 2, WN = W / MH, HALVES = KS == 1 ? 1 : 2, ROW = 4 * HALVES, STEP = 32 * ROW;
    constexpr bool RING = KS > 1;
    constexpr int D = KS >= 8 ? 3 : RING ? 2 : 1, L = STEP / 64;         // (two workgroups a compute unit but for KS from 8)
    constexpr int AT_ONCE = 64 / ROW;                    // rows of a step that a load brings
    __shared__ v4i lds[BM * ThinLds<KS>::PIECES];
    __shared__ v4i ring[RING ? W : 1][RING ? D * STEP : 16];
    // (the scales of the rows: in the first wave's last step until it is read into)
    float *const scales = reinterpret_cast<float *>(ring[0] + (RING ? D - 1 : 0) * STEP);
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int m0 = int(blockIdx.x) * BM, r = lane & 15, g = lane >> 4;
    const int steps = (p.k + 64 * HALVES - 1) / (64 * HALVES), rest = p.k % (64 * HALVES);
    int n0 = int(blockIdx.y) * part_n + wave % WN * 32;
    const int n_end = min(p.n, int(blockIdx.y + 1) * part_n), upper = wave / WN * (MT * 16);

    // order of the pieces of a row of a step (see ThinLds)
    auto key = [](int row) {
        const int q = row >> Deal<Y>::SH;
        return HALVES == 1 ? (0x78 >> ((q & 3) * 2)) & 3 : (row & 3) | ((q & 1) << 2);
    };
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring[RING ? wave : 0]));
    int next_n = n0, next_step = 0, issued = 0;          // what is read next, and how many steps have been
    v4u at_b = {0, 0, 0, 0};
    uint32_t off[L], end[L];
    auto aim = [&]() {
        at_b = buffer_at(p.b + int64_t(next_n) * p.ldb);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int row = i * AT_ONCE + lane / ROW, col = (lane % ROW ^ key(row)) * 16;
            off[i] = uint32_t(min(row, p.n - 1 - next_n)) * uint32_t(p.ldb) + uint32_t(col);
            end[i] = rest && col >= rest ? kNowhere : off[i];                // (in the last step)
        }
    };
    auto issue = [&]() {
        if (next_n >= n_end) return;
        const uint32_t to = base + uint32_t(issued % D) * uint32_t(STEP * 16);
        const bool last = next_step == steps - 1;
#pragma unroll
        for (int i = 0; i < L; ++i)
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                         ::"v"(last ? end[i] : off[i]), "s"(to + uint32_t(i * 1024)), "s"(at_b), "s"(uint32_t(next_step) * uint32_t(64 * HALVES)) : "memory");
        ++issued;
        ++next_step;
        if (last) {
            next_step = 0;
            next_n += WN * 32;
            if (next_n < n_end) aim();
        }
    };
    v4i vb[NT];
    const int piece = g * 16 < p.k ? g * 16 : 0;         // (behind k the activations are zeros)
    auto fetch = [&](int n0) {                           // (one step: to the registers)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            __builtin_memcpy(&vb[j], p.b + int64_t(min(n0 + Deal<Y>::row(j, r), p.n - 1)) * p.ldb + piece, 16);
    };
    auto start = [&]() {
        if constexpr (!RING) {
            fetch(n0);
            return;
        }
        if (next_n < n_end) aim();
#pragma unroll 1
        for (int i = 0; i < D - 1; ++i) issue();
    };

    if constexpr (sizeof(T) == 1) {
        constexpr int PIECES = ThinLds<KS>::PIECES, EACH = BM * PIECES / (W * 64);
        v4i v[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = i * (W * 64) + int(threadIdx.x);
            v[i] = load16<true>(x + int64_t(min(m0 + at / PIECES, p.m - 1)) * ldx, at % PIECES * 16, p.k);
        }
        start();
        if (threadIdx.x < BM) scales[threadIdx.x] = p.sa[min(m0 + int(threadIdx.x), p.m - 1)];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = i * (W * 64) + int(threadIdx.x);
            lds[ThinLds<KS>::at(at / PIECES, at % PIECES)] = v[i];
        }
    } else {
        Vec<T> v[ThinRows<T, KS, W, BM>::PASSES][ThinRows<T, KS, W, BM>::KEEP];
        ThinRows<T, KS, W, BM>::template load<true>(x, ldx, m0, p.m, p.k, wave, lane, v);
        start();
        ThinRows<T, KS, W, BM>::store(v, p.k, wave, lane, lds, scales);
    }
    Channels ch[NT];
    if (n0 < n_end) load_channels<Y, NT, true>(p, n0, g, ch);
    __syncthreads();
    float sa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) sa[i] = scales[upper + i * 16 + r];
    if (RING) __syncthreads();
    int landed = 0;                                      // steps that are known to be in LDS
    for (int c = 0; n0 < n_end; n0 += WN * 32) {
        const bool more = n0 + WN * 32 < n_end;
        Channels next[NT];
        if (more) load_channels<Y, NT, true>(p, n0 + WN * 32, g, next);
        v4i acc[MT][NT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = v4i{0, 0, 0, 0};
        if constexpr (!RING) {
            v4i va[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) va[i] = lds[ThinLds<KS>::at(upper + i * 16 + r, g)];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[j], va[i], acc[i][j], 0, 0, 0);
            if (more) {
                fetch(n0 + WN * 32);
#pragma unroll
                for (int j = 0; j < NT; ++j) asm volatile("" : "+v"(vb[j]));
            }
        }
#pragma unroll 1
        for (int s = 0; RING && s < steps; ++s, ++c) {
            if (c >= landed) wait_for_loads<(RING ? D - 2 : 0), L>(issued - 1 - c);
            // (the step that this one overwrites has been multiplied)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            issue();
            const v4i *const st = ring[RING ? wave : 0] + (c % D) * STEP;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                v4i va[MT];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const int row = Deal<Y>::row(j, r);
                    vb[j] = st[row * ROW + ((h * 4 + g) ^ key(row))];
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) va[i] = lds[ThinLds<KS>::at(upper + i * 16 + r, (s * HALVES + h) * 4 + g)];
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[j], va[i], acc[i][j], 0, 0, 0);
            }
        }
        // what is under way is waited for before the stores: waiting for it behind them would be waiting for them
        if (more) {
#pragma unroll
            for (int j = 0; j < NT; ++j) asm volatile("" : "+v"(next[j].scale), "+v"(next[j].bias));
        }
        if (issued > landed) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        landed = issued;
        store_tile<Y, MT, NT, true>(p, m0 + upper + r, n0, g, acc, sa, ch);
#pragma unroll
        for (int j = 0; j < NT; ++j) ch[j] = next[j];
    }
}

// Short rows that end inside a piece, or channels inside a store, or weights whose rows do not begin at multiples of
// 16 bytes: four waves, 32 rows, the weights go to the registers directly, all KS steps of the first channels before
// the activations are waited for.
template <typename T, typename Y, int KS>
__global__ void __launch_bounds__(256, KS <= 2 ? 4 : 2)
linear_i8_thin_ragged_kernel(const I8Product p, const T *__restrict__ x, int64_t ldx, int part_n)
{
    constexpr int MT = 2, W = 4, BM = 16 * MT, NT = 2, PIECES = ThinLds<KS>::PIECES;
    __shared__ v4i lds[BM * PIECES];
    __shared__ float scales[BM];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int m0 = int(blockIdx.x) * BM, r = lane & 15, g = lane >> 4;

    const int n_end = min(p.n, int(blockIdx.y + 1) * part_n);
    int n0 = int(blockIdx.y) * part_n + wave * 32;
    const bool words = rows_at_words(p.b, p.ldb);
    v4i vb[KS][NT];
    auto fetch = [&](int n0) {                           // (also behind the last channel, for nothing, so that there is no branch)
        const int8_t *b[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = p.b + int64_t(min(n0 + Deal<Y>::row(j, r), p.n - 1)) * p.ldb;
        if (words) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
                if (s * 64 + 64 <= p.k) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) __builtin_memcpy(&vb[s][j], b[j] + s * 64 + g * 16, 16);
                }
        } else {
#pragma unroll
            for (int s = 0; s < KS; ++s)
                if (s * 64 + 64 <= p.k) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) vb[s][j] = load16_loose(b[j] + s * 64 + g * 16);
                }
        }
        if (p.k % 64 != 0) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const v4i end = load16(b[j], p.k / 64 * 64 + g * 16, p.k);
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    if (s == p.k / 64) vb[s][j] = end;
            }
        }
    };
    if constexpr (sizeof(T) == 1) {
        constexpr int EACH = BM * PIECES / (W * 64);
        v4i v[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = i * (W * 64) + int(threadIdx.x), row = at / PIECES, c = at % PIECES;
            v[i] = load16(x + int64_t(min(m0 + row, p.m - 1)) * ldx, c * 16, p.k);
        }
        fetch(n0);
        if (threadIdx.x < BM) scales[threadIdx.x] = p.sa[min(m0 + int(threadIdx.x), p.m - 1)];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = i * (W * 64) + int(threadIdx.x), row = at / PIECES, c = at % PIECES;
            lds[ThinLds<KS>::at(row, c)] = v[i];
        }
    } else {
        Vec<T> v[ThinRows<T, KS, W, BM>::PASSES][ThinRows<T, KS, W, BM>::KEEP];
        ThinRows<T, KS, W, BM>::template load<false>(x, ldx, m0, p.m, p.k, wave, lane, v);
        fetch(n0);
        ThinRows<T, KS, W, BM>::store(v, p.k, wave, lane, lds, scales);
    }
    __syncthreads();
    float sa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) sa[i] = scales[i * 16 + r];
    for (; n0 < n_end; n0 += W * 32) {
        v4i acc[MT][NT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = v4i{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s * 64 >= p.k) continue;
            v4i va[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) va[i] = lds[ThinLds<KS>::at(i * 16 + r, s * 4 + g)];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[s][j], va[i], acc[i][j], 0, 0, 0);
        }
        Channels ch[NT];
        load_channels<Y, NT>(p, n0, g, ch);
        // the next weights are read before the stores: behind them they would wait for them
        if (n0 + W * 32 < n_end) fetch(n0 + W * 32);
        store_tile<Y, MT, NT>(p, m0 + r, n0, g, acc, sa, ch);
    }
}

// Few rows (up to 16): 16 channels a workgroup, whose waves share the length of k in turns of 256 bytes and add their
// sums in LDS.  Reading the weights is all of it; a wave has the next turns' under way while it multiplies: D > 0, in
// a ring of its own in LDS, past the registers (rows at multiples of 16 bytes; see linear_i8_thin_kernel), D = 0, in
// registers.  T is int8_t, or the rows come as floats, up to kFusedRows elements, and every workgroup quantises all
// of them to LDS while its first weights are on their way: less than a launch for it takes.  Bound by memory: 1x25088
// -> 4096 20.5 us, 5.0 TB/s (LONG), 1x2048 -> 1000 4.5 us.
constexpr int kRowsM = 16, kFusedRows = 32768, kRowsMost = 131072;

template <typename T, int D, bool LONG>
__global__ void __launch_bounds__(512)
linear_i8_rows_kernel(const I8Product p, const T *__restrict__ x, int64_t ldx)
{
    constexpr int WAVES = 8, TURN = 256;
    constexpr bool FUSED = sizeof(T) > 1;
    extern __shared__ v4i rows_lds[];                    // quantised rows, `pitch` bytes from one to the next
    constexpr bool RING = D > 0;
    __shared__ v4i ring[WAVES][RING ? D * 256 : 64];
    __shared__ uint32_t mosts[WAVES];
    __shared__ float scales[kRowsM];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = int(blockIdx.x) * 16, pitch = (p.k + TURN - 1) / TURN * TURN + 16;
    const int8_t *const b = p.b + int64_t(min(n0 + r, p.n - 1)) * p.ldb;
    const int whole = p.k / TURN * TURN;
    v4i vb[4];
    const bool words = rows_at_words(p.b, p.ldb);
    auto fetch = [&](v4i (&v)[4], int k0) {
        if (words) {
#pragma unroll
            for (int s = 0; s < 4; ++s) __builtin_memcpy(&v[s], b + k0 + s * 64 + g * 16, 16);
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) v[s] = load16_loose(b + k0 + s * 64 + g * 16);
        }
    };
    int k0 = wave * TURN;
    // the ring: a turn is 16 rows of 256 bytes, 16 lanes read a row together
    const v4u at_b = buffer_at(p.b + int64_t(n0) * p.ldb);
    uint32_t off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 4 + (lane >> 4);
        off[i] = uint32_t(min(row, p.n - 1 - n0)) * uint32_t(p.ldb) + uint32_t((lane & 15) ^ row) * 16u;
    }
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring[wave]));
    const int mine = whole / TURN > wave ? (whole / TURN - wave + WAVES - 1) / WAVES : 0;
    auto issue = [&](int t) {
        if (t >= mine) return;
        const uint32_t to = base + uint32_t(t % (RING ? D : 1)) * 4096u, at = uint32_t(wave + t * WAVES) * uint32_t(TURN);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                         ::"v"(off[i]), "s"(to + uint32_t(i * 1024)), "s"(at_b), "s"(at) : "memory");
    };
    if constexpr (RING) {
#pragma unroll 1
        for (int t = 0; t < D; ++t) issue(t);
    } else {
        if (k0 < whole) fetch(vb, k0);
    }
    int8_t *const q = reinterpret_cast<int8_t *>(rows_lds);
    if constexpr (FUSED) {
        constexpr int N = Vec<T>::N;
        // row m by THREADS threads, all of the workgroup or a wave, KEEP vectors each in registers
        auto quantize_row = [&](int m, int sub, auto threads, auto keep) {
            constexpr int THREADS = decltype(threads)::value, KEEP = decltype(keep)::value;
            const T *row = x + int64_t(m) * ldx;
            Vec<T> v[KEEP];
            load_row<T, THREADS, KEEP>(row, sub, p.k, v);
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < KEEP; ++i) most = most_of(v[i], most);
#pragma unroll 4
            for (int at = (KEEP * THREADS + sub) * N; at < p.k; at += THREADS * N) most = most_of(load_vec(row, at, p.k), most);
            most = most_of_lanes<64>(most);
            if (THREADS > 64) {
                __syncthreads();                         // (the maxima of the row before are read)
                if (lane == 0) mosts[wave] = most;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < WAVES; ++i) most = max(most, mosts[i]);
            }
            const RowScale s = row_scale(most);
            int8_t *to = q + m * pitch;
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                const int at = (i * THREADS + sub) * N;
                if (at >= p.k) continue;
                uint32_t w[N / 4];
                quantize_vec(v[i], s, w);
                __builtin_memcpy(to + at, w, N);
            }
#pragma unroll 2
            for (int at = (KEEP * THREADS + sub) * N; at < p.k; at += THREADS * N) {
                uint32_t w[N / 4];
                quantize_vec(load_vec(row, at, p.k), s, w);
                __builtin_memcpy(to + at, w, N);
            }
            if (sub == 0) scales[m] = s.scale;
        };
        // Long rows one after the other by all waves, else a row a wave: 2 rows of 25088 24.9 us; 16 rows of 512 19.2 us the
        // first way, 4.6 the second; 2 rows of 256 4.7 and 3.4.
        if (p.m < 4 && p.k > 64 * 4 * N) {
            for (int m = 0; m < p.m; ++m) quantize_row(m, int(threadIdx.x), std::integral_constant<int, WAVES * 64>(), std::integral_constant<int, LONG ? kFusedRows / (WAVES * 64 * N) : 4>());
        } else {
            for (int m = wave; m < p.m; m += WAVES) quantize_row(m, lane, std::integral_constant<int, 64>(), std::integral_constant<int, LONG ? 16 : 4>());
        }
        __syncthreads();
    }
    const int8_t *const a = FUSED ? q + min(r, p.m - 1) * pitch : p.a + int64_t(min(r, p.m - 1)) * p.lda;
    v4i acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if constexpr (RING) {
#pragma unroll 1
        for (int t = 0; t < mine; ++t) {
            wait_for_loads<D - 1, 4>(min(D - 1, mine - 1 - t));
            const v4i *const st = ring[wave] + (t % D) * 256;
            const int at = (wave + t * WAVES) * TURN + g * 16;
            v4i va[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                vb[s] = st[r * 16 + ((s * 4 + g) ^ r)];
                __builtin_memcpy(&va[s], a + at + s * 64, 16);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // (read, so that it may be overwritten)
            issue(t + D);
#pragma unroll
            for (int s = 0; s < 4; ++s) acc[s & 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[s], va[s], acc[s & 1], 0, 0, 0);
        }
    }
    while (!RING && k0 < whole) {
        v4i va[4], next[4];
        const int k1 = k0 + WAVES * TURN;
#pragma unroll
        for (int s = 0; s < 4; ++s) __builtin_memcpy(&va[s], a + k0 + s * 64 + g * 16, 16);
        if (k1 < whole) fetch(next, k1);
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[s & 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[s], va[s], acc[s & 1], 0, 0, 0);
#pragma unroll
        for (int s = 0; s < 4; ++s) vb[s] = next[s];
        k0 = k1;
    }
    if (whole < p.k && whole / TURN % WAVES == wave) {   // the last turn is no whole one
        v4i va[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int at = whole + s * 64 + g * 16;
            vb[s] = load16(b, at, p.k);
            // (what lies in LDS beyond k meets weights of zero)
            if (FUSED) __builtin_memcpy(&va[s], a + at, 16);
            else va[s] = load16(a, at, p.k);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[s & 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[s], va[s], acc[s & 1], 0, 0, 0);
    }
    ring[wave][lane] = acc[0] + acc[1];
    __syncthreads();
    if (wave) return;
    v4i s = ring[0][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += ring[w][lane];
    const int n = n0 + g * 4;
    if (r >= p.m || n >= p.n) return;
    const f4 v = values_of(p, s, FUSED ? scales[r] : p.sa[r], channels_at(p, n));
    if (p.y_bf16) store_channels<__bf16, 4>(p, r, n, __builtin_convertvector(v, b4));
    else store_channels<float, 4>(p, r, n, v);
}

}  // namespace

int launch_quantize_rows(const void *x, int64_t ldx, int bf16, int64_t rows, int64_t cols, int8_t *q, int64_t ldq,
                         int64_t q_cols, float *scale, void *stream, const Realign *weights)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t vecs = (q_cols + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4);
    const Realign other = weights ? *weights : Realign{};
    const int64_t pieces = int64_t(other.rows) * other.pieces;
#define PCONV_LAUNCH_AS(T, TPR, KEEP, THREADS, PASSING)                                                                        \
    hipLaunchKernelGGL((quantize_rows_kernel<T, TPR, KEEP, THREADS, PASSING>), dim3(grid + more), dim3(THREADS), 0, st,        \
                       static_cast<const T *>(x), ldx, rows, cols, q, ldq, q_cols, scale, grid, other)
#define PCONV_LAUNCH(TPR, KEEP, THREADS)                                                                                       \
    do {                                                                                                                       \
        const unsigned grid = unsigned(std::min<int64_t>((rows + (THREADS / TPR) - 1) / (THREADS / TPR), 1 << 20));            \
        const unsigned more = unsigned(std::min<int64_t>((pieces + THREADS - 1) / THREADS, 1 << 16));                          \
        const bool once = passing && vecs <= TPR * KEEP;                                                                       \
        if (bf16) { if (once) PCONV_LAUNCH_AS(__bf16, TPR, KEEP, THREADS, true); else PCONV_LAUNCH_AS(__bf16, TPR, KEEP, THREADS, false); } \
        else { if (once) PCONV_LAUNCH_AS(float, TPR, KEEP, THREADS, true); else PCONV_LAUNCH_AS(float, TPR, KEEP, THREADS, false); } \
    } while (0)
    // Activations that are read once and are more than a part of the caches are read past them, so that they do not
    // push out what the product reads (8992x9184 -> 280: 143 us without, 133).
    const bool passing = rows * cols * (bf16 ? 2 : 4) > int64_t(64) << 20;
    // Many rows: two a wave, or one with eight vectors a lane, so that more of them is under way (66 vectors, 100000
    // bf16 rows 59.7 us by a wave each and 38.4 so, 1000 rows 3.2 and 3.6; 288 vectors, 50000 fp32 rows 76.1 us by
    // 256 threads and 49.7 by a wave, 1000 rows 3.8 and 4.4).  (1024 threads for a row of 1244 vectors: 7962 rows 107
    // us, with 256 55; 300 rows 7.8 and 5.5; of 2296: 8992 rows 116 and 94)
    if (vecs <= 8) PCONV_LAUNCH(8, 1, 256);
    else if (vecs <= 16) PCONV_LAUNCH(16, 1, 256);
    else if (vecs <= 32) PCONV_LAUNCH(16, 2, 256);
    else if (vecs <= 64) PCONV_LAUNCH(16, 4, 256);
    else if (vecs <= 128 && rows > 4096) PCONV_LAUNCH(32, 4, 256);
    else if (vecs <= 128) PCONV_LAUNCH(64, 2, 256);
    else if (vecs <= 256) PCONV_LAUNCH(64, 4, 256);
    else if (vecs <= 512 && rows > 8192) PCONV_LAUNCH(64, 8, 256);
    else if (vecs <= 512) PCONV_LAUNCH(256, 2, 256);
    else if (vecs <= 1024) PCONV_LAUNCH(256, 4, 256);
    else if (vecs <= 2048 && rows >= 128) PCONV_LAUNCH(256, 8, 256);
    else if (vecs <= 4096 && rows >= 128) PCONV_LAUNCH(256, 16, 256);
    else if (vecs <= 4096) PCONV_LAUNCH(1024, 4, 1024);
    else PCONV_LAUNCH(1024, 8, 1024);
#undef PCONV_LAUNCH
#undef PCONV_LAUNCH_AS
    return check_launch("pconv_quantize_rows");
}

namespace {

// How a product of more rows than linear_i8_rows_kernel serves is cut up: the tile (an index into launch_tiles) and over how
// many workgroups the length of k is split.
struct Cut { int tile, splits; };

constexpr int kTiles = 4, kTileM[kTiles] = {32, 64, 128, 256}, kTileN[kTiles] = {128, 128, 128, 256};
constexpr int64_t kUnits = 256;                          // compute units

int64_t tiles_of(const Cut &c, int64_t m, int64_t n) { return ((m + kTileM[c.tile] - 1) / kTileM[c.tile]) * ((n + kTileN[c.tile] - 1) / kTileN[c.tile]); }

// The cheapest by a count of cycles: a compute unit takes its tiles one after the other, a stage of a tile at the rate of the
// matrix units (half of their peak) or of what 40 bytes a cycle bring from the level-2 cache, whichever is slower.
// Joining the parts of k is one more launch and reads and writes the sums.
Cut cut_of(int64_t m, int64_t n, int64_t k)
{
    constexpr int64_t stage_cycles[kTiles] = {512, 614, 1100, 4096}, start = 4000, join = 9000;
    const int64_t stages = (k + 127) / 128;
    Cut best{0, 1};
    double least = 0;
    for (int t = 0; t < kTiles; ++t)
        for (int64_t s = 1; s == 1 || (s <= 32 && s * 4 <= stages); s *= 2) {
            const int64_t tiles = tiles_of(Cut{t, int(s)}, m, n);
            double c = double((tiles * s + kUnits - 1) / kUnits) * double((stages + s - 1) / s) * double(stage_cycles[t]) + start;
            if (s > 1) c += join + double(s) * double(m) * double(n) * 8 / 2000;
            if ((t == 0 && s == 1) || c < least || (c == least && s == 1)) { least = c; best = Cut{t, int(s)}; }
        }
    return best;
}

// Sets of waves of a workgroup: two, and as many stages as LDS holds, where a compute unit has one workgroup (17x2048
// -> 1000: 8.6 us with four stages), else room for two workgroups.  The largest tile fills a compute unit with one
// set.
int sets_of(const Cut &c, int64_t tiles) { return c.tile < 3 && tiles * c.splits <= kUnits ? 2 : 1; }

template <int BM, int BN, int WM, int WN, int S, int KG>
void launch_tiles(const I8Product &p, int splits, int *part, hipStream_t st)
{
    const unsigned grid = unsigned(((int64_t(p.m) + BM - 1) / BM) * ((int64_t(p.n) + BN - 1) / BN) * splits);
    if (p.y_bf16) hipLaunchKernelGGL((matmul_i8_kernel<__bf16, BM, BN, WM, WN, S, KG>), dim3(grid), dim3(KG * WM * WN * 64), 0, st, p, splits, part);
    else hipLaunchKernelGGL((matmul_i8_kernel<float, BM, BN, WM, WN, S, KG>), dim3(grid), dim3(KG * WM * WN * 64), 0, st, p, splits, part);
}

int64_t rows_groups(int64_t n) { return (n + 15) / 16; }

template <typename T>
int launch_rows(const I8Product &p, const T *x, int64_t ldx, hipStream_t st)
{
    const size_t lds = sizeof(T) > 1 ? size_t(p.m) * ((p.k + 255) / 256 * 256 + 16) : 0;
    if (rows_groups(p.n) > kMaxGroups) return too_many_groups();
    const unsigned grid = unsigned(rows_groups(p.n));
    // The ring takes 64 KB of LDS: where a compute unit has one workgroup at most, or two fit still (1x25088 -> 1000
    // 18.3 us without it, 12.0; 2x8192 -> 8192 16.3 and, one workgroup a compute unit with it, 19.6).  There long
    // rows stay in registers between their two uses (10.9 us; 1x4096 -> 1000 4.8 us with few registers and 5.9; rows
    // that a wave has, 10x3200 -> 1856 fp32 8.8 and 10.5, 10x1168 7.2 and 6.0).
    if constexpr (sizeof(T) > 1) {
        const bool one = int64_t(grid) <= kUnits;
        if (rows_at_16(p.b, p.ldb) && (one || lds <= 14 * 1024)) {
            if (one && (p.m < 4 ? p.k > kFusedRows / 4 : p.k >= 64 * 10 * Vec<T>::N))
                hipLaunchKernelGGL((linear_i8_rows_kernel<T, 2, true>), dim3(grid), dim3(512), lds, st, p, x, ldx);
            else
                hipLaunchKernelGGL((linear_i8_rows_kernel<T, 2, false>), dim3(grid), dim3(512), lds, st, p, x, ldx);
            return check_launch("pconv_linear_i8 (few rows)");
        }
    }
    hipLaunchKernelGGL((linear_i8_rows_kernel<T, 0, false>), dim3(grid), dim3(512), lds, st, p, x, ldx);
    return check_launch("pconv_linear_i8 (few rows)");
}

// Rows of T (int8_t: quantised already, with their scales in p) times weights, k up to kThinK.
template <typename T, int KS>
int launch_thin_steps(const I8Product &p, const T *x, int64_t ldx, hipStream_t st)
{
    const bool exact = p.k > 0 && p.k % 16 == 0 && p.n % 8 == 0 && rows_at_16(p.b, p.ldb);
    const bool narrow = p.n <= 128;                      // half of the waves would have no channels: they take half of the rows
    const int rows = exact ? thin_rows(KS) : 32, channels = exact && !narrow ? 256 : 128;
    const int64_t tiles = (int64_t(p.m) + rows - 1) / rows, groups = (int64_t(p.n) + channels - 1) / channels;
    // (every part quantises the rows again: no more of them than make 512 workgroups)
    const int64_t parts = std::min<int64_t>(groups, std::max<int64_t>(1, (KS <= 8 ? 512 : 256) / tiles));
    const int part_n = int((groups + parts - 1) / parts * channels);
    if (tiles > kMaxGroups) return too_many_groups();
    const dim3 grid(unsigned(tiles), unsigned((int64_t(p.n) + part_n - 1) / part_n));
#define PCONV_LAUNCH(Y)                                                                                                        \
    do {                                                                                                                       \
        if (exact && narrow) hipLaunchKernelGGL((linear_i8_thin_kernel<T, Y, KS, 2>), grid, dim3(512), 0, st, p, x, ldx, part_n); \
        else if (exact) hipLaunchKernelGGL((linear_i8_thin_kernel<T, Y, KS, 1>), grid, dim3(512), 0, st, p, x, ldx, part_n);   \
        else if constexpr (KS <= 8) hipLaunchKernelGGL((linear_i8_thin_ragged_kernel<T, Y, KS>), grid, dim3(256), 0, st, p, x, ldx, part_n); \
    } while (0)
    if (p.y_bf16) PCONV_LAUNCH(__bf16); else PCONV_LAUNCH(float);
#undef PCONV_LAUNCH
    return check_launch("pconv_linear_i8 (short rows)");
}

template <typename T>
int launch_thin(const I8Product &p, const T *x, int64_t ldx, hipStream_t st)
{
    if (p.k <= 64) return launch_thin_steps<T, 1>(p, x, ldx, st);
    if (p.k <= 128) return launch_thin_steps<T, 2>(p, x, ldx, st);
    if (p.k <= 256) return launch_thin_steps<T, 4>(p, x, ldx, st);
    if constexpr (sizeof(T) > 1) {                       // (quantised rows of more than kThinK go in tiles)
        if (p.k > 1024) return launch_thin_steps<T, 32>(p, x, ldx, st);
        if (p.k > kThinK) return launch_thin_steps<T, 16>(p, x, ldx, st);
    }
    return launch_thin_steps<T, 8>(p, x, ldx, st);
}

}  // namespace

// The kernel for few rows up to kRowsMost activations: each of its workgroups reads all of them (16 rows of 25088:
// 33.5 us, in tiles 28.6; 4 rows 26.6 and 28.1; 16 rows of 4096 10.0 and 12.2).
static bool few(int64_t m, int64_t k) { return m <= kRowsM && m * k <= kRowsMost; }
static bool thin(int64_t m, int64_t k) { return m > kRowsM && k <= kThinK; }

// Rows of up to kThinLongK in whole pieces, quantised within the product as short rows are: one launch, no work space
// (4.9 us less on the host).  The loads, the quantising and the products of a workgroup follow each other and no
// other one is there to fill in, so that is right for few rounds of workgroups only: 1000x1024 -> 256 fp32 12.8 us,
// apart 15.3 (the GPU's part 13.0 and 9.9); 16000x768 -> 256 bf16 15 and 22; 50000x1024 -> 256 fp32 86 and 71; above
// 1024 with 32 rows a workgroup 4000x1536 -> 512 bf16 15 and 18.6, 16000x1536 -> 1024 fp32 73 and 57.
static bool thin_long(int64_t m, int64_t n, int64_t k, bool b_at_16)
{
    if (m <= kRowsM || k <= kThinK || k > kThinLongK || k % 16 != 0 || n % 8 != 0 || n > 2048 || !b_at_16) return false;
    return k <= 1024 ? m <= kUnits * 64 : (m + 31) / 32 * ((n + 255) / 256) <= 2 * kUnits;
}

bool linear_i8_fused(int64_t m, int64_t n, int64_t k, bool b_at_16)
{
    return m <= kRowsM ? m * k <= kFusedRows : thin(m, k) || thin_long(m, n, k, b_at_16);
}

int launch_linear_i8_fused(const I8Product &p, const void *x, int64_t ldx, int bf16, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (few(p.m, p.k)) return bf16 ? launch_rows(p, static_cast<const __bf16 *>(x), ldx, st) : launch_rows(p, static_cast<const float *>(x), ldx, st);
    return bf16 ? launch_thin(p, static_cast<const __bf16 *>(x), ldx, st) : launch_thin(p, static_cast<const float *>(x), ldx, st);
}

int check_linear_i8_apart(int64_t m, int64_t n, int64_t k)
{
    if (few(m, k)) return rows_groups(n) > kMaxGroups ? too_many_groups() : PCONV_OK;
    const Cut c = cut_of(m, n, k);
    return tiles_of(c, m, n) * c.splits > kMaxGroups ? too_many_groups() : PCONV_OK;
}

bool matmul_i8_aligns(int64_t m, int64_t k) { return !few(m, k) && !thin(m, k); }

Realign realigned(const int8_t *from, int64_t ld, int rows, int k, int8_t *to) { return Realign{from, to, ld, rows, k, (k + 15) / 16}; }

int64_t matmul_i8_work_bytes(int64_t m, int64_t n, int64_t k, bool a_at_16, bool b_at_16)
{
    if (!matmul_i8_aligns(m, k)) return 0;
    const Cut c = cut_of(m, n, k);
    const int64_t row = (k + 15) / 16 * 16;
    return (a_at_16 ? 0 : m * row) + (b_at_16 ? 0 : n * row) + (c.splits > 1 ? c.splits * m * ((n + 3) / 4 * 4) * 4 : 0);
}

pconv_i8_plan matmul_i8_plan(int64_t m, int64_t n, int64_t k)
{
    if (few(m, k)) return pconv_i8_plan{1, 0, 0, 0, 0};
    if (thin(m, k)) return pconv_i8_plan{2, 0, 0, 0, 0};
    const Cut c = cut_of(m, n, k);
    return pconv_i8_plan{3, kTileM[c.tile], kTileN[c.tile], sets_of(c, tiles_of(c, m, n)), c.splits};
}

int launch_matmul_i8(const I8Product &product, void *work, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    I8Product p = product;
    if (few(p.m, p.k)) return launch_rows(p, p.a, p.lda, st);
    if (thin(p.m, p.k)) return launch_thin(p, p.a, p.lda, st);
    const Cut c = cut_of(p.m, p.n, p.k);
    const int64_t tiles = tiles_of(c, p.m, p.n);
    if (tiles * c.splits > kMaxGroups) return too_many_groups();
    int8_t *at = static_cast<int8_t *>(work);
    Realign moved[2] = {};
    unsigned count = 0;
    const auto move = [&](const int8_t *&from, int64_t &ld, int rows) {
        if (rows_at_16(from, ld)) return;
        moved[count] = realigned(from, ld, rows, p.k, at);
        from = at;
        ld = int64_t(moved[count++].pieces) * 16;
        at += rows * ld;
    };
    move(p.a, p.lda, p.m);
    move(p.b, p.ldb, p.n);
    if (count) {
        const int64_t most = int64_t(std::max(moved[0].rows, moved[1].rows)) * moved[0].pieces;
        hipLaunchKernelGGL(realign_kernel, dim3(unsigned(std::min<int64_t>((most + 255) / 256, 1 << 16)), count), dim3(256), 0, st, moved[0], moved[1]);
        if (const int rc = check_launch("pconv_matmul_i8 (aligning rows)")) return rc;
    }
    int *const sums = reinterpret_cast<int *>(at);
    const bool two = sets_of(c, tiles) == 2;
    if (c.tile == 0 && two) launch_tiles<32, 128, 1, 4, 4, 2>(p, c.splits, sums, st);
    else if (c.tile == 0) launch_tiles<32, 128, 1, 4, 4, 1>(p, c.splits, sums, st);
    else if (c.tile == 1 && two) launch_tiles<64, 128, 2, 2, 3, 2>(p, c.splits, sums, st);
    else if (c.tile == 1) launch_tiles<64, 128, 2, 2, 3, 1>(p, c.splits, sums, st);
    else if (c.tile == 2 && two) launch_tiles<128, 128, 2, 2, 2, 2>(p, c.splits, sums, st);
    else if (c.tile == 2) launch_tiles<128, 128, 2, 2, 2, 1>(p, c.splits, sums, st);
    else launch_tiles<256, 256, 2, 4, 2, 1>(p, c.splits, sums, st);
    if (const int rc = check_launch("pconv_matmul_i8")) return rc;
    if (c.splits == 1) return PCONV_OK;
    const int64_t quads = (int64_t(p.n) + 3) / 4 * p.m;
    hipLaunchKernelGGL(matmul_i8_join_kernel, dim3(unsigned(std::min<int64_t>((quads + 255) / 256, 1 << 16))), dim3(256), 0, st, p, c.splits, sums);
    return check_launch("pconv_matmul_i8 (joining the parts of k)");
}

}  // namespace pconv
