// Microscaled 4-bit floats: quantising rows, and products with one power of two as the scale of each 32 values of k.
//
//   y[m][n] = act(sum_b 2^(sa[m][b] + sb[n][b] - 254) sum_(k in block b) a[m][k] b[n][k] + bias[n])
//
// A block is 16 bytes of a row, which is what a lane of the matrix instruction takes: 16 rows by 4 blocks, each lane a block
// and the byte of its scale.  The order in which k is summed is free as long as both operands have the same, so lanes
// 16 g .. take neighbouring blocks in neighbouring steps: their scales are then neighbouring bytes, read together.  The
// weights are the instruction's first operand and the activations its second, so that a lane ends up with four
// neighbouring channels of one row of y.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "pconv_internal.h"
#include "pconv_ops.h"
#include "pconv_rows.h"

namespace pconv {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

int too_many_groups()
{
    set_error("4-bit layers: too many workgroups for one launch");
    return PCONV_UNSUPPORTED;
}

// ---- quantising rows ---------------------------------------------------------------------------------------------------

// The scale's byte, X + 127, of a block whose largest magnitude has these bits: the exponent less two, at least 0; 255 where
// the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t block_scale(uint32_t most)
{
    const uint32_t e = most >> 23;
    return e >= 255u ? 255u : max(e, 2u) - 2u;
}

// 2^X as a float (2^-127 is a denormal number, which the conversion takes).
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// Eight neighbouring values of a row; 4 lanes have a block.
template <typename T> struct Eight;
template <> struct Eight<float> {
    f4 v[2];
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i / 4][i % 4]) & 0x7FFFFFFFu);
        return m;
    }
    // (the conversion divides by the scale and rounds to the nearest, ties to even, 6 at most)
    __device__ __forceinline__ uint32_t codes(float s) const
    {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][0], v[0][1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][2], v[0][3], s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[1][0], v[1][1], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[1][2], v[1][3], s, 3);
        return w;
    }
};
template <> struct Eight<__bf16> {
    b8 v;
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    __device__ __forceinline__ uint32_t most() const
    {
        Vec<__bf16> x;
        x.v = v;
        return most_of(x, 0);
    }
    __device__ __forceinline__ uint32_t codes(float s) const
    {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, b2{v[0], v[1]}, s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, b2{v[2], v[3]}, s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, b2{v[4], v[5]}, s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, b2{v[6], v[7]}, s, 3);
        return w;
    }
};

// Elements [at, at + 8) of a row of `cols`; beyond its end zero.
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T *row, int64_t at, int64_t cols)
{
    Eight<T> e;
    if (__builtin_expect(at + 8 <= cols, 1)) {
        __builtin_memcpy(&e.v, row + at, 8 * sizeof(T));
    } else {
        T all[8] = {};
        if (__builtin_expect(at < cols, 0)) {            // (a row's last eight values)
#pragma unroll
            for (int i = 0; i < 8; ++i) all[i] = at + i < cols ? row[at + i] : T(0.0f);
        }
        __builtin_memcpy(&e.v, all, 8 * sizeof(T));
    }
    return e;
}

// The largest value over the four lanes of a block.
__device__ __forceinline__ uint32_t most_of_block(uint32_t v)
{
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xF, 0xF, true)));       // the other of a pair
    return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x4E, 0xF, 0xF, true)));    // the other pair of four
}

// 32 lanes have 256 values of a row, which is a slab: 8 rows a workgroup, `slabs` of them shared by gridDim.y workgroups.
// Blocks behind the row's last one get scale 0.  Eight values a lane are one load of 16 or 32 bytes and one store of 4, and the
// conversion is an instruction: bound by memory, 8192x4096 bf16 17.4 us, 4.9 TB/s.
template <typename T>
__global__ void __launch_bounds__(256)
quantize_mx4_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int64_t cols, int64_t slabs, uint8_t *__restrict__ q,
                    int64_t ldq, uint8_t *__restrict__ scale, int64_t slab_stride)
{
    const int sub = int(threadIdx.x) & 31;
    for (int64_t r = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5); r < rows; r += int64_t(gridDim.x) * 8) {
        const T *row = x + r * ldx;
        for (int64_t s = blockIdx.y; s < slabs; s += gridDim.y) {
            const int64_t at = s * 256 + sub * 8;
            const Eight<T> e = load_eight(row, at, cols);
            const uint32_t byte = block_scale(most_of_block(e.most()));
            const uint32_t w = byte == 255u ? 0u : e.codes(scale_value(byte));
            if (at / 32 * 32 < cols) __builtin_memcpy(q + r * ldq + at / 2, &w, 4);
            if (sub % 4 == 0) scale[s * slab_stride + r * 8 + sub / 4] = uint8_t(byte);
        }
    }
}

// ---- the product --------------------------------------------------------------------------------------------------------

// Four neighbouring channels of one row of y, from n on.  ReLU keeps NaN.
__device__ __forceinline__ f4 bias_at(const Mx4Product &p, int n)
{
    f4 b = {0, 0, 0, 0};
    if (!p.bias) return b;
    if (__builtin_expect(n + 4 <= p.n, 1)) {
        __builtin_memcpy(&b, p.bias + n, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = p.bias[min(n + i, p.n - 1)];      // (what lies beyond the last channel is not stored)
    }
    return b;
}

__device__ __forceinline__ f4 values_of(const Mx4Product &p, f4 acc, f4 bias)
{
    f4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = acc[i] + bias[i];
        if (p.relu) v[i] = v[i] < 0.0f ? 0.0f : v[i];
    }
    return v;
}

template <typename Y, int N, typename V>
__device__ __forceinline__ void store_channels(const Mx4Product &p, int m, int n, V v)
{
    Y *y = static_cast<Y *>(p.y) + (int64_t(m) * p.ldy + n);
    if (__builtin_expect(n + N <= p.n, 1)) {
        if constexpr (sizeof(Y) == 2) {
            if (reinterpret_cast<uintptr_t>(y) & 2) {    // (between its ends the run lies at whole words)
                y[0] = v[0];
                __builtin_memcpy(__builtin_assume_aligned(y + 1, 4), reinterpret_cast<const Y *>(&v) + 1, (N - 2) * sizeof(Y));
                y[N - 1] = v[N - 1];
                return;
            }
        }
        __builtin_memcpy(y, &v, N * sizeof(Y));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (n + i < p.n) y[i] = v[i];
    }
}

// acc += the 16 rows of b by the 16 rows of a over 4 blocks; STEP: which of the bytes of sb and sa are the scales.
template <int STEP>
__device__ __forceinline__ f4 multiply_blocks(v4i b, v4i a, f4 acc, int sb, int sa)
{
    const v8i b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1), a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b8, a8, acc, 4, 4, STEP, sb, STEP, sa);
}

// The sums of rows m + 16 i and the NT * 16 channels from n0 on, to y or, where `splits` workgroups share k, to `part`; the lane
// has `lane & 15` in m and its group in `g`.  `inside`: all of the workgroup's tile is in y (asking for each store
// whether it is takes 8192x4096 -> 4096 from 71.1 to 75.5 us).
template <typename Y, int MT, int NT>
__device__ __forceinline__ void finish_tile(const Mx4Product &p, const f4 (&acc)[MT][NT], int m, int n0, int g, bool inside, int split, int splits, float *part)
{
    if (splits > 1) {
        const int64_t n4 = (int64_t(p.n) + 3) / 4 * 4;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = n0 + Deal<Y>::first(j, g);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (m + 16 * i < p.m && n < p.n) __builtin_memcpy(part + (int64_t(split) * p.m + m + 16 * i) * n4 + n, &acc[i][j], 16);
        }
        return;
    }
    f4 bias[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) bias[j] = bias_at(p, n0 + Deal<Y>::first(j, g));
    if (inside && sizeof(Y) == 2 && ((reinterpret_cast<uintptr_t>(p.y) | uintptr_t(p.ldy * 2)) & 2)) {
        // Rows of bf16 that begin within a word: stores there take twice as long (8192x512 -> 4095 43.8 us, and 22.5 with 4096; so 29.3).  A
        // lane takes the last channel of the one before it in place of its own last, so that it stores whole words; the wave's
        // first channel and its last go by themselves.
        const int lane = int(threadIdx.x) & 63;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            uint16_t *const row = static_cast<uint16_t *>(p.y) + (int64_t(m + 16 * i) * p.ldy + n0);
            const bool within = (reinterpret_cast<uintptr_t>(row) & 2) != 0;
            uint32_t carried = 0;
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
                const f4 v = values_of(p, acc[i][j], bias[j]), w = values_of(p, acc[i][j + 1], bias[j + 1]);
                const b8 o = __builtin_convertvector(__builtin_shufflevector(v, w, 0, 1, 2, 3, 4, 5, 6, 7), b8);
                v4u x;
                __builtin_memcpy(&x, &o, 16);
                const uint32_t other = uint32_t(__shfl(int(x.w), (lane + 48) & 63)), before = g ? other : carried;
                carried = other;
                const v4u moved = {__builtin_amdgcn_alignbit(x.x, before, 16), __builtin_amdgcn_alignbit(x.y, x.x, 16), __builtin_amdgcn_alignbit(x.z, x.y, 16),
                                   __builtin_amdgcn_alignbit(x.w, x.z, 16)};
                uint16_t *const to = row + Deal<Y>::first(j, g);
                if (within && j == 0 && g == 0) {
                    to[0] = uint16_t(x.x);
                    __builtin_memcpy(__builtin_assume_aligned(to + 1, 4), reinterpret_cast<const uint32_t *>(&moved) + 1, 12);
                } else {
                    const v4u all = within ? moved : x;
                    __builtin_memcpy(__builtin_assume_aligned(within ? to - 1 : to, 4), &all, 16);
                }
                if (within && j + 2 == NT && g == 3) to[7] = uint16_t(x.w >> 16);
            }
        }
        return;
    }
    if (inside) {
        Y *row = static_cast<Y *>(p.y) + (int64_t(m) * p.ldy + n0);
#pragma unroll
        for (int i = 0; i < MT; ++i, row += 16 * p.ldy)
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
                const f4 v = values_of(p, acc[i][j], bias[j]), w = values_of(p, acc[i][j + 1], bias[j + 1]);
                if constexpr (sizeof(Y) == 4) {
                    __builtin_memcpy(row + Deal<Y>::first(j, g), &v, 16);
                    __builtin_memcpy(row + Deal<Y>::first(j + 1, g), &w, 16);
                } else {
                    const b8 o = __builtin_convertvector(__builtin_shufflevector(v, w, 0, 1, 2, 3, 4, 5, 6, 7), b8);
                    __builtin_memcpy(row + Deal<Y>::first(j, g), &o, 16);
                }
            }
        return;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if (m + 16 * i >= p.m) continue;
#pragma unroll
        for (int j = 0; j < NT; j += 2) {
            const int n = n0 + Deal<Y>::first(j, g), n2 = n0 + Deal<Y>::first(j + 1, g);
            if (n >= p.n) continue;
            const f4 v = values_of(p, acc[i][j], bias[j]), w = values_of(p, acc[i][j + 1], bias[j + 1]);
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

// Order of the blocks of a row in LDS: place block ^ key.  A read of 16 bytes a lane goes by sixteen lanes at once: of rows 0 to 3
// and 12 to 15 with one block and 4 to 11 with that of the next group of lanes, two blocks further, and the other way round.
// Rows lie 128 bytes apart, so that the eight that begin in the same half of LDS's 256 bytes of banks need eight places: the
// first four have keys 0 to 3, which an exchange of blocks two apart keeps among themselves, the others 4 to 7.  (Keys 0 to 7 in
// order: half of the cycles in which LDS is read are conflicts.)  Activations are read row by row, weights as they are dealt.
__device__ __forceinline__ int key_of(int h) { return (h & 3) | (((h >> 1) ^ (h >> 2)) & 1) << 2; }
__device__ __forceinline__ int key_of_row(int row) { return key_of((row >> 1) & 7); }
template <typename Y> __device__ __forceinline__ int key_of_channel(int row) { return key_of(sizeof(Y) == 4 ? (row >> 1) & 7 : ((row >> 1) & 1) | ((row >> 2) & 6)); }

// Tiles of BM rows of y and BN channels, WM x WN waves, and KG such sets of waves that take the stages in turn.  A slab of
// all the tile's rows is a stage: 128 bytes of values and 8 of scales a row; S stages lie in LDS.  A row of a stage is
// eight blocks, stored in an order that depends on the row so that the eight rows that are read at once lie in different
// banks.
//
// Stages go from memory to LDS past the registers, S - 1 of them ahead of the one that is multiplied; a wave waits
// for its own loads of the next stage, and the barrier then tells it that everybody's are there and that the stage
// before is read.  In the last stage the blocks behind the end of k are zeros.
//
// `splits` workgroups share a tile, each with its part of k; their sums go to `part` [splits][m][n4], n4 = n rounded
// up to four.
//
// 8192x4096 -> 4096 takes 69 to 75 us, 3.7 to 4.0 PFLOP/s.  The matrix units alone, out of registers, do 6.0 to 6.7 PFLOP/s with codes as
// they come (45 us) and 8.9 with zeros (31), but zeros take the kernel 63 to 68: the card's power is worth some 6 us, the rest is that three pipes
// of nearly equal length, loads to LDS (2044 cycles a slab by themselves), reads of LDS (2088) and products (2272), run beside each other
// only in part from barrier to barrier (3240 to 3580 a slab, the matrix units busy for 45 % of the launch), and that all compute units store their
// outputs, 64 MiB, at the end of each of two rounds with no product under way.  Four waves of 128x128, stages of half a slab, two groups
// of waves in turn, or loads and products of a wave interleaved by hand took 69 to 75 as well.
template <typename Y, int BM, int BN, int WM, int WN, int S, int KG>
__global__ void __launch_bounds__(KG * WM * WN * 64)
matmul_mx4_kernel(const Mx4Product p, int splits, float *part)
{
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    constexpr int PA = BM / 8 / NW, PB = BN / 8 / NW;    // pieces of eight rows that a wave stages
    constexpr int PS = ((BM + BN) / 32 + NW - 1) / NW;   // and of the scales of 32 rows
    static_assert(PA * NW * 8 == BM && PB * NW * 8 == BN && BM % 32 == 0 && BN % 32 == 0 && NT % 2 == 0, "");
    constexpr int STAGE = (BM + BN) * 8 + PS * NW * 16, SUMS = NW * MT * NT * 64;        // (in pieces of 16 bytes)
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
    const int r = lane & 15, g = lane >> 4;
    // this workgroup's part of k
    const int stages = (p.blocks + 7) / 8;
    const int s_begin = int(int64_t(stages) * split / splits), s_end = int(int64_t(stages) * (split + 1) / splits);

    const int key = key_of(r >> 1);                      // (of all the rows that the lane reads)

    f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f4{0, 0, 0, 0};

    // (`have`: blocks of k from the stage's first on; of one that is not there the scale may be any byte, NaN's too)
    auto multiply = [&](const v4i *st, int have) {
        const int mask = 0xFFFF >> max(0, min(16, (2 * g + 2 - have) * 8));
        const uint16_t *const scales = reinterpret_cast<const uint16_t *>(st + (BM + BN) * 8);
        int sa[MT], sb[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = scales[(wm + i * 16 + r) * 4 + g] & mask;
#pragma unroll
        for (int j = 0; j < NT; ++j) sb[j] = scales[(BM + wn + Deal<Y>::row(j, r)) * 4 + g] & mask;
        auto step = [&](auto kk) {
            constexpr int KK = decltype(kk)::value;
            v4i a[MT], b[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int row = wm + i * 16 + r;
                a[i] = st[row * 8 + ((2 * g + KK) ^ key)];
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int row = wn + Deal<Y>::row(j, r);
                b[j] = st[BM * 8 + row * 8 + ((2 * g + KK) ^ key)];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = multiply_blocks<KK>(b[j], a[i], acc[i][j], sb[j], sa[i]);
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
    };

    const v4u at_a = buffer_at(reinterpret_cast<const int8_t *>(p.a) + int64_t(m0) * p.lda + int64_t(s_begin) * 128);
    const v4u at_b = buffer_at(reinterpret_cast<const int8_t *>(p.b) + int64_t(n0) * p.ldb + int64_t(s_begin) * 128);
    uint32_t off_a[PA], off_b[PB], off_s[PS];
    int end_a[PA], end_b[PB];                            // (a lane's block is loaded if the stage has it)
#pragma unroll
    for (int i = 0; i < PA; ++i) {
        const int row = (i * NW + wave) * 8 + (lane >> 3);
        end_a[i] = (lane & 7) ^ key_of_row(row);
        off_a[i] = uint32_t(min(row, p.m - 1 - m0)) * uint32_t(p.lda) + uint32_t(end_a[i] * 16);
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
        const int row = (i * NW + wave) * 8 + (lane >> 3);
        end_b[i] = (lane & 7) ^ key_of_channel<Y>(row);
        off_b[i] = uint32_t(min(row, p.n - 1 - n0)) * uint32_t(p.ldb) + uint32_t(end_b[i] * 16);
    }
    // 32 rows of one operand have 256 bytes of scales, a word a lane
#pragma unroll
    for (int i = 0; i < PS; ++i) {
        const int row = (i * NW + wave) * 32 + (lane >> 1);
        off_s[i] = uint32_t(row < BM ? min(row, p.m - 1 - m0) : min(row - BM, p.n - 1 - n0)) * 8u + uint32_t(lane & 1) * 4u;
    }
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)) + uint32_t(set) * uint32_t(STAGE * 16);
    const int count = s_end - s_begin;
    // (written as assembly so that the compiler does not wait for these loads before every read of LDS)
    // stage `turn` of this set is stage turn * KG + set of all
    auto stage = [&](int turn) {
        const int s = turn * KG + set;
        const uint32_t to = base + uint32_t(turn % S) * uint32_t(KG * STAGE * 16), k0 = uint32_t(s) * 128u;
        const int have = p.blocks - (s_begin + s) * 8;
#pragma unroll
        for (int i = 0; i < PA; ++i)
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                         ::"v"(end_a[i] < have ? off_a[i] : kNowhere), "s"(to + uint32_t((i * NW + wave) * 1024)), "s"(at_a), "s"(k0) : "memory");
#pragma unroll
        for (int i = 0; i < PB; ++i)
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                         ::"v"(end_b[i] < have ? off_b[i] : kNowhere), "s"(to + uint32_t(BM * 128 + (i * NW + wave) * 1024)), "s"(at_b), "s"(k0) : "memory");
#pragma unroll
        for (int i = 0; i < PS; ++i) {
            const bool of_a = (i * NW + wave) * 32 < BM;
            const uint8_t *const from = of_a ? p.sa + int64_t(s_begin + s) * p.slab_a + int64_t(m0) * 8 : p.sb + int64_t(s_begin + s) * p.slab_b + int64_t(n0) * 8;
            const v4u at_s = buffer_at(reinterpret_cast<const int8_t *>(from));
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dword %0, %2, 0 offen lds"
                         ::"v"(off_s[i]), "s"(to + uint32_t((BM + BN) * 128 + (i * NW + wave) * 256)), "s"(at_s) : "memory");
        }
    };
    constexpr int L = PA + PB + PS;
    static_assert((S - 2) * L <= 63, "");
    const int mine = (count - set + KG - 1) / KG;        // stages of this set (count >= 0, so at least 0)
    const int turns = (count + KG - 1) / KG;
#pragma unroll
    for (int t = 0; t < S - 1; ++t)
        if (t < mine) stage(t);
#pragma unroll 1
    for (int t = 0; t < turns; ++t) {
        // the loads of this turn are done when at most those of the turns behind it are under way
        wait_for_stages<S - 2, L>(min(S - 2, max(0, mine - 1 - t)));
        if (t + S - 1 < mine) stage(t + S - 1);
        if (KG == 1 || t * KG + set < count) multiply(lds + ((t % S) * KG + set) * STAGE, p.blocks - (s_begin + t * KG + set) * 8);
    }
    if constexpr (KG > 1) {                              // the sets' sums come together
        __syncthreads();
        f4 *const to = reinterpret_cast<f4 *>(lds) + wave * (MT * NT * 64) + lane;
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

    finish_tile<Y, MT, NT>(p, acc, m0 + wm + r, n0 + wn, g, m0 + BM <= p.m && n0 + BN <= p.n, split, splits, part);
}

// y of the sums of `splits` parts of k; a thread has four channels.  (32x4096 of 8 parts 3.8 us: a launch, and parts that come from
// the memory-side cache.)
__global__ void __launch_bounds__(256)
matmul_mx4_join_kernel(const Mx4Product p, int splits, const float *__restrict__ part)
{
    const int64_t quads = (int64_t(p.n) + 3) / 4, all = quads * p.m;
    for (int64_t t = int64_t(blockIdx.x) * 256 + threadIdx.x; t < all; t += int64_t(gridDim.x) * 256) {
        const int m = int(t / quads), n = int(t % quads) * 4;
        f4 s = {0, 0, 0, 0};
#pragma unroll 4
        for (int i = 0; i < splits; ++i) {
            f4 v;
            __builtin_memcpy(&v, part + (int64_t(i) * all + t) * 4, 16);
            s += v;
        }
        const f4 v = values_of(p, s, bias_at(p, n));
        if (p.y_bf16) store_channels<__bf16, 4>(p, m, n, __builtin_convertvector(v, b4));
        else store_channels<float, 4>(p, m, n, v);
    }
}

// Few rows (up to 32, RG groups of 16): 16 channels a workgroup, whose waves share k and add their sums in LDS.  Reading the weights is all
// of it; they come in turns of 16 blocks, in a ring of D turns in LDS that is the wave's own, past the registers, and no
// barrier stands in the loop.  The waves take whole turns in rounds, and what is left behind the last whole round is dealt
// out among all of them: a turn of one wave alone at the end takes a whole latency of memory (25088 -> 8192: 25.5 us with
// one turn left over, 21.5 without).  Workgroups begin with different rounds, so that rows that lie a power of two apart
// are not all read in the same places at one time (32768 -> 4096: 19.5 us if they are, 17.0).  1x25088 -> 4096 fp32 takes 11.7 us,
// 4.7 TB/s.  The rows of activations lie in LDS for all waves: they come as floats, and every workgroup quantises all of them
// while its first weights are on their way, or as blocks (T is uint8_t).
constexpr int kFewRows = 32, kTurn = 16;                 // (blocks)
constexpr size_t kFewRing = 8 * (16 * 256 + 256);        // bytes of one turn of all waves

// Rows in LDS: values, and behind all of them the scales; behind each row room for what a wave's last turn reads for nothing.
struct FewRows {
    int pitch, scales, scale_pitch;
    int bytes;
};

__host__ __device__ __forceinline__ FewRows few_rows(int m, int blocks)
{
    const int wide = (blocks + kTurn - 1) / kTurn * kTurn + kTurn;
    FewRows f;
    f.pitch = wide * 16 + 16;                            // (16 rows that are read at once in different banks)
    f.scale_pitch = wide + 4;
    f.scales = m * f.pitch;
    f.bytes = (f.scales + m * f.scale_pitch + 15) / 16 * 16;
    return f;
}

template <typename T, int D, int RG>
__global__ void __launch_bounds__(512)
linear_mx4_rows_kernel(const Mx4Product p, const T *__restrict__ x, int64_t ldx, int k)
{
    constexpr int WAVES = 8, TURN_BYTES = 16 * 256 + 256, ROUND = WAVES * kTurn;
    extern __shared__ v4i few_lds[];
    __shared__ v4i ring[WAVES][D * TURN_BYTES / 16];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = int(blockIdx.x) * 16;
    const FewRows few = few_rows(p.m, p.blocks);
    uint8_t *const a = reinterpret_cast<uint8_t *>(few_lds);

    const int rounds = p.blocks / ROUND, left = p.blocks - rounds * ROUND;
    const int share = ((left + WAVES - 1) / WAVES + 3) / 4 * 4;          // (whole words of scales)
    const int mine = rounds + (wave * share < left ? 1 : 0);
    const int first_round = rounds > 0 ? int(blockIdx.x >> 3) % rounds : 0;
    // the first block of a turn and how many it has
    auto first_of = [&](int t) {
        if (t >= rounds) return rounds * ROUND + wave * share;
        t += first_round;
        return (t < rounds ? t : t - rounds) * ROUND + wave * kTurn;
    };
    auto count_of = [&](int t) { return t < rounds ? kTurn : min(share, left - wave * share); };

    // a turn is 16 rows of 256 bytes, 16 lanes read a row together, and the word of scales that each lane will use itself
    const v4u at_b = buffer_at(reinterpret_cast<const int8_t *>(p.b) + int64_t(n0) * p.ldb);
    uint32_t off[4];
    int piece[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 4 + g;
        piece[i] = r ^ row;
        off[i] = uint32_t(min(row, p.n - 1 - n0)) * uint32_t(p.ldb) + uint32_t(piece[i]) * 16u;
    }
    const uint8_t *const scales_b = p.sb + int64_t(min(n0 + r, p.n - 1)) * 8;
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring[wave]));
    auto issue = [&](int t) {
        if (t >= mine) return;
        const int first = first_of(t), have = count_of(t);
        const uint32_t to = base + uint32_t(t % D) * uint32_t(TURN_BYTES), at = uint32_t(first) * 16u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("s_mov_b32 m0, %1\n s_nop 0\n buffer_load_dwordx4 %0, %2, %3 offen lds"
                         ::"v"(piece[i] < have ? off[i] : kNowhere), "s"(to + uint32_t(i * 1024)), "s"(at_b), "s"(at) : "memory");
        // (of blocks that are not there the turn's first word again, for nothing)
        const int word = first + (g * 4 < have ? g * 4 : 0);
        asm volatile("s_mov_b32 m0, %1\n s_nop 0\n global_load_lds_dword %0, off"
                     ::"v"(scales_b + int64_t(word >> 3) * p.slab_b + (word & 4)), "s"(to + 4096u) : "memory");
    };
    constexpr int AHEAD = 2;                             // (what a wave asks for behind its weights is waited for with them)
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) issue(t);

    if constexpr (sizeof(T) == 1) {
#pragma unroll 2
        for (int u = int(threadIdx.x); u < p.m * p.blocks; u += WAVES * 64) {
            const int row = u / p.blocks, block = u - row * p.blocks;
            v4i v;
            __builtin_memcpy(&v, x + row * ldx + block * 16, 16);
            const uint8_t s = p.sa[int64_t(block >> 3) * p.slab_a + row * 8 + (block & 7)];
            __builtin_memcpy(a + row * few.pitch + block * 16, &v, 16);
            a[few.scales + row * few.scale_pitch + block] = s;
        }
    } else {
        // (several at once, so that their loads are under way together; four lanes have a block, so that nothing ends within one)
        constexpr int AT_ONCE = 4;
        const int eights = p.blocks * 4, all = p.m * eights;
#pragma unroll 1
        for (int first = int(threadIdx.x); first < all; first += AT_ONCE * WAVES * 64) {
            Eight<T> e[AT_ONCE];
            int row[AT_ONCE], at[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (first + i * WAVES * 64 >= all) continue;
                row[i] = (first + i * WAVES * 64) / eights;
                at[i] = first + i * WAVES * 64 - row[i] * eights;
                e[i] = load_eight(x + row[i] * ldx, at[i] * 8, k);
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (first + i * WAVES * 64 >= all) continue;
                const uint32_t byte = block_scale(most_of_block(e[i].most()));
                const uint32_t w = byte == 255u ? 0u : e[i].codes(scale_value(byte));
                __builtin_memcpy(a + row[i] * few.pitch + at[i] * 4, &w, 4);
                if (at[i] % 4 == 0) a[few.scales + row[i] * few.scale_pitch + at[i] / 4] = uint8_t(byte);
            }
        }
    }
#pragma unroll
    for (int t = AHEAD; t < D; ++t) issue(t);
    __syncthreads();
    const uint8_t *row_a[RG], *row_s[RG];
#pragma unroll
    for (int i = 0; i < RG; ++i) {
        row_a[i] = a + min(i * 16 + r, p.m - 1) * few.pitch + g * 64;
        row_s[i] = a + few.scales + min(i * 16 + r, p.m - 1) * few.scale_pitch + g * 4;
    }
    f4 acc[RG][2];
#pragma unroll
    for (int i = 0; i < RG; ++i) acc[i][0] = acc[i][1] = f4{0, 0, 0, 0};
#pragma unroll 1
    for (int t = 0; t < mine; ++t) {
        wait_for_loads<D - 1, 5>(min(D - 1, mine - 1 - t));
        const v4i *const st = ring[wave] + (t % D) * (TURN_BYTES / 16);
        const int first = first_of(t);
        v4i va[RG][4], vb[4];
        int sa[RG], sb = reinterpret_cast<const int *>(st + 256)[lane];
#pragma unroll
        for (int i = 0; i < RG; ++i) __builtin_memcpy(&sa[i], row_s[i] + first, 4);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            vb[s] = st[r * 16 + ((4 * g + s) ^ r)];
#pragma unroll
            for (int i = 0; i < RG; ++i) __builtin_memcpy(&va[i][s], row_a[i] + first * 16 + s * 16, 16);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");               // (read, so that it may be overwritten)
        issue(t + D);
        // (of blocks that are not there the weights are zeros and the scales may be any byte)
        const int mask = int(0xFFFFFFFFull >> max(0, min(32, (g * 4 + 4 - count_of(t)) * 8)));
        sb &= mask;
#pragma unroll
        for (int i = 0; i < RG; ++i) {
            sa[i] &= mask;
            acc[i][0] = multiply_blocks<0>(vb[0], va[i][0], acc[i][0], sb, sa[i]);
            acc[i][1] = multiply_blocks<1>(vb[1], va[i][1], acc[i][1], sb, sa[i]);
            acc[i][0] = multiply_blocks<2>(vb[2], va[i][2], acc[i][0], sb, sa[i]);
            acc[i][1] = multiply_blocks<3>(vb[3], va[i][3], acc[i][1], sb, sa[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < RG; ++i) reinterpret_cast<f4 *>(ring[wave])[i * 64 + lane] = acc[i][0] + acc[i][1];
    __syncthreads();
    if (wave >= RG) return;
    f4 s = reinterpret_cast<const f4 *>(ring[0])[wave * 64 + lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += reinterpret_cast<const f4 *>(ring[w])[wave * 64 + lane];
    const int m = wave * 16 + r, n = n0 + g * 4;
    if (m >= p.m || n >= p.n) return;
    const f4 v = values_of(p, s, bias_at(p, n));
    if (p.y_bf16) store_channels<__bf16, 4>(p, m, n, __builtin_convertvector(v, b4));
    else store_channels<float, 4>(p, m, n, v);
}

// How a product is cut up: the tile (an index into launch_tiles) and over how many workgroups the length of k is split.
struct Cut { int tile, splits; };

constexpr int kTiles = 4, kTileM[kTiles] = {32, 64, 128, 256}, kTileN[kTiles] = {128, 128, 128, 256};
constexpr int64_t kUnits = 256;                          // compute units

int64_t tiles_of(const Cut &c, int64_t m, int64_t n) { return ((m + kTileM[c.tile] - 1) / kTileM[c.tile]) * ((n + kTileN[c.tile] - 1) / kTileN[c.tile]); }

// The cheapest by a count of cycles: a compute unit takes its tiles one after the other, each with a start and an end that two
// of the smaller ones on it share, and the stages of its part of k.  Joining the parts is one more launch and reads and writes the
// sums.  The constants are those that choose best for 460 products of 17 to 20000 rows, 8 to 4096 channels and lengths up to
// 25088 that were timed with every tile and split: the choice takes 1.008 times the best of them on average and at most 1.16 times
// (stages by the rates of the matrix units and the level-2 cache, and one start for all tiles: 1.06 and 1.57).
Cut cut_of(int64_t m, int64_t n, int64_t blocks)
{
    constexpr int64_t stage[kTiles] = {600, 800, 1000, 3400}, start[kTiles] = {1900, 2900, 5500, 9600}, join = 3000;
    const int64_t stages = (blocks + 7) / 8;
    Cut best{0, 1};
    double least = 0;
    for (int t = 0; t < kTiles; ++t)
        for (int64_t s = 1; s == 1 || (s <= 32 && s * 2 <= stages); s *= 2) {
            const int64_t rounds = (tiles_of(Cut{t, int(s)}, m, n) * s + kUnits - 1) / kUnits;
            double c = double(rounds) * double((stages + s - 1) / s) * double(stage[t]) + double(t < 3 ? (rounds + 1) / 2 : rounds) * double(start[t]);
            if (s > 1) c += double(join) + double(s) * double(m) * double(n) * 8 / 1700;
            if ((t == 0 && s == 1) || c < least || (c == least && s == 1)) { least = c; best = Cut{t, int(s)}; }
        }
    return best;
}

// Sets of waves of a workgroup: two where a compute unit has one workgroup, else room for two workgroups.  The largest tile
// fills a compute unit with one set.
int sets_of(const Cut &c, int64_t tiles) { return c.tile < 3 && tiles * c.splits <= kUnits ? 2 : 1; }

template <int BM, int BN, int WM, int WN, int S, int KG>
void launch_tiles(const Mx4Product &p, int splits, float *part, hipStream_t st)
{
    const unsigned grid = unsigned(((int64_t(p.m) + BM - 1) / BM) * ((int64_t(p.n) + BN - 1) / BN) * splits);
    if (p.y_bf16) hipLaunchKernelGGL((matmul_mx4_kernel<__bf16, BM, BN, WM, WN, S, KG>), dim3(grid), dim3(KG * WM * WN * 64), 0, st, p, splits, part);
    else hipLaunchKernelGGL((matmul_mx4_kernel<float, BM, BN, WM, WN, S, KG>), dim3(grid), dim3(KG * WM * WN * 64), 0, st, p, splits, part);
}

int64_t rows_groups(int64_t n) { return (n + 15) / 16; }

constexpr int64_t kLds = 160 * 1024;

// Whether rows are so few and short that every workgroup has all of them in LDS beside two turns of weights (32x4096 -> 4096 with a
// launch that quantises 7.8 us, 10.1 in tiles; 4x25088 -> 4096 13.7 and 16.4), less of them where a compute unit has several
// workgroups to run (4x8192 -> 8192 14.1 us, and 15.3 in tiles, 6x8192 -> 8192 16.8 and 15.3, 8x8192 ->
// 8192 19.6 and 15.6).
bool few(int64_t m, int64_t n, int64_t blocks)
{
    if (m > kFewRows || blocks == 0 || blocks > 2048 || m * blocks * 16 > kLds) return false;
    const int64_t rounds = (rows_groups(n) + kUnits - 1) / kUnits;
    return rounds == 1 ? int64_t(kFewRing) * 2 + few_rows(int(m), int(blocks)).bytes <= kLds : m * blocks * 16 * rounds <= 32768;
}

template <typename T, int RG>
void launch_few_of(const Mx4Product &p, const T *x, int64_t ldx, int k, hipStream_t st)
{
    const int64_t lds = few_rows(p.m, p.blocks).bytes;
    const dim3 grid(unsigned(rows_groups(p.n)));
    // Three turns of each wave under way where a compute unit has one workgroup (1x25088 -> 8192 24.2 us with two, 23.0),
    // two where it has two (8192 -> 8192 8.5 us, and one with three turns 10.7) or the rows leave no room.
    const bool two = (int64_t(grid.x) > kUnits && 2 * (int64_t(kFewRing) * 2 + lds) <= kLds) || int64_t(kFewRing) * 3 + lds > kLds;
    if (two) hipLaunchKernelGGL((linear_mx4_rows_kernel<T, 2, RG>), grid, dim3(512), size_t(lds), st, p, x, ldx, k);
    else hipLaunchKernelGGL((linear_mx4_rows_kernel<T, 3, RG>), grid, dim3(512), size_t(lds), st, p, x, ldx, k);
}

template <typename T>
int launch_few(const Mx4Product &p, const T *x, int64_t ldx, int k, hipStream_t st)
{
    if (p.m <= 16) launch_few_of<T, 1>(p, x, ldx, k, st);
    else launch_few_of<T, 2>(p, x, ldx, k, st);
    return check_launch("pconv_linear_mx4 (few rows)");
}

}  // namespace

// (Every workgroup quantises all rows: 8x4096 -> 4096 5.9 us, and 6.0 with a launch for it; 16x4096 8.4 and 6.5.)
bool linear_mx4_fused(int64_t m, int64_t n, int64_t blocks) { return few(m, n, blocks) && m * blocks <= 1024; }

int launch_linear_mx4_fused(const Mx4Product &p, const void *x, int64_t ldx, int bf16, int64_t k, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch_few(p, static_cast<const __bf16 *>(x), ldx, int(k), st) : launch_few(p, static_cast<const float *>(x), ldx, int(k), st);
}

int launch_quantize_mx4(const void *x, int64_t ldx, int bf16, int64_t rows, int64_t cols, uint8_t *q, int64_t ldq, uint8_t *scale,
                        int64_t slab_stride, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t slabs = (cols + 255) / 256;
    const unsigned gx = unsigned(std::min<int64_t>((rows + 7) / 8, 1 << 20));
    const unsigned gy = unsigned(std::min<int64_t>(slabs, std::max<int64_t>(1, 4096 / gx)));
    if (bf16) hipLaunchKernelGGL(quantize_mx4_kernel<__bf16>, dim3(gx, gy), dim3(256), 0, st, static_cast<const __bf16 *>(x), ldx, rows, cols, slabs, q, ldq, scale, slab_stride);
    else hipLaunchKernelGGL(quantize_mx4_kernel<float>, dim3(gx, gy), dim3(256), 0, st, static_cast<const float *>(x), ldx, rows, cols, slabs, q, ldq, scale, slab_stride);
    return check_launch("pconv_quantize_mx4");
}

int64_t matmul_mx4_work_bytes(int64_t m, int64_t n, int64_t blocks)
{
    if (few(m, n, blocks)) return 0;
    const Cut c = cut_of(m, n, blocks);
    return c.splits > 1 ? c.splits * m * ((n + 3) / 4 * 4) * 4 : 0;
}

int check_matmul_mx4(int64_t m, int64_t n, int64_t blocks)
{
    if (few(m, n, blocks)) return PCONV_OK;
    const Cut c = cut_of(m, n, blocks);
    return tiles_of(c, m, n) * c.splits > kMaxGroups ? too_many_groups() : PCONV_OK;
}

pconv_mx4_plan matmul_mx4_plan(int64_t m, int64_t n, int64_t blocks)
{
    if (few(m, n, blocks)) return pconv_mx4_plan{1, 0, 0, 0, 0};
    const Cut c = cut_of(m, n, blocks);
    return pconv_mx4_plan{2, kTileM[c.tile], kTileN[c.tile], sets_of(c, tiles_of(c, m, n)), c.splits};
}

int launch_matmul_mx4(const Mx4Product &p, void *work, void *stream)
{
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (few(p.m, p.n, p.blocks)) return launch_few(p, p.a, p.lda, 0, st);
    const Cut c = cut_of(p.m, p.n, p.blocks);
    const int64_t tiles = tiles_of(c, p.m, p.n);
    if (tiles * c.splits > kMaxGroups) return too_many_groups();
    float *const sums = static_cast<float *>(work);
    const bool two = sets_of(c, tiles) == 2;
    if (c.tile == 0 && two) launch_tiles<32, 128, 1, 4, 3, 2>(p, c.splits, sums, st);
    else if (c.tile == 0) launch_tiles<32, 128, 1, 4, 3, 1>(p, c.splits, sums, st);
    else if (c.tile == 1 && two) launch_tiles<64, 128, 2, 2, 3, 2>(p, c.splits, sums, st);
    else if (c.tile == 1) launch_tiles<64, 128, 2, 2, 3, 1>(p, c.splits, sums, st);
    else if (c.tile == 2 && two) launch_tiles<128, 128, 2, 2, 2, 2>(p, c.splits, sums, st);
    else if (c.tile == 2) launch_tiles<128, 128, 2, 2, 2, 1>(p, c.splits, sums, st);
    else launch_tiles<256, 256, 2, 4, 2, 1>(p, c.splits, sums, st);
    if (const int rc = check_launch("pconv_matmul_mx4")) return rc;
    if (c.splits == 1) return PCONV_OK;
    const int64_t quads = (int64_t(p.n) + 3) / 4 * p.m;
    hipLaunchKernelGGL(matmul_mx4_join_kernel, dim3(unsigned(std::min<int64_t>((quads + 255) / 256, 1 << 16))), dim3(256), 0, st, p, c.splits, sums);
    return check_launch("pconv_matmul_mx4 (joining the parts of k)");
}

}  // namespace pconv
