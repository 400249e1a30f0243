// Products in 8-bit floating point with a power-of-two scale for each block of 128 (ts_matmul_fp8), and the codes and
// scales that they take (ts_quantize_fp8).
//
// A scale that is a power of two is a biased exponent in one byte, which is what gfx950 takes beside the codes, in its matrix
// instructions and where it converts codes, so a block's scale costs no instruction of its own and no rounding.  (A fp32
// scale would have to be multiplied into every block's partial sums: four multiply-adds per lane for each matrix
// instruction of 32 cycles.)
//
// The result's type chooses between the two.  The matrix instructions of 8-bit codes (16 x 128 by 128 x 16) bring eight products
// along K at a time to the exponent of the largest and cut off what lies more than 13 bits below it before they add in fp32
// (found with single products of known size): on normal data the result is 1.5e-5 of its norm off, whatever K is.
// That is a hundredth of what a bf16 result loses by its own rounding, and 100 times what a fp32 result should lose.  So a bf16 result is
// made by them; for a fp32 result the codes are converted to bf16, scale included, which is exact, and multiplied by the bf16
// matrix instructions (16 x 32 by 32 x 16, half the rate), whose products are exact and whose sums are fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ts_densify.h"
#include "ts_workspace.h"

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = TS_FP8_BLOCK;

__host__ __device__ constexpr int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
__host__ __device__ constexpr int64_t code_row(int64_t k) { return round_up(k, kBlock); }
__host__ __device__ constexpr int64_t scale_row(int64_t k) { return round_up((k + kBlock - 1) / kBlock, 4); }

__device__ __forceinline__ uint32_t narrow2(float x, float y)
{
    const f2 v = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}

// The t-th tile.  Work-groups b, b + 8, b + 16, ... run on one of eight XCDs with an L2 each: every XCD takes neighbouring tiles, STRIP of them along
// M before the next along N, so that those it works on at one time share their operands, and write long stretches of the result's rows.
// (Codes and scales are made in strips of 3: 2-3 % before 2 and 4, whose rows' addresses fall on fewer memory channels.)
// 8192 x 32768 x 1024 to bf16 with strips of 1 / 2 / 4 / 8 / 16: 310 / 299 / 290 / 325 / 327 us, 8192^3 487 / 459 / 460 / 469 / 470.
template <int STRIP = 4>
__device__ __forceinline__ void place(int64_t wg, int64_t m_tiles, int64_t n_tiles, int64_t* mt, int64_t* nt)
{
    const int64_t tiles = m_tiles * n_tiles, each = tiles >> 3, rest = tiles & 7, x = wg & 7;
    const int64_t t = x * each + (x < rest ? x : rest) + (wg >> 3);
    const int64_t strip = STRIP * n_tiles, s = t / strip, at = t - s * strip;
    const int64_t high = m_tiles - s * STRIP < STRIP ? m_tiles - s * STRIP : STRIP;
    *nt = at / high;
    *mt = s * STRIP + (at - *nt * high);
}

// ------------------------------------------------------------------ codes and scales
// Byte of the scale of a block whose largest finite magnitude has these bits: e + 127 for the smallest e >= -127 with
// most <= MAX 2^e, where MAX is 1.75 * 2^8 (e4m3) or 1.75 * 2^15 (e5m2).
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    const int e = (int)(most >> 23) - (FMT == TS_FP8_E4M3 ? 8 : 15) + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)(e < 0 ? 0 : e);
}

constexpr uint32_t kInfinite = 0x7F800000u;          // bits of magnitudes: infinities and NaN lie above all numbers
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// The largest of sixteen neighbouring lanes, by rotations within them.
template <int N>
__device__ __forceinline__ uint32_t rotated(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t largest_of_16(uint32_t x)
{
    x = larger(x, rotated<8>(x));
    x = larger(x, rotated<4>(x));
    x = larger(x, rotated<2>(x));
    return larger(x, rotated<1>(x));
}
// The largest of lanes i, i + 16, i + 32 and i + 48.
template <int WIDE>
__device__ __forceinline__ uint32_t largest_of_rows(uint32_t x)
{
    if constexpr (WIDE == 1) {
        const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = larger(a[0], a[1]);
    }
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return larger(b[0], b[1]);
}

// Four codes of x * 2^(127 - byte).  (byte <= 247, so the factor is a normal number.)
template <int FMT>
__device__ __forceinline__ uint32_t codes4(f4 x, uint32_t byte)
{
    const float f = __uint_as_float((254u - byte) << 23);
    int w = 0;
    if (FMT == TS_FP8_E4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x.x * f, x.y * f, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x.z * f, x.w * f, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(x.x * f, x.y * f, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(x.z * f, x.w * f, w, true);
    }
    return (uint32_t)w;
}

struct Quantize {
    const void* x;
    uint8_t *q, *q_scales, *qt, *qt_scales;
    int64_t rows, cols;
    int64_t tile_first;
    int64_t row_tiles, col_tiles;
};

// Eight rows of eight elements as they lie in memory, at any address that is aligned to one; and the bits of the largest magnitudes of a row and of all columns,
// which show whether a value is no finite number.
template <typename T>
struct Part;

template <>
struct Part<float> {
    f4 v[8][2];

    __device__ __forceinline__ void clear(int i) { v[i][0] = v[i][1] = (f4)(0.0f); }
    __device__ __forceinline__ void load(int i, const float* p)
    {
        typedef f4 __attribute__((aligned(4))) any_f4;
#pragma unroll
        for (int h = 0; h < 2; ++h) v[i][h] = __builtin_nontemporal_load(reinterpret_cast<const any_f4*>(p) + h);
    }
    __device__ __forceinline__ void set(int i, int c, float x) { v[i][c >> 2][c & 3] = x; }
    __device__ __forceinline__ float value(int i, int c) const { return v[i][c >> 2][c & 3]; }
    __device__ __forceinline__ f4 four(int i, int h) const { return v[i][h]; }
    // (two magnitudes in one instruction, of which any NaN makes a NaN, whose bits lie above all numbers'; v_max3_f32 passes over a signalling NaN
    // together with the value beside it)
    static __device__ __forceinline__ float larger3(float most, float a, float b)
    {
        asm("v_maximum3_f32 %0, |%1|, |%2|, %3" : "=v"(most) : "v"(a), "v"(b), "v"(most));
        return most;
    }
    __device__ __forceinline__ uint32_t row_size(int i) const
    {
        float m = 0.0f;
#pragma unroll
        for (int c = 0; c < 8; c += 2) m = larger3(m, value(i, c), value(i, c + 1));
        return __float_as_uint(m) & 0x7FFFFFFFu;
    }
    __device__ __forceinline__ void column_sizes(uint32_t (&most)[8]) const
    {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i += 2) m = larger3(m, value(i, c), value(i + 1, c));
            most[c] = __float_as_uint(m) & 0x7FFFFFFFu;
        }
    }
};

template <>
struct Part<uint16_t> {
    typedef uint16_t h2 __attribute__((ext_vector_type(2)));
    u4 v[8];

    __device__ __forceinline__ void clear(int i) { v[i] = (u4)(0u); }
    __device__ __forceinline__ void load(int i, const uint16_t* p)
    {
        typedef u4 __attribute__((aligned(2))) any_u4;
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const any_u4*>(p));
    }
    __device__ __forceinline__ void set(int i, int c, uint16_t x) { v[i][c >> 1] = c & 1 ? v[i][c >> 1] | (uint32_t)x << 16 : x; }
    __device__ __forceinline__ float value(int i, int c) const { return __uint_as_float(c & 1 ? v[i][c >> 1] & 0xFFFF0000u : v[i][c >> 1] << 16); }
    __device__ __forceinline__ f4 four(int i, int h) const { return f4{value(i, 4 * h), value(i, 4 * h + 1), value(i, 4 * h + 2), value(i, 4 * h + 3)}; }
    // (two magnitudes in one instruction, as 16-bit numbers)
    static __device__ __forceinline__ uint32_t larger2(uint32_t most, uint32_t w)
    {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(h2, most), __builtin_bit_cast(h2, w & 0x7FFF7FFFu)));
    }
    __device__ __forceinline__ uint32_t row_size(int i) const
    {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) m = larger2(m, v[i][k]);
        return larger(m << 16, m & 0xFFFF0000u);
    }
    __device__ __forceinline__ void column_sizes(uint32_t (&most)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = larger2(m, v[i][k]);
            most[2 * k] = m << 16;
            most[2 * k + 1] = m & 0xFFFF0000u;
        }
    }
};

__device__ __forceinline__ uint32_t finite_size(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < kInfinite ? b : 0u;
}

// A work-group takes WIDE tiles of 128 x 128 elements that lie side by side, a thread 8 x 8 elements.  A row's block is in the registers of sixteen
// neighbouring lanes; a column's in those of every (16 * WIDE)th thread.  Where a largest magnitude is that of an infinity or NaN, the elements are
// looked at again without them.  Bound by memory, and so by how many tiles a compute unit holds: bf16 elements stay as they are, two to a register.
// 8192 x 32768 bf16 to e5m2, both ways / rows only: 203 us = 5.3 TB/s / 142 = 5.7 (261 / 181 with fp32 in the registers and every magnitude by itself).
// Two tiles, whose stretches are twice as long, against one: 205 / 210 us there, 8320 x 33152 219 / 234; against two below each other 205 / 212 and 219 / 226.
// Rows of any length, whose 16-byte loads begin anywhere: 10001 x 10003 rows only / both ways 59 / 88 us of bf16, 116 / 141 of fp32, 5.3 and 4.8 TB/s by what is counted
// rows only, of which lines that are read twice are 5 and 15 %.
// Wavefronts to a SIMD: five of bf16, four of fp32, of which a fifth one makes more requests than memory takes well (8192 x 32768 rows only 273 us, so 281).
template <typename T, int FMT, bool WHOLE, int WIDE>
__global__ __launch_bounds__(256 * WIDE) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 5 : 4, sizeof(T) == 2 ? 5 : 4))) void quantize_kernel(Quantize p)
{
    __shared__ __align__(16) uint32_t most_of[4 * WIDE][WIDE * kBlock];
    __shared__ __align__(16) uint8_t turned[WIDE * kBlock][kBlock + 8];
    constexpr int ACROSS = 16 * WIDE;        // threads beside each other
    int64_t r_tile, c_wide;
    place<3>(p.tile_first + blockIdx.x, p.row_tiles, (p.col_tiles + WIDE - 1) / WIDE, &r_tile, &c_wide);
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int r8 = tid / ACROSS * 8, c8 = tid % ACROSS * 8;       // the thread's place
    const int64_t r0 = r_tile * kBlock + r8, c0 = c_wide * (WIDE * kBlock) + c8;
    const int64_t c_tile = c_wide * WIDE + c8 / kBlock;
    const bool here = WIDE == 1 || c_tile < p.col_tiles;
    Part<T> x;
    const int64_t left = here ? p.cols - c0 : 0, below = p.rows - r0;
    const T* const from = (const T*)p.x + r0 * p.cols + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x.clear(i);
        if (left >= 8 && i < below) x.load(i, from + i * p.cols);
    }
    // A row's end inside eight elements: one by one, all of them asked for before one is looked at (7118 x 948 bf16 rows only 6.7 us, one
    // row's after the other 12.3).
    if (!WHOLE && left > 0 && left < 8 && below > 0) {
        T e[8][8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < 8; ++c) e[i][c] = from[(i < below ? i : 0) * p.cols + (c < left ? c : 0)];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < 8; ++c) x.set(i, c, i < below && c < left ? e[i][c] : T(0));
    }
    if (p.q) {
        const int64_t ld = code_row(p.cols), lds = scale_row(p.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t most = largest_of_16(x.row_size(i));
            if (__any(most >= kInfinite)) {
                most = 0;
#pragma unroll
                for (int c = 0; c < 8; ++c) most = larger(most, finite_size(x.value(i, c)));
                most = largest_of_16(most);
            }
            const uint32_t byte = scale_byte<FMT>(most);
            if (r0 + i < p.rows && here) {
                const u2 w = {codes4<FMT>(x.four(i, 0), byte), codes4<FMT>(x.four(i, 1), byte)};
                __builtin_nontemporal_store(w, reinterpret_cast<u2*>(p.q + (r0 + i) * ld + c0));
                // lane 0 of the sixteen writes the block's byte; behind the last block, lanes 1 to 3 the zeros
                const int64_t at = c_tile + (lane & 15);
                if ((lane & 15) == 0) p.q_scales[(r0 + i) * lds + at] = (uint8_t)byte;
                else if (c_tile == p.col_tiles - 1 && at < lds) p.q_scales[(r0 + i) * lds + at] = 0;
            }
        }
    }
    if (!p.qt) return;
    uint32_t most[8];
    x.column_sizes(most);
    uint32_t all = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        most[c] = largest_of_rows<WIDE>(most[c]);
        all = larger(all, most[c]);
    }
    if (__any(all >= kInfinite)) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            most[c] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) most[c] = larger(most[c], finite_size(x.value(i, c)));
            most[c] = largest_of_rows<WIDE>(most[c]);
        }
    }
    if (lane < ACROSS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<u4*>(&most_of[wave][c8 + 4 * h]) = u4{most[4 * h], most[4 * h + 1], most[4 * h + 2], most[4 * h + 3]};
    }
    __syncthreads();
    const int64_t ld = code_row(p.rows), lds = scale_row(p.rows);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u4 m = (u4)(0u);
#pragma unroll
        for (int w = 0; w < 4 * WIDE; ++w) {
            const u4 a = *reinterpret_cast<const u4*>(&most_of[w][c8 + 4 * h]);
#pragma unroll
            for (int j = 0; j < 4; ++j) m[j] = larger(m[j], a[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 4 * h + j;
            const uint32_t byte = scale_byte<FMT>(m[j]);
            const f4 lo = {x.value(0, c), x.value(1, c), x.value(2, c), x.value(3, c)}, hi = {x.value(4, c), x.value(5, c), x.value(6, c), x.value(7, c)};
            *reinterpret_cast<u2*>(&turned[c8 + c][r8]) = u2{codes4<FMT>(lo, byte), codes4<FMT>(hi, byte)};
            if (r8 == 0 && c0 + c < p.cols) {
                uint8_t* const s = p.qt_scales + (c0 + c) * lds;
                s[r_tile] = (uint8_t)byte;
                if (r_tile == p.row_tiles - 1)
                    for (int64_t at = p.row_tiles; at < lds; ++at) s[at] = 0;
            }
        }
    }
    __syncthreads();
    // eight lanes to a row of 128 codes
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 32 * WIDE + (tid >> 3), at = (tid & 7) * 16;
        const int64_t row = c_wide * (WIDE * kBlock) + c;
        const u2 lo = *reinterpret_cast<const u2*>(&turned[c][at]), hi = *reinterpret_cast<const u2*>(&turned[c][at + 8]);
        if (row < p.cols)
            __builtin_nontemporal_store(__builtin_shufflevector(lo, hi, 0, 1, 2, 3), reinterpret_cast<u4*>(p.qt + row * ld + r_tile * kBlock + at));
    }
}

// ------------------------------------------------------------------ product
struct Matmul {
    const uint8_t *a, *a_scales, *b, *b_scales;
    const float* c_in;
    void* out;
    int64_t M, N;
    int64_t ld, lds;            // bytes of a row of codes and of scales
    int32_t blocks;             // of 128 along K
    int32_t parts, part_blocks; // tiles beyond the first `full` are computed in parts of so many blocks, a multiple of four
    int64_t full;
    f4* sums;                   // [parts][those tiles][wavefronts][fragments][64]: the parts' sums as the registers hold them
    int64_t m_tiles, n_tiles;
    int64_t n_first;            // first column of a launch of rows_kernel
};

// 32 codes of one row as four operands of eight bf16 values, exactly (a value below 2^-133 is cut at bf16's last bit).
template <int FMT>
__device__ __forceinline__ void widen(i8 codes, uint32_t scale, b8 (&out)[4])
{
    const float f = __uint_as_float(scale << 23);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        b2 v[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int w = codes[2 * q + h];
            if (FMT == TS_FP8_E4M3) {
                v[2 * h] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, false);
                v[2 * h + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, true);
            } else {
                v[2 * h] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, f, false);
                v[2 * h + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, f, true);
            }
        }
        out[q] = __builtin_shufflevector(__builtin_shufflevector(v[0], v[1], 0, 1, 2, 3), __builtin_shufflevector(v[2], v[3], 0, 1, 2, 3),
                                         0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// 16 bytes of a row of the result, at an address that is aligned to an element.
template <bool HALF>
struct Out;
template <>
struct Out<true> {
    typedef u4 Vec;
};
template <>
struct Out<false> {
    typedef f4 Vec;
};

template <bool HALF>
__device__ __forceinline__ void store_row(const Matmul& p, int64_t m, int64_t n, typename Out<HALF>::Vec v)
{
    if (n >= p.N) return;
    const int64_t at = m * p.N + n;
    if constexpr (HALF) {
        typedef u4 __attribute__((aligned(2))) any_u4;
        uint16_t* const out = (uint16_t*)p.out + at;
        if (n + 8 <= p.N) {
            __builtin_nontemporal_store(v, reinterpret_cast<any_u4*>(out));
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (n + j < p.N) out[j] = (uint16_t)(v[j >> 1] >> (j & 1) * 16);
        }
    } else {
        typedef f4 __attribute__((aligned(4))) any_f4;
        float* const out = (float*)p.out + at;
        if (n + 4 <= p.N) {
            if (p.c_in) v += *reinterpret_cast<const any_f4*>(p.c_in + at);
            __builtin_nontemporal_store(v, reinterpret_cast<any_f4*>(out));
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (n + j < p.N) out[j] = p.c_in ? v[j] + p.c_in[at + j] : v[j];
        }
    }
}

// Four elements of a row of the result.
template <bool HALF>
__device__ __forceinline__ void store4(const Matmul& p, int64_t m, int64_t n, f4 v)
{
    if constexpr (!HALF) {
        store_row<false>(p, m, n, v);
    } else {
        typedef u2 __attribute__((aligned(2))) any_u2;
        uint16_t* const out = (uint16_t*)p.out + m * p.N + n;
        const u2 w = {narrow2(v.x, v.y), narrow2(v.z, v.w)};
        if (n + 4 <= p.N) {
            *reinterpret_cast<any_u2*>(out) = w;
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (n + j < p.N) out[j] = (uint16_t)(w[j >> 1] >> (j & 1) * 16);
        }
    }
}

__device__ __forceinline__ i8 load_codes(const uint8_t* p)
{
    const i4 lo = *reinterpret_cast<const i4*>(p), hi = *reinterpret_cast<const i4*>(p + 16);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// ---- few rows: codes straight into registers
// A wavefront computes 16 * NF columns of the result in MF * 16 rows: lane l holds 32 codes of row l % 16 of a fragment.  It takes every kw-th run of four
// blocks, all of whose codes it asks for at once; the kw wavefronts of one place add their sums up in LDS, in their order.  Bound by reading B once:
// one row, N = 32768, K = 1024 6.9 us = 4.9 TB/s, a launch of 2 us included; and, with more rows, by the L1 caches: neighbouring lanes' codes lie in different
// rows and so in different lines.
template <int FA, int FB, bool HALF, int MF, int NF>
__global__ __launch_bounds__(256) void rows_kernel(Matmul p, int log_kw)
{
    __shared__ f4 sums[4][NF * MF][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int kw = 1 << log_kw, part = wave & (kw - 1), places = (int)(blockDim.x >> 6) >> log_kw;
    const int64_t n0 = p.n_first + ((int64_t)blockIdx.x * places + (wave >> log_kw)) * (16 * NF);
    const uint8_t *b[NF], *sb[NF], *a[MF], *sa[MF];
    f4 acc[NF][MF];
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        const int64_t n = n0 + f * 16 + i, rb = n < p.N ? n : p.N - 1;                 // rows past the end: the last one again
        b[f] = p.b + rb * p.ld + g * 32;
        sb[f] = p.b_scales + rb * p.lds;
    }
#pragma unroll
    for (int h = 0; h < MF; ++h) {
        const int64_t m = h * 16 + i, ra = m < p.M ? m : p.M - 1;
        a[h] = p.a + ra * p.ld + g * 32;
        sa[h] = p.a_scales + ra * p.lds;
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[f][h] = (f4)(0.0f);
    }
    for (int k = part * 4; k < p.blocks; k += kw * 4) {
        uint32_t wb[NF], wa[MF];
#pragma unroll
        for (int f = 0; f < NF; ++f) wb[f] = *reinterpret_cast<const uint32_t*>(sb[f] + k);
#pragma unroll
        for (int h = 0; h < MF; ++h) wa[h] = *reinterpret_cast<const uint32_t*>(sa[h] + k);
        i8 u[4][NF], v[4][MF];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t at = (int64_t)(k + q < p.blocks ? k + q : p.blocks - 1) * kBlock;      // (behind the last block: it again, unused)
#pragma unroll
            for (int f = 0; f < NF; ++f) u[q][f] = load_codes(b[f] + at);
#pragma unroll
            for (int h = 0; h < MF; ++h) v[q][h] = load_codes(a[h] + at);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (k + q >= p.blocks) break;
            if constexpr (HALF) {
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int h = 0; h < MF; ++h)
                        acc[f][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u[q][f], v[q][h], acc[f][h], FB, FA, 0, (int)(wb[f] >> 8 * q), 0, (int)(wa[h] >> 8 * q));
            } else {
                b8 x[NF][4];
#pragma unroll
                for (int f = 0; f < NF; ++f) widen<FB>(u[q][f], (wb[f] >> 8 * q) & 255u, x[f]);
#pragma unroll
                for (int h = 0; h < MF; ++h) {
                    b8 y[4];
                    widen<FA>(v[q][h], (wa[h] >> 8 * q) & 255u, y);
#pragma unroll
                    for (int f = 0; f < NF; ++f)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[f][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[f][r], y[r], acc[f][h], 0, 0, 0);
                }
            }
        }
    }
    if (kw > 1) {
        if (part > 0) {
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int h = 0; h < MF; ++h) sums[wave][f * MF + h][lane] = acc[f][h];
        }
        __syncthreads();
        if (part > 0) return;
        for (int w = 1; w < kw; ++w)
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int h = 0; h < MF; ++h) acc[f][h] += sums[wave + w][f * MF + h][lane];
    }
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int h = 0; h < MF; ++h) {
            const int64_t m = h * 16 + i;
            if (m < p.M) store4<HALF>(p, m, n0 + f * 16 + g * 4, acc[f][h]);
        }
}

// ---- large products: tiles through LDS
typedef __attribute__((address_space(3))) void* lds_ptr;

// Waits for this wavefront's reads from LDS and for all but the LATER last of its accesses to memory, which end in their order, loads into LDS among
// them; then for the work-group's other wavefronts.
template <int LATER = 0>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER < 63 ? LATER : 63) : "memory");
}
// The same with WITH_STORES where stores lie among the accesses behind the loads in question, else with LATER.  (In one statement: a branch would end the run of
// instructions that keeps its order.)
template <int LATER, int WITH_STORES>
__device__ __forceinline__ void meet_behind_stores(bool behind)
{
    static_assert(LATER <= WITH_STORES, "the second wait adds nothing to the first");
    asm volatile("s_cmp_lg_u32 %2, 0\n\ts_cbranch_scc1 .Lstores_%=\n\ts_waitcnt vmcnt(%0)\n.Lstores_%=:\n\ts_waitcnt vmcnt(%1) lgkmcnt(0)\n\ts_barrier"
                 ::"n"(LATER < 63 ? LATER : 63), "n"(WITH_STORES < 63 ? WITH_STORES : 63), "s"(__builtin_amdgcn_readfirstlane((int)behind)) : "memory", "scc");
}

#ifdef __HIP_DEVICE_COMPILE__     // (a buffer's type is none of the host compiler's)
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

// A part of an operand as a buffer: reads beyond `bytes` give zeros.  What is added to a load's own offset is never more than `bytes`.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const uint8_t* p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, (int)(uint32_t)bytes, 0x00020000);
}
#endif

// Sizes that the host needs, too.  LDS: S stages (2 or 4) of [ROWS][128] codes, two of [ROWS] words of scales, 1 KiB that nobody reads, and eight rows of
// the result for every wavefront.
template <bool HALF, int WN, int WM, int NF, int MF, int S>
struct Tile {
    static constexpr int TN = 16 * WN * NF, TM = 16 * WM * MF, ROWS = TN + TM, STAGE = ROWS * kBlock, SCALES = S * STAGE, UNREAD = SCALES + 2 * ROWS * 4;
    static constexpr int EF = HALF ? NF : NF / 2, PITCH = EF * 16 * (HALF ? 2 : 4) + 16;       // fragments of a turn of the result; bytes of a row
    static constexpr int RESULT = UNREAD + 1024, LDS = RESULT + WN * WM * 8 * PITCH;
};

// A work-group of WN x WM wavefronts computes tiles of TN columns by TM rows of the result, a wavefront NF x MF fragments of 16 x 16, whose sums stay in
// its registers; it takes tile after tile, as many work-groups as the GPU holds.  Codes go from memory into LDS past the registers, in S stages: up to S - 1
// blocks of 128 along K ahead.  Bound by the matrix instructions, the loads' latencies between them and, where K is short, by writing the result (256 x 256):
//                                       us       TFLOP/s    without any loads / without any accesses
//   8192^3 to bf16                      401      2740       319 / 272 us
//   8192 x 32768 x 1024 to bf16         283      1940       203 / 181, without stores 233
//   8192^3 to fp32                      731      1504
// What else was measured and lost: a ring of four half-blocks with 32 x 32 x 64 products (500 and 317 us: half lines of 64 bytes, twice the requests to L2),
// 128 x 128 tiles everywhere (540 and 343), four wavefronts of 128 x 128 (431 and 302), work-groups that begin one after the other, so that not all
// store at a time (8192^3 15 % slower).
template <int FA, int FB, bool HALF, bool ONTO, int WN, int WM, int NF, int MF, int S>
__global__ __launch_bounds__(64 * WN * WM, 2) void tile_kernel([[maybe_unused]] Matmul p)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef Tile<HALF, WN, WM, NF, MF, S> T;
    constexpr int TN = T::TN, TM = T::TM, ROWS = T::ROWS, STAGE = T::STAGE, SCALES = T::SCALES, WAVES = WN * WM;
    constexpr int LB = TN / (8 * WAVES), LA = TM / (8 * WAVES);     // loads of 1 KiB by a wavefront, for one block
    static_assert(TN % (8 * WAVES) == 0 && TM % (8 * WAVES) == 0 && TN % 64 == 0 && TM % 64 == 0, "whole loads");
    extern __shared__ __align__(1024) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wm = wave / WN, i = lane & 15, g = lane >> 4;
    // Row r of a stage: of B for r < TN, else of A; its 16-byte chunk c lies in slot c ^ key(r), so that sixteen lanes that read
    // one chunk of sixteen rows meet no bank twice.  With a bf16 result, rows of two fragments of B are interleaved by fours (n_of), and the
    // four columns that a lane has of each lie side by side.
    const auto n_of = [&](int f) { return HALF ? (f >> 1) * 32 + (i >> 2) * 8 + (f & 1) * 4 + (i & 3) : f * 16 + i; };
    const uint32_t ld = (uint32_t)p.ld, rb = (uint32_t)(wave * LB * 8 + (lane >> 3)), ra = (uint32_t)(wave * LA * 8 + (lane >> 3));
    const uint32_t key_b = HALF ? (rb & 3) | ((rb >> 1) & 4) : rb & 7;
    const uint32_t from_b = rb * ld + (((lane & 7) ^ key_b) << 4), from_a = ra * ld + (((lane & 7) ^ (ra & 7)) << 4);
    uint32_t row_b[LB], row_a[LA];
#pragma unroll
    for (int j = 0; j < LB; ++j) row_b[j] = (HALF && (j & 1) ? from_b ^ 64 : from_b) + j * 8 * ld;    // (eight rows on, the key's third bit is the other one)
#pragma unroll
    for (int j = 0; j < LA; ++j) row_a[j] = from_a + j * 8 * ld;
    // the tile that is fetched
    int64_t m0, n0, m_here, n_here;
    const uint8_t *a, *b, *sa_from, *sb_from;
    int64_t a_bytes, b_bytes, words_bytes;
    int blocks;
    const int64_t rest = p.m_tiles * p.n_tiles - p.full, all = p.full + rest * p.parts;
    const auto turn_to = [&](int64_t t) {
        int64_t mt, nt;
        int k0 = 0;
        blocks = p.blocks;
        if (t >= p.full && p.parts > 1) {
            const int part = (int)((t - p.full) / rest);
            t -= part * rest;
            k0 = part * p.part_blocks;
            blocks = p.blocks - k0 < p.part_blocks ? p.blocks - k0 : p.part_blocks;
        }
        place(t, p.m_tiles, p.n_tiles, &mt, &nt);
        m0 = mt * TM;
        n0 = nt * TN;
        m_here = p.M - m0 < TM ? p.M - m0 : TM;
        n_here = p.N - n0 < TN ? p.N - n0 : TN;
        a = p.a + m0 * p.ld + (int64_t)k0 * kBlock;
        b = p.b + n0 * p.ld + (int64_t)k0 * kBlock;
        sa_from = p.a_scales + m0 * p.lds + k0;
        sb_from = p.b_scales + n0 * p.lds + k0;
        a_bytes = m_here * p.ld - (int64_t)k0 * kBlock;
        b_bytes = n_here * p.ld - (int64_t)k0 * kBlock;
        words_bytes = -k0;
    };
    // Load j of this wavefront's share of block k (codes of B, of A, words of four scales), into stage k % 2.  Behind the last block: zeros, without
    // a question, so that the loop below stays one run of instructions that keeps its order.
    constexpr int LS = (ROWS / 64 + WAVES - 1) / WAVES, LOADS = LB + LA + LS;
    const auto fetch = [&](int k, int j, bool wanted = true) {
        const bool there = wanted && k < blocks;
        uint8_t* const to = wanted ? lds + (k & (S - 1)) * STAGE : nullptr;          // (a load that was made before: to where nobody looks)
        uint8_t* const unread = lds + T::UNREAD;
        const int at_k = there ? k * kBlock : 0;            // (never more than a buffer's length)
        if (j < LB) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(b, there ? b_bytes : 0), (lds_ptr)(wanted ? to + (wave * LB + j) * 1024 : unread), 16, row_b[j], at_k, 0, 0);
        } else if (j < LB + LA) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(a, there ? a_bytes : 0), (lds_ptr)(wanted ? to + TN * kBlock + (wave * LA + j - LB) * 1024 : unread), 16,
                                                     row_a[j - LB], at_k, 0, 0);
        } else {
            // every fourth block has new words; else nothing is read, and zeros go where nobody looks
            const bool words = there && (k & 3) == 0;
            const int at = (wave + (j - LB - LA) * WAVES) % (ROWS / 64);        // (more wavefronts than words: some are fetched twice)
            const bool of_b = at * 64 < TN;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(of_b ? sb_from : sa_from, words ? (of_b ? n_here : m_here) * p.lds + words_bytes : 0),
                                                     (lds_ptr)(words ? lds + SCALES + (k >> 2 & 1) * ROWS * 4 + at * 256 : unread), 4,
                                                     (uint32_t)(at * 64 + lane - (of_b ? 0 : TN)) * (uint32_t)p.lds, words ? k : 0, 0, 0);
        }
    };
    // places of this lane's codes in a stage, chunk g and chunk g + 4 of a row
    const int at_b = (wn * NF * 16 + n_of(0)) * kBlock, at_a = (TN + wm * MF * 16 + i) * kBlock, lo = (g ^ (i & 7)) << 4, hi = lo ^ 64;
    const auto codes = [&](int at) {
        const i4 x = *reinterpret_cast<const i4*>(lds + at + lo), y = *reinterpret_cast<const i4*>(lds + at + hi);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const auto codes_b = [&](int stage, int f) { return codes(stage + at_b + (HALF ? (f >> 1) * 32 + (f & 1) * 4 : f * 16) * kBlock); };
    const auto codes_a = [&](int stage, int h) { return codes(stage + at_a + h * 16 * kBlock); };
    uint32_t sb[NF], sa[MF];
    const auto scales = [&](int k) {
        const uint8_t* const at = lds + SCALES + (k >> 2 & 1) * ROWS * 4;
#pragma unroll
        for (int f = 0; f < NF; ++f) sb[f] = *reinterpret_cast<const uint32_t*>(at + (wn * NF * 16 + n_of(f)) * 4);
#pragma unroll
        for (int h = 0; h < MF; ++h) sa[h] = *reinterpret_cast<const uint32_t*>(at + (TN + (wm * MF + h) * 16 + i) * 4);
    };
    // The loads of a block are spread over the multiplication of the one before, so that none of them holds up a read from LDS that a product
    // waits for.  A stage is free for them once the block in it has been read, from the middle of its multiplication on (bf16 result), or but for its
    // last fragment of B (fp32, whose widened codes leave no registers for half a block's).
    constexpr int SPREAD = HALF ? NF : NF > 4 ? NF / 2 : NF - 1, AT_ONCE = (LOADS + SPREAD - 1) / SPREAD;
    typedef typename Out<HALF>::Vec Vec;
    constexpr int PER_VEC = HALF ? 8 : 4, EF = T::EF, VECS = EF * 16 / PER_VEC, PITCH = T::PITCH, TURN = 64 / VECS;
    static_assert(64 % VECS == 0 && 8 % TURN == 0, "whole rows");
    constexpr int NT = 2;           // nontemporal
    constexpr int STORES = MF * (NF / EF) * (16 / TURN);
    // loads of the block after the next that are made before the next one begins
    constexpr int FIRST = !HALF ? 0 : NF / 2 * AT_ONCE < LOADS ? NF / 2 * AT_ONCE : LOADS;
    constexpr int AHEAD_K = HALF ? S : S - 1;        // blocks that are asked for before the first is multiplied
    int64_t tile = blockIdx.x;
    turn_to(tile);
#pragma unroll
    for (int k = 0; k < AHEAD_K; ++k)
#pragma unroll
        for (int j = 0; j < LOADS; ++j) fetch(k, j);
    wait_and_meet<(AHEAD_K - 1) * LOADS>();
    bool behind = false;        // stores of the last tile lie between the loads
    for (;;) {
        f4 acc[NF][MF];
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int h = 0; h < MF; ++h) acc[f][h] = (f4)(0.0f);
        scales(0);
        i8 u = codes_b(0, 0), v[MF];
        b8 wide[MF][4];
#pragma unroll
        for (int h = 0; h < MF; ++h) v[h] = codes_a(0, h);
        if constexpr (!HALF) {
#pragma unroll
            for (int h = 0; h < MF; ++h) widen<FA>(v[h], sa[h] & 255u, wide[h]);
        }
        for (int k = 0; k < blocks; ++k) {
            const int stage = (k & (S - 1)) * STAGE, next = ((k + 1) & (S - 1)) * STAGE;
            if constexpr (HALF) {
                // First half of the fragments of B: each is multiplied while the one after it is read, and the second half's are read besides.
                constexpr int H = NF / 2;
                i8 w[H];
#pragma unroll
                for (int f = 0; f < H; ++f) {
                    i8 un = u;
                    if (f + 1 < H) un = codes_b(stage, f + 1);
                    w[f] = codes_b(stage, H + f);
                    keep_order();
#pragma unroll
                    for (int j = (H + f) * AT_ONCE; j < (H + f + 1) * AT_ONCE; ++j)
                        if (j < LOADS) fetch(k + S - 1, j, k > 0);
#pragma unroll
                    for (int h = 0; h < MF; ++h)
                        acc[f][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v[h], acc[f][h], FB, FA, 0, (int)sb[f], 0, (int)sa[h]);
                    keep_order();
                    u = un;
                }
                // All of this stage is in registers: it is given back.  Second half: as soon as a fragment of A is done with, the next block's is read.
                meet_behind_stores<(S - 2) * LOADS, (S - 2) * LOADS + STORES + LOADS - FIRST>(behind && k == 0);
                u = codes_b(next, 0);
#pragma unroll
                for (int h = 0; h < MF; ++h) {
                    keep_order();
#pragma unroll
                    for (int j = h * H * AT_ONCE / MF; j < (h + 1) * H * AT_ONCE / MF; ++j)
                        if (j < LOADS) fetch(k + S, j);
#pragma unroll
                    for (int f = 0; f < H; ++f)
                        acc[H + f][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[f], v[h], acc[H + f][h], FB, FA, 0, (int)sb[H + f], 0, (int)sa[h]);
                    keep_order();
                    v[h] = codes_a(next, h);
                }
            } else {
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    if (f + 1 == NF) wait_and_meet<(S - 2) * LOADS>();
                    const i8 un = f + 1 < NF ? codes_b(stage, f + 1) : codes_b(next, 0);
                    keep_order();
#pragma unroll
                    for (int j = f * AT_ONCE; j < (f + 1) * AT_ONCE; ++j)
                        if (j < LOADS) fetch(k + S - 1, j);
                    b8 x[4];
                    widen<FB>(u, sb[f] & 255u, x);
#pragma unroll
                    for (int h = 0; h < MF; ++h) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[f][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[q], wide[h][q], acc[f][h], 0, 0, 0);
                        if (f + 1 == NF) {
                            keep_order();
                            v[h] = codes_a(next, h);
                            keep_order();
                        }
                    }
                    keep_order();
                    u = un;
                }
            }
            scales(k + 1);
            const int shift = ((k + 1) & 3) * 8;
#pragma unroll
            for (int f = 0; f < NF; ++f) sb[f] >>= shift;
#pragma unroll
            for (int h = 0; h < MF; ++h) sa[h] >>= shift;
            if constexpr (!HALF) {
#pragma unroll
                for (int h = 0; h < MF; ++h) widen<FA>(v[h], sa[h] & 255u, wide[h]);
            }
        }
        // The next tile's first blocks are asked for before this tile's result leaves through LDS, eight rows at a time, so that a wavefront stores whole
        // stretches of 256 bytes; each has a place of its own, and waits for nobody.  Results and loads overlap in the smaller tiles only.  256 x 256 tiles
        // want more registers than there are (spilled: 8 to bf16, 2 to fp32, 28 onto a tensor), and what is read back behind the loads waits for them:
        // nothing leaves before the blocks have arrived.
        wait_and_meet();
        const int64_t m_out = m0 + wm * MF * 16 + lane / VECS, n_out = n0 + wn * NF * 16 + (lane % VECS) * PER_VEC;
        const bool whole_tile = m_here == TM && n_here == TN, whole = whole_tile && !ONTO;
        const int64_t done = tile;
        const bool in_parts = done >= p.full && p.parts > 1;
        // c_in of a whole tile is asked for sixteen rows at a time (asked for where it is added, every store waited for it: 33801 x 1024 x 4987 onto fp32
        // 331 us, so 305), by way of a buffer, whose addresses are one register for all rows.  (The stores' offsets are one for each row; in 256 x 256 tiles
        // they are among what is spilled, and most stores wait behind a reload for the store before them.)
        const bool ahead = ONTO && whole_tile && p.N <= 1 << 20;
        const int64_t corner = (m0 + wm * MF * 16) * p.N + n0 + wn * NF * 16;
        const uint32_t row_bytes = (uint32_t)p.N * 4, from_corner = (uint32_t)(lane / VECS) * row_bytes + (uint32_t)(lane % VECS) * 16;
        tile += gridDim.x;
        if (tile < all) {
            turn_to(tile);
#pragma unroll
            for (int k = 0; k < AHEAD_K; ++k)
#pragma unroll
                for (int j = 0; j < LOADS; ++j) fetch(k, j);
        }
        if (in_parts) {
            f4* const to = p.sums + ((done - p.full) * WAVES + wave) * (NF * MF * 64) + lane;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int h = 0; h < MF; ++h) to[(f * MF + h) * 64] = acc[f][h];
            if (tile >= all) return;
            behind = false;
            wait_and_meet();
            continue;
        }
        uint8_t* const mine = lds + T::RESULT + wave * 8 * PITCH;
        const auto leave = [&](auto in_advance) {
            constexpr bool AHEAD = decltype(in_advance)::value;
#pragma unroll
            for (int h = 0; h < MF; ++h) {
                [[maybe_unused]] f4 c[NF / EF][16 / TURN];
                if constexpr (AHEAD) {
                    const __amdgpu_buffer_rsrc_t onto = buffer((const uint8_t*)(p.c_in + corner), 0x7FFFFFFF);
                    keep_order();
#pragma unroll
                    for (int e = 0; e < NF; e += EF)
#pragma unroll
                        for (int t = 0; t < 16 / TURN; ++t)
                            c[e / EF][t] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(onto, from_corner, (h * 16 + t * TURN) * row_bytes + e * 64, NT));
                }
#pragma unroll
                for (int e = 0; e < NF; e += EF) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if ((i >> 3) == half) {
#pragma unroll
                            for (int f = e; f < e + EF; ++f) {
                                if constexpr (HALF) {
                                    if (f & 1) {
                                        const u4 w = {narrow2(acc[f - 1][h].x, acc[f - 1][h].y), narrow2(acc[f - 1][h].z, acc[f - 1][h].w),
                                                      narrow2(acc[f][h].x, acc[f][h].y), narrow2(acc[f][h].z, acc[f][h].w)};
                                        *reinterpret_cast<u4*>(mine + (i & 7) * PITCH + ((f >> 1) * 32 + g * 8) * 2) = w;
                                    }
                                } else {
                                    *reinterpret_cast<f4*>(mine + (i & 7) * PITCH + ((f - e) * 16 + g * 4) * 4) = acc[f][h];
                                }
                            }
                        }
                        __builtin_amdgcn_wave_barrier();
                        Vec out[8 / TURN];
#pragma unroll
                        for (int t = 0; t < 8 / TURN; ++t) out[t] = *reinterpret_cast<const Vec*>(mine + (t * TURN + lane / VECS) * PITCH + (lane % VECS) * 16);
#pragma unroll
                        for (int t = 0; t < 8 / TURN; ++t) {
                            const int64_t m = m_out + h * 16 + half * 8 + t * TURN;
                            if constexpr (AHEAD) {
                                // (All of the offset in the vector register: behind a store of 16 bytes with a scalar register for an offset the compiler
                                // leaves no wait before the data's registers are written again, and the store has taken what was written.)
                                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, out[t] + c[e / EF][half * (8 / TURN) + t]),
                                                                       buffer((const uint8_t*)((const float*)p.out + corner), 0x7FFFFFFF),
                                                                       from_corner + (uint32_t)(h * 16 + half * 8 + t * TURN) * row_bytes + e * 64, 0, NT);
                            } else if (m < p.M) {
                                store_row<HALF>(p, m, n_out + e * 16, out[t]);
                            }
                        }
                        __builtin_amdgcn_wave_barrier();
                    }
                }
            }
        };
        if constexpr (ONTO) {
            if (ahead) leave(std::true_type());
            else leave(std::false_type());
        } else {
            leave(std::false_type());
        }
        if (tile >= all) return;
        // the loads are older than the stores: where every store was made, these may still be on their way
        behind = whole;
        if (whole) wait_and_meet<(AHEAD_K - 1) * LOADS + STORES>();
        else wait_and_meet();
    }
#endif
}

// The tiles that were computed in parts: their sums, in the parts' order, and c_in.  A work-group takes one fragment of each wavefront of a tile.
template <bool HALF, int WN, int WM, int NF, int MF, int S>
__global__ __launch_bounds__(64 * WN * WM) void parts_kernel(Matmul p)
{
    typedef Tile<HALF, WN, WM, NF, MF, S> T;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wn = wave % WN, wm = wave / WN, i = lane & 15, g = lane >> 4;
    const int64_t rest = p.m_tiles * p.n_tiles - p.full, t = blockIdx.x / (NF * MF);
    const int fh = (int)(blockIdx.x % (NF * MF)), f = fh / MF, h = fh - f * MF;
    int64_t mt, nt;
    place(p.full + t, p.m_tiles, p.n_tiles, &mt, &nt);
    const int64_t m = mt * T::TM + (wm * MF + h) * 16 + i;
    const int64_t n = nt * T::TN + wn * NF * 16 + (HALF ? (f >> 1) * 32 + g * 8 + (f & 1) * 4 : f * 16 + g * 4);
    if (m >= p.M || n >= p.N) return;
    constexpr int64_t ONE = WN * WM * NF * MF * 64;
    const f4* const from = p.sums + t * ONE + (wave * NF * MF + fh) * 64 + lane;
    f4 v = from[0];
#pragma unroll 4
    for (int s = 1; s < p.parts; ++s) v += from[s * rest * ONE];
    store4<HALF>(p, m, n, v);
}

// K = 0: out = c_in, or zeros; an element to a lane.
__global__ __launch_bounds__(256) void copy_kernel(const float* c_in, void* out, int64_t n, int elem, int64_t first_wg)
{
    const int64_t at = (first_wg + blockIdx.x) * 256 + threadIdx.x;
    if (at >= n) return;
    if (elem == 2) ((uint16_t*)out)[at] = 0;
    else ((float*)out)[at] = c_in ? c_in[at] : 0.0f;
}

constexpr int64_t kMaxWgs = 1 << 22;      // work-groups per launch (a launch has less than 2^32 threads)

template <typename F>
void in_launches(int64_t wgs, int64_t most, F&& launch)
{
    for (int64_t at = 0; at < wgs; at += most) launch(at, (unsigned)(wgs - at < most ? wgs - at : most));
}

// Compute units of the current GPU.
int compute_units()
{
    static int of[16];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 16) return 256;
    if (of[dev] == 0) of[dev] = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0 ? n : 256;
    return of[dev];
}

template <typename T, int FMT, int WIDE>
void launch_quantize(Quantize p, hipStream_t stream)
{
    const dim3 threads(256 * WIDE);
    in_launches(p.row_tiles * ((p.col_tiles + WIDE - 1) / WIDE), kMaxWgs, [&](int64_t at, unsigned n) {
        p.tile_first = at;
        if (p.cols % 8 == 0) hipLaunchKernelGGL((quantize_kernel<T, FMT, true, WIDE>), dim3(n), threads, 0, stream, p);
        else hipLaunchKernelGGL((quantize_kernel<T, FMT, false, WIDE>), dim3(n), threads, 0, stream, p);
    });
}

// bf16 rows in pairs of tiles once every compute unit has four: both ways 4096 x 4096 15.4 us in pairs, 16.0 in single tiles, 5000 x 6000 29.3 / 30.8, but 4987 x
// 2048 12.9 / 11.3, and 1021 x 512 rows only 4.4 / 4.1.  fp32 rows have stretches of 512 bytes anyway: 8192 x 8192 87 / 84, 5000 x 6000 47.6 / 45.6.
template <int FMT>
void launch_quantize(const Quantize& p, bool half, hipStream_t stream)
{
    if (!half) launch_quantize<float, FMT, 1>(p, stream);
    else if (p.row_tiles * p.col_tiles >= 1024) launch_quantize<uint16_t, FMT, 2>(p, stream);
    else launch_quantize<uint16_t, FMT, 1>(p, stream);
}

// How a product is computed.  The form and the number of parts fix the order of additions, so they follow from the sizes and the result's type alone,
// as if for a GPU of 256 compute units.
enum { FORM_ROWS, FORM_LOW, FORM_DEEP, FORM_SMALL, FORM_LARGE };
struct Way {
    int form;
    int parts, part_blocks;
    int64_t full, rest;     // tiles that are computed whole, and in parts
    int log_kw;             // FORM_ROWS: wavefronts that share a place
    bool two;               // FORM_ROWS: places of 32 columns
};

// A form's tiles, how many of them a compute unit computes at a time, and the microseconds that these take: per block of 128 along K (half / full: for a
// bf16 / fp32 result), for the tiles' beginning and results, and with a part's sums instead.  Measured on products of 20 to 1100 GFLOP; two small
// tiles on a compute unit take 1 / 0.7 times as long as one.
struct Form {
    int tm, tn, beside;
    double block[2], tile[2], part;
};
constexpr Form kForms[] = {{0, 0, 0, {0, 0}, {0, 0}, 0},
                           {64, 128, 2, {1.10, 0.80}, {4.0, 2.5}, 2.5},
                           {64, 128, 1, {0.75, 0.33}, {3.5, 2.2}, 2.0},       // four stages
                           {128, 128, 2, {1.70, 1.15}, {6.0, 3.0}, 3.0},
                           {256, 256, 1, {2.75, 1.55}, {14.0, 6.0}, 6.0}};
constexpr int kUnits = 256;

// Rounds of work-groups on the compute units, the last of which may not find a second one on its.
double rounds_us(const Form& c, int64_t wgs, double each)
{
    const int64_t per_unit = (wgs + kUnits - 1) / kUnits, whole = per_unit / c.beside;
    return whole * each + (per_unit % c.beside ? 0.7 * each : 0.0);
}

// A work-group that has a compute unit to itself waits for its loads with two stages; with four it does not, 64 x 128 1239 x 1024 x 3419 to bf16 13.3 us / 20.3, 7135
// x 104 x 15275 30.1 / 36.9, 562 x 80 x 39483 to fp32 19.0 / 21.5.  Two beside each other hide their waits as well: four stages, which leave room for one, lose there.
// What was measured (us) / what one tile size for all would take, without parts: 33801 x 1024 x 4987 to fp32 269 / 322 (256 x 256: its third round has 20 tiles), 300 x 1024 x 20000
// to fp32 29 / 366, 1000 x 512 x 8000 to bf16 18 / 75, 12000 x 500 x 4000 to fp32 59 / 86, 8192 x 1024 x 32768 to fp32 391 (256 x 256 in two parts) / 477 (128 x 128).
Way way_for(int64_t M, int64_t N, int64_t K, bool half)
{
    const int blocks = (int)(code_row(K) / kBlock);
    Way w{FORM_ROWS, 1, blocks, 0, 0, 0, false};
    // Up to 32 rows the matrix instructions are idle anyway: B is read past LDS.  One wavefront has work for its latencies with eight blocks; where there are
    // few places, up to four share one.  32 rows / 33 rows, in tiles, us to bf16 and to fp32: 7003 x 512 5.3 / 6.0 and 5.6 / 7.2, 32768 x 1024 10.7 / 6.9 and
    // 10.0 / 11.4, 1024 x 32768 55 / 16 and 49 / 18.  The limit is no part of the costs below; it loses where K is long, and at 32768 x 1024 to bf16.
    if (M <= 32) {
        const int64_t places = (N + 15) / 16;
        while (w.log_kw < 2 && (places << w.log_kw) < 2048 && (4 << w.log_kw) < blocks) ++w.log_kw;
        // Places of 32 columns ask for A's codes half as often, where there are wavefronts enough and that is much of the work, us with 32 / 16: 32 x 32768 x 1024
        // to bf16 11.2 / 13.3, to fp32 10.1 / 13.4, 16 rows 9.1 / 9.5 and 8.1 / 9.6, one 8.3 / 6.8 and 7.1 / 7.0; 8192 x 4096, one row 9.1 / 10.4 and 8.7 /
        // 10.5; 10000 x 512, 32 rows 6.1 / 4.8.
        w.two = (places << w.log_kw) >= 1500 && (M > 16 || blocks >= 32 || (!half && M > 1 && blocks >= 8));
        return w;
    }
    double best = 1e30;
    for (int form = FORM_LOW; form <= FORM_LARGE; ++form) {
        const Form& c = kForms[form];
        const int64_t tiles = (M + c.tm - 1) / c.tm * ((N + c.tn - 1) / c.tn), room = (int64_t)c.beside * kUnits;
        const double block = c.block[half], whole = blocks * block + c.tile[half];
        // all tiles whole; or those of the last, unfinished round in parts
        const double us = rounds_us(c, tiles, whole);
        if (us < best) {
            best = us;
            w = Way{form, 1, blocks, tiles, 0, 0, false};
        }
        const int64_t rest = tiles % room ? tiles % room : tiles == room ? room : 0;
        for (int parts = 2; rest > 0 && parts <= 64 && parts * 4 <= blocks + 3; ++parts) {
            const int per = ((blocks + parts - 1) / parts + 3) / 4 * 4;
            if ((blocks + per - 1) / per != parts) continue;
            const double us = rounds_us(c, tiles - rest, whole) + rounds_us(c, rest * parts, per * block + c.part) + 3 + (double)(rest * c.tm * c.tn) * (4 * parts + 4) / 4e6;
            if (us < best) {
                best = us;
                w = Way{form, parts, per, tiles - rest, rest, 0, false};
            }
        }
    }
    return w;
}

int64_t parts_bytes(const Way& w) { return w.parts > 1 ? w.rest * w.parts * kForms[w.form].tm * kForms[w.form].tn * 4 : 0; }

template <int FA, int FB, bool HALF, int WN, int WM, int NF, int MF, int S>
void launch_tiles(Matmul p, hipStream_t stream)
{
    typedef Tile<HALF, WN, WM, NF, MF, S> T;
    p.n_tiles = (p.N + T::TN - 1) / T::TN;
    p.m_tiles = (p.M + T::TM - 1) / T::TM;
    const auto kernel = !HALF && p.c_in ? tile_kernel<FA, FB, HALF, !HALF, WN, WM, NF, MF, S> : tile_kernel<FA, FB, HALF, false, WN, WM, NF, MF, S>;
    const int lds = T::LDS;
    const int64_t rest = p.m_tiles * p.n_tiles - p.full, all = p.full + rest * p.parts;
    const int64_t most = (int64_t)compute_units() * (160 * 1024 / lds);          // as many work-groups as there is room for
    hipLaunchKernelGGL(kernel, dim3((unsigned)(all < most ? all : most)), dim3(64 * WN * WM), lds, stream, p);
    if (p.parts > 1) hipLaunchKernelGGL((parts_kernel<HALF, WN, WM, NF, MF, S>), dim3((unsigned)(rest * NF * MF)), dim3(64 * WN * WM), 0, stream, p);
}

template <int FA, int FB, bool HALF, int MF, int NF>
void launch_rows(Matmul p, int log_kw, hipStream_t stream)
{
    constexpr int waves = 4;
    const int columns = 16 * NF * (waves >> log_kw);
    in_launches((p.N + columns - 1) / columns, kMaxWgs / 2, [&](int64_t at, unsigned n) {
        p.n_first = at * columns;
        hipLaunchKernelGGL((rows_kernel<FA, FB, HALF, MF, NF>), dim3(n), dim3(64 * waves), 0, stream, p, log_kw);
    });
}

template <int FA, int FB, bool HALF>
void launch_matmul(const Matmul& p, const Way& w, hipStream_t stream)
{
    if (w.form == FORM_LARGE) launch_tiles<FA, FB, HALF, 2, 4, 8, 4, 2>(p, stream);
    else if (w.form == FORM_SMALL) launch_tiles<FA, FB, HALF, 2, 2, 4, 4, 2>(p, stream);
    else if (w.form == FORM_LOW) launch_tiles<FA, FB, HALF, 2, 2, 4, 2, 2>(p, stream);
    else if (w.form == FORM_DEEP) launch_tiles<FA, FB, HALF, 2, 2, 4, 2, 4>(p, stream);
    else if (p.M <= 16 && !w.two) launch_rows<FA, FB, HALF, 1, 1>(p, w.log_kw, stream);
    else if (p.M <= 16) launch_rows<FA, FB, HALF, 1, 2>(p, w.log_kw, stream);
    else if (!w.two) launch_rows<FA, FB, HALF, 2, 1>(p, w.log_kw, stream);
    else launch_rows<FA, FB, HALF, 2, 2>(p, w.log_kw, stream);
}

template <int FA, int FB>
void launch_matmul(const Matmul& p, bool half, const Way& w, hipStream_t stream)
{
    if (half) launch_matmul<FA, FB, true>(p, w, stream);
    else launch_matmul<FA, FB, false>(p, w, stream);
}

bool unaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
bool bad_format(int32_t f) { return f != TS_FP8_E4M3 && f != TS_FP8_E5M2; }
constexpr int64_t kSizeMax = (int64_t)1 << 31, kKMax = ((int64_t)1 << 24) - kBlock;      // (256 rows of codes: below 2^32 bytes)

}  // namespace

extern "C" {

int ts_fp8_layout(int64_t K, int64_t* code_bytes, int64_t* scale_bytes)
{
    if (!code_bytes || !scale_bytes) return TS_ERR_NULL;
    if (K < 0) return TS_ERR_SHAPE;
    if (K >= kSizeMax) return TS_ERR_OVERFLOW;
    *code_bytes = code_row(K);
    *scale_bytes = scale_row(K);
    return TS_OK;
}

int ts_quantize_fp8(const void* x, int32_t x_dtype, int64_t rows, int64_t cols, int32_t format, uint8_t* q, uint8_t* q_scales,
                    uint8_t* qt, uint8_t* qt_scales, void* stream)
{
    if (rows < 0 || cols < 0 || bad_format(format) || (x_dtype != TS_ROW_FP32 && x_dtype != TS_ROW_BF16)) return TS_ERR_SHAPE;
    if (rows >= kSizeMax || cols >= kSizeMax) return TS_ERR_OVERFLOW;
    if (rows == 0 || cols == 0) return TS_OK;           // (an empty tensor has no address)
    if ((!q && !qt) || (!q != !q_scales) || (!qt != !qt_scales)) return TS_ERR_NULL;
    if (unaligned(x, 16) || unaligned(q, 16) || unaligned(qt, 16) || unaligned(q_scales, 4) || unaligned(qt_scales, 4)) return TS_ERR_ALIGN;
    if (!x) return TS_ERR_NULL;
    Quantize p;
    p.x = x;
    p.q = q;
    p.q_scales = q_scales;
    p.qt = qt;
    p.qt_scales = qt_scales;
    p.rows = rows;
    p.cols = cols;
    p.row_tiles = (rows + kBlock - 1) / kBlock;
    p.col_tiles = (cols + kBlock - 1) / kBlock;
    const hipStream_t s = (hipStream_t)stream;
    if (format == TS_FP8_E4M3) launch_quantize<TS_FP8_E4M3>(p, x_dtype == TS_ROW_BF16, s);
    else launch_quantize<TS_FP8_E5M2>(p, x_dtype == TS_ROW_BF16, s);
    return hipGetLastError() == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int ts_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t* bytes)
{
    if (!bytes) return TS_ERR_NULL;
    if (M < 0 || N < 0 || K < 0) return TS_ERR_SHAPE;
    if (M >= kSizeMax || N >= kSizeMax || K > kKMax) return TS_ERR_OVERFLOW;
    if (M == 0 || N == 0 || K == 0) {
        *bytes = 0;
        return TS_OK;
    }
    const int64_t half = parts_bytes(way_for(M, N, K, true)), full = parts_bytes(way_for(M, N, K, false));
    *bytes = half > full ? half : full;
    return TS_OK;
}

int ts_matmul_fp8(const uint8_t* a, const uint8_t* a_scales, int32_t a_format, const uint8_t* b, const uint8_t* b_scales,
                  int32_t b_format, int64_t M, int64_t N, int64_t K, const float* c_in, void* out, int32_t out_dtype, void* stream)
{
    if (M < 0 || N < 0 || K < 0 || bad_format(a_format) || bad_format(b_format)) return TS_ERR_SHAPE;
    if ((out_dtype != TS_OUT_FP32 && out_dtype != TS_OUT_BF16) || (out_dtype == TS_OUT_BF16 && c_in)) return TS_ERR_SHAPE;
    if (M >= kSizeMax || N >= kSizeMax || K > kKMax) return TS_ERR_OVERFLOW;
    if (unaligned(a, 16) || unaligned(b, 16) || unaligned(a_scales, 4) || unaligned(b_scales, 4) || unaligned(c_in, 16) || unaligned(out, 16))
        return TS_ERR_ALIGN;
    if (M == 0 || N == 0) return TS_OK;
    if (!out || (K > 0 && (!a || !b || !a_scales || !b_scales))) return TS_ERR_NULL;
    Matmul p;
    p.a = a;
    p.a_scales = a_scales;
    p.b = b;
    p.b_scales = b_scales;
    p.c_in = c_in;
    p.out = out;
    p.M = M;
    p.N = N;
    p.ld = code_row(K);
    p.lds = scale_row(K);
    p.blocks = (int32_t)(p.ld / kBlock);
    p.m_tiles = p.n_tiles = p.n_first = 0;
    const bool half = out_dtype == TS_OUT_BF16;
    const hipStream_t s = (hipStream_t)stream;
    if (K == 0) {           // nothing to add up, and no operands to look at
        in_launches((M * N + 255) / 256, kMaxWgs, [&](int64_t at, unsigned n) {
            hipLaunchKernelGGL(copy_kernel, dim3(n), dim3(256), 0, s, c_in, out, M * N, half ? 2 : 4, at);
        });
        return hipGetLastError() == hipSuccess ? TS_OK : TS_ERR_HIP;
    }
    const Way w = way_for(M, N, K, half);
    p.parts = w.parts;
    p.part_blocks = w.part_blocks;
    p.full = w.full;
    p.sums = nullptr;
    if (w.parts > 1) {
        void* ws = nullptr;
        const int rc = ts_workspace::take(parts_bytes(w), &ws);
        if (rc != TS_OK) return rc;
        p.sums = (f4*)ws;
    }
    if (a_format == TS_FP8_E4M3 && b_format == TS_FP8_E4M3) launch_matmul<TS_FP8_E4M3, TS_FP8_E4M3>(p, half, w, s);
    else if (a_format == TS_FP8_E4M3) launch_matmul<TS_FP8_E4M3, TS_FP8_E5M2>(p, half, w, s);
    else if (b_format == TS_FP8_E4M3) launch_matmul<TS_FP8_E5M2, TS_FP8_E4M3>(p, half, w, s);
    else launch_matmul<TS_FP8_E5M2, TS_FP8_E5M2>(p, half, w, s);
    return hipGetLastError() == hipSuccess ? TS_OK : TS_ERR_HIP;
}

}  // extern "C"
