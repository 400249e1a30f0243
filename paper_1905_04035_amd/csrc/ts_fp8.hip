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

// ------------------------------------------------------------------ codes and scales
// Byte of the scale of a block whose largest finite magnitude is `most`: e + 127 for the smallest e >= -127 with
// most <= MAX 2^e, where MAX is 1.75 * 2^8 (e4m3) or 1.75 * 2^15 (e5m2).
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(float most)
{
    const uint32_t b = __float_as_uint(most);
    const int e = (int)(b >> 23) - (FMT == TS_FP8_E4M3 ? 8 : 15) + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)(e < 0 ? 0 : e);
}

__device__ __forceinline__ float finite_size(float x)
{
    const float a = fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;
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
    int64_t col_tiles;
};

__device__ __forceinline__ float widen1(const float* p) { return *p; }
__device__ __forceinline__ float widen1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ f4 widen4(const float* p) { return *reinterpret_cast<const f4*>(p); }
__device__ __forceinline__ f4 widen4(const uint16_t* p)
{
    const u2 b = *reinterpret_cast<const u2*>(p);
    f4 r;
    r.x = __uint_as_float(b.x << 16);
    r.y = __uint_as_float(b.x & 0xFFFF0000u);
    r.z = __uint_as_float(b.y << 16);
    r.w = __uint_as_float(b.y & 0xFFFF0000u);
    return r;
}

// A work-group takes a tile of 128 x 128 elements, a thread 8 x 8 of them.  A row's block is in the registers of sixteen
// neighbouring lanes; a column's in those of every sixteenth thread.
template <typename T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void quantize_kernel(Quantize p)
{
    __shared__ float most_of[4][kBlock];
    __shared__ __align__(16) uint8_t turned[kBlock][kBlock + 16];
    const int64_t tile = p.tile_first + blockIdx.x;
    const int64_t r_tile = tile / p.col_tiles, c_tile = tile - r_tile * p.col_tiles;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int r8 = (tid >> 4) * 8, c8 = (tid & 15) * 8;       // the thread's place in the tile
    const int64_t r0 = r_tile * kBlock + r8, c0 = c_tile * kBlock + c8;
    f4 v[8][2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const T* const row = (const T*)p.x + (r0 + i) * p.cols + c0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[i][h] = (f4)(0.0f);
            if (r0 + i < p.rows) {
                if (VEC) {
                    if (c0 + 4 * h < p.cols) v[i][h] = widen4(row + 4 * h);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (c0 + 4 * h + j < p.cols) v[i][h][j] = widen1(row + 4 * h + j);
                }
            }
        }
    }
    if (p.q) {
        const int64_t ld = code_row(p.cols), lds = scale_row(p.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float most = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) most = fmaxf(most, finite_size(v[i][h][j]));
#pragma unroll
            for (int m = 1; m < 16; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
            const uint32_t byte = scale_byte<FMT>(most);
            if (r0 + i < p.rows) {
                u2 w;
                w.x = codes4<FMT>(v[i][0], byte);
                w.y = codes4<FMT>(v[i][1], byte);
                *reinterpret_cast<u2*>(p.q + (r0 + i) * ld + c0) = w;
                // lane 0 of the sixteen writes the block's byte; behind the last block, lanes 1 to 3 the zeros
                const int64_t at = c_tile + (lane & 15);
                if ((lane & 15) == 0) p.q_scales[(r0 + i) * lds + at] = (uint8_t)byte;
                else if (c_tile == p.col_tiles - 1 && at < lds) p.q_scales[(r0 + i) * lds + at] = 0;
            }
        }
    }
    if (!p.qt) return;
    f4 most[2] = {(f4)(0.0f), (f4)(0.0f)};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) most[h][j] = fmaxf(most[h][j], finite_size(v[i][h][j]));
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            most[h][j] = fmaxf(most[h][j], __shfl_xor(most[h][j], 16));
            most[h][j] = fmaxf(most[h][j], __shfl_xor(most[h][j], 32));
            if (lane < 16) most_of[wave][c8 + 4 * h + j] = most[h][j];
        }
    __syncthreads();
    const int64_t ld = code_row(p.rows), lds = scale_row(p.rows), row_tiles = (p.rows + kBlock - 1) / kBlock;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c8 + 4 * h + j;
            const float m = fmaxf(fmaxf(most_of[0][c], most_of[1][c]), fmaxf(most_of[2][c], most_of[3][c]));
            const uint32_t byte = scale_byte<FMT>(m);
            const f4 lo = {v[0][h][j], v[1][h][j], v[2][h][j], v[3][h][j]}, hi = {v[4][h][j], v[5][h][j], v[6][h][j], v[7][h][j]};
            u2 w;
            w.x = codes4<FMT>(lo, byte);
            w.y = codes4<FMT>(hi, byte);
            *reinterpret_cast<u2*>(&turned[c][r8]) = w;
            if (r8 == 0 && c0 + 4 * h + j < p.cols) {
                uint8_t* const s = p.qt_scales + (c0 + 4 * h + j) * lds;
                s[r_tile] = (uint8_t)byte;
                if (r_tile == row_tiles - 1)
                    for (int64_t at = row_tiles; at < lds; ++at) s[at] = 0;
            }
        }
    __syncthreads();
    // eight lanes to a row of 128 codes
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 32 + (tid >> 3), at = (tid & 7) * 16;
        if (c_tile * kBlock + c < p.cols)
            *reinterpret_cast<u4*>(p.qt + (c_tile * kBlock + c) * ld + r_tile * kBlock + at) = *reinterpret_cast<const u4*>(&turned[c][at]);
    }
}

// ------------------------------------------------------------------ product
#define LOAD16(base, off, to) \
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)((base) + (off)), \
                                     (__attribute__((address_space(3))) void*)(lds + (to)), 16, 0, 0)

struct Matmul {
    const uint8_t *a, *a_scales, *b, *b_scales;
    const float* c_in;
    void* out;
    int64_t M, N;
    int64_t ld, lds;            // bytes of a row of codes and of scales
    int32_t blocks;             // of 128 along K
    int64_t tile_first;
    int64_t n_tiles;
};

// Stores out[m][n .. n + 3].
template <bool BF16>
__device__ __forceinline__ void store4(const Matmul& p, int64_t m, int64_t n, f4 v)
{
    if (m >= p.M || n >= p.N) return;
    const int64_t at = m * p.N + n;
    if ((p.N & 3) == 0) {
        if (p.c_in) v += *reinterpret_cast<const f4*>(p.c_in + at);
        if (BF16) {
            u2 w;
            w.x = narrow2(v.x, v.y);
            w.y = narrow2(v.z, v.w);
            *reinterpret_cast<u2*>((uint16_t*)p.out + at) = w;
        } else {
            *reinterpret_cast<f4*>((float*)p.out + at) = v;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i >= p.N) return;
        const float x = p.c_in ? v[i] + p.c_in[at + i] : v[i];
        if (BF16) ((uint16_t*)p.out)[at + i] = (uint16_t)narrow2(x, x);
        else ((float*)p.out)[at + i] = x;
    }
}

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

__device__ __forceinline__ i8 load_codes(const uint8_t* p)
{
    const i4 lo = *reinterpret_cast<const i4*>(p), hi = *reinterpret_cast<const i4*>(p + 16);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A wavefront computes 16 columns of the result in 16 rows: lane l holds 32 codes of row l % 16 of either operand.
template <int FA, int FB, bool BF16>
__global__ __launch_bounds__(256) void matmul_kernel(Matmul p)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tile = p.tile_first + blockIdx.x;
    const int64_t m0 = tile / p.n_tiles * 16, n0 = (tile % p.n_tiles) * 64 + wave * 16;
    const int64_t m = m0 + (lane & 15), n = n0 + (lane & 15);
    const int64_t ra = m < p.M ? m : p.M - 1, rb = n < p.N ? n : p.N - 1;       // rows past the end: the last one again
    const uint8_t *a = p.a + ra * p.ld + (lane >> 4) * 32, *b = p.b + rb * p.ld + (lane >> 4) * 32;
    const uint8_t *sa = p.a_scales + ra * p.lds, *sb = p.b_scales + rb * p.lds;
    f4 acc = (f4)(0.0f);
    for (int k = 0; k < p.blocks; ++k) {
        const i8 u = load_codes(b + (int64_t)k * kBlock), v = load_codes(a + (int64_t)k * kBlock);
        if (BF16) {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v, acc, FB, FA, 0, sb[k], 0, sa[k]);
        } else {
            b8 x[4], y[4];
            widen<FB>(u, sb[k], x);
            widen<FA>(v, sa[k], y);
#pragma unroll
            for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[q], y[q], acc, 0, 0, 0);
        }
    }
    store4<BF16>(p, m, n0 + (lane >> 4) * 4, acc);
}

// ---- large products: tiles through LDS
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int FA, int FB, bool BF16, int WN, int WM, int NF, int MF>
__global__ __launch_bounds__(64 * WN * WM) void tile_kernel(Matmul p)
{
    constexpr int TN = 16 * WN * NF, TM = 16 * WM * MF, ROWS = TN + TM, WAVES = WN * WM;
    constexpr int LOADS = ROWS / (8 * WAVES);                 // of 1 KiB by a wavefront, for one block
    extern __shared__ __align__(1024) uint8_t lds[];          // [2][ROWS][128]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wm = wave / WN;
    const int64_t tile = p.tile_first + blockIdx.x;
    const int64_t m0 = tile / p.n_tiles * TM, n0 = tile % p.n_tiles * TN;

    const auto key = [](int row, bool of_b) { return BF16 && of_b ? (row & 3) | ((row >> 1) & 4) : row & 7; };
    // where this lane's 16 bytes of each load come from
    uint32_t from[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int row = (wave * LOADS + j) * 8 + (lane >> 3);
        const bool of_b = (wave * LOADS + j) * 8 < TN;
        const int r = of_b ? row : row - TN;
        const int64_t last = of_b ? p.N - 1 - n0 : p.M - 1 - m0;
        const int64_t at = r < last ? r : last;
        from[j] = (uint32_t)(at * p.ld) + (uint32_t)(((lane & 7) ^ key(r, of_b)) * 16);
    }
    const uint8_t *const a = p.a + m0 * p.ld, *const b = p.b + n0 * p.ld;
    const auto fetch = [&](int k, int stage) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const bool of_b = (wave * LOADS + j) * 8 < TN;
            const uint8_t* const base = (of_b ? b : a) + (int64_t)k * kBlock;
            const uint32_t to = (uint32_t)(stage * ROWS * kBlock + (wave * LOADS + j) * 1024);
            LOAD16(base, from[j], to);
        }
    };
    // scales: four blocks to a word
    const uint32_t *sb_at[NF], *sa_at[MF];
    uint32_t sb[NF], sa[MF], sb_next[NF], sa_next[MF];
    const int i = lane & 15, g = lane >> 4;
    const auto n_of = [&](int f) { return BF16 ? (f >> 1) * 32 + (i >> 2) * 8 + (f & 1) * 4 + (i & 3) : f * 16 + i; };
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        const int64_t n = n0 + wn * NF * 16 + n_of(f);
        sb_at[f] = (const uint32_t*)(p.b_scales + (n < p.N ? n : p.N - 1) * p.lds);
        sb_next[f] = *sb_at[f];
    }
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int64_t m = m0 + (wm * MF + f) * 16 + i;
        sa_at[f] = (const uint32_t*)(p.a_scales + (m < p.M ? m : p.M - 1) * p.lds);
        sa_next[f] = *sa_at[f];
    }
    const uint8_t* const read_b = lds + (wn * NF * 16 + n_of(0)) * kBlock + ((g ^ (i & 7)) << 4);
    const uint8_t* const read_a = lds + (TN + wm * MF * 16 + i) * kBlock + ((g ^ (i & 7)) << 4);
    const uint8_t* const read_b4 = lds + (wn * NF * 16 + n_of(0)) * kBlock + (((g ^ (i & 7)) ^ 4) << 4);
    const uint8_t* const read_a4 = lds + (TN + wm * MF * 16 + i) * kBlock + (((g ^ (i & 7)) ^ 4) << 4);
    const auto codes = [&](const uint8_t* lo, const uint8_t* hi, int at) {
        const i4 x = *reinterpret_cast<const i4*>(lo + at), y = *reinterpret_cast<const i4*>(hi + at);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    f4 acc[NF][MF];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int h = 0; h < MF; ++h) acc[f][h] = (f4)(0.0f);

    fetch(0, 0);
    for (int k = 0; k < p.blocks; ++k) {
        wait_and_meet();
        if ((k & 3) == 0) {
#pragma unroll
            for (int f = 0; f < NF; ++f) sb[f] = sb_next[f];
#pragma unroll
            for (int f = 0; f < MF; ++f) sa[f] = sa_next[f];
        }
        if (k + 1 < p.blocks) {
            fetch(k + 1, (k + 1) & 1);
            if ((k & 3) == 3) {
#pragma unroll
                for (int f = 0; f < NF; ++f) sb_next[f] = sb_at[f][(k + 1) >> 2];
#pragma unroll
                for (int f = 0; f < MF; ++f) sa_next[f] = sa_at[f][(k + 1) >> 2];
            }
        }
        const int stage = (k & 1) * ROWS * kBlock, shift = (k & 3) * 8;
        if constexpr (BF16) {
            i8 v[MF];
#pragma unroll
            for (int h = 0; h < MF; ++h) v[h] = codes(read_a, read_a4, stage + h * 16 * kBlock);
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const i8 u = codes(read_b, read_b4, stage + (f >> 1) * 32 * kBlock + (f & 1) * 4 * kBlock);
#pragma unroll
                for (int h = 0; h < MF; ++h)
                    acc[f][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v[h], acc[f][h], FB, FA, 0, (int)(sb[f] >> shift), 0, (int)(sa[h] >> shift));
            }
        } else {
            b8 v[MF][4];
#pragma unroll
            for (int h = 0; h < MF; ++h) widen<FA>(codes(read_a, read_a4, stage + h * 16 * kBlock), (sa[h] >> shift) & 255u, v[h]);
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                b8 u[4];
                widen<FB>(codes(read_b, read_b4, stage + f * 16 * kBlock), (sb[f] >> shift) & 255u, u);
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int h = 0; h < MF; ++h) acc[f][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u[q], v[h][q], acc[f][h], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int h = 0; h < MF; ++h) {
        const int64_t m = m0 + (wm * MF + h) * 16 + i;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int64_t n = n0 + wn * NF * 16 + (BF16 ? (f >> 1) * 32 + g * 8 + (f & 1) * 4 : f * 16 + g * 4);
            store4<BF16>(p, m, n, acc[f][h]);
        }
    }
}

constexpr int64_t kMaxWgs = 1 << 22;      // work-groups per launch (a launch has less than 2^32 threads)

template <typename F>
void in_launches(int64_t tiles, F&& launch)
{
    for (int64_t at = 0; at < tiles; at += kMaxWgs) launch(at, (unsigned)(tiles - at < kMaxWgs ? tiles - at : kMaxWgs));
}

template <typename T, int FMT>
void launch_quantize(Quantize p, int64_t tiles, hipStream_t stream)
{
    in_launches(tiles, [&](int64_t at, unsigned n) {
        p.tile_first = at;
        if (p.cols % 4 == 0) hipLaunchKernelGGL((quantize_kernel<T, FMT, true>), dim3(n), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((quantize_kernel<T, FMT, false>), dim3(n), dim3(256), 0, stream, p);
    });
}

template <int FA, int FB, bool BF16, int WN, int WM, int NF, int MF>
void launch_tiles(Matmul p, hipStream_t stream)
{
    constexpr int TN = 16 * WN * NF, TM = 16 * WM * MF;
    p.n_tiles = (p.N + TN - 1) / TN;
    const int lds = 2 * (TN + TM) * kBlock;
    const auto kernel = tile_kernel<FA, FB, BF16, WN, WM, NF, MF>;
    in_launches((p.M + TM - 1) / TM * p.n_tiles, [&](int64_t at, unsigned n) {
        p.tile_first = at;
        hipLaunchKernelGGL(kernel, dim3(n), dim3(64 * WN * WM), lds, stream, p);
    });
}

template <int FA, int FB>
void launch_matmul(Matmul p, bool bf16, hipStream_t stream)
{
    if (p.blocks > 0 && p.M > 64 && p.N > 64) {          // (a tile's first block is fetched without a question)
        if (bf16) launch_tiles<FA, FB, true, 2, 4, 8, 4>(p, stream);
        else launch_tiles<FA, FB, false, 2, 2, 4, 4>(p, stream);
        return;
    }
    p.n_tiles = (p.N + 63) / 64;
    in_launches((p.M + 15) / 16 * p.n_tiles, [&](int64_t at, unsigned n) {
        p.tile_first = at;
        if (bf16) hipLaunchKernelGGL((matmul_kernel<FA, FB, true>), dim3(n), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((matmul_kernel<FA, FB, false>), dim3(n), dim3(256), 0, stream, p);
    });
}

bool unaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
bool bad_format(int32_t f) { return f != TS_FP8_E4M3 && f != TS_FP8_E5M2; }
constexpr int64_t kSizeMax = (int64_t)1 << 31, kKMax = (int64_t)1 << 24;

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
    if ((!q && !qt) || (!q != !q_scales) || (!qt != !qt_scales)) return TS_ERR_NULL;
    if (unaligned(x, 16) || unaligned(q, 16) || unaligned(qt, 16) || unaligned(q_scales, 4) || unaligned(qt_scales, 4)) return TS_ERR_ALIGN;
    if (rows == 0 || cols == 0) return TS_OK;
    if (!x) return TS_ERR_NULL;
    Quantize p;
    p.x = x;
    p.q = q;
    p.q_scales = q_scales;
    p.qt = qt;
    p.qt_scales = qt_scales;
    p.rows = rows;
    p.cols = cols;
    p.col_tiles = (cols + kBlock - 1) / kBlock;
    const int64_t tiles = (rows + kBlock - 1) / kBlock * p.col_tiles;
    const hipStream_t s = (hipStream_t)stream;
    if (x_dtype == TS_ROW_BF16 && format == TS_FP8_E4M3) launch_quantize<uint16_t, TS_FP8_E4M3>(p, tiles, s);
    else if (x_dtype == TS_ROW_BF16) launch_quantize<uint16_t, TS_FP8_E5M2>(p, tiles, s);
    else if (format == TS_FP8_E4M3) launch_quantize<float, TS_FP8_E4M3>(p, tiles, s);
    else launch_quantize<float, TS_FP8_E5M2>(p, tiles, s);
    return hipGetLastError() == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int ts_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t* bytes)
{
    if (!bytes) return TS_ERR_NULL;
    if (M < 0 || N < 0 || K < 0) return TS_ERR_SHAPE;
    if (M >= kSizeMax || N >= kSizeMax || K > kKMax) return TS_ERR_OVERFLOW;
    *bytes = 0;
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
    const bool bf16 = out_dtype == TS_OUT_BF16;
    const hipStream_t s = (hipStream_t)stream;
    if (a_format == TS_FP8_E4M3 && b_format == TS_FP8_E4M3) launch_matmul<TS_FP8_E4M3, TS_FP8_E4M3>(p, bf16, s);
    else if (a_format == TS_FP8_E4M3) launch_matmul<TS_FP8_E4M3, TS_FP8_E5M2>(p, bf16, s);
    else if (b_format == TS_FP8_E4M3) launch_matmul<TS_FP8_E5M2, TS_FP8_E4M3>(p, bf16, s);
    else launch_matmul<TS_FP8_E5M2, TS_FP8_E5M2>(p, bf16, s);
    return hipGetLastError() == hipSuccess ? TS_OK : TS_ERR_HIP;
}

}  // extern "C"
