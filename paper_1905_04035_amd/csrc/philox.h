// The generator behind dropout, and how a mask follows from it.  Shared by the forward kernels (ts_dropout.hip) and the
// densify kernels that make the same mask again for the gradient (ts_densify.hip).
//
// Philox4x32 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011): a counter of four
// 32-bit words goes through rounds of two 32 x 32 -> 64 bit products; any element's bits follow from its place and the key
// alone, so nothing is stored and no order of evaluation matters.  Seven rounds: the fewest that pass the whole BigCrush
// battery according to that paper (ten is its margin).  A round costs a lane two wide products, each four times as long as
// an addition, per four elements (thirteen in all: one of the first round's is the same for all lanes); ten rounds would take 1.5
// times as long where the products bound a kernel.
#ifndef TS_PHILOX_H
#define TS_PHILOX_H

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ts_densify.h"

namespace ts_mask {

constexpr int kRounds = 7;

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));

// What a kernel needs of a ts_dropout_mask.
struct Mask {
    uint64_t offset;
    const uint64_t* step;       // its value when the kernel runs is added to offset; or NULL
    uint32_t key0, key1;
    uint32_t threshold;         // an element is kept if its word is at least this; 0: all are kept, no word is made
    float factor;               // of the kept elements
};

// One instruction, which the compiler does not form by itself (two exclusive ors take
// the dropout of 65536 x 1024 bf16 with a residual from 66.4 to 67.3 us, and ts_densify_dropout of 131072 x 1024 bf16 from 121.6 to 128.1).
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// Words of elements 4 * group .. 4 * group + 3.
__device__ __forceinline__ u4 words(uint64_t group, uint64_t offset, uint32_t k0, uint32_t k1)
{
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor3((uint32_t)(q >> 32), c1, k0);
        c1 = (uint32_t)q;
        c2 = xor3((uint32_t)(p >> 32), c3, k1);
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    u4 w;
    w.x = c0;
    w.y = c1;
    w.z = c2;
    w.w = c3;
    return w;
}

__device__ __forceinline__ uint64_t offset_now(const Mask& m) { return m.offset + (m.step ? *m.step : 0ull); }

// x * factor + add where the element is kept, add where it is dropped (whatever x is there, NaN and infinities included).
template <bool ADD>
__device__ __forceinline__ f4 apply(f4 x, f4 add, uint64_t group, uint64_t offset, const Mask& m)
{
    f4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = ADD ? fmaf(x[i], m.factor, add[i]) : x[i] * m.factor;
    if (m.threshold == 0) return y;
    const u4 w = words(group, offset, m.key0, m.key1);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = w[i] >= m.threshold ? y[i] : (ADD ? add[i] : 0.0f);
    return y;
}

// The host's side: checks a mask and works its constants out.  scale: a further factor of the kept elements.
inline int make(const ts_dropout_mask* from, float scale, Mask* to)
{
    if (!from) return TS_ERR_NULL;
    if (!(from->p >= 0.0f && from->p < 1.0f) || !isfinite(scale)) return TS_ERR_SHAPE;
    if ((uintptr_t)from->step & 7u) return TS_ERR_ALIGN;
    to->offset = from->offset;
    to->step = from->step;
    to->key0 = (uint32_t)from->seed;
    to->key1 = (uint32_t)(from->seed >> 32);
    to->threshold = (uint32_t)((double)from->p * 4294967296.0);
    to->factor = (float)((double)scale / (1.0 - (double)from->p));
    return isfinite(to->factor) ? TS_OK : TS_ERR_SHAPE;
}

}  // namespace ts_mask

#endif  // TS_PHILOX_H
