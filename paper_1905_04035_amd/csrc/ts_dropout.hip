// Dropout with a mask that is made from a counter and never stored: on its own (ts_dropout) and on the embedding lookup
// whose gradient the densify calls take (ts_lookup_dropout).  What an element's fate follows from stands in philox.h.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "philox.h"
#include "ts_densify.h"

namespace {

using ts_mask::f4;
using ts_mask::Mask;
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int64_t kMaxWgs = 1 << 22;      // work-groups per launch (a launch has less than 2^32 threads)

// Four consecutive elements as fp32.
__device__ __forceinline__ f4 load4(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const f4*>(p)); }
__device__ __forceinline__ f4 widen4(u2 b)
{
    f4 r;
    r.x = __uint_as_float(b.x << 16);
    r.y = __uint_as_float(b.x & 0xFFFF0000u);
    r.z = __uint_as_float(b.y << 16);
    r.w = __uint_as_float(b.y & 0xFFFF0000u);
    return r;
}
__device__ __forceinline__ f4 load4(const uint16_t* p) { return widen4(__builtin_nontemporal_load(reinterpret_cast<const u2*>(p))); }

// The same for rows that are read again: those of hot ids, and of positions.
__device__ __forceinline__ f4 load4_kept(const float* p) { return *reinterpret_cast<const f4*>(p); }
__device__ __forceinline__ f4 load4_kept(const uint16_t* p) { return widen4(*reinterpret_cast<const u2*>(p)); }

// bf16, nearest with ties to even: one instruction for two elements.
__device__ __forceinline__ uint32_t narrow2(float x, float y)
{
    const f2 v = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}
__device__ __forceinline__ void store4(float* p, f4 v) { __builtin_nontemporal_store(v, reinterpret_cast<f4*>(p)); }
__device__ __forceinline__ void store4(uint16_t* p, f4 v)
{
    u2 b;
    b.x = narrow2(v.x, v.y);
    b.y = narrow2(v.z, v.w);
    __builtin_nontemporal_store(b, reinterpret_cast<u2*>(p));
}

// out[e] = add[e] + (kept ? x[e] * factor : 0) over a flat array, four elements per lane: those of one counter, so that no bit is made twice and no
// lane waits for another.  Bound by memory: nothing is read again, so all accesses are nontemporal.  With a residual, 65536 x 1024 bf16 66.5 us =
// 6.1 TB/s (a copy kernel reaches 6.2 to 6.4 here), 4987 x 516 fp32 6.2 us, of which 2 are the launch.
template <typename T, bool ADD>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* x, const T* add, T* out, int64_t groups, int64_t g_first, Mask m)
{
    const int64_t g = g_first + (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (g >= groups) return;
    const f4 v = load4(x + 4 * g), a = ADD ? load4(add + 4 * g) : (f4)(0.0f);
    store4(out + 4 * g, ts_mask::apply<ADD>(v, a, (uint64_t)g, ts_mask::offset_now(m), m));
}

struct Lookup {
    const int32_t *ids, *pos_ids;
    const void *weight, *pos;
    void* out;
    int64_t n, row_first;
    int32_t d, V, n_pos;
    float scale;
    Mask m;
};

// out[t] = dropout(scale * weight[ids[t]] + pos[pos_ids[t]]).  A row belongs to `lanes` neighbouring lanes (a power of two), a
// work-group takes 4 * 64 / lanes rows and, where rows are wider than 64 lanes, one block of CH * 256 of their columns: a lane then asks for all its
// parts of a row before it needs one (rows' addresses come from ids, which is a second latency).  Bound by memory: 16384 rows of 1024 from an fp32
// weight of 32768 rows, positions and a bf16 result 12.6 us = 5.8 TB/s of 39 MB read, as counted, and 33 written (28 us with one load per lane in
// flight).  The rows that are used and the positions are 25 MB, but hot ones are read into the L2 of each of eight XCDs.  One row 4.3 us, a launch.
template <typename W, typename O, int CH>
__global__ __launch_bounds__(kThreads) void lookup_kernel(Lookup p, int log_lanes)
{
    const int64_t t = p.row_first + ((int64_t)blockIdx.x * (kThreads >> log_lanes) + (threadIdx.x >> log_lanes));
    const int col0 = ((int)blockIdx.y * (64 * CH) + (int)(threadIdx.x & ((1u << log_lanes) - 1u))) * 4;
    if (t >= p.n || col0 >= p.d) return;
    const int32_t id = p.ids[t];
    const int32_t at = p.pos ? p.pos_ids[t] : -1;
    const bool has_row = (uint32_t)id < (uint32_t)p.V, has_pos = (uint32_t)at < (uint32_t)p.n_pos;
    f4 v[CH], q[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = col0 + c * 256;
        v[c] = q[c] = (f4)(0.0f);
        if (has_row && col < p.d) v[c] = load4_kept((const W*)p.weight + (size_t)id * p.d + col);
        if (has_pos && col < p.d) q[c] = load4_kept((const W*)p.pos + (size_t)at * p.d + col);
    }
    const uint64_t offset = ts_mask::offset_now(p.m);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = col0 + c * 256;
        if (col >= p.d) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[c][i] = fmaf(v[c][i], p.scale, q[c][i]);
        const int64_t e = t * p.d + col;
        store4((O*)p.out + e, ts_mask::apply<false>(v[c], (f4)(0.0f), (uint64_t)e >> 2, offset, p.m));
    }
}

template <typename T>
void launch_dropout(const void* x, const void* add, void* out, int64_t groups, const Mask& m, hipStream_t stream)
{
    for (int64_t at = 0; at < groups;) {
        const int64_t wgs = (groups - at + kThreads - 1) / kThreads;
        const dim3 grid((unsigned)(wgs < kMaxWgs ? wgs : kMaxWgs));
        if (add)
            hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(kThreads), 0, stream, (const T*)x, (const T*)add, (T*)out, groups, at, m);
        else
            hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(kThreads), 0, stream, (const T*)x, (const T*)nullptr, (T*)out, groups, at, m);
        at += (int64_t)grid.x * kThreads;
    }
}

template <typename W, typename O>
void launch_lookup(Lookup p, hipStream_t stream)
{
    int log_lanes = 0;
    while (log_lanes < 6 && (4 << log_lanes) < p.d) ++log_lanes;
    const int rows = kThreads >> log_lanes;
    const bool wide = p.d > 256;
    const unsigned blocks = (unsigned)(wide ? (p.d + 1023) / 1024 : 1);
    const int64_t most = kMaxWgs / blocks > 0 ? kMaxWgs / blocks : 1;
    for (int64_t at = 0; at < p.n;) {
        const int64_t wgs = (p.n - at + rows - 1) / rows;
        const dim3 grid((unsigned)(wgs < most ? wgs : most), blocks);
        p.row_first = at;
        if (wide) hipLaunchKernelGGL((lookup_kernel<W, O, 4>), grid, dim3(kThreads), 0, stream, p, log_lanes);
        else hipLaunchKernelGGL((lookup_kernel<W, O, 1>), grid, dim3(kThreads), 0, stream, p, log_lanes);
        at += (int64_t)grid.x * rows;
    }
}

bool unaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }
bool bad_type(int32_t t) { return t != TS_ROW_FP32 && t != TS_ROW_BF16; }

}  // namespace

extern "C" {

int ts_dropout(const void* x, const void* add, int64_t n, int32_t d, int32_t dtype, const ts_dropout_mask* mask, void* out, void* stream)
{
    if (n < 0 || d <= 0 || d % 4 != 0 || bad_type(dtype)) return TS_ERR_SHAPE;
    if (n >= (int64_t)1 << 31) return TS_ERR_OVERFLOW;
    Mask m;
    const int rc = ts_mask::make(mask, 1.0f, &m);
    if (rc != TS_OK) return rc;
    if (n == 0) return TS_OK;
    if (!x || !out) return TS_ERR_NULL;
    if (unaligned(x) || unaligned(add) || unaligned(out)) return TS_ERR_ALIGN;
    const int64_t groups = n * d / 4;
    if (dtype == TS_ROW_BF16) launch_dropout<uint16_t>(x, add, out, groups, m, (hipStream_t)stream);
    else launch_dropout<float>(x, add, out, groups, m, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int ts_lookup_dropout(const int32_t* ids, int64_t n, const void* weight, int32_t weight_dtype, int32_t d, int32_t V, float scale,
                      const void* pos, const int32_t* pos_ids, int32_t n_pos, const ts_dropout_mask* mask, void* out,
                      int32_t out_dtype, void* stream)
{
    if (n < 0 || d <= 0 || d % 4 != 0 || V <= 0 || n_pos < 0 || bad_type(weight_dtype) || bad_type(out_dtype) || !isfinite(scale))
        return TS_ERR_SHAPE;
    if (n >= (int64_t)1 << 31 || (d - 1) / 256 >= 65535) return TS_ERR_OVERFLOW;     // (the grid's second dimension)
    Lookup p;
    const int rc = ts_mask::make(mask, 1.0f, &p.m);
    if (rc != TS_OK) return rc;
    if (n == 0) return TS_OK;
    if (!ids || !weight || !out || (pos && !pos_ids) || (!pos && n_pos > 0)) return TS_ERR_NULL;
    if (unaligned(weight) || unaligned(out) || unaligned(pos) || ((uintptr_t)ids & 3u) || ((uintptr_t)pos_ids & 3u)) return TS_ERR_ALIGN;
    p.ids = ids;
    p.pos_ids = pos_ids;
    p.weight = weight;
    p.pos = pos;
    p.out = out;
    p.n = n;
    p.d = d;
    p.V = V;
    p.n_pos = n_pos;
    p.scale = scale;
    const hipStream_t s = (hipStream_t)stream;
    if (weight_dtype == TS_ROW_BF16 && out_dtype == TS_OUT_BF16) launch_lookup<uint16_t, uint16_t>(p, s);
    else if (weight_dtype == TS_ROW_BF16) launch_lookup<uint16_t, float>(p, s);
    else if (out_dtype == TS_OUT_BF16) launch_lookup<float, uint16_t>(p, s);
    else launch_lookup<float, float>(p, s);
    return hipGetLastError() == hipSuccess ? TS_OK : TS_ERR_HIP;
}

}  // extern "C"
