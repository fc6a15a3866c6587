// dropout.hip -- dropout of rows [m][c] whose mask is never stored, with an
// optional addition behind it.
//
//   words = Philox4x32-10 of the counter (ch / 8, row, site, step), key = seed
//   bits  = the (ch % 8)-th of the words' eight halves, low halves first
//   y     = (bits >= t ? x * 65536 / (65536 - t) : 0) + add,   t = round(65536 p)
//
// The generator is Philox4x32-10 of Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3" (2011): ten rounds of two 32 x 32 products.  An
// element's bits depend on its row, channel, site and step alone, not on strides,
// types or the launch, so the backward applies the forward's mask by forming it
// again.  Sixteen bits an element halve the generator's work per element: with 32 it
// would take as long as the memory accesses of bf16 rows (quarter-rate products).
// The scale is that of the rounded probability, so E[y] = x exactly.
//
// A thread takes eight channels of a row: one call of the generator.  Any stride and
// alignment: the eight elements move as one 16-byte access (two in float32), which
// gfx950 allows at element alignment, and one by one at a row's ragged end.  Bound by
// HBM: 8192 bf16 rows of 4096 with an addition 36.4 us = 5.5 TB/s on buffers that take turns
// (two, four and eight blocks a thread, whose loads all come first: 2, 5 and 9 us more), rows
// of 4095, none of them aligned, 47.7 us: an access of a wave ends inside a line, which the
// next one moves again.
#include "common.hpp"
#include "kernels.hpp"
#include "trace.hpp"

namespace bnr {

namespace {

__device__ __forceinline__ void philox4x32(uint32_t x[4], uint32_t k0, uint32_t k1)
{
    #pragma unroll
    for (int r = 0; r < 10; r++) {
        const uint64_t a = (uint64_t)x[0] * 0xD2511F53u, b = (uint64_t)x[2] * 0xCD9E8D57u;
        const uint32_t y0 = (uint32_t)(b >> 32) ^ x[1] ^ k0, y2 = (uint32_t)(a >> 32) ^ x[3] ^ k1;
        x[0] = y0; x[1] = (uint32_t)b; x[2] = y2; x[3] = (uint32_t)a;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
}

// Eight elements of storage type T, as they lie in memory.
template <typename T> struct Eight { T e[8]; };

template <bool WHOLE, typename T> __device__ __forceinline__ Eight<T> load8(const T *p, int n)
{
    Eight<T> v;
    if (WHOLE || n == 8) {
        __builtin_memcpy(&v, p, sizeof v);       // element-aligned: one 16-byte access each half KiB of a wave
    } else {
        #pragma unroll
        for (int i = 0; i < 8; i++) v.e[i] = i < n ? p[i] : (T)0;
    }
    return v;
}
template <bool WHOLE, typename T> __device__ __forceinline__ void store8(T *p, const Eight<T> &v, int n)
{
    if (WHOLE || n == 8) {
        __builtin_memcpy(p, &v, sizeof v);
    } else {
        #pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = v.e[i];
    }
}

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return bf2f(v); }
__device__ __forceinline__ void narrow(float v, float &o) { o = v; }
__device__ __forceinline__ void narrow(float v, bf16_t &o) { o = f2bf(v); }

// Thread t of a workgroup: block (first + t) % blocks of row (first + t) / blocks; the
// workgroup's own first item is divided once, the rest by a product (t + a block number
// stays below 2^31).  WHOLE: rows of whole blocks (c a multiple of eight), without the
// code of ragged ends.
template <typename T, bool ADD, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutParams p)
{
    const uint64_t first = (uint64_t)wide_block() * kThreads;
    const uint64_t row0 = first / p.blocks;
    const uint32_t col0 = (uint32_t)(first - row0 * p.blocks);
    const uint32_t step = p.step_dev ? *p.step_dev : p.step;
    const uint32_t k0 = (uint32_t)p.seed, k1 = (uint32_t)(p.seed >> 32);
    const T *x = (const T *)p.x, *add = (const T *)p.add;
    T *y = (T *)p.y;
    const uint32_t t = col0 + threadIdx.x, q = (uint32_t)(((uint64_t)t * p.magic) >> p.shift);
    const uint64_t r = row0 + q;
    const uint32_t blk = t - q * p.blocks, row = (uint32_t)r;
    if (r >= (uint64_t)p.m) return;
    const int n = WHOLE ? 8 : min(8, p.c - (int)blk * 8);
    const Eight<T> vx = load8<WHOLE>(x + (int64_t)row * p.x_ldc + blk * 8, n);
    Eight<T> va;
    if constexpr (ADD) va = load8<WHOLE>(add + (int64_t)row * p.add_ldc + blk * 8, n);
    uint32_t w[4] = {blk, row, p.site, step};
    philox4x32(w, k0, k1);
    Eight<T> o;
    #pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t bits = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
        const float a = ADD ? widen(va.e[i]) : 0.f, v = widen(vx.e[i]);
        // (a dropped infinity or NaN adds nothing)
        narrow(bits >= p.limit ? (ADD ? __builtin_fmaf(v, p.scale, a) : v * p.scale) : a, o.e[i]);
    }
    store8<WHOLE>(y + (int64_t)row * p.y_ldc + blk * 8, o, n);
}

template <typename T>
void go(const DropoutParams &p, dim3 g, hipStream_t s)
{
    const dim3 b(kThreads);
    if (p.c % 8 == 0) {
        if (p.add) hipLaunchKernelGGL((k_dropout<T, true, true>), g, b, 0, s, p);
        else hipLaunchKernelGGL((k_dropout<T, false, true>), g, b, 0, s, p);
    } else {
        if (p.add) hipLaunchKernelGGL((k_dropout<T, true, false>), g, b, 0, s, p);
        else hipLaunchKernelGGL((k_dropout<T, false, false>), g, b, 0, s, p);
    }
}

}  // namespace

int64_t dropout_groups(int64_t m, int c)
{
    const int64_t per = kThreads, blocks = (c + 7LL) / 8;
    return m > INT64_MAX / 2 / blocks ? INT64_MAX : (m * blocks + per - 1) / per;
}

hipError_t launch_dropout(int dtype, DropoutParams p, hipStream_t s)
{
    p.blocks = (uint32_t)((p.c + 7LL) / 8);
    // t / blocks = t magic >> shift for every t below 2^31: magic = ceil(2^shift / blocks), shift = 31 + ceil(log2 blocks)
    p.shift = 31;
    while ((1ull << (p.shift - 31)) < p.blocks) p.shift++;
    p.magic = (uint32_t)(((1ull << p.shift) + p.blocks - 1) / p.blocks);
    const double es = dtype == DT_BF16 ? 2 : 4, n = (double)p.m * p.c * es;
    TraceScope tr(KC_SWEEP, KID_DROPOUT, s, (p.add ? 3.0 : 2.0) * n, 0.0);
    const dim3 grid = wide_grid(dropout_groups(p.m, p.c));
    if (dtype == DT_BF16) go<bf16_t>(p, grid, s);
    else go<float>(p, grid, s);
    return hipGetLastError();
}

}  // namespace bnr
