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
// A thread takes eight channels of a row (one call of the generator), kDropWays of
// them with their loads issued ahead of the generator.  Any stride and alignment:
// the eight elements move as one 16-byte access (two in float32), which gfx950
// allows at element alignment, and one by one at a row's ragged end.
#include "common.hpp"
#include "kernels.hpp"
#include "trace.hpp"

namespace bnr {

namespace {

constexpr int kDropWays = 4;

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

template <typename T> __device__ __forceinline__ Eight<T> load8(const T *p, int n)
{
    Eight<T> v;
    if (n == 8) {
        __builtin_memcpy(&v, p, sizeof v);       // element-aligned: one 16-byte access each half KiB of a wave
    } else {
        #pragma unroll
        for (int i = 0; i < 8; i++) v.e[i] = i < n ? p[i] : (T)0;
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store8(T *p, const Eight<T> &v, int n)
{
    if (n == 8) {
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

// Work item i of a workgroup's kDropWays * kThreads: block (first + i) % blocks of row
// (first + i) / blocks; the workgroup's own first item is divided once, the rest by a
// product (i + a block number stays below 2^31).
template <typename T, bool ADD>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutParams p)
{
    const uint64_t first = (uint64_t)blockIdx.x * (kDropWays * kThreads);
    const uint64_t row0 = first / p.blocks;
    const uint32_t col0 = (uint32_t)(first - row0 * p.blocks);
    const uint32_t step = p.step_dev ? *p.step_dev : p.step;
    const uint32_t k0 = (uint32_t)p.seed, k1 = (uint32_t)(p.seed >> 32);
    const T *x = (const T *)p.x, *add = (const T *)p.add;
    T *y = (T *)p.y;
    Eight<T> vx[kDropWays], va[kDropWays];
    uint32_t row[kDropWays], blk[kDropWays];
    int n[kDropWays];
    #pragma unroll
    for (int u = 0; u < kDropWays; u++) {
        const uint32_t t = col0 + u * kThreads + threadIdx.x;
        const uint32_t q = (uint32_t)(((uint64_t)t * p.magic) >> p.shift);
        const uint64_t r = row0 + q;
        blk[u] = t - q * p.blocks;
        row[u] = (uint32_t)r;
        n[u] = r < (uint64_t)p.m ? min(8, p.c - (int)blk[u] * 8) : 0;
        if (n[u] > 0) {
            vx[u] = load8(x + (int64_t)row[u] * p.x_ldc + blk[u] * 8, n[u]);
            if constexpr (ADD) va[u] = load8(add + (int64_t)row[u] * p.add_ldc + blk[u] * 8, n[u]);
        }
    }
    #pragma unroll
    for (int u = 0; u < kDropWays; u++) {
        if (n[u] <= 0) continue;
        uint32_t w[4] = {blk[u], row[u], p.site, step};
        philox4x32(w, k0, k1);
        Eight<T> o;
        #pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t bits = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
            const float a = ADD ? widen(va[u].e[i]) : 0.f, v = widen(vx[u].e[i]);
            // (a dropped infinity or NaN adds nothing)
            narrow(bits >= p.limit ? (ADD ? __builtin_fmaf(v, p.scale, a) : v * p.scale) : a, o.e[i]);
        }
        store8(y + (int64_t)row[u] * p.y_ldc + blk[u] * 8, o, n[u]);
    }
}

template <typename T>
void go(const DropoutParams &p, unsigned grid, hipStream_t s)
{
    if (p.add) hipLaunchKernelGGL((k_dropout<T, true>), dim3(grid), dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((k_dropout<T, false>), dim3(grid), dim3(kThreads), 0, s, p);
}

}  // namespace

int64_t dropout_groups(int64_t m, int c)
{
    const int64_t per = kDropWays * kThreads, blocks = (c + 7LL) / 8;
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
    const unsigned grid = (unsigned)dropout_groups(p.m, p.c);
    if (dtype == DT_BF16) go<bf16_t>(p, grid, s);
    else go<float>(p, grid, s);
    return hipGetLastError();
}

}  // namespace bnr
