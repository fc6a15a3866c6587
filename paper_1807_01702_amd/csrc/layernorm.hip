// layernorm.hip -- layer normalisation over the channels of each row (pixel,
// token), forward and backward, for float32 and bf16 rows of up to kLnMaxC
// channels.
//
//   forward   s = x, or the stored x + res;  mean = sum(s)/c,
//             var = sum((s - mean)^2)/c,  rstd = (var + eps)^-1/2,
//             y = (s - mean) rstd gamma + beta
//   backward  g = dy gamma,  xhat = (x - mean) rstd,
//             dx = rstd (g - sum(g)/c - xhat sum(g xhat)/c)  (+ dsum),
//             dgamma = sum over rows of dy xhat,  dbeta = sum over rows of dy
//
// Both passes are bound by HBM: every input is read once and every output
// written once, with the row held in registers between the reductions.  The
// forward adds a row in float64 and takes differences from the unrounded mean
// (as two float32 parts), so a mean far from zero costs them no accuracy and a
// row of one repeated value differs from its mean by nothing; the rest is
// float32.  The stored mean is rounded to float32, and the backward's xhat
// carries that rounding, 2^-24 |mean| rstd.
// Measured: forward, 8192 bf16 rows of 4096 with a residual, 43.4 us = 6.2 TB/s
// (part of it from the last-level cache); backward there 50.3 us, 401408 rows of
// 256 154 to 158 us = 5.2 to 5.3 TB/s, where a copy of 4 GiB runs at 5.44.
//
// A row is held by TPR threads with NV loads of V elements each: V is the
// 16-byte vector where pointers, strides and the channel count allow it, else
// one element.  (The 1024-thread forward of more than 8192 single elements spills 64
// registers of its row.)  Rows of up to 64 TPR-lanes reduce with cross-lane shuffles and
// need no barrier; longer rows take a workgroup of 256 or 1024 threads.
#include "common.hpp"
#include "kernels.hpp"
#include "tiles.hpp"
#include "trace.hpp"

#include <type_traits>

namespace bnr {

namespace {

// V elements at p as floats (V = 1 or one 16-byte vector)
template <typename T, int V> struct LnVec;
template <> struct LnVec<float, 1> {
    typedef float raw;
    __device__ static __forceinline__ raw load(const float *p) { return *p; }
    __device__ static __forceinline__ void unpack(raw r, float *f) { f[0] = r; }
    __device__ static __forceinline__ void store(float *p, const float *f) { *p = f[0]; }
};
template <> struct LnVec<bf16_t, 1> {
    typedef bf16_t raw;
    __device__ static __forceinline__ raw load(const bf16_t *p) { return *p; }
    __device__ static __forceinline__ void unpack(raw r, float *f) { f[0] = bf2f(r); }
    __device__ static __forceinline__ void store(bf16_t *p, const float *f) { *p = f2bf(f[0]); }
};
template <typename T> struct LnVec16 {
    typedef vec16 raw;
    __device__ static __forceinline__ raw load(const T *p) { return ldg16(p); }
    __device__ static __forceinline__ void unpack(const raw &r, float *f) { Elem<T>::unpack(r, f); }
    __device__ static __forceinline__ void store(T *p, const float *f) { stg16(p, Elem<T>::pack(f)); }
};
template <> struct LnVec<float, 4> : LnVec16<float> {};
template <> struct LnVec<bf16_t, 8> : LnVec16<bf16_t> {};

// V per-channel parameters at p (16-byte aligned where V > 1), or the constant
// `other` where there are none
template <int V>
__device__ __forceinline__ void ln_param(const float *p, int c, float other, float *f)
{
    if constexpr (V == 1) {
        f[0] = p ? p[c] : other;
    } else {
        #pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 t = p ? *reinterpret_cast<const float4 *>(p + c + i) : make_float4(other, other, other, other);
            f[i] = t.x; f[i + 1] = t.y; f[i + 2] = t.z; f[i + 3] = t.w;
        }
    }
}

// N sums over the TPR threads of a row (every thread gets them).  Rows longer
// than a wave go through red[N][waves], which the next call may not reuse
// before a barrier: callers alternate between two or more areas.
template <int TPR, int N, typename A>
__device__ __forceinline__ void row_sums(A (&v)[N], A *red)
{
    constexpr int W = TPR < 64 ? TPR : 64;
    #pragma unroll
    for (int o = W / 2; o > 0; o >>= 1)
        #pragma unroll
        for (int k = 0; k < N; k++) v[k] += __shfl_xor(v[k], o, 64);
    if constexpr (TPR > 64) {
        constexpr int NW = TPR / 64;
        const int wave = threadIdx.x / 64, first = wave / NW * NW;      // waves of this row
        if (threadIdx.x % 64 == 0)
            #pragma unroll
            for (int k = 0; k < N; k++) red[wave * N + k] = v[k];
        __syncthreads();
        #pragma unroll
        for (int k = 0; k < N; k++) {
            A t = 0;
            #pragma unroll
            for (int q = 0; q < NW; q++) t += red[(first + q) * N + k];
            v[k] = t;
        }
    }
}

// U rows at a time per row group, GR row groups per workgroup; a workgroup takes
// row sets b, b + grid, ... (one, unless there are more than a grid holds).
template <typename T, int V, int TPR, int NV, int U, bool RES>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_ln_fwd(LnParams p)
{
    constexpr int WG = TPR > kThreads ? TPR : kThreads, GR = WG / TPR;
    typedef LnVec<T, V> L;
    __shared__ double red[WG / 64 * U];
    __shared__ float red_sq[WG / 64 * U];
    const int lane = threadIdx.x % TPR, grp = threadIdx.x / TPR;
    const int nvec = p.c / V;
    const T *x = (const T *)p.x, *res = (const T *)p.res;
    T *sum = (T *)p.sum, *y = (T *)p.y;
    for (int64_t base = (int64_t)blockIdx.x * (GR * U); base < p.m; base += (int64_t)gridDim.x * (GR * U)) {
        const int64_t row0 = base + grp;
        typename L::raw rx[U][NV], rr[U][NV];
        float f[U][NV][V], gam[NV][V], bet[NV][V], mean[U], sq[U];
        double acc[U];
        #pragma unroll
        for (int u = 0; u < U; u++) {
            // rows and vectors past the end read the last ones and are dropped
            const int64_t row = row0 + u * GR < p.m ? row0 + u * GR : p.m - 1;
            #pragma unroll
            for (int j = 0; j < NV; j++) {
                const int v = j * TPR + lane < nvec ? j * TPR + lane : nvec - 1;
                rx[u][j] = L::load(x + row * p.x_ldc + (int64_t)v * V);
                if (RES) rr[u][j] = L::load(res + row * p.res_ldc + (int64_t)v * V);
            }
        }
        #pragma unroll
        for (int j = 0; j < NV; j++) {
            const int v = j * TPR + lane < nvec ? j * TPR + lane : nvec - 1;
            ln_param<V>(p.gamma, v * V, 1.f, gam[j]);
            ln_param<V>(p.beta, v * V, 0.f, bet[j]);
        }
        #pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t row = row0 + u * GR;
            acc[u] = 0.0;
            #pragma unroll
            for (int j = 0; j < NV; j++) {
                const bool in = j * TPR + lane < nvec;
                L::unpack(rx[u][j], f[u][j]);
                if (RES) {
                    float r[V];
                    L::unpack(rr[u][j], r);
                    // what is normalised is the sum as it is stored
                    #pragma unroll
                    for (int i = 0; i < V; i++) f[u][j][i] = Elem<T>::round(f[u][j][i] + r[i]);
                    if (in && row < p.m) L::store(sum + row * p.sum_ldc + (int64_t)(j * TPR + lane) * V, f[u][j]);
                }
                if (in)
                    #pragma unroll
                    for (int i = 0; i < V; i++) acc[u] += (double)f[u][j][i];
            }
        }
        row_sums<TPR, U>(acc, red);
        #pragma unroll
        for (int u = 0; u < U; u++) {
            // acc / c: the product's remainder makes an exact quotient exact (NaN beside an infinity)
            double mu = acc[u] * p.inv_c;
            const double rem = fma(-mu, (double)p.c, acc[u]);
            if (rem == rem) mu = fma(rem, p.inv_c, mu);
            mean[u] = (float)mu;
            const float low = (float)(mu - (double)mean[u]);
            sq[u] = 0.f;
            #pragma unroll
            for (int j = 0; j < NV; j++)
                if (j * TPR + lane < nvec)
                    #pragma unroll
                    for (int i = 0; i < V; i++) {
                        f[u][j][i] = f[u][j][i] - mean[u] - low;
                        sq[u] += f[u][j][i] * f[u][j][i];
                    }
        }
        row_sums<TPR, U>(sq, red_sq);
        #pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t row = row0 + u * GR;
            if (row >= p.m) continue;
            const float rstd = 1.f / sqrtf(sq[u] * (float)p.inv_c + p.eps);
            if (lane == 0) {
                p.mean[row] = mean[u];
                p.rstd[row] = rstd;
            }
            #pragma unroll
            for (int j = 0; j < NV; j++) {
                const int v = j * TPR + lane;
                if (v >= nvec) continue;
                float o[V];
                #pragma unroll
                for (int i = 0; i < V; i++) o[i] = f[u][j][i] * rstd * gam[j][i] + bet[j][i];
                L::store(y + row * p.y_ldc + (int64_t)v * V, o);
            }
        }
    }
}

// Backward: workgroup b takes row sets b, b + grid, ...; each thread keeps the
// sums of dy and dy xhat of its own channels in registers over all its rows
// and the workgroup writes one partial row [2][c] at the end (float32 sums of
// at most kLnChain terms; k_ln_combine adds the partial rows in float64 in a
// fixed order).  The next row set is loaded before the current one reduces,
// and gamma stays in registers, except in the widest rows (512 threads, up to 32
// channels each), which do not hold both beside the sums (1024 threads of 16
// channels and 128 registers spilled more): those read gamma again, and load
// ahead only where a vector holds 8 values.  (Widths past 8192 in single elements
// still spill 130 to 163 registers, and 256 threads of 32 bf16 channels with dsum 15.)
template <typename T, int V, int TPR, int NV, int WG, bool RES>
__global__ __launch_bounds__(WG) void k_ln_bwd(LnParams p)
{
    constexpr int GR = WG / TPR;
    constexpr bool WIDE = TPR >= 512, AHEAD = !WIDE || V == 8, GAM = !WIDE;
    typedef LnVec<T, V> L;
    __shared__ float red[2][WG / 64 * 2];
    __shared__ float cols[GR > 1 ? 2 * WG * V : 1];
    const int lane = threadIdx.x % TPR, grp = threadIdx.x / TPR;
    const int nvec = p.c / V;
    const T *x = (const T *)p.x, *dy = (const T *)p.dy, *dsum = (const T *)p.res;
    T *dx = (T *)p.y;
    float gam[GAM ? NV : 1][V], sb[NV][V], sg[NV][V];
    int col[NV];
    #pragma unroll
    for (int j = 0; j < NV; j++) {
        const int v = j * TPR + lane;
        col[j] = v < nvec ? v * V : -1;
        if (GAM) ln_param<V>(p.gamma, (v < nvec ? v : nvec - 1) * V, 1.f, gam[GAM ? j : 0]);
        #pragma unroll
        for (int i = 0; i < V; i++) {
            sb[j][i] = 0.f;
            sg[j][i] = 0.f;
        }
    }
    const float inv_c = (float)p.inv_c;
    const int64_t step = (int64_t)gridDim.x * GR;
    const int64_t sets = (p.m + step - 1) / step;
    int64_t row = (int64_t)blockIdx.x * GR + grp;
    typename L::raw rx[NV], rd[NV], rs[RES ? NV : 1];
    float mean = 0.f, rstd = 0.f;
    auto load = [&](int64_t r) __attribute__((always_inline)) {
        if (r >= p.m) r = p.m - 1;                    // read and dropped
        mean = p.mean[r];
        rstd = p.rstd[r];
        #pragma unroll
        for (int j = 0; j < NV; j++) {
            const int64_t c = col[j] >= 0 ? col[j] : (nvec - 1) * V;
            rx[j] = L::load(x + r * p.x_ldc + c);
            rd[j] = L::load(dy + r * p.dy_ldc + c);
            if (RES) rs[j] = L::load(dsum + r * p.res_ldc + c);
        }
    };
    if (AHEAD) load(row);
    for (int64_t it = 0; it < sets; it++, row += step) {
        if (!AHEAD) load(row);
        float xh[NV][V], d[NV][V], s[2] = {0.f, 0.f};
        typename L::raw e[RES ? NV : 1];
        const float rs0 = rstd, mu0 = mean;
        const bool live = row < p.m;
        #pragma unroll
        for (int j = 0; j < NV; j++) {
            L::unpack(rx[j], xh[j]);
            L::unpack(rd[j], d[j]);
            if (RES) e[j] = rs[j];
        }
        if (AHEAD && it + 1 < sets) load(row + step);
        #pragma unroll
        for (int j = 0; j < NV; j++)
            if (col[j] >= 0) {
                float g[V];
                if (!GAM) ln_param<V>(p.gamma, col[j], 1.f, g);
                #pragma unroll
                for (int i = 0; i < V; i++) {
                    xh[j][i] = (xh[j][i] - mu0) * rs0;
                    if (live) {
                        sb[j][i] += d[j][i];
                        sg[j][i] += d[j][i] * xh[j][i];
                    }
                    d[j][i] *= GAM ? gam[GAM ? j : 0][i] : g[i];
                    s[0] += d[j][i];
                    s[1] += d[j][i] * xh[j][i];
                }
            }
        row_sums<TPR, 2>(s, red[it & 1]);
        if (live) {
            const float a = s[0] * inv_c, b = s[1] * inv_c;
            #pragma unroll
            for (int j = 0; j < NV; j++) {
                if (col[j] < 0) continue;
                float o[V], f[V];
                if (RES) L::unpack(e[j], f);
                #pragma unroll
                for (int i = 0; i < V; i++) {
                    o[i] = rs0 * (d[j][i] - a - xh[j][i] * b);
                    if (RES) o[i] += f[i];
                }
                L::store(dx + row * p.y_ldc + col[j], o);
            }
        }
    }
    if (!p.part) return;
    float *part = p.part + (int64_t)blockIdx.x * 2 * p.c;
    #pragma unroll
    for (int j = 0; j < NV; j++) {
        if constexpr (GR == 1) {
            if (col[j] >= 0)
                #pragma unroll
                for (int i = 0; i < V; i++) {
                    part[col[j] + i] = sb[j][i];
                    part[p.c + col[j] + i] = sg[j][i];
                }
        } else {
            // column sums over the row groups, in a fixed order
            constexpr int CW = TPR * V;
            if (j) __syncthreads();
            #pragma unroll
            for (int i = 0; i < V; i++) {
                cols[grp * CW + lane * V + i] = sb[j][i];
                cols[WG * V + grp * CW + lane * V + i] = sg[j][i];
            }
            __syncthreads();
            for (int k = threadIdx.x; k < 2 * CW; k += WG) {
                const int half = k >= CW, q = k - half * CW, c = j * CW + q;
                if (c < p.c) {
                    float t = 0.f;
                    #pragma unroll
                    for (int g = 0; g < GR; g++) t += cols[half * WG * V + g * CW + q];
                    part[half * p.c + c] = t;
                }
            }
        }
    }
}

// dbeta and dgamma (either may be NULL) from the partial rows [R][2 c], added in
// float64 in a fixed order: a workgroup takes COLS of the 2 c columns with
// 1024 / COLS row groups, eight rows in flight a thread, then adds the groups.
// 64 columns are 256-byte reads of long rows; 16 columns keep enough workgroups
// where rows are short.
template <int COLS>
__global__ __launch_bounds__(1024) void k_ln_combine(const float *__restrict__ part, int64_t R, int c, float *dbeta,
                                                         float *dgamma)
{
    constexpr int GROUPS = 1024 / COLS, U = 8;
    __shared__ double red[GROUPS][COLS + 1];
    const int tx = threadIdx.x % COLS, ty = threadIdx.x / COLS;
    const int64_t width = 2 * (int64_t)c, k = (int64_t)blockIdx.x * COLS + tx;
    const float *src = part + (k < width ? k : width - 1);
    double acc = 0.0;
    for (int64_t r = ty; r < R; r += U * GROUPS) {
        float v[U];
        #pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t rr = r + u * GROUPS;           // rows past the last are read again and left out
            v[u] = src[(rr < R ? rr : R - 1) * width];
        }
        #pragma unroll
        for (int u = 0; u < U; u++) acc += r + u * GROUPS < R ? (double)v[u] : 0.0;
    }
    red[ty][tx] = acc;
    __syncthreads();
    if (ty == 0 && k < width) {
        double t = 0.0;
        #pragma unroll
        for (int g = 0; g < GROUPS; g++) t += red[g][tx];
        float *out = k < c ? dbeta : dgamma;
        if (out) out[k < c ? k : k - c] = (float)t;
    }
}

// The row layout of a call: threads per row, loads per thread, and in the
// backward pass the workgroup.  As few threads as hold a row in a few loads each:
// they reduce in fewer steps, and no lane idles (2^25 values, forward / backward in
// us: 64 bf16 channels by 8 threads 28 / 41, by 32 threads 71 / 90; 1024 by 64
// threads 28 / 43, by 256 45 / 54; 4096 by 256 28 / 49, by 1024 (512) 106 / 74; 201
// float32 channels by 64 62 / 77, by 256 335 / 213; 1001 by 256 81 / 84, by 1024
// (512) 409 / 249).
struct LnPlan { bool vec; int tpr, nv, wg; };

LnPlan ln_plan(int dtype, int c, bool vec)
{
    if (!vec) {
        if (c <= 256) return {false, 64, 4, 256};
        if (c <= 2048) return {false, 256, 8, 256};
        if (c <= 8192) return {false, 1024, 8, 1024};
        return {false, 1024, 16, 1024};
    }
    const int n = c / stats_vec(dtype);
    if (n <= 8) return {true, 8, 1, 256};
    if (n <= 16) return {true, 16, 1, 256};
    if (n <= 32) return {true, 32, 1, 256};
    if (n <= 64) return {true, 64, 1, 256};
    if (n <= 128) return {true, 64, 2, 256};
    if (n <= 256) return {true, 256, 1, 512};
    if (n <= 512) return {true, 256, 2, 512};
    if (n <= 1024) return {true, 256, 4, 512};
    return {true, 1024, n <= 2048 ? 2 : 4, 1024};
}

// The backward's: the rows of 1024 threads take 512 and twice the loads.
LnPlan ln_bwd_plan(int dtype, int c, bool vec)
{
    LnPlan q = ln_plan(dtype, c, vec);
    return q.tpr == 1024 ? LnPlan{q.vec, 512, 2 * q.nv, 512} : q;
}

template <bool BWD, typename F>
hipError_t ln_dispatch(const LnPlan &q, int dtype, F &&go)
{
    auto with = [&](auto tag, auto v, auto tpr, auto nv, auto wg) { return go(tag, v, tpr, nv, wg); };
#define LN_I(N) std::integral_constant<int, N>{}
#define LN_CASE(T, V, TPR, NV, WG) \
    if (q.tpr == TPR && q.nv == NV) return with((T *)nullptr, LN_I(V), LN_I(TPR), LN_I(NV), LN_I(WG))
#define LN_WIDE(T, V, NV) \
    if constexpr (BWD) { LN_CASE(T, V, 512, 2 * NV, 512); } else { LN_CASE(T, V, 1024, NV, 1024); }
#define LN_VECTORS(T, V) \
    LN_CASE(T, V, 8, 1, 256);   LN_CASE(T, V, 16, 1, 256);  LN_CASE(T, V, 32, 1, 256);  LN_CASE(T, V, 64, 1, 256); \
    LN_CASE(T, V, 64, 2, 256);  LN_CASE(T, V, 256, 1, 512); LN_CASE(T, V, 256, 2, 512); LN_CASE(T, V, 256, 4, 512); \
    LN_WIDE(T, V, 2)
#define LN_SCALARS(T) \
    LN_CASE(T, 1, 64, 4, 256); LN_CASE(T, 1, 256, 8, 256); LN_WIDE(T, 1, 8); LN_WIDE(T, 1, 16)
    if (dtype == DT_BF16) {
        if (q.vec) { LN_VECTORS(bf16_t, 8); }
        else { LN_SCALARS(bf16_t); }
    } else {
        if (q.vec) { LN_VECTORS(float, 4); LN_WIDE(float, 4, 4); }
        else { LN_SCALARS(float); }
    }
#undef LN_SCALARS
#undef LN_VECTORS
#undef LN_WIDE
#undef LN_CASE
#undef LN_I
    return hipErrorInvalidValue;
}

}  // namespace

// Partial rows (= workgroups) of the backward: enough workgroups to fill the
// chip, few enough that writing and adding the partial rows stays small next
// to the data (c = 4096: 512 rows are 16 MiB), and so many that no thread adds
// more than kLnChain rows in float32 (the partial rows are then at most 1/64 of
// the data).
int64_t ln_bwd_groups(int dtype, int64_t m, int c, bool vec)
{
    const LnPlan q = ln_bwd_plan(dtype, c, vec);
    const int64_t sets = ceil_div(m, q.wg / q.tpr);
    const int64_t most = q.wg == 256 ? 1024 : (q.tpr == 256 ? 512 : 256);
    const int64_t enough = ceil_div(sets, kLnChain) > most ? ceil_div(sets, kLnChain) : most;
    const int64_t groups = sets < enough ? sets : enough;
    return groups < kLnMaxGrid ? groups : kLnMaxGrid;
}

hipError_t launch_ln_fwd(int dtype, const LnParams &p, bool vec, hipStream_t s)
{
    const LnPlan q = ln_plan(dtype, p.c, vec);
    const double n = (double)p.m * p.c * (dtype == DT_BF16 ? 2 : 4);
    TraceScope tr(KC_SWEEP, KID_LAYERNORM, s, (p.res ? 4.0 : 2.0) * n + 8.0 * p.m + 8.0 * p.c, 0.0);
    return ln_dispatch<false>(q, dtype, [&](auto *tag, auto v, auto tpr, auto nv, auto) {
        using T = std::remove_pointer_t<decltype(tag)>;
        constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, V = decltype(v)::value;
        constexpr int WG = TPR > kThreads ? TPR : kThreads, U = NV == 1 && TPR <= 64 ? 2 : 1;
        const int64_t sets = ceil_div(p.m, WG / TPR * U);
        const dim3 grid((unsigned)(sets < kLnMaxGrid ? sets : kLnMaxGrid));
        if (p.res) hipLaunchKernelGGL((k_ln_fwd<T, V, TPR, NV, U, true>), grid, dim3(WG), 0, s, p);
        else hipLaunchKernelGGL((k_ln_fwd<T, V, TPR, NV, U, false>), grid, dim3(WG), 0, s, p);
        return hipGetLastError();
    });
}

hipError_t launch_ln_combine(const float *part, int64_t R, int c, float *dbeta, float *dgamma, hipStream_t s)
{
    TraceScope tr(KC_SMALL, KID_COMBINE, s, (double)R * 2 * c * 4 + 8.0 * c, 0.0);
    const int64_t width = 2 * (int64_t)c;
    if (c > 1024) hipLaunchKernelGGL(k_ln_combine<64>, dim3((unsigned)ceil_div(width, 64)), dim3(1024), 0, s, part, R, c,
                                     dbeta, dgamma);
    else hipLaunchKernelGGL(k_ln_combine<16>, dim3((unsigned)ceil_div(width, 16)), dim3(1024), 0, s, part, R, c,
                            dbeta, dgamma);
    return hipGetLastError();
}

hipError_t launch_ln_bwd(int dtype, const LnParams &p, bool vec, hipStream_t s)
{
    const LnPlan q = ln_bwd_plan(dtype, p.c, vec);
    const double n = (double)p.m * p.c * (dtype == DT_BF16 ? 2 : 4);
    const int64_t R = ln_bwd_groups(dtype, p.m, p.c, vec);
    TraceScope tr(KC_SWEEP, KID_LAYERNORM, s, (p.res ? 4.0 : 3.0) * n + 8.0 * p.m + 4.0 * p.c + 8.0 * R * p.c, 0.0);
    return ln_dispatch<true>(q, dtype, [&](auto *tag, auto v, auto tpr, auto nv, auto wg) {
        using T = std::remove_pointer_t<decltype(tag)>;
        constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, V = decltype(v)::value;
        constexpr int WG = decltype(wg)::value;
        if (p.res) hipLaunchKernelGGL((k_ln_bwd<T, V, TPR, NV, WG, true>), dim3((unsigned)R), dim3(WG), 0, s, p);
        else hipLaunchKernelGGL((k_ln_bwd<T, V, TPR, NV, WG, false>), dim3((unsigned)R), dim3(WG), 0, s, p);
        return hipGetLastError();
    });
}

}  // namespace bnr
