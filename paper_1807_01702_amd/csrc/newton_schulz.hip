// newton_schulz.hip -- orthogonalisation of a list of matrices by Newton-Schulz
// products, alone or as the optimizer step built on it.
//
//   u = the matrix itself, or the momentum update of its gradient
//   X = u / (||u||_F + eps), the shorter side first: X is [p][q], p <= q
//   `steps` times:  G = X X^T,  R = a I + b G + c G G,  X <- R X
//   out = X, or  w <- w (1 - lr decay) - lr scale X
//
// Precision.  The products run on the fp16 matrix cores at float32 accuracy:
// every operand v is held as a pair hi = fp16(S v), lo = fp16(S v - hi), 22
// bits together, and a product of two operands is three matrix products,
// hi hi' + hi lo' + lo hi', accumulated in float32 (the dropped lo lo' is below
// 2^-22 of the term).  The factor S = 2^12 keeps both parts inside fp16's range:
// the spectral norm of X, G and R stays below 16 (the caller's coefficients are
// checked for that), so no |S v| reaches 65504, and what is lost below fp16's
// smallest step is 2^-37 of the norm of X.  Three fp16 products run at 2.6 times
// the rate of one float32 matrix product on this chip and carry the same error.
//
// Layout.  A pair matrix with K columns is [rows][K / 32][hi 32 | lo 32]: the 32
// columns of one k step are one 128-byte line, so a tile row is one line per
// step.  Every product is of the form C[i][j] = sum_k P[i][k] Q[j][k] with both
// operands contiguous along k: G = X X^T as it is, G G because G is symmetric,
// and R X from X's transpose, which each R X writes beside X for the next step.
// Rows and columns are padded to whole tiles with zeros, which every product
// keeps, so the main loops have no bounds to check.
//
// A list runs through every stage in one launch: a stage's workgroups find
// their matrix by the running count of tiles.
#include "common.hpp"
#include "kernels.hpp"
#include "tiles.hpp"
#include "trace.hpp"

namespace bnr {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t h16;                                // fp16 storage word

constexpr float kS = 4096.f, kInvS = 1.f / 4096.f;   // see the precision note
constexpr int kTile = kNsTile;

// one matrix of the list on the device: the caller's arguments and its place in the workspace
struct NsDev {
    NsIn in;
    int p, q, P, Q, flip;          // short and long side, padded; flip: X is the transpose of the caller's matrix
    int parts;                     // partial sums of squares
    double *sq;                    // [parts]
    h16 *x, *xt[2], *g, *r;        // pair matrices [P][Q], [Q][P], [P][P]
};
// the device table: the matrices and the running counts of work items per stage
struct NsTable { NsDev *items; int *pre[4]; };
enum { PRE_SQ = 0, PRE_PREP = 1, PRE_GRAM = 2, PRE_APPLY = 3 };

// Sizes of one matrix, the same on the host (workspace, grids) and on the device.
struct NsSize {
    int p, q, P, Q, flip, parts;
    int64_t work[4];               // work items per stage
    int64_t bytes;                 // workspace
};
__host__ __device__ inline NsSize ns_size(int rows, int cols)
{
    NsSize z;
    z.flip = rows > cols;
    z.p = z.flip ? cols : rows;
    z.q = z.flip ? rows : cols;
    z.P = (z.p + kTile - 1) / kTile * kTile;
    z.Q = (z.q + kTile - 1) / kTile * kTile;
    // 16384 values a partial sum, whole rows, at most 256 partial sums
    int64_t n = ((int64_t)rows * cols + 16383) / 16384;
    if (n > 256) n = 256;
    if (n > rows) n = rows;
    const int rp = (int)((rows + n - 1) / n);
    z.parts = (rows + rp - 1) / rp;
    const int64_t tp = z.P / kTile, tq = z.Q / kTile;
    z.work[PRE_SQ] = z.parts;
    z.work[PRE_PREP] = (int64_t)(z.P / 64) * (z.Q / 64);
    z.work[PRE_GRAM] = tp * (tp + 1) / 2;
    z.work[PRE_APPLY] = tp * tq;
    z.bytes = 256 * 8 + (int64_t)z.P * z.Q * 4 * 3 + (int64_t)z.P * z.P * 4 * 2;
    return z;
}

struct NsChunk {                   // by value: the next matrices of the list
    int first, count;
    int64_t at;                    // workspace offset and running counts in front of them
    int work[4];
    NsIn in[kNsChunk];
};

__global__ __launch_bounds__(64) void k_ns_table(NsChunk c, NsTable t, char *base)
{
    const int i = threadIdx.x;
    if (i >= c.count) return;
    int64_t at = c.at;
    int work[4] = {c.work[0], c.work[1], c.work[2], c.work[3]};
    for (int j = 0; j < i; j++) {
        const NsSize z = ns_size(c.in[j].rows, c.in[j].cols);
        at += z.bytes;
        for (int k = 0; k < 4; k++) work[k] += (int)z.work[k];
    }
    const NsSize z = ns_size(c.in[i].rows, c.in[i].cols);
    NsDev d;
    d.in = c.in[i];
    d.p = z.p; d.q = z.q; d.P = z.P; d.Q = z.Q; d.flip = z.flip; d.parts = z.parts;
    char *b = base + at;
    const int64_t pq = (int64_t)z.P * z.Q * 4, pp = (int64_t)z.P * z.P * 4;
    d.sq = (double *)b;
    b += 256 * 8;
    d.x = (h16 *)b;
    d.xt[0] = (h16 *)(b + pq);
    d.xt[1] = (h16 *)(b + 2 * pq);
    d.g = (h16 *)(b + 3 * pq);
    d.r = (h16 *)(b + 3 * pq + pp);
    t.items[c.first + i] = d;
    for (int k = 0; k < 4; k++) t.pre[k][c.first + i] = work[k];
}

// The matrix a work item belongs to: the last one whose running count is not
// past it (the counts ascend; the wave compares 64 of them at a time).
__device__ __forceinline__ int ns_find(const int *pre, int count, int item)
{
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int base = 0; base < count; base += 64) {
        const bool in = base + lane < count && pre[base + lane] <= item;
        const unsigned long long m = __ballot(in);
        n += __popcll(m);
        if (m != ~0ull) break;
    }
    return __builtin_amdgcn_readfirstlane(n - 1);
}

template <typename T> __device__ __forceinline__ float ns_load(const void *p, int64_t i)
{
    if constexpr (sizeof(T) == 4) return ((const float *)p)[i];
    else return bf2f(((const bf16_t *)p)[i]);
}

// u of element i of a gradient row: the gradient itself, or what the momentum step makes of it
__device__ __forceinline__ float ns_u(float g, float buf, const NsStep &s)
{
    return !s.update ? g : (s.nesterov ? __builtin_fmaf(s.momentum, buf, g) : buf);
}

// Stage 1: the momentum (buf <- momentum buf + g) and the partial sums of u^2
// (in float64: the squares of float32 values neither overflow nor vanish there).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_ns_squares(NsTable t, int count, NsStep s)
{
    __shared__ double red[kThreads / 64];
    const int it = ns_find(t.pre[PRE_SQ], count, blockIdx.x);
    const NsDev &d = t.items[it];
    const int part = blockIdx.x - t.pre[PRE_SQ][it];
    const int rows = d.in.rows, cols = d.in.cols, rp = (rows + d.parts - 1) / d.parts;
    const int r0 = part * rp, r1 = min(rows, r0 + rp);
    double acc = 0.0;
    const int64_t n = (int64_t)(r1 - r0) * cols;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
        const int64_t r = r0 + i / cols;
        const int c = (int)(i % cols);
        const float g = ns_load<T>(d.in.src, r * d.in.ld_src + c);
        float b = 0.f;
        if (s.update) {
            float *pb = d.in.buf + r * d.in.ld_buf + c;
            b = __builtin_fmaf(s.momentum, *pb, g);
            *pb = b;
        }
        const double u = (double)ns_u(g, b, s);
        acc += u * u;
    }
    for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o, 64);
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = acc;
    __syncthreads();
    if (threadIdx.x == 0) d.sq[part] = red[0] + red[1] + red[2] + red[3];
}

// The pair of a value already scaled by S.  The empty asm makes v one float32
// value: without it the compiler fuses the product that formed v into one of the
// two roundings to fp16 (v_fma_mixlo_f16), and where v lies half way between two
// fp16 values the hi that is stored and the hi that lo is relative to differ.
__device__ __forceinline__ void ns_pair(float v, h16 &hi, h16 &lo)
{
    asm("" : "+v"(v));
    const _Float16 h = (_Float16)v;
    const _Float16 l = (_Float16)(v - (float)h);
    hi = __builtin_bit_cast(h16, h);
    lo = __builtin_bit_cast(h16, l);
}
// element offset of (row, k) of a pair matrix with K columns: hi there, lo 32 further on
__device__ __forceinline__ int64_t ns_at(int64_t row, int k, int K)
{
    return row * 2 * K + (k >> 5) * 64 + (k & 31);
}

// Stage 2: X and its transpose as pairs, from u / (||u||_F + eps); 64 x 64
// values a workgroup, turned through LDS; zeros past the matrix.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_ns_prepare(NsTable t, int count, NsStep s)
{
    __shared__ float tile[64][65];
    __shared__ double red[kThreads / 64];
    const int it = ns_find(t.pre[PRE_PREP], count, blockIdx.x);
    const NsDev &d = t.items[it];
    const int w = blockIdx.x - t.pre[PRE_PREP][it];
    // blocks over the caller's orientation [rows][cols], padded
    const int RP = d.flip ? d.Q : d.P, CP = d.flip ? d.P : d.Q;
    const int rb = w / (CP / 64) * 64, cb = w % (CP / 64) * 64;
    const int tid = threadIdx.x;
    double acc = tid < d.parts ? d.sq[tid] : 0.0;
    for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o, 64);
    if (tid % 64 == 0) red[tid / 64] = acc;
    for (int e = tid; e < 64 * 64; e += kThreads) {
        const int r = rb + e / 64, c = cb + e % 64;
        float u = 0.f;
        if (r < d.in.rows && c < d.in.cols) {
            const float g = ns_load<T>(d.in.src, (int64_t)r * d.in.ld_src + c);
            u = ns_u(g, s.update ? d.in.buf[(int64_t)r * d.in.ld_buf + c] : 0.f, s);
        }
        tile[e / 64][e % 64] = u;
    }
    __syncthreads();
    const double norm = sqrt(((red[0] + red[1]) + red[2]) + red[3]);
    const float scale = (float)((double)kS / (norm + (double)s.eps));
    // as it is: [RP rows][K = CP]; turned: [CP rows][K = RP]
    h16 *straight = d.flip ? d.xt[0] : d.x, *turned = d.flip ? d.x : d.xt[0];
    for (int v = tid; v < 64 * 8; v += kThreads) {
        const int a = v / 8, k8 = v % 8 * 8;
        __align__(16) h16 hi[8], lo[8];
        for (int i = 0; i < 8; i++) ns_pair(tile[a][k8 + i] * scale, hi[i], lo[i]);
        h16 *o = straight + ns_at(rb + a, cb + k8, CP);
        *reinterpret_cast<vec16 *>(o) = *reinterpret_cast<vec16 *>(hi);
        *reinterpret_cast<vec16 *>(o + 32) = *reinterpret_cast<vec16 *>(lo);
        for (int i = 0; i < 8; i++) ns_pair(tile[k8 + i][a] * scale, hi[i], lo[i]);
        o = turned + ns_at(cb + a, rb + k8, RP);
        *reinterpret_cast<vec16 *>(o) = *reinterpret_cast<vec16 *>(hi);
        *reinterpret_cast<vec16 *>(o + 32) = *reinterpret_cast<vec16 *>(lo);
    }
}

// One product stage over the whole list.
//   NS_GRAM    G = X X^T            (lower-triangle tiles, mirrored)
//   NS_SQUARE  R = a I + b G + c G G (likewise)
//   NS_APPLY   X, X^T <- R X
//   NS_LAST    R X into the caller's matrix
enum { NS_GRAM = 0, NS_SQUARE = 1, NS_APPLY = 2, NS_LAST = 3 };

// Workgroup: BT x BT outputs by WM x WN waves.  Two LDS stages of 2 BT rows of
// 128 bytes (one k step of both operands); the 16-byte chunks of a row are
// stored in the order chunk ^ (row % 8), so the 16 rows of a fragment read lie
// in different banks.  The next step's lines are loaded straight into LDS while
// the current step multiplies.
template <int BT, int WM, int WN, int MODE, typename W>
__global__ __launch_bounds__(WM * WN * 64) void k_ns_product(NsTable t, int count, NsStep s, int turn)
{
    constexpr int NT = WM * WN * 64, TM = BT / WM, TN = BT / WN, MI = TM / 16, NI = TN / 16;
    constexpr int kRow = 128, kStage = 2 * BT * kRow, kLoads = kStage / (NT * 16);
    constexpr bool SYM = MODE == NS_GRAM || MODE == NS_SQUARE;
    __shared__ __align__(16) unsigned char lds0[kStage], lds1[kStage];
    const int work = xcd_remap(blockIdx.x, gridDim.x);
    const int *pre = t.pre[SYM ? PRE_GRAM : PRE_APPLY];
    const int it = ns_find(pre, count, work);
    const NsDev &d = t.items[it];
    const int w = work - pre[it];
    const int P = d.P, Q = d.Q;
    int ti, tj;
    if (SYM) {                                   // row i of the triangle starts at i (i + 1) / 2
        ti = (int)((sqrtf(8.f * (float)w + 1.f) - 1.f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= w) ti++;
        while (ti * (ti + 1) / 2 > w) ti--;
        tj = w - ti * (ti + 1) / 2;
    } else {
        ti = w % (P / BT);
        tj = w / (P / BT);
    }
    const int K = MODE == NS_GRAM ? Q : P;
    const h16 *pa = MODE == NS_GRAM ? d.x : (MODE == NS_SQUARE ? d.g : d.r);
    const h16 *pb = MODE == NS_GRAM ? d.x : (MODE == NS_SQUARE ? d.g : d.xt[turn]);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // this thread's chunk of load l: row (l NT + tid) / 8 of the stage, position tid % 8
    const int lrow = tid / 8, lchunk = (tid % 8) ^ (lrow % 8);
    const char *src[kLoads];
    #pragma unroll
    for (int l = 0; l < kLoads; l++) {
        const int row = l * (NT / 8) + lrow;
        const h16 *base = row < BT ? pa + (int64_t)(ti * BT + row) * 2 * K : pb + (int64_t)(tj * BT + row - BT) * 2 * K;
        src[l] = (const char *)base + lchunk * 16;
    }
    auto load = [&](unsigned char *stage, int step) __attribute__((always_inline)) {
        #pragma unroll
        for (int l = 0; l < kLoads; l++)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(src[l] + (int64_t)step * kRow),
                                             (__attribute__((address_space(3))) uint32_t *)(stage + (l * NT + wave * 64) * 16),
                                             16, 0, 0);
    };
    const int wm = wave / WN, wn = wave % WN;
    const int fr = lane % 16, fc = lane / 16;    // fragment row and k chunk of this lane
    f32x4 acc[MI][NI];
    #pragma unroll
    for (int i = 0; i < MI; i++)
        #pragma unroll
        for (int j = 0; j < NI; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto frag = [&](const unsigned char *stage, int row, int part) __attribute__((always_inline)) {
        const int r = row + fr;
        return *reinterpret_cast<const f16x8 *>(stage + r * kRow + ((part * 4 + fc) ^ (r % 8)) * 16);
    };
    auto multiply = [&](const unsigned char *stage) __attribute__((always_inline)) {
        f16x8 ah[MI], al[MI], bh[NI], bl[NI];
        #pragma unroll
        for (int i = 0; i < MI; i++) {
            ah[i] = frag(stage, wm * TM + i * 16, 0);
            al[i] = frag(stage, wm * TM + i * 16, 1);
        }
        #pragma unroll
        for (int j = 0; j < NI; j++) {
            bh[j] = frag(stage, BT + wn * TN + j * 16, 0);
            bl[j] = frag(stage, BT + wn * TN + j * 16, 1);
        }
        #pragma unroll
        for (int i = 0; i < MI; i++)
            #pragma unroll
            for (int j = 0; j < NI; j++) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bl[j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[i], bh[j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bh[j], acc[i][j], 0, 0, 0);
            }
    };
    const int steps = K / 32;                    // even: K is a multiple of 64
    load(lds0, 0);
    __syncthreads();
    for (int k = 0; k < steps; k += 2) {
        load(lds1, k + 1);
        multiply(lds0);
        __syncthreads();
        if (k + 2 < steps) load(lds0, k + 2);
        multiply(lds1);
        __syncthreads();
    }

    // lane l holds rows 4 (l / 16) .. + 3 of column l % 16 of each 16 x 16 block
    const int i0 = ti * BT + wm * TM + 4 * fc, j0 = tj * BT + wn * TN + fr;
    #pragma unroll
    for (int mi = 0; mi < MI; mi++)
        #pragma unroll
        for (int nj = 0; nj < NI; nj++) {
            const int i = i0 + mi * 16, j = j0 + nj * 16;
            float v[4];
            #pragma unroll
            for (int e = 0; e < 4; e++) v[e] = acc[mi][nj][e] * kInvS;        // S times the product
            if constexpr (MODE == NS_LAST) {
                if (j >= d.q) continue;
                const float lr = s.update ? (s.lr_dev ? *s.lr_dev : s.lr) : 0.f;
                #pragma unroll
                for (int e = 0; e < 4; e++) {
                    if (i + e >= d.p) continue;
                    const float o = v[e] * kInvS;
                    const int64_t r = d.flip ? j : i + e, c = d.flip ? i + e : j;
                    W *dst = (W *)d.in.dst + r * d.in.ld_dst + c;
                    float res = o;
                    if (s.update) {
                        const float old = ns_load<W>(dst, 0);
                        res = __builtin_fmaf(-lr * d.in.scale, o, old * (1.f - lr * s.decay));
                        if (d.in.copy) d.in.copy[r * d.in.ld_copy + c] = f2bf(res);
                    }
                    if constexpr (sizeof(W) == 4) *dst = res;
                    else *dst = f2bf(res);
                }
            } else {
                // straight: [i][j] with j along k; turned: [j][i]
                h16 *st = MODE == NS_GRAM ? d.g : (MODE == NS_SQUARE ? d.r : d.x);
                h16 *tu = MODE == NS_GRAM ? d.g : (MODE == NS_SQUARE ? d.r : d.xt[turn ^ 1]);
                const int ks = SYM ? P : Q;
                if constexpr (MODE == NS_SQUARE) {
                    #pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const h16 *g = d.g + ns_at(i + e, j, P);
                        const float gv = (float)__builtin_bit_cast(_Float16, g[0]) + (float)__builtin_bit_cast(_Float16, g[32]);
                        v[e] = __builtin_fmaf(s.c, v[e], s.b * gv) + (i + e == j ? s.a * kS : 0.f);
                    }
                }
                h16 hi[4], lo[4];
                #pragma unroll
                for (int e = 0; e < 4; e++) ns_pair(v[e], hi[e], lo[e]);
                #pragma unroll
                for (int e = 0; e < 4; e++) {
                    h16 *o = st + ns_at(i + e, j, ks);
                    o[0] = hi[e];
                    o[32] = lo[e];
                }
                if (!SYM || ti != tj) {
                    h16 *o = tu + ns_at(j, i, P);
                    *reinterpret_cast<uint2 *>(o) = make_uint2(hi[0] | (uint32_t)hi[1] << 16, hi[2] | (uint32_t)hi[3] << 16);
                    *reinterpret_cast<uint2 *>(o + 32) = make_uint2(lo[0] | (uint32_t)lo[1] << 16, lo[2] | (uint32_t)lo[3] << 16);
                }
            }
        }
}

size_t table_bytes(int count)
{
    const size_t a = (size_t)count * sizeof(NsDev), b = (size_t)count * 4 * sizeof(int);
    return (a + b + 255) / 256 * 256;
}

}  // namespace

void ns_plan_add(NsPlan &p, int rows, int cols)
{
    const NsSize z = ns_size(rows, cols);
    p.count++;
    p.bytes += z.bytes;
    for (int k = 0; k < 4; k++) p.work[k] += z.work[k];
    p.flops += (double)z.p * (z.p + 1) * z.q + (double)z.p * z.p * (z.p + 1) + 2.0 * z.p * z.p * z.q;
    p.values += (double)rows * cols;
}

size_t ns_plan_bytes(const NsPlan &p) { return table_bytes(p.count) + (size_t)p.bytes; }

namespace {

NsTable ns_table(void *ws, int count)
{
    NsTable t;
    t.items = (NsDev *)ws;
    int *pre = (int *)((char *)ws + (size_t)count * sizeof(NsDev));
    for (int k = 0; k < 4; k++) t.pre[k] = pre + (size_t)k * count;
    return t;
}

template <int MODE, typename W>
hipError_t ns_product(const NsPlan &p, const NsTable &t, const NsStep &s, int turn, double flops, hipStream_t st)
{
    const int64_t work = p.work[MODE == NS_GRAM || MODE == NS_SQUARE ? PRE_GRAM : PRE_APPLY];
    TraceScope tr(KC_CONV, KID_ORTHO, st, 0.0, flops);
    hipLaunchKernelGGL((k_ns_product<kTile, 2, 2, MODE, W>), dim3((unsigned)work), dim3(256), 0, st, t, p.count, s, turn);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ns(const NsPlan &p, NsFill fill, const void *arg, const NsStep &s, int src_dtype, int dst_dtype,
                     void *ws, hipStream_t st)
{
    const NsTable t = ns_table(ws, p.count);
    NsChunk c;
    c.at = (int64_t)table_bytes(p.count);
    for (int k = 0; k < 4; k++) c.work[k] = 0;
    for (c.first = 0; c.first < p.count; c.first += kNsChunk) {
        c.count = p.count - c.first < kNsChunk ? p.count - c.first : kNsChunk;
        for (int i = 0; i < c.count; i++) c.in[i] = fill(arg, c.first + i);
        TraceScope tr(KC_SMALL, KID_ORTHO, st, (double)c.count * sizeof(NsDev), 0.0);
        hipLaunchKernelGGL(k_ns_table, dim3(1), dim3(64), 0, st, c, t, (char *)ws);
        if (hipError_t e = hipGetLastError()) return e;
        for (int i = 0; i < c.count; i++) {
            const NsSize z = ns_size(c.in[i].rows, c.in[i].cols);
            c.at += z.bytes;
            for (int k = 0; k < 4; k++) c.work[k] += (int)z.work[k];
        }
    }
    const double es = src_dtype == DT_BF16 ? 2.0 : 4.0;
    {
        TraceScope tr(KC_SWEEP, KID_ORTHO, st, p.values * (es + (s.update ? 8.0 : 0.0)), 0.0);
        auto kern = src_dtype == DT_BF16 ? k_ns_squares<bf16_t> : k_ns_squares<float>;
        hipLaunchKernelGGL(kern, dim3((unsigned)p.work[PRE_SQ]), dim3(kThreads), 0, st, t, p.count, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    {
        TraceScope tr(KC_SWEEP, KID_ORTHO, st, p.values * (es + (s.update ? 4.0 : 0.0) + 8.0), 0.0);
        auto kern = src_dtype == DT_BF16 ? k_ns_prepare<bf16_t> : k_ns_prepare<float>;
        hipLaunchKernelGGL(kern, dim3((unsigned)p.work[PRE_PREP]), dim3(kThreads), 0, st, t, p.count, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    for (int k = 0, turn = 0; k < s.steps; k++, turn ^= 1) {
        hipError_t e = ns_product<NS_GRAM, float>(p, t, s, turn, 0.0, st);
        if (e == hipSuccess) e = ns_product<NS_SQUARE, float>(p, t, s, turn, 0.0, st);
        if (e == hipSuccess) {
            if (k + 1 < s.steps) e = ns_product<NS_APPLY, float>(p, t, s, turn, p.flops, st);
            else if (dst_dtype == DT_BF16) e = ns_product<NS_LAST, bf16_t>(p, t, s, turn, p.flops, st);
            else e = ns_product<NS_LAST, float>(p, t, s, turn, p.flops, st);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace bnr
