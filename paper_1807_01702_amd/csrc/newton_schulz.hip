// newton_schulz.hip -- orthogonalisation of a list of matrices by Newton-Schulz
// products, alone or as the optimizer step built on it.
//
//   u = the matrix itself, or the momentum update of its gradient
//   X = u / (||u||_F + eps), the shorter side first: X is [p][q], p <= q
//   `steps` times:  G = X X^T,  R = a I + b G + c G G,  X <- R X
//   out = X, or  w <- w (1 - lr decay) - lr scale X
//
// Precision.  The products run on the fp16 matrix cores: every operand v is held as
// a pair hi = fp16(S v), lo = fp16(S v - hi), off by at most 2^-23 of v (float32:
// 2^-24), and a product of two operands is three matrix products,
// hi hi' + hi lo' + lo hi', accumulated in float32; the dropped lo lo', below 2^-22
// of the term, is added where sums are short (nw_four, nw_third).  The factor S = 2^12 keeps
// both parts inside fp16's range: the spectral norm of X, G and R stays below 16 (the
// caller's coefficients are checked for that), so no |S v| reaches 65504, and what is
// lost below fp16's smallest step is 2^-37, where X's norm is at most 1.  Against
// float64 the results are 0.2 to 1.2 times as far off as those of float32 products,
// for noise, strong directions, rows of different scale and decaying spectra of
// 8 x 8 to 4096 x 4096.  A library's large product reaches 1330 TFLOP/s in fp16 and
// 150 in float32 on this chip: three fp16 products run at 2.9 times float32's rate.
//
// Measured: 4096 x 4096, five steps, 3.5 ms = 393 of the 443 TFLOP/s that pairs can
// reach (the matrix cores bound it); twelve bf16 weights of 1024 x 4096 2.9 ms; all
// 119 filters of DenseNet-121 412 us and 128 x 128 56 us (dependent short stages).
//
// Layout.  A pair matrix lies in the order of the fragments that the matrix
// instructions take (ns_at): a fragment is one KiB, whether it goes to registers
// or, straight from memory, to LDS, and an LDS read of it has no bank conflicts.  (A CU
// reads whole KiB at 105 to 124 GB/s from its L2, 16 rows of 64 bytes at 50.)
// Every product is of the form C[i][j] = sum_k P[i][k] Q[j][k] with both
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
#include "mfma.hpp"
#include "trace.hpp"

#include <atomic>
#include <type_traits>

namespace bnr {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t h16;                                // fp16 storage word

constexpr float kS = 4096.f, kInvS = 1.f / 4096.f;   // see the precision note
constexpr int kSub = 64;                             // wide matrices are padded to multiples of it

// Stages of a call and their work items: momentum and squares; the narrow
// matrices' blocks and the sums of their partial Gram matrices; the wide ones'
// conversion, symmetric product tiles and general product tiles, and the same in
// larger and smaller tiles; the matrices of a single block, whole.
enum { PRE_SQ = 0, PRE_NARROW = 1, PRE_SUM = 2, PRE_PREP = 3, PRE_GRAM = 4, PRE_APPLY = 5, PRE_GRAM_L = 6, PRE_APPLY_L = 7,
       PRE_GRAM_S = 8, PRE_APPLY_S = 9, PRE_TINY = 10, PRE_GRAM_T = 11, PRE_APPLY_T = 12, kPre = kNsStages };

// one matrix of the list on the device: the caller's arguments and its place in the workspace
struct NsDev {
    NsIn in;
    int p, q, P, Q, flip;          // short and long side, padded; flip: X is the transpose of the caller's matrix
    int parts, blocks;             // partial sums of squares; column blocks of a narrow matrix (0: wide)
    double *sq;                    // [parts]
    h16 *x, *xt[2], *g, *r;        // wide: pair matrices [P][Q], [Q][P] twice, [P][P] twice; narrow: xt[0] = the blocks
    float *part[2], *sum;          // narrow: partial Gram matrices [blocks][P][P], their sum
};
// the device table: the matrices and the running counts of work items per stage
struct NsTable { NsDev *items; int *pre[kPre]; };

// Sizes of one matrix, the same on the host (workspace, grids) and on the device.
struct NsSize {
    int p, q, P, Q, flip, parts, blocks;
    int work[kPre];                // work items per stage
    int64_t bytes;                 // workspace
};
// the stage that counts the symmetric tiles of a size; the general tiles' is the next
__host__ __device__ constexpr int ns_gram_stage(int bt)
{
    return bt == 32 ? PRE_GRAM_T : (bt == 64 ? PRE_GRAM_S : (bt == 128 ? PRE_GRAM : PRE_GRAM_L));
}
constexpr int kMaxParts = 1024;    // partial sums of squares of a matrix
// short sides up to this take the narrow path (128 x 4096 106 us, sixteen of 128 x
// 1024 128; the wide path's 136 x 4096 161, sixteen of 136 x 1024 214)
constexpr int kNarrow = 128;
constexpr int kBlock = 16384;      // values of a narrow matrix's block: [kBlock / P][P]
// Blocks of one narrow matrix up to which every block adds the partial Gram
// matrices itself; past it a launch of its own adds them once (five steps, own
// additions against launches: 128 x 512, 4 blocks, 95 us against 100, sixteen of
// them 97 against 113; 128 x 1024, 8 blocks, 109 against 101; 64 x 2048, 8
// blocks, 75 against 85; 32 x 8192, 16 blocks, 70 against 76).
__host__ __device__ inline bool ns_summed(int blocks, int P) { return blocks > (P == 128 ? 4 : (P == 64 ? 8 : 32)); }

// whole: a matrix of a single block runs as a launch of its own over all steps.
__host__ __device__ inline NsSize ns_size(int rows, int cols, int whole)
{
    NsSize z;
    z.flip = rows > cols;
    z.p = z.flip ? cols : rows;
    z.q = z.flip ? rows : cols;
    // 16384 values a partial sum, whole rows, at most kMaxParts partial sums
    const int64_t want = ((int64_t)rows * cols + 16383) >> 14;
    unsigned n = want > kMaxParts ? kMaxParts : (unsigned)want;
    if (n > (unsigned)rows) n = rows;
    const unsigned rp = ((unsigned)rows + n - 1) / n;
    z.parts = (int)(((unsigned)rows + rp - 1) / rp);
    for (int k = 0; k < kPre; k++) z.work[k] = 0;
    z.work[PRE_SQ] = z.parts;
    z.blocks = 0;
    if (z.p <= kNarrow) {
        z.P = z.p <= 32 ? 32 : (z.p <= 64 ? 64 : 128);
        const int qb = kBlock / z.P;
        z.blocks = (z.q + qb - 1) / qb;
        z.Q = z.blocks * qb;
        if (z.blocks == 1 && whole) {            // nothing of it passes through the workspace
            z.work[PRE_SQ] = 0;
            z.work[PRE_TINY] = 1;
            z.bytes = 0;
            return z;
        }
        z.work[PRE_NARROW] = z.blocks;
        if (ns_summed(z.blocks, z.P)) z.work[PRE_SUM] = z.P * z.P / 256;
        z.bytes = kMaxParts * 8 + (int64_t)z.blocks * (kBlock * 4 + 2 * z.P * z.P * 4) + z.P * z.P * 4;
        return z;
    }
    const int up = (z.p + 63) / 64, uq = (z.q + 63) / 64;
    z.P = up * 64;
    z.Q = uq * 64;
    z.work[PRE_PREP] = up * uq;
    for (int l = 0; l < 4; l++) {                // tiles of 32, 64, 128, 256
        const int tp = l ? (up + (1 << l >> 1) - 1) >> (l - 1) : 2 * up, tq = l ? (uq + (1 << l >> 1) - 1) >> (l - 1) : 2 * uq;
        const int at = ns_gram_stage(32 << l);
        z.work[at] = tp * (tp + 1) / 2;
        z.work[at + 1] = tp * tq;
    }
    z.bytes = kMaxParts * 8 + (int64_t)z.P * z.Q * 4 * 3 + (int64_t)z.P * z.P * 4 * 2;
    return z;
}

struct NsChunk {                   // by value: the next matrices of the list
    int first, count, whole;
    int64_t at;                    // workspace offset and running counts in front of them
    int work[kPre];
    NsIn in[kNsChunk];
};

static_assert(sizeof(NsChunk) + sizeof(NsTable) + sizeof(void *) <= 4096, "kernel arguments");

// One wave, one matrix a lane; the places come from running sums across the lanes.
__global__ __launch_bounds__(64) void k_ns_table(NsChunk c, NsTable t, char *base)
{
    const int i = threadIdx.x;
    const bool in = i < c.count;
    NsDev d;
    d.in = c.in[in ? i : 0];
    NsSize z = ns_size(d.in.rows, d.in.cols, c.whole);
    int64_t at = in ? z.bytes : 0;
    int work[kPre];
    for (int k = 0; k < kPre; k++) work[k] = in ? z.work[k] : 0;
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t a = __shfl_up((long long)at, o, 64);
        if (i >= o) at += a;
        for (int k = 0; k < kPre; k++) {
            const int w = __shfl_up(work[k], o, 64);
            if (i >= o) work[k] += w;
        }
    }
    if (!in) return;
    d.p = z.p; d.q = z.q; d.P = z.P; d.Q = z.Q; d.flip = z.flip; d.parts = z.parts; d.blocks = z.blocks;
    char *b = base + c.at + at - z.bytes;
    d.sq = (double *)b;
    b += kMaxParts * 8;
    d.x = d.xt[0] = d.xt[1] = d.g = d.r = nullptr;
    d.part[0] = d.part[1] = d.sum = nullptr;
    const int64_t pp = (int64_t)z.P * z.P * 4;
    if (z.blocks) {
        d.xt[0] = (h16 *)b;
        b += (int64_t)z.blocks * kBlock * 4;
        d.part[0] = (float *)b;
        d.part[1] = (float *)(b + z.blocks * pp);
        d.sum = (float *)(b + 2 * z.blocks * pp);
    } else {
        const int64_t pq = (int64_t)z.P * z.Q * 4;
        d.x = (h16 *)b;
        d.xt[0] = (h16 *)(b + pq);
        d.xt[1] = (h16 *)(b + 2 * pq);
        d.g = (h16 *)(b + 3 * pq);
        d.r = (h16 *)(b + 3 * pq + pp);
    }
    t.items[c.first + i] = d;
    for (int k = 0; k < kPre; k++) t.pre[k][c.first + i] = c.work[k] + work[k] - z.work[k];
}

// The matrix a work item belongs to: the last one whose running count is not
// past it (the counts ascend, matrices without work in a stage repeat their
// successor's; the wave compares 64 of them at a time).
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

// Accesses through a pointer that was read from memory (the table's), or chosen
// between two LDS arrays: the compiler does not know its address space and would
// make flat accesses, which wait for the global and the LDS side both (250 ns a
// step where LDS reads and global stores alternate).  These name the space.
#define NS_GLOBAL __attribute__((address_space(1)))
typedef __attribute__((address_space(3))) unsigned char lds_byte;
template <typename V> __device__ __forceinline__ V gld(const void *p) { return *(const NS_GLOBAL V *)p; }
template <typename V> __device__ __forceinline__ void gst(void *p, V v) { *(NS_GLOBAL V *)p = v; }
template <typename V> __device__ __forceinline__ V lld(const lds_byte *p) { return *(const __attribute__((address_space(3))) V *)p; }
template <typename V> __device__ __forceinline__ void lst(lds_byte *p, V v) { *(__attribute__((address_space(3))) V *)p = v; }

template <typename T> __device__ __forceinline__ float ns_load(const void *p, int64_t i)
{
    if constexpr (sizeof(T) == 4) return gld<float>((const float *)p + i);
    else return bf2f(gld<bf16_t>((const bf16_t *)p + i));
}

// u of element i of a gradient row: the gradient itself, or what the momentum step makes of it
__device__ __forceinline__ float ns_u(float g, float buf, const NsStep &s)
{
    return !s.update ? g : (s.nesterov ? __builtin_fmaf(s.momentum, buf, g) : buf);
}

// Stage 1: the momentum (buf <- momentum buf + g) and the partial sums of u^2
// (in float64: the squares of float32 values neither overflow nor vanish there).
// A thread takes every 256th value of the part's rows, eight in flight, and
// steps its row and column along without dividing.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_ns_squares(NsTable t, int count, NsStep s)
{
    constexpr int U = 8;
    __shared__ double red[kThreads / 64];
    const int it = ns_find(t.pre[PRE_SQ], count, blockIdx.x);
    const NsDev &d = t.items[it];
    const int part = blockIdx.x - t.pre[PRE_SQ][it];
    const int rows = d.in.rows, cols = d.in.cols, rp = (rows + d.parts - 1) / d.parts;
    const int r1 = min(rows, part * rp + rp);
    const int dr = kThreads / cols, dc = kThreads % cols;
    int r = part * rp + (int)threadIdx.x / cols, c = (int)threadIdx.x % cols;
    const void *src = d.in.src;
    float *buf = d.in.buf;
    const int64_t ls = d.in.ld_src, lb = d.in.ld_buf;
    double acc = 0.0;
    while (r < r1) {
        float g[U], b[U];
        int64_t at[U];
        bool in[U];
        #pragma unroll
        for (int u = 0; u < U; u++) {
            in[u] = r < r1;
            const int rr = in[u] ? r : r1 - 1, cc = in[u] ? c : 0;       // read and dropped
            g[u] = ns_load<T>(src, rr * ls + cc);
            at[u] = rr * lb + cc;
            b[u] = s.update ? gld<float>(buf + at[u]) : 0.f;
            r += dr;
            c += dc;
            if (c >= cols) { c -= cols; r++; }
        }
        #pragma unroll
        for (int u = 0; u < U; u++) {
            if (!in[u]) continue;
            if (s.update) {
                b[u] = __builtin_fmaf(s.momentum, b[u], g[u]);
                gst(buf + at[u], b[u]);
            }
            const double v = (double)ns_u(g[u], b[u], s);
            acc += v * v;
        }
    }
    for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o, 64);
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = acc;
    __syncthreads();
    if (threadIdx.x == 0) gst(d.sq + part, red[0] + red[1] + red[2] + red[3]);
}

// S / (||u||_F + eps) of a matrix, by all threads of the workgroup; red: one
// double per wave.  Starts and ends without a barrier of its own around the
// caller's LDS; contains one.
template <int NT>
__device__ __forceinline__ float ns_factor(const NsDev &d, float eps, double *red)
{
    double acc = 0.0;
    for (int i = threadIdx.x; i < d.parts; i += NT) acc += gld<double>(d.sq + i);
    for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o, 64);
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = acc;
    __syncthreads();
    double sum = red[0];
    for (int i = 1; i < NT / 64; i++) sum += red[i];
    return (float)((double)kS / (sqrt(sum) + (double)eps));
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
// the pairs of four values, hi and lo as two words each
__device__ __forceinline__ void ns_pair4(const float *v, u32x2_t &hi, u32x2_t &lo)
{
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    #pragma unroll
    for (int k = 0; k < 2; k++) {
        float a = v[2 * k], b = v[2 * k + 1];
        asm("" : "+v"(a), "+v"(b));
        const f16x2 h = __builtin_convertvector(f32x2_t{a, b}, f16x2);
        const f16x2 l = __builtin_convertvector(f32x2_t{a - (float)h[0], b - (float)h[1]}, f16x2);
        hi[k] = __builtin_bit_cast(uint32_t, h);
        lo[k] = __builtin_bit_cast(uint32_t, l);
    }
}
// Element offset of (row, k) of a pair matrix with K columns: hi there, lo kLo
// further on.  The order is the one in which the matrix instructions' fragments
// are read: 16 rows x 32 columns of hi are one KiB, 8 columns of one row together,
// 16 rows of them, four times that; then the lo ones; four such blocks make the 64
// rows of one k step, then the next step follows.
constexpr int kFrag = 512, kLo = kFrag, kBlk = 2 * kFrag, kStep = 4 * kBlk;      // halves
__device__ __forceinline__ int64_t ns_at(int row, int k, int K)
{
    return ((int64_t)(row >> 6) * (K >> 5) + (k >> 5)) * kStep + ((row >> 4) & 3) * kBlk + ((k >> 3) & 3) * 128 +
           (row & 15) * 8 + (k & 7);
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
    constexpr int U = 64 * 64 / kThreads;
    float gv[U], bv[U];
    #pragma unroll
    for (int u = 0; u < U; u++) {                // all loads before the first use
        const int e = tid + u * kThreads, r = rb + e / 64, c = cb + e % 64;
        const bool in = r < d.in.rows && c < d.in.cols;
        gv[u] = in ? ns_load<T>(d.in.src, (int64_t)r * d.in.ld_src + c) : 0.f;
        bv[u] = in && s.update ? gld<float>(d.in.buf + (int64_t)r * d.in.ld_buf + c) : 0.f;
    }
    #pragma unroll
    for (int u = 0; u < U; u++) {
        const int e = tid + u * kThreads;
        tile[e / 64][e % 64] = ns_u(gv[u], bv[u], s);
    }
    const float scale = ns_factor<kThreads>(d, s.eps, red);              // (its barrier covers the tile)
    // as it is: [RP rows][K = CP]; turned: [CP rows][K = RP]
    h16 *straight = d.flip ? d.xt[0] : d.x, *turned = d.flip ? d.x : d.xt[0];
    // a thread makes 8 columns of one row: lane, then 16-row block, then k step
    for (int v = tid; v < 64 * 8; v += kThreads) {
        const int a = (v >> 6 & 3) * 16 + (v & 15), k8 = (v >> 8) * 32 + (v >> 4 & 3) * 8;
        u32x2_t hi[2], lo[2];
        float f[8];
        for (int i = 0; i < 8; i++) f[i] = tile[a][k8 + i] * scale;
        ns_pair4(f, hi[0], lo[0]);
        ns_pair4(f + 4, hi[1], lo[1]);
        h16 *o = straight + ns_at(rb + a, cb + k8, CP);
        gst(o, u32x4{hi[0][0], hi[0][1], hi[1][0], hi[1][1]});
        gst(o + kLo, u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]});
        for (int i = 0; i < 8; i++) f[i] = tile[k8 + i][a] * scale;
        ns_pair4(f, hi[0], lo[0]);
        ns_pair4(f + 4, hi[1], lo[1]);
        o = turned + ns_at(cb + a, rb + k8, RP);
        gst(o, u32x4{hi[0][0], hi[0][1], hi[1][0], hi[1][1]});
        gst(o + kLo, u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]});
    }
}

// The result o of element (row, col) of the caller's matrix: itself, or the
// weight it steps (and the weight's bf16 copy).  lr is 0 without an update.
template <typename W>
__device__ __forceinline__ void ns_result(const NsIn &in, const NsStep &s, float lr, int64_t row, int col, float o)
{
    W *dst = (W *)in.dst + row * in.ld_dst + col;
    float res = o;
    if (s.update) {
        res = __builtin_fmaf(-lr * in.scale, o, ns_load<W>(dst, 0) * (1.f - lr * s.decay));
        if (in.copy) gst(in.copy + row * in.ld_copy + col, f2bf(res));
    }
    if constexpr (sizeof(W) == 4) gst<float>(dst, res);
    else gst<bf16_t>(dst, f2bf(res));
}
// Whether four results side by side, the first at a multiple of four columns,
// can move as one access in every matrix that the results touch.
template <typename W>
__device__ __forceinline__ bool ns_fours(const NsIn &in, const NsStep &s)
{
    const bool dst = ((uintptr_t)in.dst & (4 * sizeof(W) - 1)) == 0 && (in.ld_dst & 3) == 0;
    return dst && (!s.update || !in.copy || (((uintptr_t)in.copy & 7) == 0 && (in.ld_copy & 3) == 0));
}
// Four of them: one read, one write and one copy instead of four each (twelve bf16
// weights of 1024 x 4096, last stage: 480 us in single accesses, 405 in these).
template <typename W>
__device__ __forceinline__ void ns_result4(const NsIn &in, const NsStep &s, float lr, int64_t row, int col, const float (&o)[4])
{
    W *dst = (W *)in.dst + row * in.ld_dst + col;
    typedef std::conditional_t<sizeof(W) == 4, f32x4, u32x2_t> raw;
    union { raw v; W e[4]; } t;
    float res[4] = {o[0], o[1], o[2], o[3]};
    if (s.update) {
        t.v = gld<raw>(dst);
        #pragma unroll
        for (int e = 0; e < 4; e++) {
            float old;
            if constexpr (sizeof(W) == 4) old = t.e[e]; else old = bf2f(t.e[e]);
            res[e] = __builtin_fmaf(-lr * in.scale, o[e], old * (1.f - lr * s.decay));
        }
        if (in.copy) {
            union { u32x2_t v; bf16_t e[4]; } c;
            #pragma unroll
            for (int e = 0; e < 4; e++) c.e[e] = f2bf(res[e]);
            gst(in.copy + row * in.ld_copy + col, c.v);
        }
    }
    #pragma unroll
    for (int e = 0; e < 4; e++)
        if constexpr (sizeof(W) == 4) t.e[e] = res[e]; else t.e[e] = f2bf(res[e]);
    gst(dst, t.v);
}
__device__ __forceinline__ float ns_rate(const NsStep &s) { return !s.update ? 0.f : (s.lr_dev ? gld<float>(s.lr_dev) : s.lr); }

// A product's sums: hi hi' in acc and the two smaller products apart in low, joined
// at the end.  A matrix instruction adds its 32 terms in four roundings, so one
// chain of all three products takes twelve a k step at the sum's full size; with
// low, whose roundings are 2^-11 of that, it takes four.  (1023 x 4093 with singular
// values over five decades: 1.56 times the error of float32 products in one chain,
// 0.97 apart; 413 us and 421.  Tiles of 256 have no registers for both: 4096 x 4096
// is 1.13 times as far off as float32 products.)
template <int MI, int NI>
__device__ __forceinline__ void ns_zero(f32x4 (&acc)[MI][NI])
{
    #pragma unroll
    for (int i = 0; i < MI; i++)
        #pragma unroll
        for (int j = 0; j < NI; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}
template <int MI, int NI>
__device__ __forceinline__ void ns_join(f32x4 (&acc)[MI][NI], const f32x4 (&low)[MI][NI])
{
    #pragma unroll
    for (int i = 0; i < MI; i++)
        #pragma unroll
        for (int j = 0; j < NI; j++)
            #pragma unroll
            for (int e = 0; e < 4; e++) acc[i][j][e] += low[i][j][e];
}

// One product stage over the whole list.
//   NS_GRAM    G = X X^T            (lower-triangle tiles, mirrored)
//   NS_SQUARE  R = a I + b G + c G G (likewise)
//   NS_APPLY   X, X^T <- R X
//   NS_LAST    R X into the caller's matrix
enum { NS_GRAM = 0, NS_SQUARE = 1, NS_APPLY = 2, NS_LAST = 3 };
constexpr bool ns_sym(int mode) { return mode == NS_GRAM || mode == NS_SQUARE; }

// How a stage's tiles run.  The chip holds ns_slots workgroups of the product
// kernel at once (512 of the small tile, two a CU, 256 of the large).  Whole tiles fill as many rounds of that as they can; the rest
// (tiles [whole, tiles)) would leave most of the chip idle for a round, so each
// of them is cut into `pieces` along k: a piece's float32 sums go to the
// workspace and k_ns_finish adds them in a fixed order.
struct NsCut { int bt, tiles, whole, pieces; float *part; };

// the tile of a stage: its matrix and its block row and column
struct NsPlace { int it, ti, tj; };
template <int BT, int MODE>
__device__ __forceinline__ NsPlace ns_place(const NsTable &t, int count, int tile)
{
    const int *pre = t.pre[ns_gram_stage(BT) + !ns_sym(MODE)];
    NsPlace pl;
    pl.it = ns_find(pre, count, tile);
    const int w = tile - pre[pl.it];
    if (ns_sym(MODE)) {                          // row i of the triangle starts at i (i + 1) / 2
        int ti = (int)((sqrtf(8.f * (float)w + 1.f) - 1.f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= w) ti++;
        while (ti * (ti + 1) / 2 > w) ti--;
        pl.ti = ti;
        pl.tj = w - ti * (ti + 1) / 2;
    } else {
        const int tp = (t.items[pl.it].P + BT - 1) / BT;
        pl.ti = w % tp;
        pl.tj = w / tp;
    }
    return pl;
}

// Orders a wave's LDS accesses of other lanes' values (the wave's own area: no barrier needed).
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// 64 x 64 results in LDS, turned: row j holds the 64 i as pairs (two k blocks of
// [hi 32 | lo 32], 256 bytes) or as float32, its 16-byte chunks in the order
// chunk ^ (j % 16), so that 16 rows of one column lie in different banks.
constexpr int kSubBytes = kSub * 256;
__device__ __forceinline__ int sub_at(int j, int byte) { return j * 256 + ((byte >> 4 ^ (j & 15)) << 4) + (byte & 15); }

// Results [MI][NI] of 16 x 16 blocks (a lane holds rows 4 g .. + 3 of column q;
// S^2 times the product) into the sub-tile from its block (mi0, nj0) on.
template <int MODE, int MI, int NI>
__device__ __forceinline__ void sub_put(lds_byte *sub, const f32x4 (&acc)[MI][NI], int mi0, int nj0, const NsDev &d,
                                        const NsStep &s, int i0, int j0)
{
    const int lane = threadIdx.x & 63, g = lane / 16, q = lane % 16;
    #pragma unroll
    for (int nj = 0; nj < NI; nj++)
        #pragma unroll
        for (int mi = 0; mi < MI; mi++) {
            const int i = (mi0 + mi) * 16 + 4 * g, j = (nj0 + nj) * 16 + q;
            float v[4];
            #pragma unroll
            for (int e = 0; e < 4; e++) v[e] = acc[mi][nj][e] * kInvS;
            if constexpr (MODE == NS_SQUARE) {
                float gg[4];                     // G is symmetric: row j holds the four i together
                const h16 *p = d.g + ns_at(j0 + j, i0 + i, d.P);
                const f16x4 hi = gld<f16x4>(p), lo = gld<f16x4>(p + kLo);
                #pragma unroll
                for (int e = 0; e < 4; e++) {
                    gg[e] = (float)hi[e] + (float)lo[e];
                    v[e] = __builtin_fmaf(s.c, v[e], s.b * gg[e]) + (i0 + i + e == j0 + j ? s.a * kS : 0.f);
                }
            }
            if constexpr (MODE == NS_LAST) {
                f32x4 o = {v[0] * kInvS, v[1] * kInvS, v[2] * kInvS, v[3] * kInvS};
                lst(sub + sub_at(j, i * 4), o);
            } else {
                u32x2_t hi, lo;
                ns_pair4(v, hi, lo);
                const int byte = (i >> 5) * 128 + (i & 31) * 2;
                lst(sub + sub_at(j, byte), hi);
                lst(sub + sub_at(j, byte + 64), lo);
            }
        }
}

// The SB x SB sub-tile to memory by NW waves, w this wave's number among them:
// its rows as they lie, and the other orientation through transposing reads.
// i0, j0: the sub-tile's place in the result.
template <int MODE, int SB, int NW, typename W>
__device__ __forceinline__ void sub_out(const lds_byte *sub, int w, const NsDev &d, const NsStep &s, int turn,
                                        bool mirror, int i0, int j0)
{
    const int lane = threadIdx.x & 63, g = lane / 16, q = lane % 16;
    if constexpr (MODE == NS_LAST) {
        const float lr = ns_rate(s);
        const int rows = d.flip ? d.q - j0 : d.p - i0, cols = d.flip ? d.p - i0 : d.q - j0;
        const int64_t row0 = d.flip ? j0 : i0;
        const int col0 = d.flip ? i0 : j0;
        if (!ns_fours<W>(d.in, s)) {
            #pragma unroll 4
            for (int k = w; k < SB * SB / 64; k += NW) {         // along rows of the caller's matrix
                const int r = k * (64 / SB) + lane / SB, c = lane % SB;
                const float o = lld<float>(d.flip ? sub + sub_at(r, c * 4) : sub + sub_at(c, r * 4));
                if (r < rows && c < cols) ns_result<W>(d.in, s, lr, row0 + r, col0 + c, o);
            }
            return;
        }
        #pragma unroll 4
        for (int k = w; k < SB * SB / 256; k += NW) {            // the same, four columns a lane: a quarter of the accesses
            const int r = k * (256 / SB) + lane / (SB / 4), c = lane % (SB / 4) * 4;
            float o[4];
            #pragma unroll
            for (int e = 0; e < 4; e++) o[e] = lld<float>(d.flip ? sub + sub_at(r, (c + e) * 4) : sub + sub_at(c + e, r * 4));
            if (r >= rows || c >= cols) continue;
            if (c + 4 <= cols) ns_result4<W>(d.in, s, lr, row0 + r, col0 + c, o);
            else
                for (int e = 0; e < 4 && c + e < cols; e++) ns_result<W>(d.in, s, lr, row0 + r, col0 + c + e, o[e]);
        }
    } else {
        h16 *straight = MODE == NS_GRAM ? d.g : (MODE == NS_SQUARE ? d.r : d.x);
        h16 *turned = MODE == NS_APPLY ? d.xt[turn ^ 1] : straight;
        const int ks = ns_sym(MODE) ? d.P : d.Q;
        // a fragment a step: 16 rows, 32 columns, hi or lo; a lane has 8 columns of row q
        constexpr int FRAGS = SB / 16 * (SB / 32) * 2;
        #pragma unroll
        for (int k = w; k < FRAGS; k += NW) {
            const int part = k & 1, j = (k >> 1) / (SB / 32) * 16 + q, i = (k >> 1) % (SB / 32) * 32;
            gst(turned + ns_at(j0 + j, i0 + i + 8 * g, d.P) + part * kLo, lld<u32x4>(sub + sub_at(j, i * 4 + part * 64 + g * 16)));
        }
        if (!mirror) return;
        #pragma unroll
        for (int k = w; k < FRAGS; k += NW) {
            const int part = k & 1, jb = (k >> 1) % (SB / 32) * 32, i = (k >> 1) / (SB / 32) * 16;
            const int byte = (i >> 5) * 128 + (i & 31) * 2 + part * 64 + 8 * (q % 4), j = jb + 8 * g + q / 4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(sub + sub_at(j, byte)));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(sub + sub_at(j + 4, byte)));
            const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            gst(straight + ns_at(i0 + i + q, j0 + jb + 8 * g, ks) + part * kLo, v);
        }
    }
}

// Workgroup: a tile of BT x BT outputs, or a piece of one.  BT = 128: 2 x 2
// waves of 64 x 64, two workgroups a CU; BT = 256: 2 x 4 waves of 128 x 64, one a
// CU, for which a k step's operands are half of the lines per product and its
// fragment reads three quarters (a tile may hang over the matrix by 128 rows or
// columns: those rows are read again from inside and not written).  Two LDS
// stages of BT / 4 fragments (one k step of both operands), each a KiB as it lies
// in memory, hi and lo of 16 rows in turn.  The next step's fragments are loaded
// straight into LDS while the current step multiplies.
// (For 128-tiles alone on their CUs, reading the next step's fragments from LDS
// ahead of the products and memory four steps ahead through registers was no
// faster: 256 tiles of 32 steps 44 us against 41.)
template <int BT, int MODE, typename W>
__global__ __launch_bounds__(BT * 2, 2) void k_ns_product(NsTable t, int count, NsStep s, int turn, NsCut cut)
{
    constexpr int NT = BT * 2, WN = BT / 64, TM = BT / 2, TN = 64, MI = TM / 16, NI = TN / 16;
    constexpr int kStage = BT / 4 * 1024, kLoads = kStage / (NT * 16);
    static_assert(kStage == NT / 128 * kSubBytes, "half of the waves' results fit a stage");
    __shared__ __align__(16) unsigned char lds0[kStage], lds1[kStage];
    int tile, piece = 0, pieces = 1;
    if ((int)blockIdx.x < cut.whole) {
        tile = xcd_remap(blockIdx.x, cut.whole);
    } else {
        const int u = blockIdx.x - cut.whole;
        pieces = cut.pieces;
        tile = cut.whole + u / pieces;
        piece = u % pieces;
    }
    const NsPlace pl = ns_place<BT, MODE>(t, count, tile);
    const NsDev &d = t.items[pl.it];
    const int P = d.P, Q = d.Q, ti = pl.ti, tj = pl.tj;
    const int K = MODE == NS_GRAM ? Q : P;
    const h16 *pa = MODE == NS_GRAM ? d.x : (MODE == NS_SQUARE ? d.g : d.r);
    const h16 *pb = MODE == NS_GRAM ? d.x : (MODE == NS_SQUARE ? d.g : d.xt[turn]);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // fragment of this wave's load l: l (NT / 64) + wave of the stage
    const char *src[kLoads];
    #pragma unroll
    for (int l = 0; l < kLoads; l++) {
        const int f = l * (NT / 64) + wave, row = f / 2 * 16;
        const int end_a = P - 16, end_b = (ns_sym(MODE) ? P : Q) - 16;
        const h16 *base = row < BT ? pa + ns_at(min(ti * BT + row, end_a), 0, K) : pb + ns_at(min(tj * BT + row - BT, end_b), 0, K);
        src[l] = (const char *)(base + f % 2 * kLo + lane * 8);
    }
    auto load = [&](unsigned char *stage, int step) __attribute__((always_inline)) {
        #pragma unroll
        for (int l = 0; l < kLoads; l++)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(src[l] + (int64_t)step * (kStep * 2)),
                                             (__attribute__((address_space(3))) uint32_t *)(stage + (l * NT + wave * 64) * 16),
                                             16, 0, 0);
        __builtin_amdgcn_sched_barrier(0);       // (the scheduler would sink them to the barrier that waits for them)
    };
    const int wm = wave / WN, wn = wave % WN;
    constexpr bool APART = BT == 128;
    f32x4 acc[MI][NI], low[APART ? MI : 1][APART ? NI : 1];
    ns_zero(acc);
    ns_zero(low);
    auto frag = [&](const unsigned char *stage, int row, int part) __attribute__((always_inline)) {
        return *reinterpret_cast<const f16x8 *>(stage + (row / 8 + part) * 1024 + lane * 16);
    };
    struct Frags { f16x8 ah[MI], al[MI], bh[NI], bl[NI]; };
    auto read = [&](Frags &f, const unsigned char *stage) __attribute__((always_inline)) {
        #pragma unroll
        for (int i = 0; i < MI; i++) {
            f.ah[i] = frag(stage, wm * TM + i * 16, 0);
            f.al[i] = frag(stage, wm * TM + i * 16, 1);
        }
        #pragma unroll
        for (int j = 0; j < NI; j++) {
            f.bh[j] = frag(stage, BT + wn * TN + j * 16, 0);
            f.bl[j] = frag(stage, BT + wn * TN + j * 16, 1);
        }
    };
    // the three products of a sum are far apart, except where the registers do not
    // hold all fragments (256-tiles: spills, 140 -> 179 us)
    auto multiply = [&](const Frags &f) __attribute__((always_inline)) {
        if constexpr (APART) {
            #pragma unroll
            for (int term = 0; term < 3; term++)
                #pragma unroll
                for (int i = 0; i < MI; i++)
                    #pragma unroll
                    for (int j = 0; j < NI; j++) {
                        f32x4 &to = term < 2 ? low[i][j] : acc[i][j];
                        to = __builtin_amdgcn_mfma_f32_16x16x32_f16(term == 1 ? f.al[i] : f.ah[i],
                                                                    term == 0 ? f.bl[j] : f.bh[j], to, 0, 0, 0);
                    }
        } else {
            #pragma unroll
            for (int i = 0; i < MI; i++)
                #pragma unroll
                for (int j = 0; j < NI; j++) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.ah[i], f.bl[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.al[i], f.bh[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.ah[i], f.bh[j], acc[i][j], 0, 0, 0);
                }
        }
    };
    // steps in pairs (K is a multiple of 64); a piece may have none
    const int pairs = K / 64, k0 = piece * pairs / pieces * 2, k1 = (piece + 1) * pairs / pieces * 2;
    if (k0 < k1) {
        load(lds0, k0);
        __syncthreads();
        for (int k = k0; k < k1; k += 2) {
            Frags f;
            load(lds1, k + 1);
            read(f, lds0);
            multiply(f);
            __syncthreads();
            if (k + 2 < k1) load(lds0, k + 2);
            read(f, lds1);
            multiply(f);
            __syncthreads();
        }
    }
    if constexpr (APART) ns_join(acc, low);
    if (pieces > 1) {                            // in the order of the fragments: [wave][block][lane]
        float *o = cut.part + (int64_t)(blockIdx.x - cut.whole) * (BT * BT) + wave * (TM * TN);
        #pragma unroll
        for (int i = 0; i < MI; i++)
            #pragma unroll
            for (int j = 0; j < NI; j++)
                gst(o + ((j * MI + i) * 64 + lane) * 4, acc[i][j]);
        return;
    }
    // every wave stages 64 x 64 results at a time in its own part of the stages
    lds_byte *sub = (wave < NT / 128 ? (lds_byte *)lds0 : (lds_byte *)lds1) + wave % (NT / 128) * kSubBytes;
    const int j0 = tj * BT + wn * TN;
    const bool in = j0 < (ns_sym(MODE) ? P : Q);
    #pragma unroll
    for (int h = 0; h < TM / kSub; h++) {
        const int i0 = ti * BT + wm * TM + h * kSub;
        if (!in || i0 >= P) continue;
        f32x4 part[4][NI];
        #pragma unroll
        for (int i = 0; i < 4; i++)
            #pragma unroll
            for (int j = 0; j < NI; j++) part[i][j] = acc[h * 4 + i][j];
        sub_put<MODE>(sub, part, 0, 0, d, s, i0, j0);
        wave_sync();
        // both orientations already
        sub_out<MODE, kSub, 1, W>(sub, 0, d, s, turn, !ns_sym(MODE) || ti != tj, i0, j0);
        wave_sync();
    }
}

// The results of the tiles that ran in pieces: a workgroup adds the pieces of
// 64 x 64 results, wave w their block column w, in order.
template <int BT, int MODE, typename W>
__global__ __launch_bounds__(256) void k_ns_finish(NsTable t, int count, NsStep s, int turn, NsCut cut)
{
    constexpr int WN = BT / 64, TM = BT / 2, MI = TM / 16, kSubs = BT * BT / (kSub * kSub), kHalves = TM / kSub;
    __shared__ __align__(16) unsigned char sub[kSubBytes];
    const int tile = cut.whole + blockIdx.x / kSubs, q = blockIdx.x % kSubs, from = q / kHalves, h = q % kHalves;
    const NsPlace pl = ns_place<BT, MODE>(t, count, tile);
    const NsDev &d = t.items[pl.it];
    const int i0 = pl.ti * BT + from / WN * TM + h * kSub, j0 = pl.tj * BT + from % WN * kSub;
    if (i0 >= d.P || j0 >= (ns_sym(MODE) ? d.P : d.Q)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float *src = cut.part + (int64_t)(blockIdx.x / kSubs) * cut.pieces * (BT * BT) + from * (TM * 64) +
                       ((wave * MI + h * 4) * 64 + lane) * 4;
    f32x4 acc[4][1];
    #pragma unroll
    for (int i = 0; i < 4; i++) acc[i][0] = gld<f32x4>(src + i * 256);
    #pragma unroll 4
    for (int k = 1; k < cut.pieces; k++)
        #pragma unroll
        for (int i = 0; i < 4; i++) {
            const f32x4 v = gld<f32x4>(src + (int64_t)k * (BT * BT) + i * 256);
            acc[i][0][0] += v[0]; acc[i][0][1] += v[1]; acc[i][0][2] += v[2]; acc[i][0][3] += v[3];
        }
    sub_put<MODE>((lds_byte *)sub, acc, 0, wave, d, s, i0, j0);
    __syncthreads();
    sub_out<MODE, kSub, 4, W>((lds_byte *)sub, wave, d, s, turn, !ns_sym(MODE) || pl.ti != pl.tj, i0, j0);
}

// Workgroup: a tile of BT x BT outputs (64 or 32) whose k steps are split over
// its four waves.  Nothing is shared between the waves, so the operands'
// fragments are loaded straight into registers, AHEAD steps ahead, without LDS or
// barriers: for few tiles, where the time of a stage is what one CU loads (30 to
// 50 GB/s).  The waves' sums are added through LDS in a fixed order.
template <int BT, int MODE, typename W>
__global__ __launch_bounds__(256, 1) void k_ns_direct(NsTable t, int count, NsStep s, int turn)
{
    constexpr int B = BT / 16, AHEAD = 16 / B;
    __shared__ __align__(16) unsigned char lds[BT == 64 ? 4 * kSubBytes : kSubBytes];
    const NsPlace pl = ns_place<BT, MODE>(t, count, xcd_remap(blockIdx.x, gridDim.x));
    const NsDev &d = t.items[pl.it];
    const int K = MODE == NS_GRAM ? d.Q : d.P;
    const h16 *pa = MODE == NS_GRAM ? d.x : (MODE == NS_SQUARE ? d.g : d.r);
    const h16 *pb = MODE == NS_GRAM ? d.x : (MODE == NS_SQUARE ? d.g : d.xt[turn]);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i0 = pl.ti * BT, j0 = pl.tj * BT;
    const int steps = K / 32, k0 = wave * steps / 4, n = (wave + 1) * steps / 4 - k0;
    const h16 *a = pa + ns_at(i0, k0 * 32, K) + lane * 8, *b = pb + ns_at(j0, k0 * 32, K) + lane * 8;
    f16x8 f[AHEAD][4 * B];                       // a hi, lo; b hi, lo of B blocks each
    auto load = [&](f16x8 (&o)[4 * B], int k) __attribute__((always_inline)) {
        #pragma unroll
        for (int i = 0; i < B; i++) {
            const h16 *p = a + i * kBlk + (int64_t)k * kStep, *q = b + i * kBlk + (int64_t)k * kStep;
            o[2 * i] = gld<f16x8>(p);
            o[2 * i + 1] = gld<f16x8>(p + kLo);
            o[2 * B + 2 * i] = gld<f16x8>(q);
            o[2 * B + 2 * i + 1] = gld<f16x8>(q + kLo);
        }
    };
    f32x4 acc[B][B], low[B][B];
    ns_zero(acc);
    ns_zero(low);
    #pragma unroll
    for (int u = 0; u < AHEAD; u++)
        if (u < n) load(f[u], u);
    for (int k = 0; k < n; k += AHEAD)
        #pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            if (k + u < n)
                #pragma unroll
                for (int i = 0; i < B; i++)
                    #pragma unroll
                    for (int j = 0; j < B; j++) {
                        const f16x8 &ah = f[u][2 * i], &al = f[u][2 * i + 1], &bh = f[u][2 * B + 2 * j], &bl = f[u][2 * B + 2 * j + 1];
                        low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bl, low[i][j], 0, 0, 0);
                        low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, bh, low[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bh, acc[i][j], 0, 0, 0);
                    }
            if (k + u + AHEAD < n) load(f[u], k + u + AHEAD);
        }
    ns_join(acc, low);
    // in the order of the fragments, [wave][block][lane]; wave w adds the B B / 4 blocks from w B B / 4 on
    constexpr int MINE = B * B / 4;
    f32x4 *red = reinterpret_cast<f32x4 *>(lds);
    #pragma unroll
    for (int j = 0; j < B; j++)
        #pragma unroll
        for (int i = 0; i < B; i++) red[(wave * B * B + j * B + i) * 64 + lane] = acc[i][j];
    __syncthreads();
    f32x4 sum[MINE][1];
    #pragma unroll
    for (int i = 0; i < MINE; i++) {
        sum[i][0] = red[(wave * MINE + i) * 64 + lane];
        #pragma unroll
        for (int w = 1; w < 4; w++) {
            const f32x4 v = red[(w * B * B + wave * MINE + i) * 64 + lane];
            sum[i][0][0] += v[0]; sum[i][0][1] += v[1]; sum[i][0][2] += v[2]; sum[i][0][3] += v[3];
        }
    }
    __syncthreads();
    sub_put<MODE>((lds_byte *)lds, sum, wave * MINE % B, wave * MINE / B, d, s, i0, j0);
    __syncthreads();
    sub_out<MODE, BT, 4, W>((lds_byte *)lds, wave, d, s, turn, !ns_sym(MODE) || pl.ti != pl.tj, i0, j0);
}

// ---- narrow matrices (short side up to 128) --------------------------------
// A workgroup owns a block of kBlock / P columns of X and keeps it, transposed,
// in LDS ([column][P] pairs, 64 KiB) together with G or R.  One launch is one
// whole step: the workgroup adds the partial Gram matrices of all blocks of its
// matrix, forms R = a I + b G + c G G (each block for itself: 128^3 products
// cost less than a launch), Y = R X over its block and the block's partial Gram
// matrix of Y for the next step.  So a list of narrow matrices of any number
// takes one launch per step where the wide path takes three.
constexpr int kNwThreads = 512;
template <int P> struct Nw {
    static constexpr int QB = kBlock / P;
    // row pitches in halves: 16 and 32 bytes past the pairs, so that the 16 rows
    // of a fragment and the rows of a transposing read start in different banks
    static constexpr int GP = 2 * P + 8, XP = 2 * P + 16;
    // G's third parts (nw_third), one a value
    static constexpr int MP = P + 8, MBytes = P <= 32 ? P * MP * 2 : 0;
    static constexpr int XBytes = QB * XP * 2, LBytes = XBytes + P * GP * 2 + MBytes;
    // waves over a P x P product and over R X
    static constexpr int TM = P == 128 ? 32 : 16, TN = P == 128 ? 64 : (P == 64 ? 32 : 16), WN = P / TN;
    static constexpr int YM = 32, YN = 64, YWN = QB / YN;
    static_assert(P / YM * YWN == kNwThreads / 64, "R X tiles fill the waves");
};
constexpr int nw_max(int a, int b) { return a > b ? a : b; }
constexpr int kNwLds = nw_max(Nw<128>::LBytes, nw_max(Nw<64>::LBytes, Nw<32>::LBytes));

// halves offset of k (0 .. K) within a pair row
__device__ __forceinline__ int nw_k(int k) { return (k >> 5) * 64 + (k & 31); }

// In sums of few terms no other rounding covers those of the pairs.  Up to 64 rows
// lo lo' is added too; up to 32 the square takes G in three parts, hi + lo + what those
// leave, with the third ones' products with hi.  Times the error of float32 products,
// without and with: 8 x 8 with rows of different scale 1.7 and 0.9, 16 x 40 of rank 4
// and noise 1.33 and 1.16, 64 x 4096 1.28 and 1.05 (without the third parts, which do not
// lower it and cost 4 %).  Time: 1 to 4 %.  Past 64 rows the errors are at most 1.12
// times float32's without, and the fourth product costs 5 to 7 %.
constexpr bool nw_four(int P) { return P <= 64; }
constexpr bool nw_third(int P) { return P <= 32; }

__device__ __forceinline__ f16x8 nw_frag(const h16 *p) { return *reinterpret_cast<const f16x8 *>(p); }

// acc += A B^T over KS k steps, A rows at a, B rows at b (both contiguous along k);
// with THIRD also A's hi times B's third parts (rows at bm) and the reverse
template <int MI, int NI, int KS, bool THIRD = false>
__device__ __forceinline__ void nw_product(const h16 *a, int pa, const h16 *b, int pb, f32x4 (&acc)[MI][NI],
                                           const h16 *am = nullptr, const h16 *bm = nullptr, int pm = 0)
{
    const int lane = threadIdx.x & 63, fr = lane % 16, fc = lane / 16;
    f32x4 low[MI][NI];
    ns_zero(low);
    a += fr * pa + fc * 8;
    b += fr * pb + fc * 8;
    if (THIRD) {
        am += fr * pm + fc * 8;
        bm += fr * pm + fc * 8;
    }
    #pragma unroll
    for (int k = 0; k < KS; k++) {
        f16x8 ah[MI], al[MI], bh[NI], bl[NI];
        #pragma unroll
        for (int i = 0; i < MI; i++) {
            ah[i] = nw_frag(a + i * 16 * pa + k * 64);
            al[i] = nw_frag(a + i * 16 * pa + k * 64 + 32);
        }
        #pragma unroll
        for (int j = 0; j < NI; j++) {
            bh[j] = nw_frag(b + j * 16 * pb + k * 64);
            bl[j] = nw_frag(b + j * 16 * pb + k * 64 + 32);
        }
        #pragma unroll
        for (int i = 0; i < MI; i++)
            #pragma unroll
            for (int j = 0; j < NI; j++) {
                if constexpr (THIRD) {
                    low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], nw_frag(bm + j * 16 * pm + k * 32), low[i][j], 0, 0, 0);
                    low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(nw_frag(am + i * 16 * pm + k * 32), bh[j], low[i][j], 0, 0, 0);
                }
                if (nw_four(KS * 32)) low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[i], bl[j], low[i][j], 0, 0, 0);
                low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bl[j], low[i][j], 0, 0, 0);
                low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[i], bh[j], low[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bh[j], acc[i][j], 0, 0, 0);
            }
    }
    ns_join(acc, low);
}

// four consecutive values of a pair row
__device__ __forceinline__ void nw_store4(h16 *p, const float *v)
{
    u32x2_t hi, lo;
    ns_pair4(v, hi, lo);
    *reinterpret_cast<u32x2_t *>(p) = hi;
    *reinterpret_cast<u32x2_t *>(p + 32) = lo;
}

// The block's partial Gram matrix over `steps` k steps of 32 columns (S^2 times
// it): the wave's tile in acc.  False for a wave without one (P = 32: four waves
// have a tile).
// between(k) runs ahead of step k.
template <int P, int MI, int NI, typename F>
__device__ __forceinline__ bool nw_gram(const h16 *xs, int steps, f32x4 (&acc)[MI][NI], F &&between)
{
    using N = Nw<P>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / N::WN, wn = wave % N::WN;
    if (wm * N::TM >= P) return false;
    f32x4 low[MI][NI];
    ns_zero(acc);
    ns_zero(low);
    // fragments of 8 consecutive block columns of one row of X: transposing reads
    const int g = lane / 16, q = lane % 16;
    const h16 *base = xs + (8 * g + q / 4) * N::XP + 4 * (q % 4);
    auto frag = [&](int k, int i, int part_) __attribute__((always_inline)) {
        return __builtin_bit_cast(f16x8, tr_frag(base + k * 32 * N::XP + nw_k(i) + part_ * 32, N::XP));
    };
    #pragma unroll 4
    for (int k = 0; k < steps; k++) {
        between(k);
        f16x8 ah[MI], al[MI], bh[NI], bl[NI];
        #pragma unroll
        for (int i = 0; i < MI; i++) {
            ah[i] = frag(k, wm * N::TM + i * 16, 0);
            al[i] = frag(k, wm * N::TM + i * 16, 1);
        }
        #pragma unroll
        for (int j = 0; j < NI; j++) {
            bh[j] = frag(k, wn * N::TN + j * 16, 0);
            bl[j] = frag(k, wn * N::TN + j * 16, 1);
        }
        #pragma unroll
        for (int i = 0; i < MI; i++)
            #pragma unroll
            for (int j = 0; j < NI; j++) {
                if (nw_four(P)) low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[i], bl[j], low[i][j], 0, 0, 0);
                low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bl[j], low[i][j], 0, 0, 0);
                low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[i], bh[j], low[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bh[j], acc[i][j], 0, 0, 0);
            }
    }
    ns_join(acc, low);
    return true;
}

// What a symmetric P x P product's tiles hold at (i, j) goes to row j, where a
// lane's four i are consecutive: put(row, col, values).
template <int P, int MI, int NI, typename F>
__device__ __forceinline__ void nw_tiles(const f32x4 (&acc)[MI][NI], F &&put)
{
    using N = Nw<P>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane / 16, q = lane % 16;
    const int wm = wave / N::WN, wn = wave % N::WN;
    #pragma unroll
    for (int i = 0; i < MI; i++)
        #pragma unroll
        for (int j = 0; j < NI; j++) put(wn * N::TN + j * 16 + q, wm * N::TM + i * 16 + 4 * g, acc[i][j]);
}

// The block in LDS to the workspace, and its partial Gram matrix; the stores
// (64 KiB, 2.5 us at what a CU writes) go out between the product's steps.
template <int P>
__device__ __forceinline__ void nw_leave(const NsDev &d, int block, const h16 *xs, float *part)
{
    using N = Nw<P>;
    constexpr int XL = kBlock * 4 / 16 / kNwThreads, STEPS = N::QB / 32, EACH = (XL + STEPS - 1) / STEPS;
    const int tid = threadIdx.x;
    h16 *out = d.xt[0] + (int64_t)block * kBlock * 2;
    auto store = [&](int l) __attribute__((always_inline)) {
        const int v = l * kNwThreads + tid, row = v / (P / 4), c = v % (P / 4);
        gst(out + (int64_t)v * 8, *reinterpret_cast<const u32x4 *>(xs + row * N::XP + c * 8));
    };
    constexpr int MI = N::TM / 16, NI = N::TN / 16;
    f32x4 acc[MI][NI];
    float *o = part + (int64_t)block * P * P;
    const bool has = nw_gram<P>(xs, STEPS, acc, [&](int k) __attribute__((always_inline)) {
        #pragma unroll
        for (int e = 0; e < EACH; e++)
            if (k * EACH + e < XL) store(k * EACH + e);
    });
    if (has) {
        // in the order of the fragments, [wave][block][lane]: the next step's waves take the same tiles
        #pragma unroll
        for (int i = 0; i < MI; i++)
            #pragma unroll
            for (int j = 0; j < NI; j++) gst(o + (((tid >> 6) * MI * NI + i * NI + j) * 64 + (tid & 63)) * 4, acc[i][j]);
    } else {
        for (int l = 0; l < XL; l++) store(l);
    }
}

// Stage 2 of a narrow matrix: X's block as pairs, and its partial Gram matrix.
template <int P, typename T>
__device__ __forceinline__ void nw_prepare(const NsDev &d, int block, const NsStep &s, h16 *xs, double *red)
{
    using N = Nw<P>;
    const int tid = threadIdx.x, j0 = block * N::QB;
    const float scale = ns_factor<kNwThreads>(d, s.eps, red);
    // e runs along the caller's rows: over P where X is its transpose, else over the block's columns
    constexpr int U = 8;
    for (int e0 = tid; e0 < kBlock; e0 += U * kNwThreads) {
        float u[U];
        #pragma unroll
        for (int k = 0; k < U; k++) {
            const int e = e0 + k * kNwThreads;
            const int i = d.flip ? e % P : e / N::QB, j = d.flip ? e / P : e % N::QB;
            const bool in = i < d.p && j0 + j < d.q;
            const int64_t r = in ? (d.flip ? j0 + j : i) : 0, c = in ? (d.flip ? i : j0 + j) : 0;
            const float g = ns_load<T>(d.in.src, r * d.in.ld_src + c);
            const float b = s.update ? gld<float>(d.in.buf + r * d.in.ld_buf + c) : 0.f;
            u[k] = in ? ns_u(g, b, s) : 0.f;
        }
        #pragma unroll
        for (int k = 0; k < U; k++) {
            const int e = e0 + k * kNwThreads;
            const int i = d.flip ? e % P : e / N::QB, j = d.flip ? e / P : e % N::QB;
            h16 hi, lo;
            ns_pair(u[k] * scale, hi, lo);
            h16 *o = xs + j * N::XP + nw_k(i);
            o[0] = hi;
            o[32] = lo;
        }
    }
    __syncthreads();
    nw_leave<P>(d, block, xs, d.part[0]);
}

// G's pairs into LDS from the wave's tile of it (raw: S^2 times G, as the
// product leaves it), and its third parts behind them (nw_third).
template <int P, int MI, int NI>
__device__ __forceinline__ void nw_put(h16 *gs, const f32x4 (&raw)[MI][NI])
{
    using N = Nw<P>;
    nw_tiles<P>(raw, [&](int row, int col, const f32x4 &v) {
        float f[4] = {v[0] * kInvS, v[1] * kInvS, v[2] * kInvS, v[3] * kInvS};
        h16 *o = gs + row * N::GP + nw_k(col);
        nw_store4(o, f);
        if constexpr (nw_third(P)) {
            const f16x4 hi = *reinterpret_cast<const f16x4 *>(o), lo = *reinterpret_cast<const f16x4 *>(o + 32);
            f16x4 m;
            #pragma unroll
            for (int e = 0; e < 4; e++) m[e] = (_Float16)(f[e] - (float)hi[e] - (float)lo[e]);
            *reinterpret_cast<f16x4 *>(gs + P * N::GP + row * N::MP + col) = m;
        }
    });
}

// R = a I + b G + c G G over G's place in LDS; raw: this wave's tile of G as in
// nw_put (has: it has one).  Starts after a barrier, ends with one.
template <int P, int MI, int NI>
__device__ __forceinline__ void nw_polynomial(const NsStep &s, h16 *gs, bool has, const f32x4 (&raw)[MI][NI])
{
    using N = Nw<P>;
    const int lane = threadIdx.x & 63, g = lane / 16, q = lane % 16;
    const int wave = threadIdx.x >> 6, wm = wave / N::WN, wn = wave % N::WN;
    f32x4 acc[MI][NI];
    ns_zero(acc);
    const h16 *gm = gs + P * N::GP;
    if (has) nw_product<MI, NI, P / 32, nw_third(P)>(gs + wm * N::TM * N::GP, N::GP, gs + wn * N::TN * N::GP, N::GP, acc,
                                                    gm + wm * N::TM * N::MP, gm + wn * N::TN * N::MP, N::MP);
    __syncthreads();
    if (has)
        #pragma unroll
        for (int i = 0; i < MI; i++)
            #pragma unroll
            for (int j = 0; j < NI; j++) {
                const int row = wn * N::TN + j * 16, col = wm * N::TM + i * 16;
                float v[4];
                #pragma unroll
                for (int e = 0; e < 4; e++) v[e] = __builtin_fmaf(s.c, acc[i][j][e], s.b * raw[i][j][e]) * kInvS;
                if (row == col)                  // a block of the diagonal
                    #pragma unroll
                    for (int e = 0; e < 4; e++) v[e] += q == 4 * g + e ? s.a * kS : 0.f;
                nw_store4(gs + (row + q) * N::GP + nw_k(col + 4 * g), v);
            }
    __syncthreads();
}

// Y = R X of the block: this wave's YM x YN tile.
template <int P, int MI, int NI>
__device__ __forceinline__ void nw_apply(const h16 *xs, const h16 *gs, f32x4 (&acc)[MI][NI])
{
    using N = Nw<P>;
    const int wave = threadIdx.x >> 6, ym = wave / N::YWN * N::YM, yn = wave % N::YWN * N::YN;
    ns_zero(acc);
    nw_product<MI, NI, P / 32>(gs + ym * N::GP, N::GP, xs + yn * N::XP, N::XP, acc);
}
// Y over X's place.  The caller has had a barrier since the last read of X.
template <int P, int MI, int NI>
__device__ __forceinline__ void nw_keep(h16 *xs, const f32x4 (&acc)[MI][NI])
{
    using N = Nw<P>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane / 16, q = lane % 16;
    const int ym = wave / N::YWN * N::YM, yn = wave % N::YWN * N::YN;
    #pragma unroll
    for (int i = 0; i < MI; i++)
        #pragma unroll
        for (int j = 0; j < NI; j++) {
            float v[4];
            #pragma unroll
            for (int e = 0; e < 4; e++) v[e] = acc[i][j][e] * kInvS;
            nw_store4(xs + (yn + j * 16 + q) * N::XP + nw_k(ym + i * 16 + 4 * g), v);
        }
}
// Y into the caller's matrix, through X's place so that rows are written whole
// (the same barrier as above).
template <int P, typename W, int MI, int NI>
__device__ __forceinline__ void nw_result(const NsDev &d, int block, const NsStep &s, h16 *xs, const f32x4 (&acc)[MI][NI])
{
    using N = Nw<P>;
    constexpr int FP = P + 1;
    static_assert(N::QB * FP * 4 <= N::XBytes, "the results fit the block's place");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane / 16, q = lane % 16;
    const int ym = wave / N::YWN * N::YM, yn = wave % N::YWN * N::YN;
    float *fs = (float *)xs;
    #pragma unroll
    for (int i = 0; i < MI; i++)
        #pragma unroll
        for (int j = 0; j < NI; j++)
            #pragma unroll
            for (int e = 0; e < 4; e++)
                fs[(yn + j * 16 + q) * FP + ym + i * 16 + 4 * g + e] = acc[i][j][e] * (kInvS * kInvS);
    __syncthreads();
    const float lr = ns_rate(s);
    const int j0 = block * N::QB;
    #pragma unroll 4
    for (int e = tid; e < kBlock; e += kNwThreads) {
        const int i = d.flip ? e % P : e / N::QB, j = d.flip ? e / P : e % N::QB;
        if (i < d.p && j0 + j < d.q)
            ns_result<W>(d.in, s, lr, d.flip ? j0 + j : i, d.flip ? i : j0 + j, fs[j * FP + i]);
    }
}

template <int P, bool LAST, typename W>
__device__ __forceinline__ void nw_step(const NsDev &d, int block, const NsStep &s, int turn, h16 *xs)
{
    using N = Nw<P>;
    const int tid = threadIdx.x;
    h16 *gs = xs + N::QB * N::XP;
    // the block and the partial sums, all loads before the first use
    constexpr int XL = kBlock * 4 / 16 / kNwThreads;
    u32x4 xv[XL];
    const h16 *xin = d.xt[0] + (int64_t)block * kBlock * 2;
    #pragma unroll
    for (int l = 0; l < XL; l++) xv[l] = gld<u32x4>(xin + (int64_t)(l * kNwThreads + tid) * 8);
    const bool summed = ns_summed(d.blocks, P);
    const float *part = summed ? d.sum : d.part[turn];
    const int np = summed ? 1 : d.blocks;
    constexpr int MI = N::TM / 16, NI = N::TN / 16;
    const int lane = tid & 63, wave = tid >> 6;
    const bool has = wave / N::WN * N::TM < P;
    f32x4 raw[MI][NI];                           // this wave's tile of G, summed over the blocks
    ns_zero(raw);
    if (has) {
        const float *from = part + (wave * MI * NI * 64 + lane) * 4;
        #pragma unroll (P == 128 ? 1 : 4)        // (a tile of 128's G is 32 registers: 98 us against 94 unrolled)
        for (int b = 0; b < np; b++)
            #pragma unroll
            for (int i = 0; i < MI; i++)
                #pragma unroll
                for (int j = 0; j < NI; j++) {
                    const f32x4 w = gld<f32x4>(from + (int64_t)b * P * P + (i * NI + j) * 256);
                    raw[i][j][0] += w[0]; raw[i][j][1] += w[1]; raw[i][j][2] += w[2]; raw[i][j][3] += w[3];
                }
    }
    #pragma unroll
    for (int l = 0; l < XL; l++) {
        const int v = l * kNwThreads + tid, row = v / (P / 4), c = v % (P / 4);
        *reinterpret_cast<u32x4 *>(xs + row * N::XP + c * 8) = xv[l];
    }
    if (has) nw_put<P>(gs, raw);
    __syncthreads();
    nw_polynomial<P>(s, gs, has, raw);
    f32x4 acc[N::YM / 16][N::YN / 16];
    nw_apply<P>(xs, gs, acc);
    __syncthreads();
    if constexpr (!LAST) {
        nw_keep<P>(xs, acc);
        __syncthreads();
        nw_leave<P>(d, block, xs, d.part[turn ^ 1]);
    } else {
        nw_result<P, W>(d, block, s, xs, acc);
    }
}

// A matrix of one block, all of it in one workgroup: momentum, norm, every step
// and the result, X and G in LDS throughout.
template <int P, typename T, typename W>
__device__ __forceinline__ void nw_tiny(const NsDev &d, const NsStep &s, h16 *xs, double *red)
{
    using N = Nw<P>;
    const int tid = threadIdx.x;
    h16 *gs = xs + N::QB * N::XP;
    constexpr int U = kBlock / kNwThreads;
    float u[U], b[U];
    auto at = [&](int k, int &i, int &j) __attribute__((always_inline)) {
        const int e = tid + k * kNwThreads;      // along the caller's rows
        i = d.flip ? e % P : e / N::QB;
        j = d.flip ? e / P : e % N::QB;
        return i < d.p && j < d.q;
    };
    #pragma unroll
    for (int k = 0; k < U; k++) {
        int i, j;
        const bool in = at(k, i, j);
        const int64_t r = in ? (d.flip ? j : i) : 0, c = in ? (d.flip ? i : j) : 0;
        u[k] = ns_load<T>(d.in.src, r * d.in.ld_src + c);
        b[k] = s.update ? gld<float>(d.in.buf + r * d.in.ld_buf + c) : 0.f;
    }
    double sum = 0.0;
    #pragma unroll
    for (int k = 0; k < U; k++) {
        int i, j;
        if (!at(k, i, j)) {
            u[k] = 0.f;
            continue;
        }
        if (s.update) {
            b[k] = __builtin_fmaf(s.momentum, b[k], u[k]);
            gst(d.in.buf + (int64_t)(d.flip ? j : i) * d.in.ld_buf + (d.flip ? i : j), b[k]);
        }
        u[k] = ns_u(u[k], b[k], s);
        sum += (double)u[k] * (double)u[k];
    }
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (tid % 64 == 0) red[tid / 64] = sum;
    __syncthreads();
    sum = red[0];
    for (int w = 1; w < kNwThreads / 64; w++) sum += red[w];
    const float scale = (float)((double)kS / (sqrt(sum) + (double)s.eps));
    #pragma unroll
    for (int k = 0; k < U; k++) {
        int i, j;
        at(k, i, j);
        h16 hi, lo;
        ns_pair(u[k] * scale, hi, lo);
        h16 *o = xs + j * N::XP + nw_k(i);
        o[0] = hi;
        o[32] = lo;
    }
    __syncthreads();
    const int columns = (d.q + 31) / 32;
    for (int k = 0; k < s.steps; k++) {
        f32x4 gram[N::TM / 16][N::TN / 16];
        const bool has = nw_gram<P>(xs, columns, gram, [](int) {});
        if (has) nw_put<P>(gs, gram);
        __syncthreads();
        nw_polynomial<P>(s, gs, has, gram);
        f32x4 acc[N::YM / 16][N::YN / 16];
        nw_apply<P>(xs, gs, acc);
        __syncthreads();
        if (k + 1 < s.steps) {
            nw_keep<P>(xs, acc);
            __syncthreads();
        } else {
            nw_result<P, W>(d, 0, s, xs, acc);
        }
    }
}

enum { NW_PREPARE = 0, NW_STEP = 1, NW_LAST = 2 };

// T: the source type (NW_PREPARE) or the result type (NW_LAST)
template <int STAGE, typename T>
__global__ __launch_bounds__(kNwThreads) void k_ns_narrow(NsTable t, int count, NsStep s, int turn)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ double red[kNwThreads / 64];
    h16 *xs = (h16 *)smem;
    const int work = xcd_remap(blockIdx.x, gridDim.x);
    const int it = ns_find(t.pre[PRE_NARROW], count, work);
    const NsDev &d = t.items[it];
    const int block = work - t.pre[PRE_NARROW][it];
    auto go = [&](auto tag) __attribute__((always_inline)) {
        constexpr int P = decltype(tag)::value;
        if constexpr (STAGE == NW_PREPARE) nw_prepare<P, T>(d, block, s, xs, red);
        else nw_step<P, STAGE == NW_LAST, T>(d, block, s, turn, xs);
    };
    if (d.P == 128) go(std::integral_constant<int, 128>{});
    else if (d.P == 64) go(std::integral_constant<int, 64>{});
    else go(std::integral_constant<int, 32>{});
}

// T: source type, W: result type
template <typename T, typename W>
__global__ __launch_bounds__(kNwThreads) void k_ns_tiny(NsTable t, int count, NsStep s)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ double red[kNwThreads / 64];
    const int it = ns_find(t.pre[PRE_TINY], count, blockIdx.x);
    const NsDev &d = t.items[it];
    if (d.P == 128) nw_tiny<128, T, W>(d, s, (h16 *)smem, red);
    else if (d.P == 64) nw_tiny<64, T, W>(d, s, (h16 *)smem, red);
    else nw_tiny<32, T, W>(d, s, (h16 *)smem, red);
}

// The sum of a narrow matrix's partial Gram matrices: 64 float4 outputs a
// workgroup, each added by four threads over a quarter of the blocks.
__global__ __launch_bounds__(kThreads) void k_ns_sum(NsTable t, int count, int turn)
{
    __shared__ f32x4 red[kThreads];
    const int it = ns_find(t.pre[PRE_SUM], count, blockIdx.x);
    const NsDev &d = t.items[it];
    const int w = blockIdx.x - t.pre[PRE_SUM][it], tid = threadIdx.x;
    const int64_t pp = (int64_t)d.P * d.P;
    const float *src = d.part[turn] + ((int64_t)w * 64 + tid % 64) * 4;
    const int quarter = tid / 64;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    #pragma unroll 4
    for (int b = quarter; b < d.blocks; b += 4) {
        const f32x4 v = gld<f32x4>(src + b * pp);
        acc[0] += v[0]; acc[1] += v[1]; acc[2] += v[2]; acc[3] += v[3];
    }
    red[tid] = acc;
    __syncthreads();
    if (tid < 64) {
        f32x4 o = red[tid];
        for (int k = 1; k < 4; k++)
            for (int e = 0; e < 4; e++) o[e] += red[k * 64 + tid][e];
        gst(d.sum + ((int64_t)w * 64 + tid) * 4, o);
    }
}

size_t table_bytes(int count)
{
    const size_t a = (size_t)count * sizeof(NsDev), b = (size_t)count * kPre * sizeof(int);
    return (a + b + 255) / 256 * 256;
}

constexpr int ns_slots(int bt) { return bt == 128 ? kNsSlots : kNsSlots / 2; }
int64_t cut_bytes(const NsCut &c) { return c.pieces > 1 ? (int64_t)(c.tiles - c.whole) * c.pieces * c.bt * c.bt * 4 : 0; }

// The time of a stage in us as measured (kernel traces of 256 x 256 to
// 4096 x 4096, alone and in lists; before the smaller products had sums of their
// own, which add 0 to 3 %): the launch, and per round of workgroups a
// part for finding the matrix, the first loads and leaving the results, and a
// part per k step, which depends on whether the CUs are shared; for cut tiles the
// launch that adds the pieces.  Measured, tiles of 32, 64, 128, 256:
//   256 x 256, X X^T (8 steps)      4.7    6.8   13.3         12.8 + 4.0
//   512 x 512 (16 steps)            6.0    8.8    8.6 + 4.6   13.3 + 5.2
//   1024 x 1024 (32 steps)         17.2   12.0   12.1 + 6.4   20.0 + 6.5
//   four 2048 x 2048, R X (64)      703    380    214          164
double cut_time(const NsCut &c, int steps)
{
    const int slots = ns_slots(c.bt), rest = c.tiles - c.whole;
    if (c.bt <= 64) {
        const int rounds = (c.tiles + slots - 1) / slots;
        return c.bt == 32 ? 2.5 + rounds * (1.3 + steps * (rounds > 1 ? 0.15 : 0.09))
                          : 3.0 + rounds * (2.0 + steps * (rounds > 1 ? 0.31 : 0.19));
    }
    const double step = c.bt == 128 ? 1.5 : 2.35, alone = c.bt == 128 ? 0.8 : 2.0, leave = c.bt == 128 ? 9.0 : 14.0;
    const int units = rest * c.pieces;
    double t = 2.0 + c.whole / slots * (leave + step * steps);
    if (units) t += leave + (steps + c.pieces - 1) / c.pieces * (units * 2 <= slots ? alone : step);
    if (c.pieces > 1) t += 4.5 + cut_bytes(c) * 0.23e-6;
    return t;
}

// The tile and the cut of a stage: tiles are counted over the whole list, steps
// are those of the longest product.  Small tiles spread the operands of few
// products over many CUs; large ones read and stage fewer bytes a product.
NsCut ns_stage(const NsPlan &p, int sym, int steps)
{
    NsCut best{};
    double least = 1e30;
    for (int bt = 32; bt <= 256; bt *= 2) {
        const int tiles = (int)p.work[ns_gram_stage(bt) + !sym];
        if (tiles > kNsMaxGrid && bt < 256) continue;
        const int rest = tiles % ns_slots(bt), most = bt <= 64 || !rest ? 1 : ns_slots(bt) / rest;
        for (int pieces = 1; pieces <= most && (pieces == 1 || pieces * 4 <= steps); pieces += (pieces + 3) / 4) {
            const NsCut c{bt, tiles, bt <= 64 ? tiles : tiles - rest, pieces, nullptr};
            const double t = cut_time(c, steps);
            if (t < least) {
                least = t;
                best = c;
            }
        }
    }
    if (best.pieces == 1) best.whole = best.tiles;
    return best;
}

struct NsCuts { NsCut gram, square, apply; };
NsCuts ns_cuts(const NsPlan &p)
{
    return NsCuts{ns_stage(p, 1, p.long_side / 32), ns_stage(p, 1, p.short_side / 32), ns_stage(p, 0, p.short_side / 32)};
}

}  // namespace

void ns_plan_add(NsPlan &p, int rows, int cols)
{
    // Single-block matrices run whole (128 x 128: 57 us against 85 in a launch a
    // step), unless the list has narrow matrices of several blocks: those take a
    // launch a step anyway, and the others ride along (dense block 1's filters:
    // 105 us against 163 with a launch of their own first).
    const NsSize z = ns_size(rows, cols, !p.stepwise);
    if (z.blocks > 1 && !p.stepwise) {
        p.stepwise = 1;
        for (int k = 0; k < kPre; k++) p.work[k] += p.ride_work[k];
        p.work[PRE_TINY] = 0;
        p.bytes += p.ride_bytes;
    }
    p.count++;
    p.bytes += z.bytes;
    for (int k = 0; k < kPre; k++) p.work[k] += z.work[k];
    if (z.work[PRE_TINY]) {
        const NsSize r = ns_size(rows, cols, 0);
        p.ride_bytes += r.bytes;
        for (int k = 0; k < kPre; k++) p.ride_work[k] += r.work[k];
    }
    (z.blocks ? p.narrow_flops : p.flops) += (double)z.p * (z.p + 1) * z.q + (double)z.p * z.p * (z.p + 1) + 2.0 * z.p * z.p * z.q;
    p.values += (double)rows * cols;
    if (z.blocks) return;
    if (z.P > p.short_side) p.short_side = z.P;
    if (z.Q > p.long_side) p.long_side = z.Q;
}

bool ns_plan_fits(const NsPlan &p)
{
    for (int k = 0; k < kPre; k++) {
        const bool choice = k == PRE_GRAM || k == PRE_APPLY || k >= PRE_GRAM_S;      // larger tiles can take it
        if (p.work[k] > (choice && k != PRE_TINY ? (int64_t)1 << 30 : kNsMaxGrid)) return false;
    }
    return true;
}

size_t ns_plan_bytes(const NsPlan &p)
{
    const NsCuts c = ns_cuts(p);
    int64_t part = 0;
    for (const NsCut *k : {&c.gram, &c.square, &c.apply}) part = cut_bytes(*k) > part ? cut_bytes(*k) : part;
    return table_bytes(p.count) + (size_t)p.bytes + (size_t)part;
}

namespace {

NsTable ns_table(void *ws, int count)
{
    NsTable t;
    t.items = (NsDev *)ws;
    int *pre = (int *)((char *)ws + (size_t)count * sizeof(NsDev));
    for (int k = 0; k < kPre; k++) t.pre[k] = pre + (size_t)k * count;
    return t;
}

template <int BT, int MODE, typename W>
hipError_t ns_product_bt(const NsPlan &p, const NsTable &t, const NsStep &s, int turn, const NsCut &cut, hipStream_t st)
{
    const int rest = cut.tiles - cut.whole;
    {
        TraceScope tr(KC_CONV, KID_ORTHO, st, 0.0, ns_sym(MODE) ? 0.0 : p.flops);
        const int units = cut.whole + rest * cut.pieces;
        hipLaunchKernelGGL((k_ns_product<BT, MODE, W>), dim3((unsigned)units), dim3(BT * 2), 0, st, t, p.count, s, turn, cut);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (cut.pieces == 1) return hipSuccess;
    TraceScope tr(KC_SMALL, KID_ORTHO, st, (double)cut_bytes(cut), 0.0);
    hipLaunchKernelGGL((k_ns_finish<BT, MODE, W>), dim3((unsigned)rest * (BT * BT / (kSub * kSub))), dim3(256), 0, st, t,
                       p.count, s, turn, cut);
    return hipGetLastError();
}
template <int MODE, typename W>
hipError_t ns_product(const NsPlan &p, const NsTable &t, const NsStep &s, int turn, const NsCut &cut, hipStream_t st)
{
    if (cut.bt == 128) return ns_product_bt<128, MODE, W>(p, t, s, turn, cut, st);
    if (cut.bt == 256) return ns_product_bt<256, MODE, W>(p, t, s, turn, cut, st);
    TraceScope tr(KC_CONV, KID_ORTHO, st, 0.0, ns_sym(MODE) ? 0.0 : p.flops);
    if (cut.bt == 64) hipLaunchKernelGGL((k_ns_direct<64, MODE, W>), dim3((unsigned)cut.tiles), dim3(256), 0, st, t, p.count, s, turn);
    else hipLaunchKernelGGL((k_ns_direct<32, MODE, W>), dim3((unsigned)cut.tiles), dim3(256), 0, st, t, p.count, s, turn);
    return hipGetLastError();
}

// Lets a kernel take kNwLds bytes of LDS, more than the default limit, on the current device.
template <typename K>
hipError_t allow_lds(K kern, std::atomic<uint64_t> &ready)
{
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (ready.load(std::memory_order_relaxed) & bit) return hipSuccess;
    if (hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kNwLds)) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
    return hipSuccess;
}

template <typename T, typename W>
hipError_t ns_tiny(const NsPlan &p, const NsTable &t, const NsStep &s, hipStream_t st)
{
    auto kern = k_ns_tiny<T, W>;
    static std::atomic<uint64_t> ready{0};       // one bit per device
    if (hipError_t e = allow_lds(kern, ready)) return e;
    TraceScope tr(KC_CONV, KID_ORTHO, st, 0.0, 0.0);
    hipLaunchKernelGGL(kern, dim3((unsigned)p.work[PRE_TINY]), dim3(kNwThreads), kNwLds, st, t, p.count, s);
    return hipGetLastError();
}

// one stage of the narrow matrices
template <int STAGE, typename T>
hipError_t ns_narrow(const NsPlan &p, const NsTable &t, const NsStep &s, int turn, hipStream_t st)
{
    auto kern = k_ns_narrow<STAGE, T>;
    static std::atomic<uint64_t> ready{0};       // one bit per device
    if (hipError_t e = allow_lds(kern, ready)) return e;
    TraceScope tr(KC_CONV, KID_ORTHO, st, 0.0, STAGE == NW_PREPARE ? 0.0 : p.narrow_flops);
    hipLaunchKernelGGL(kern, dim3((unsigned)p.work[PRE_NARROW]), dim3(kNwThreads), kNwLds, st, t, p.count, s, turn);
    return hipGetLastError();
}

// the sums in front of a narrow step, where a matrix has many blocks
hipError_t ns_sum(const NsPlan &p, const NsTable &t, int turn, hipStream_t st)
{
    if (!p.work[PRE_SUM]) return hipSuccess;
    TraceScope tr(KC_SMALL, KID_ORTHO, st, 0.0, 0.0);
    hipLaunchKernelGGL(k_ns_sum, dim3((unsigned)p.work[PRE_SUM]), dim3(kThreads), 0, st, t, p.count, turn);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ns(const NsPlan &p, NsFill fill, const void *arg, const NsStep &s, int src_dtype, int dst_dtype,
                     void *ws, hipStream_t st)
{
    const NsTable t = ns_table(ws, p.count);
    NsChunk c;
    c.whole = !p.stepwise;
    c.at = (int64_t)table_bytes(p.count);
    for (int k = 0; k < kPre; k++) c.work[k] = 0;
    for (c.first = 0; c.first < p.count; c.first += kNsChunk) {
        c.count = p.count - c.first < kNsChunk ? p.count - c.first : kNsChunk;
        for (int i = 0; i < c.count; i++) c.in[i] = fill(arg, c.first + i);
        TraceScope tr(KC_SMALL, KID_ORTHO, st, (double)c.count * sizeof(NsDev), 0.0);
        hipLaunchKernelGGL(k_ns_table, dim3(1), dim3(64), 0, st, c, t, (char *)ws);
        if (hipError_t e = hipGetLastError()) return e;
        for (int i = 0; i < c.count; i++) {
            const NsSize z = ns_size(c.in[i].rows, c.in[i].cols, c.whole);
            c.at += z.bytes;
            for (int k = 0; k < kPre; k++) c.work[k] += z.work[k];
        }
    }
    if (p.work[PRE_TINY]) {
        const bool b = dst_dtype == DT_BF16;
        const hipError_t e = src_dtype == DT_BF16 ? (b ? ns_tiny<bf16_t, bf16_t>(p, t, s, st) : ns_tiny<bf16_t, float>(p, t, s, st))
                                                  : (b ? ns_tiny<float, bf16_t>(p, t, s, st) : ns_tiny<float, float>(p, t, s, st));
        if (e != hipSuccess) return e;
    }
    if (!p.work[PRE_SQ]) return hipSuccess;
    const double es = src_dtype == DT_BF16 ? 2.0 : 4.0;
    {
        TraceScope tr(KC_SWEEP, KID_ORTHO, st, p.values * (es + (s.update ? 8.0 : 0.0)), 0.0);
        auto kern = src_dtype == DT_BF16 ? k_ns_squares<bf16_t> : k_ns_squares<float>;
        hipLaunchKernelGGL(kern, dim3((unsigned)p.work[PRE_SQ]), dim3(kThreads), 0, st, t, p.count, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (p.work[PRE_NARROW]) {
        hipError_t e = src_dtype == DT_BF16 ? ns_narrow<NW_PREPARE, bf16_t>(p, t, s, 0, st)
                                            : ns_narrow<NW_PREPARE, float>(p, t, s, 0, st);
        for (int k = 0, turn = 0; k < s.steps && e == hipSuccess; k++, turn ^= 1) {
            e = ns_sum(p, t, turn, st);
            if (e != hipSuccess) break;
            if (k + 1 < s.steps) e = ns_narrow<NW_STEP, float>(p, t, s, turn, st);
            else if (dst_dtype == DT_BF16) e = ns_narrow<NW_LAST, bf16_t>(p, t, s, turn, st);
            else e = ns_narrow<NW_LAST, float>(p, t, s, turn, st);
        }
        if (e != hipSuccess) return e;
    }
    if (!p.work[PRE_GRAM]) return hipSuccess;
    {
        TraceScope tr(KC_SWEEP, KID_ORTHO, st, p.values * (es + (s.update ? 4.0 : 0.0) + 8.0), 0.0);
        auto kern = src_dtype == DT_BF16 ? k_ns_prepare<bf16_t> : k_ns_prepare<float>;
        hipLaunchKernelGGL(kern, dim3((unsigned)p.work[PRE_PREP]), dim3(kThreads), 0, st, t, p.count, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    NsCuts cuts = ns_cuts(p);
    float *part = (float *)((char *)ws + table_bytes(p.count) + p.bytes);
    for (NsCut *k : {&cuts.gram, &cuts.square, &cuts.apply}) k->part = part;
    for (int k = 0, turn = 0; k < s.steps; k++, turn ^= 1) {
        hipError_t e = ns_product<NS_GRAM, float>(p, t, s, turn, cuts.gram, st);
        if (e == hipSuccess) e = ns_product<NS_SQUARE, float>(p, t, s, turn, cuts.square, st);
        if (e == hipSuccess) {
            if (k + 1 < s.steps) e = ns_product<NS_APPLY, float>(p, t, s, turn, cuts.apply, st);
            else if (dst_dtype == DT_BF16) e = ns_product<NS_LAST, bf16_t>(p, t, s, turn, cuts.apply, st);
            else e = ns_product<NS_LAST, float>(p, t, s, turn, cuts.apply, st);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace bnr
