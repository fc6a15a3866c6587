// linear_ce.hip -- the last linear layer and its softmax cross entropy over many
// classes, whose logits are never kept, and its gradients.
//
//   l[i][v] = sum_k h[i][k] w[v][k] + bias[v],   lse[i] = log sum_v exp l[i][v]
//   loss[i] = lse - (1 - s) l[i][label] - (s / V) sum_v l[i][v] + z lse^2
//   g[i][v] = r[i] (exp(l - lse) (1 + 2 z lse) - (1 - s) [v = label] - s / V)
//   dh = g w,  dw = g^T h,  dbias = column sums of g
//
// r[i] is the loss's gradient (1 / rows that count for the mean).  Rows of the
// ignored label are left out of every product: the first launch (k_ce_list) copies
// the rows that count together, so padding costs nothing and what stands in it
// reaches nothing.
//
// Forward: one matrix product whose tiles never leave the registers as logits; a
// tile's epilogue gives each row's maximum and sum of exponentials over its columns,
// and k_ce_rows joins them.  Backward: the classes in pieces; a piece's logits are
// formed again, g is written in the storage type (the operand type of the two
// products that follow, as every stored gradient of this library), then the piece's
// rows of dw and its share of dh are formed.  dh adds up over pieces in float32.
//
// Every product is k_ce_gemm: C[i][j] = sum_k I[i][k] J[j][k] with operands that lie
// along k ("rows") or across it ("columns"); matrix instructions take the weights'
// side as their rows, so that a lane holds four neighbouring results of one row.
#include "common.hpp"
#include "kernels.hpp"
#include "mfma.hpp"
#include "trace.hpp"

#include <type_traits>

namespace bnr {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

// exp(x) by the base-2 instruction: its product's one rounding puts it off by about |x| 2^-24
// of itself, next to the c 2^-24 sum |h w| that the logits are off by (gradients of 128 x 1024
// x 1000 in float32: 4.9e-7 of their norm off float64, elementary float32 operations 3.6e-7).
__device__ __forceinline__ float ce_exp(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// A row's entry of g from its probability e
__device__ __forceinline__ float ce_g(float e, const CeRow &r, const CeGemm &p, bool label)
{
    return __builtin_fmaf(e, r.scale * (1.f + 2.f * p.z * r.lse), -r.scale * p.flat) - (label ? r.scale * p.hit : 0.f);
}

// ---- rows that count -------------------------------------------------------
constexpr int kListRows = 4;               // rows a workgroup of k_ce_list takes, one a wave
constexpr int kOwnRows = 128;              // rows a workgroup of k_ce_own takes at most
constexpr int kCountRows = 4096;           // rows a workgroup of k_ce_count takes

__device__ __forceinline__ int ce_counted(const int32_t *labels, int64_t from, int64_t to, int ignore, int tid)
{
    int n = 0;
    #pragma unroll 8
    for (int64_t i = from + tid; i < to; i += kThreads) n += labels[i] != ignore;
    return n;
}

__device__ __forceinline__ int ce_group_sum(int n, int *red, int tid)
{
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    if ((tid & 63) == 0) red[tid >> 6] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kThreads / 64; w++) n += red[w];
    return n;
}

__global__ __launch_bounds__(kThreads) void k_ce_count(CeList p)
{
    __shared__ int red[kThreads / 64];
    const int64_t from = (int64_t)blockIdx.x * kCountRows;
    const int n = ce_group_sum(ce_counted(p.labels, from, min(from + kCountRows, p.m), p.ignore, threadIdx.x), red, threadIdx.x);
    if (threadIdx.x == 0) p.counts[blockIdx.x] = n;
}

// The list of rows that count, in order, with what the products' epilogues need of
// each; their features copied together; zeros in the other rows' results.
__global__ __launch_bounds__(kThreads) void k_ce_list(CeList p)
{
    __shared__ int red[kThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t first = (int64_t)blockIdx.x * kListRows;
    int n = 0;
    int64_t from = 0;
    if (p.counts) {
        const int whole = (int)(first / kCountRows);
        for (int b = tid; b < whole; b += kThreads) n += p.counts[b];
        from = (int64_t)whole * kCountRows;
    }
    n += ce_counted(p.labels, from, first, p.ignore, tid);
    const int before = ce_group_sum(n, red, tid);
    // The gradient of the mean, dloss[0] / n, multiplies every g.  Its significand is kept
    // apart and multiplies the sums in float32: g's rounding to bf16 would otherwise shift
    // the many values that are the same (-1 / n at the labels of a model that knows
    // little yet) by the same error.
    float mean = 0.f, factor = 1.f;
    if (p.lse) {
        mean = (p.dloss ? p.dloss[0] : 1.f) / p.lse[0];
        const uint32_t bits = __float_as_uint(mean), exponent = bits >> 23 & 255;
        if (exponent && exponent < 255) factor = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
        if (tid == 0 && blockIdx.x == 0) *p.factor = factor;
    }
    const int64_t row = first + lane;
    const bool mine = lane < kListRows && row < p.m;
    const int label = mine ? p.labels[row] : p.ignore;
    const uint64_t here = __ballot(mine && label != p.ignore);
    if (wave == 0 && mine) {
        if (label != p.ignore) {
            CeRow r;
            r.row = (int)row;
            r.label = label;
            r.lse = r.scale = 0.f;
            if (p.lse) {
                r.lse = p.lse[1 + row];
                r.scale = (p.dloss ? mean + p.dloss[1 + row] : mean) / factor;
                if ((uint32_t)label >= (uint32_t)p.classes) r.scale = NAN;
            }
            p.rows[before + __popcll(here & ((1ull << lane) - 1))] = r;
        } else if (p.zero_loss) {
            p.zero_loss[1 + row] = 0.f;
            p.zero_lse[1 + row] = 0.f;
        }
    }
    if (tid == 0 && first + kListRows >= p.m) *p.count = before + __popcll(here);
    const int vecs = p.row_bytes / 16;
    for (int k = wave; k < kListRows; k += kThreads / 64) {
        if (first + k >= p.m) break;
        if (here >> k & 1) {
            const char *src = (const char *)p.h + (first + k) * p.h_ld;
            char *dst = (char *)p.copy + (int64_t)(before + __popcll(here & ((1ull << k) - 1))) * p.row_bytes;
            #pragma unroll 4
            for (int i = lane; i < vecs; i += 64) stg16(dst + i * 16, ldg16(src + i * 16));
        } else if (p.zero) {
            char *dst = (char *)p.zero + (first + k) * p.zero_ld;
            for (int i = lane; i < vecs; i += 64) stg16(dst + i * 16, zero16());
        }
    }
}

// ---- the product -----------------------------------------------------------
// Operand tiles in LDS, 128 bytes for each of a stage's rows or columns:
//   rows     B rows of 128 bytes along k, as 16-byte chunks in the order
//            chunk ^ (row / 2 % 8), so that 16 rows of one chunk lie in different banks
//   columns  the stage's k one after another, B values each; in bf16 the chunks of a
//            k in the order chunk ^ 2 (k % 4 + 4 (k / 8 % 2)), for the transposing reads
// The order is made by the addresses that the lanes load straight into LDS from.
template <typename T, int B, int NT, bool COLS>
struct CeLoad {
    static constexpr int kLoads = B * 128 / (NT * 16), BK = 128 / sizeof(T);
    // a thread's loads lie kStep rows (k) apart; the order repeats every 16
    static constexpr uint32_t kRow = COLS ? B * sizeof(T) : 128, kStep = NT * 16 / kRow;
    static_assert(kStep % (COLS ? (sizeof(T) == 2 ? 8 : 1) : 16) == 0, "two places at most");
    uint32_t off, odd, at;                         // of even loads, of odd ones; at: the chunk's place along k (rows)
    __device__ __forceinline__ void init(int64_t ld, int tid)
    {
        const uint32_t row = tid * 16 / kRow, slot = tid * 16 % kRow / 16;
        const uint32_t turn = COLS ? (sizeof(T) == 2 ? 2 * (row % 4 + 4 * (row / 8 % 2)) : 0) : row / 2 % 8;
        at = COLS ? 0 : (slot ^ turn) * 16;
        off = row * (uint32_t)ld + (slot ^ turn) * 16;
        odd = COLS && sizeof(T) == 2 && kStep % 16 ? row * (uint32_t)ld + (slot ^ turn ^ 8) * 16 : off;
    }
    // stage `k0` of an operand whose tile starts at base, with `extent` rows (columns) left;
    // past k no address is read and zeros arrive
    struct Stage { const char *src; uint32_t bytes, o, odd, step; };
    __device__ __forceinline__ Stage stage(const char *base, int64_t ld, int extent, int k0, int k) const
    {
        const int left = min(k - k0, BK), wide = min(extent, B);
        const char *src = base + (COLS ? k0 * ld : k0 * (int64_t)sizeof(T));
        // (c is a multiple of the 16-byte vector, and g's rows are whole vectors: a column tile's last vector is read whole)
        const int bytes = COLS ? (left - 1) * (int)ld + (wide * (int)sizeof(T) + 15) / 16 * 16
                               : (wide - 1) * (int)ld + left * (int)sizeof(T);
        Stage s;
        s.src = src;
        s.bytes = __builtin_amdgcn_readfirstlane(left > 0 ? bytes : 0);
        s.o = off;
        s.odd = odd;
        if constexpr (!COLS) s.o = s.odd = (int)at < left * (int)sizeof(T) ? off : kBufOff;
        s.step = kStep * (uint32_t)ld;
        return s;
    }
    __device__ __forceinline__ void load(const Stage &s, unsigned char *lds, int l, int wave) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf_view(s.src, s.bytes),
                                                 (__attribute__((address_space(3))) void *)(lds + (l * NT + wave * 64) * 16),
                                                 16, (l % 2 ? s.odd : s.o) + l * s.step, 0, 0, 0);
    }
};

// Fragments of NB blocks of 16 rows (columns) from w0 on, of sub-step `sub` (64 bytes
// along k), read in NB parts.  Block b's lane value q stands for row 16 b + q, in float32 columns for
// NB q + b (a lane's neighbouring values, one read).
template <typename T, int B, int NB, bool COLS> struct CeFrags;
template <int B, int NB> struct CeFrags<bf16_t, B, NB, false> {
    uint32_t at;
    __device__ __forceinline__ void init(int w0, int lane) { at = (w0 + lane % 16) * 128; }
    __device__ __forceinline__ void read(const unsigned char *lds, int sub, int lane, bf16x8 *f, int part) const
    {
        f[part] = *reinterpret_cast<const bf16x8 *>(lds + at + ((sub * 4 + lane / 16) ^ (lane % 16 / 2)) * 16 + part * 2048);
    }
};
template <int B, int NB> struct CeFrags<float, B, NB, false> {
    uint32_t at;
    __device__ __forceinline__ void init(int w0, int lane) { at = (w0 + lane % 16) * 128; }
    __device__ __forceinline__ void read(const unsigned char *lds, int sub, int lane, f32x4 *f, int part) const
    {
        f[part] = *reinterpret_cast<const f32x4 *>(lds + at + ((sub * 4 + lane / 16) ^ (lane % 16 / 2)) * 16 + part * 2048);
    }
};
template <int B, int NB> struct CeFrags<bf16_t, B, NB, true> {
    static_assert(B >= 128, "the order of a k's chunks spans 256 bytes");
    uint32_t at[NB];
    __device__ __forceinline__ void init(int w0, int lane)
    {
        const uint32_t q = lane % 16, k = 8 * (lane / 16) + q / 4, turn = 2 * (k % 4 + 4 * (k / 8 % 2));
        #pragma unroll
        for (int b = 0; b < NB; b++) at[b] = k * (B * 2) + ((((w0 + 16 * b) / 8 + q % 4 / 2) ^ turn) * 16) + q % 2 * 8;
    }
    __device__ __forceinline__ void read(const unsigned char *lds, int sub, int lane, bf16x8 *f, int part) const
    {
        f[part] = tr_frag((const bf16_t *)(lds + at[part] + sub * 32 * B * 2), B);
    }
};
template <int B, int NB> struct CeFrags<float, B, NB, true> {
    static_assert(NB == 4 || NB == 2, "the blocks' values are one read");
    typedef __attribute__((ext_vector_type(NB))) float vec;
    uint32_t at;
    __device__ __forceinline__ void init(int w0, int lane) { at = 4 * (lane / 16) * (B * 4) + (w0 + NB * (lane % 16)) * 4; }
    __device__ __forceinline__ void read(const unsigned char *lds, int sub, int lane, f32x4 *f, int part) const
    {
        const vec v = *reinterpret_cast<const vec *>(lds + at + (sub * 16 + part) * (B * 4));
        #pragma unroll
        for (int b = 0; b < NB; b++) f[b][part] = v[b];
    }
};

__device__ __forceinline__ void ce_mma(f32x4 &c, bf16x8 a, bf16x8 b) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void ce_mma(f32x4 &c, f32x4 a, f32x4 b)
{
    #pragma unroll
    for (int t = 0; t < 4; t++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[t], b[t], c, 0, 0, 0);
}

template <int N, int M> __device__ __forceinline__ void ce_zero(f32x4 (&v)[N][M])
{
    #pragma unroll
    for (int b = 0; b < N; b++)
        #pragma unroll
        for (int a = 0; a < M; a++) v[b][a] = f32x4{0.f, 0.f, 0.f, 0.f};
}
// total += part, part = 0
template <int N, int M> __device__ __forceinline__ void ce_fold(f32x4 (&total)[N][M], f32x4 (&part)[N][M])
{
    #pragma unroll
    for (int b = 0; b < N; b++)
        #pragma unroll
        for (int a = 0; a < M; a++)
            #pragma unroll
            for (int r = 0; r < 4; r++) { total[b][a][r] += part[b][a][r]; part[b][a][r] = 0.f; }
}

// A wave's LDS accesses up to here are done before those that follow (its own area: no barrier).
__device__ __forceinline__ void ce_wave_sync()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

typedef __attribute__((address_space(3))) unsigned char lds_char;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

// The sum over eight neighbouring lanes, in every one of them: neighbours, pairs, and the
// mirrored half row (no LDS).
template <int CTRL> __device__ __forceinline__ float ce_lane(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float ce_sum8(float v)
{
    v += ce_lane<0xB1>(v);                           // quad_perm 1 0 3 2
    v += ce_lane<0x4E>(v);                           // quad_perm 2 3 0 1
    return v + ce_lane<0x141>(v);                    // row_half_mirror
}

// neighbouring results
__device__ __forceinline__ void ce_store4(float *p, const float *v) { *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void ce_store4(bf16_t *p, const float *v)
{
    *reinterpret_cast<u32x2_t *>(p) = u32x2_t{pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
}

__device__ __forceinline__ void ce_store8(float *p, const float *v) { ce_store4(p, v); ce_store4(p + 4, v + 4); }
__device__ __forceinline__ void ce_store8(bf16_t *p, const float *v) { stg16(p, Elem<bf16_t>::pack(v)); }

// A workgroup's tile: tiles of one k range first; four row tiles take turns over the
// column tiles, so that the 32 workgroups of an XCD share both operands in its L2
// (8192 x 32768 x 4096, weight gradient: 1.58 ms with four, 1.67 with eight, 1.77 with 16).
struct CePlace { int ti, tj, part; };
__device__ __forceinline__ bool ce_place(CePlace &pl, int block, int nti, int ntj, int parts)
{
    const int tiles = nti * ntj, total = tiles * parts;
    if (block >= total) return false;
    const int id = xcd_remap(block, total);
    pl.part = id / tiles;
    const int t = id - pl.part * tiles, per = 4 * ntj, first = t / per * 4, n = min(4, nti - first), r = t % per;
    pl.ti = first + r % n;
    pl.tj = r / n;
    return true;
}

// The sums acc of a wave: its blocks of a BI x BJ tile over the stages [s0, s1) along k.
// Operand tiles start at i0 and j0, with ni, nj rows (columns) left and k_i, k_j values
// along k.  Starts without, ends with a barrier.
template <typename T, int BI, int BJ, int WI, int WJ, bool ICOLS, bool JCOLS>
__device__ __forceinline__ void ce_product(f32x4 (&acc)[BJ / WJ / 16][BI / WI / 16], const char *i0, int64_t i_ld, int ni,
                                           int k_i, const char *j0, int64_t j_ld, int nj, int k_j, int s0, int s1,
                                           unsigned char *lds0, unsigned char *lds1)
{
    constexpr int NT = WI * WJ * 64, TI = BI / WI, TJ = BJ / WJ, MI = TI / 16, NJ = TJ / 16, BK = 128 / sizeof(T);
    typedef typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type frag;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    typedef CeLoad<T, BI, NT, ICOLS> LoadI;
    typedef CeLoad<T, BJ, NT, JCOLS> LoadJ;
    LoadI li;
    LoadJ lj;
    li.init(i_ld, tid);
    lj.init(j_ld, tid);
    CeFrags<T, BI, MI, ICOLS> ri;
    CeFrags<T, BJ, NJ, JCOLS> rj;
    ri.init(wave / WJ * TI, lane);
    rj.init(wave % WJ * TJ, lane);
    ce_zero(acc);
    // float32 sums in two levels, 64 terms and then those: a chain of all terms, one
    // rounding each, left the gradients of 128 x 1024 x 1000 7 times as far off float64
    // as a library's product does
    constexpr bool kFold = sizeof(T) == 4;
    f32x4 total[kFold ? NJ : 1][kFold ? MI : 1];
    if constexpr (kFold) ce_zero(total);
    const int end = s1 * BK;
    k_i = min(k_i, end);
    k_j = min(k_j, end);
    // A stage has two sub-steps.  Between two barriers a wave multiplies the second
    // sub-step of the stage before, whose fragments it already holds, and the first of
    // this one; meanwhile it reads this stage's fragments and the next stage is loaded
    // into the LDS that the stage before has left.  Products, reads and loads alternate.
    struct Frags { frag i[MI], j[NJ]; } f0, f1;
    constexpr int kPi = ICOLS && sizeof(T) == 4 ? 4 : MI, kPj = JCOLS && sizeof(T) == 4 ? 4 : NJ;     // reads of a sub-step
    constexpr int kLi = LoadI::kLoads, kLj = LoadJ::kLoads, kParts = kPi > kPj ? kPi : kPj,
                  kEach = MI > 2 ? (kLi + kLj) * 2 / MI : kLi + kLj;
    auto load = [&](unsigned char *lds, const typename LoadI::Stage &a, const typename LoadJ::Stage &b, int from, int to)
        __attribute__((always_inline)) {
        #pragma unroll
        for (int l = from; l < to; l++) {
            if (l < kLi) li.load(a, lds, l, wave);
            else lj.load(b, lds + BI * 128, l - kLi, wave);
        }
    };
    auto read = [&](Frags &f, const unsigned char *lds, int sub, int part) __attribute__((always_inline)) {
        if (part < kPj) rj.read(lds + BI * 128, sub, lane, f.j, part);
        if (part < kPi) ri.read(lds, sub, lane, f.i, part);
    };
    auto multiply = [&](const Frags &f, int a) __attribute__((always_inline)) {
        #pragma unroll
        for (int b = 0; b < NJ; b++) ce_mma(acc[b][a], f.j[b], f.i[a]);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto stage = [&](const unsigned char *now, unsigned char *other, int s, bool first) __attribute__((always_inline)) {
        const typename LoadI::Stage sa = li.stage(i0, i_ld, ni, (s + 1) * BK, k_i);
        const typename LoadJ::Stage sb = lj.stage(j0, j_ld, nj, (s + 1) * BK, k_j);
        #pragma unroll
        for (int a = 0; a < MI; a++) {
            #pragma unroll
            for (int b = a; b < (a + 1 < MI ? a + 1 : kParts); b++) read(f0, now, 0, b);
            load(other, sa, sb, min(a * kEach, kLi + kLj), min((a + 1) * kEach, kLi + kLj));
            if (!first) multiply(f1, a);
        }
        #pragma unroll
        for (int a = 0; a < MI; a++) {
            #pragma unroll
            for (int b = a; b < (a + 1 < MI ? a + 1 : kParts); b++) read(f1, now, 1, b);
            multiply(f0, a);
        }
        __syncthreads();
    };
    if (s0 < s1) {
        load(lds0, li.stage(i0, i_ld, ni, s0 * BK, k_i), lj.stage(j0, j_ld, nj, s0 * BK, k_j), 0, kLi + kLj);
        __syncthreads();
        stage(lds0, lds1, s0, true);
        for (int s = s0 + 1; s < s1; s += 2) {
            stage(lds1, lds0, s, false);
            if (s + 1 < s1) stage(lds0, lds1, s + 1, false);
            if constexpr (kFold) ce_fold(total, acc);
        }
        #pragma unroll
        for (int a = 0; a < MI; a++) multiply(f1, a);
    }
    if constexpr (kFold) {
        ce_fold(total, acc);
        #pragma unroll
        for (int b = 0; b < NJ; b++)
            #pragma unroll
            for (int a = 0; a < MI; a++) acc[b][a] = total[b][a];
    }
    __syncthreads();
}

// LDS of a workgroup: two stages, and what the epilogue needs of the tile's rows and columns
#define CE_LDS(BI, BJ)                                                                  \
    __shared__ __align__(16) unsigned char lds0[(BI + BJ) * 128], lds1[(BI + BJ) * 128]; \
    __shared__ CeRow rows[BI];                                                          \
    __shared__ float bias[BJ], others[WJ * BI]

// One tile of a product, by workgroup `block` of its grid.
template <typename T, int BI, int BJ, int WI, int WJ, int MODE>
__device__ __forceinline__ void ce_tile_of(const CeGemm &p, int block, unsigned char *lds0, unsigned char *lds1, CeRow *rows,
                                           float *bias, float *others)
{
#ifdef __HIP_DEVICE_COMPILE__              // (the host pass cannot instantiate the matrix instructions twice)
    constexpr bool ICOLS = MODE == CE_DW, JCOLS = MODE == CE_DW || MODE == CE_DH;
    constexpr int NT = WI * WJ * 64, TI = BI / WI, TJ = BJ / WJ, MI = TI / 16, NJ = TJ / 16, BK = 128 / sizeof(T);
    constexpr int kStage = (BI + BJ) * 128;
    const int count = *p.count;
    const int ni = MODE == CE_DW ? p.classes : (MODE == CE_DH && p.gt ? 2 * count : count), nj = MODE == CE_DW || MODE == CE_DH ? p.c : p.classes;
    const int K = MODE == CE_DW ? count : (MODE == CE_DH ? p.classes : p.c);
    CePlace pl;
    if (!ce_place(pl, block, (ni + BI - 1) / BI, (nj + BJ - 1) / BJ, p.parts)) return;
    const int i0 = pl.ti * BI, j0 = pl.tj * BJ;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / WJ, wj = wave % WJ;
    const char *ibase = (const char *)p.i + (ICOLS ? (int64_t)i0 * sizeof(T) : i0 * p.i_ld);
    const char *jbase = (const char *)p.j + (JCOLS ? (int64_t)j0 * sizeof(T) : j0 * p.j_ld);
    const int steps = (K + BK - 1) / BK;
    const int s0 = (int)((int64_t)pl.part * steps / p.parts), s1 = (int)((int64_t)(pl.part + 1) * steps / p.parts);
    // (there before the products are done)
    if constexpr (MODE != CE_DW) {
        for (int i = tid; i < BI; i += NT) rows[i] = i0 + i < count ? p.rows[i0 + i] : CeRow{0, -1, 0.f, 0.f};
    }
    if constexpr (MODE == CE_STATS || MODE == CE_GRAD) {
        for (int j = tid; j < BJ; j += NT)
            bias[j] = j0 + j < nj ? (p.bias ? p.bias[j0 + j] : 0.f) : (MODE == CE_STATS ? -INFINITY : 0.f);
    }
    f32x4 acc[NJ][MI];
    // (g's rows are whole vectors of zeros past the classes: their last vector is read whole)
    ce_product<T, BI, BJ, WI, WJ, ICOLS, JCOLS>(acc, ibase, p.i_ld, ni - i0, MODE == CE_DH ? (K + 7) / 8 * 8 : K, jbase,
                                                p.j_ld, nj - j0, K, s0, s1, lds0, lds1);

    // (the lane hidden from the compiler, which would form addresses ahead of the loop)
    int late = lane;
    asm volatile("" : "+v"(late));
    const int q = late % 16, g = late / 16;
    const int iw = i0 + wi * TI, jw = j0 + wj * TJ;
    if constexpr (MODE == CE_STATS) {
        // each row's maximum, sum of exponentials and sum over the tile's columns
        float *red = reinterpret_cast<float *>(lds0);
        if (p.bias || j0 + BJ > nj) {                // (classes past the last are -infinity)
            #pragma unroll
            for (int b = 0; b < NJ; b++)
                #pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float add = bias[wj * TJ + 16 * b + 4 * g + r];
                    #pragma unroll
                    for (int a = 0; a < MI; a++) acc[b][a][r] += add;
                }
        }
        #pragma unroll
        for (int a = 0; a < MI; a++) {
            const int row = wi * TI + 16 * a + q, at = rows[row].label - jw;   // the label's column here
            float mx = -INFINITY, sum = 0.f, all = 0.f;
            #pragma unroll
            for (int b = 0; b < NJ; b++)
                #pragma unroll
                for (int r = 0; r < 4; r++) mx = fmaxf(mx, acc[b][a][r]);
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float base = mx == -INFINITY ? 0.f : mx;
            #pragma unroll
            for (int b = 0; b < NJ; b++)
                #pragma unroll
                for (int r = 0; r < 4; r++) sum += ce_exp(acc[b][a][r] - base);
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (p.sums) {
                #pragma unroll
                for (int b = 0; b < NJ; b++)
                    #pragma unroll
                    for (int r = 0; r < 4; r++) all += jw + 16 * b + 4 * g + r < nj ? acc[b][a][r] : 0.f;
                all += __shfl_xor(all, 16, 64);
                all += __shfl_xor(all, 32, 64);
            }
            if (__any((uint32_t)at < TJ)) {
                float hit = 0.f;
                #pragma unroll
                for (int b = 0; b < NJ; b++)
                    #pragma unroll
                    for (int r = 0; r < 4; r++) hit = at == 16 * b + 4 * g + r ? acc[b][a][r] : hit;
                if ((uint32_t)at < TJ && at / 4 % 4 == g && jw + at < nj) p.picked[i0 + row] = hit;
            }
            if (g == 0) {
                float *o = red + (wj * BI + row) * 3;
                o[0] = mx; o[1] = sum; o[2] = all;
            }
        }
        __syncthreads();
        for (int i = tid; i < BI; i += NT) {
            if (i0 + i >= ni) break;
            float mx = -INFINITY, sum = 0.f, all = 0.f;
            #pragma unroll
            for (int w = 0; w < WJ; w++) mx = fmaxf(mx, red[(w * BI + i) * 3]);
            const float base = mx == -INFINITY ? 0.f : mx;
            #pragma unroll
            for (int w = 0; w < WJ; w++) {
                sum += red[(w * BI + i) * 3 + 1] * ce_exp(red[(w * BI + i) * 3] - base);
                all += red[(w * BI + i) * 3 + 2];
            }
            const int64_t o = (int64_t)pl.tj * p.m + i0 + i;
            p.stats[o] = float2{mx, sum};
            if (p.sums) p.sums[o] = all;
        }
    } else {
        // The results through LDS, 64 x 64 of a wave at a time in its own 16 KiB (a row's
        // 16-byte chunks in the order chunk ^ row % 16), so that a lane goes on with eight
        // neighbouring columns: whole lines are stored, in a short loop over the rows.
        // i = 16 a + q and j = 16 b + 4 g + r, in float32 columns i = MI q + a, j = NJ (4 g + r) + b.
        constexpr bool IP = ICOLS && sizeof(T) == 4, JP = JCOLS && sizeof(T) == 4;
        constexpr int kHalf = NT / 128;
        constexpr int kSub = TI < 64 ? TI : 64, kWaveOut = kSub * 64 * 4;
        static_assert(kStage >= kHalf * kWaveOut && (!IP || TI == kSub) && (!JP || TJ == 64), "a wave's part of the stages");
        lds_char *mine = (wave < kHalf ? (lds_char *)lds0 : (lds_char *)lds1) + wave % kHalf * kWaveOut;
        const int lrow = late / 8, lcol = late % 8 * 8;
        // (parts are multiplied when they are added)
        const float factor = MODE == CE_GRAD || p.part_stride ? 1.f : *p.factor;
        #pragma unroll
        for (int c = 0; c < TJ / 64; c++) {
        const int j = jw + 64 * c + lcol;
        float col[8];
        if constexpr (MODE == CE_GRAD) {
            #pragma unroll
            for (int e = 0; e < 8; e++) col[e] = 0.f;
        }
        #pragma unroll
        for (int h = 0; h < TI / kSub; h++) {
            #pragma unroll
            for (int a = 0; a < kSub / 16; a++)
                #pragma unroll
                for (int b = 0; b < 4; b++) {
                    const int row = IP ? MI * q + a : 16 * a + q, chunk = JP ? 4 * g + b : 4 * b + g;
                    const f32x4 v = JP ? f32x4{acc[0][4 * h + a][b], acc[1][4 * h + a][b], acc[2][4 * h + a][b], acc[3][4 * h + a][b]}
                                       : acc[4 * c + b][4 * h + a];
                    *(lds_f32x4 *)(mine + row * 256 + ((chunk ^ (row % 16)) * 16)) = v;
                }
            ce_wave_sync();
            #pragma unroll 2
            for (int it = 0; it < kSub / 8; it++) {
                const int row = it * 8 + lrow, i = iw + kSub * h + row;
                float v[8];
                #pragma unroll
                for (int k = 0; k < 2; k++) {
                    const f32x4 u = *(const lds_f32x4 *)(mine + row * 256 + (((lcol / 4 + k) ^ (row % 16)) * 16));
                    #pragma unroll
                    for (int r = 0; r < 4; r++) v[4 * k + r] = u[r];
                }
                if (i >= ni) continue;
                if constexpr (MODE == CE_GRAD) {
                    const CeRow r = rows[i - i0];
                    const int at = r.label - p.first - j;
                    const float grow = r.scale * (1.f + 2.f * p.z * r.lse), flat = r.scale * p.flat;
                    if (p.bias) {
                        #pragma unroll
                        for (int e = 0; e < 8; e++) v[e] += bias[j + e - j0];
                    }
                    #pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = ce_exp(v[e] - r.lse);
                    if (p.others) {                  // (eight lanes share a row's 64 columns)
                        if (j0 + BJ > nj) {
                            #pragma unroll
                            for (int e = 0; e < 8; e++) v[e] = j + e < nj ? v[e] : 0.f;
                        }
                        float sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
                        if ((uint32_t)at < 8) {
                            float prob = 0.f;
                            sum = 0.f;
                            #pragma unroll
                            for (int e = 0; e < 8; e++) {
                                sum += e == at ? 0.f : v[e];
                                prob = e == at ? v[e] : prob;
                            }
                            if (j + at < nj) p.prob[i] = prob;
                        }
                        sum = ce_sum8(sum);
                        if (lcol == 0) others[wj * BI + i - i0] = sum;
                    }
                    #pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = __builtin_fmaf(v[e], grow, -flat);
                    if ((uint32_t)at < 8) {
                        const float hit = r.scale * p.hit;
                        #pragma unroll
                        for (int e = 0; e < 8; e++) v[e] -= e == at ? hit : 0.f;
                    }
                    if (j0 + BJ > nj) {
                        #pragma unroll
                        for (int e = 0; e < 8; e++) v[e] = j + e < nj ? v[e] : 0.f;
                    }
                    if (p.colsum) {
                        #pragma unroll
                        for (int e = 0; e < 8; e++) col[e] += v[e];
                    }
                    ce_store8((T *)p.g + (int64_t)i * p.g_ld + j, v);
                } else if (j < nj) {                 // (the second half of a vector that c cuts, in float32: below)
                    const int64_t row_out = MODE == CE_DW || p.part_stride ? i : rows[MODE == CE_DW ? 0 : i - i0].row;
                    const bool whole = sizeof(T) == 2 || j + 4 < nj;
                    #pragma unroll
                    for (int e = 0; e < 8; e++) v[e] *= factor;
                    if (p.out_f32) {
                        float *o = (float *)p.out + (int64_t)pl.part * p.part_stride + row_out * p.out_ld + j;
                        if (p.add) {
                            #pragma unroll
                            for (int k = 0; k < 2; k++) {
                                if (k && !whole) break;
                                const f32x4 old = *reinterpret_cast<const f32x4 *>(o + 4 * k);
                                #pragma unroll
                                for (int r = 0; r < 4; r++) v[4 * k + r] += old[r];
                            }
                        }
                        ce_store4(o, v);
                        if (whole) ce_store4(o + 4, v + 4);
                    } else {
                        bf16_t *o = (bf16_t *)p.out + row_out * p.out_ld + j;
                        if (whole) ce_store8(o, v);
                        else ce_store4(o, v);
                    }
                }
            }
            ce_wave_sync();
        }
        if constexpr (MODE == CE_GRAD) {
            static_assert(MODE != CE_GRAD || TJ == 64, "a row's others of a wave");
            if (p.colsum) {                          // the wave's rows; then the tile's, of all its waves
                #pragma unroll
                for (int e = 0; e < 8; e++) {
                    for (int o = 8; o < 64; o *= 2) col[e] += __shfl_xor(col[e], o, 64);
                    if (lrow == 0 && j + e < nj) p.colsum[(int64_t)(pl.ti * WI + wi) * p.colsum_ld + j + e] = col[e];
                }
            }
        }
        }
        if constexpr (MODE == CE_GRAD) {
            if (p.others) {                          // the tile's columns
                __syncthreads();
                for (int i = tid; i < min(BI, ni - i0); i += NT) {
                    float sum = others[i];
                    #pragma unroll
                    for (int w = 1; w < WJ; w++) sum += others[w * BI + i];
                    p.others[(int64_t)pl.tj * p.m + i0 + i] = sum;
                }
            }
        }
    }
#endif
}

template <typename T, int BI, int BJ, int WI, int WJ, int MODE>
__global__ __launch_bounds__(WI * WJ * 64, 2) void k_ce_gemm(CeGemm p)
{
    CE_LDS(BI, BJ);
    ce_tile_of<T, BI, BJ, WI, WJ, MODE>(p, (int)wide_block(), lds0, lds1, rows, bias, others);
}

// dh and dw of a piece, which do not need each other, in one launch: dh's longer tiles
// first (`first` workgroups, a multiple of the eight XCDs), and dw's fill the chip as
// they end.
template <typename T, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(WI * WJ * 64, 2) void k_ce_pair(CeGemm dh, CeGemm dw, int first)
{
    CE_LDS(BI, BJ);
    const int block = (int)wide_block();
    if (block < first) ce_tile_of<T, BI, BJ, WI, WJ, CE_DH>(dh, block, lds0, lds1, rows, bias, others);
    else ce_tile_of<T, BI, BJ, WI, WJ, CE_DW>(dw, block - first, lds0, lds1, rows, bias, others);
}

// ---- few rows, or few tiles ---------------------------------------------------
// Logits of 16 MI x 16 NJ by one workgroup, its four waves each a quarter of k.  Nothing
// is shared, so the fragments are loaded straight into registers, kAhead steps ahead;
// the waves' sums are added through LDS in order.  With few rows this is a stream of the
// weights, with few tiles it spreads them over the chip.  Sums in two levels, four steps
// and then those: where few classes make the model sure of its labels, g is a difference
// of numbers near 1 and shows every rounding of the logits.
template <typename T, int MI, int NJ, int MODE>
__global__ __launch_bounds__(kThreads) void k_ce_small(CeGemm p)
{
    constexpr int BI = 16 * MI, BJ = 16 * NJ, kAhead = 20 / (MI + NJ), kPitch = BJ + 4, BK = 64 / sizeof(T);
    constexpr int kGroups = 4 * NJ, kLanes = 16 / MI;        // groups of four columns of a row, threads of a row
    typedef typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type frag;
    __shared__ __align__(16) float part[4][BI * kPitch];
    const int ni = p.rows ? *p.count : (int)p.m, nj = p.classes;
    CePlace pl;
    if (!ce_place(pl, (int)wide_block(), (ni + BI - 1) / BI, (nj + BJ - 1) / BJ, 1)) return;
    const int i0 = pl.ti * BI, j0 = pl.tj * BJ;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane % 16, g = lane / 16;
    const int width = p.c * (int)sizeof(T);
    const __amdgpu_buffer_rsrc_t ri = buf_view((const char *)p.i + i0 * p.i_ld, (min(ni - i0, BI) - 1) * (int)p.i_ld + width);
    const __amdgpu_buffer_rsrc_t rj = buf_view((const char *)p.j + j0 * p.j_ld, (min(nj - j0, BJ) - 1) * (int)p.j_ld + width);
    const int steps = (p.c + BK - 1) / BK, s0 = wave * steps / 4, s1 = (wave + 1) * steps / 4;
    frag fi[kAhead][MI], fj[kAhead][NJ];
    auto load = [&](int d, int s) __attribute__((always_inline)) {
        const uint32_t at = s * 64 + g * 16, in = s < s1 && (int)at < width ? at : kBufOff;
        #pragma unroll
        for (int b = 0; b < NJ; b++) fj[d][b] = __builtin_bit_cast(frag, bld16(rj, in + (16 * b + q) * (uint32_t)p.j_ld));
        #pragma unroll
        for (int a = 0; a < MI; a++) fi[d][a] = __builtin_bit_cast(frag, bld16(ri, in + (16 * a + q) * (uint32_t)p.i_ld));
    };
    // kLanes threads a row, group after group of its columns: what they will need of them
    constexpr int kTurns = (kGroups + kLanes - 1) / kLanes;
    const int row = tid / kLanes, i = i0 + row, li = tid % kLanes;
    CeRow info = CeRow{0, -1, 0.f, 0.f};
    if (i < ni) {
        if (p.rows) info = p.rows[i];
        else info.label = p.labels[i];
    }
    float bias[kTurns][4];
    #pragma unroll
    for (int u = 0; u < kTurns; u++)
        #pragma unroll
        for (int r = 0; r < 4; r++) {
            const int j = j0 + (u * kLanes + li) * 4 + r;
            bias[u][r] = p.bias ? p.bias[min(j, nj - 1)] : 0.f;
        }
    f32x4 acc[NJ][MI], total[NJ][MI];
    ce_zero(acc);
    ce_zero(total);
    #pragma unroll
    for (int d = 0; d < kAhead; d++) load(d, s0 + d);
    for (int s = s0; s < s1; s += kAhead) {
        #pragma unroll
        for (int d = 0; d < kAhead; d++) {
            #pragma unroll
            for (int a = 0; a < MI; a++)
                #pragma unroll
                for (int b = 0; b < NJ; b++) ce_mma(acc[b][a], fj[d][b], fi[d][a]);
            load(d, s + kAhead + d);
            if (d % 4 == 3 || d == kAhead - 1) ce_fold(total, acc);
        }
    }
    #pragma unroll
    for (int a = 0; a < MI; a++)
        #pragma unroll
        for (int b = 0; b < NJ; b++)
            *reinterpret_cast<f32x4 *>(&part[wave][(16 * a + q) * kPitch + 16 * b + 4 * g]) = total[b][a];
    __syncthreads();
    float mx = -INFINITY, sum = 0.f, all = 0.f, v[kTurns][4];
    float others = 0.f;                              // CE_GRAD: the sum of the classes' probabilities without the label's
    #pragma unroll
    for (int u = 0; u < kTurns; u++) {
        const int c = (u * kLanes + li) * 4;
        #pragma unroll
        for (int r = 0; r < 4; r++) v[u][r] = -INFINITY;
        if (c >= BJ) continue;
        const float *o = &part[0][row * kPitch + c];
        #pragma unroll
        for (int r = 0; r < 4; r++) {
            float l = o[r];
            #pragma unroll
            for (int w = 1; w < 4; w++) l += o[w * BI * kPitch + r];
            const int j = j0 + c + r;
            l += bias[u][r];
            v[u][r] = j < nj ? l : -INFINITY;
            if constexpr (MODE == CE_STATS) {
                mx = fmaxf(mx, v[u][r]);
                all += j < nj ? l : 0.f;
                if (j == info.label && j < nj && i < ni) p.picked[i] = l;
            } else {
                const float e = ce_exp(l - info.lse);
                v[u][r] = j < nj && i < ni ? ce_g(e, info, p, j + p.first == info.label) : 0.f;
                if (j < nj && j + p.first != info.label) others += e;
                else if (j < nj && i < ni && p.others) p.prob[i] = e;
            }
        }
        if constexpr (MODE == CE_GRAD) {
            if (i < ni) {
                T *to = (T *)p.g + (int64_t)i * p.g_ld + j0 + c;
                ce_store4(to, v[u]);
                if (sizeof(T) == 2 && p.gt) {            // what the rounding left, as rows of their own
                    float rest[4];
                    #pragma unroll
                    for (int r = 0; r < 4; r++) rest[r] = v[u][r] - bf2f(f2bf(v[u][r]));
                    ce_store4(to + ni * p.g_ld, rest);
                }
            }
        }
    }
    if constexpr (MODE == CE_STATS) {
        #pragma unroll
        for (int o = 1; o < kLanes; o *= 2) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        const float base = mx == -INFINITY ? 0.f : mx;
        #pragma unroll
        for (int u = 0; u < kTurns; u++)
            #pragma unroll
            for (int r = 0; r < 4; r++) sum += ce_exp(v[u][r] - base);
        #pragma unroll
        for (int o = 1; o < kLanes; o *= 2) {
            sum += __shfl_xor(sum, o, 64);
            all += __shfl_xor(all, o, 64);
        }
        if (li == 0 && i < ni) {
            const int64_t o = (int64_t)pl.tj * p.m + i;
            p.stats[o] = float2{mx, sum};
            if (p.sums) p.sums[o] = all;
        }
    } else if (p.others) {
        #pragma unroll
        for (int o = 1; o < kLanes; o *= 2) others += __shfl_xor(others, o, 64);
        if (li == 0 && i < ni) p.others[(int64_t)pl.tj * p.m + i] = others;
    }
    if (MODE == CE_GRAD && (p.colsum || p.gt)) {
        __syncthreads();
        #pragma unroll
        for (int u = 0; u < kTurns; u++) {
            const int c = (u * kLanes + li) * 4;
            if (c < BJ) *reinterpret_cast<f32x4 *>(&part[0][row * kPitch + c]) = f32x4{v[u][0], v[u][1], v[u][2], v[u][3]};
        }
        __syncthreads();
        if (sizeof(T) == 2 && p.gt) {                    // a class's 16 rows together, then what they left
            for (int e = tid; e < BJ * 4 * MI; e += kThreads) {
                const int col = e / (4 * MI), a = e / 4 % MI, quarter = e % 4;
                float f[8];
                #pragma unroll
                for (int r = 0; r < 8; r++) {
                    const float t = part[0][(16 * a + quarter % 2 * 8 + r) * kPitch + col];
                    f[r] = quarter < 2 ? t : t - bf2f(f2bf(t));
                }
                stg16((char *)p.gt + ((int64_t)(j0 + col) * p.gt_rows + pl.ti * MI + a) * 64 + quarter * 16, Elem<bf16_t>::pack(f));
            }
        }
        if (p.colsum && tid < BJ && j0 + tid < nj) {
            float t = 0.f;
            #pragma unroll
            for (int r = 0; r < BI; r++) t += part[0][r * kPitch + tid];
            p.colsum[(int64_t)pl.ti * p.colsum_ld + j0 + tid] = t;
        }
    }
}

// The labels' own entries of g once more.  Where a row is sure of its label, p - 1 is what
// the roundings of l and lse left of it: 1e-6 of an lse of 8, a thousandth of a g of 1e-3.
// The others' probabilities are each right relative to themselves and their sum is 1 - p, so
// beyond p = 1/2 the entry is formed from that sum (while the two agree: an lse that is not
// these logits' stays as it was given).  A workgroup takes the rows of one of dbias's partial
// sums, each in NT / tile slices of the column parts; the partial sums are mended by the first
// row of each label, in the rows' order.
// 64 x 2192 of 6 classes in float32: dh off by 3.3e-7 of its norm, without it by 1.8e-6, and
// a row of 1488 of 3 classes with p = 0.9995 by 1.5e-6 and 2.2e-3.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void k_ce_own(CeGemm p, int tile, int parts)
{
    __shared__ double sums[NT];
    __shared__ int labels[kOwnRows], before[NT];
    __shared__ float changes[kOwnRows];
    const int tid = threadIdx.x, first = blockIdx.x * tile, r = tid % tile, slice = tid / tile, slices = NT / tile, i = first + r;
    const int64_t at = min((int64_t)i, p.m - 1);     // (the loads do not wait for the count: what lies behind it is left unused)
    const int ni = *p.count;
    double others = 0.0;
    for (int t = slice; t < parts; t += 8 * slices) {
        float part[8];
        #pragma unroll
        for (int u = 0; u < 8; u++) part[u] = p.others[min(t + u * slices, parts - 1) * p.m + at];
        #pragma unroll
        for (int u = 0; u < 8; u++) others += t + u * slices < parts ? part[u] : 0.f;
    }
    CeRow info = CeRow{0, -1, 0.f, 0.f};
    float prob = 0.f, old = 0.f;
    if (tid < tile) {
        info = p.rows[at];
        prob = p.prob[at];
    }
    if (first >= ni) return;
    // (a label outside the classes has left no probability)
    const bool known = tid < tile && i < ni && (uint32_t)info.label < (uint32_t)p.classes;
    float *sum_to = p.colsum + (int64_t)blockIdx.x * p.colsum_ld + (known ? info.label : 0);
    if (known && p.colsum) old = *sum_to;
    sums[tid] = others;
    __syncthreads();
    int label = -1;
    if (tid < tile) {
        float change = 0.f;
        for (int s = 1; s < slices; s++) others += sums[s * tile + r];
        if (known && prob > 0.5f && fabs(prob + others - 1.0) < 1e-3) {
            label = info.label;
            const double grow = 1.0 + 2.0 * p.z * info.lse;
            const float v = (float)(info.scale * (grow * (1.0 - others) - p.hit - p.flat));
            change = v - ce_g(prob, info, p, true);
            T *to = (T *)p.g + (int64_t)i * p.g_ld + label;
            if constexpr (sizeof(T) == 2) {
                *to = f2bf(v);
                if (p.gt) {
                    const bf16_t rest = f2bf(v - bf2f(f2bf(v)));
                    to[ni * p.g_ld] = rest;
                    bf16_t *t = (bf16_t *)p.gt + ((int64_t)label * p.gt_rows + i / 16) * 32 + i % 16;
                    t[0] = f2bf(v);
                    t[16] = rest;
                }
            } else {
                *to = v;
            }
        }
        labels[r] = label;
        changes[r] = change;
    }
    if (!p.colsum || !__syncthreads_or(label >= 0)) return;
    // the rows of each row's label, in as many slices
    const int mine = labels[r], per = (tile + slices - 1) / slices;
    double sum = 0.0;
    bool earlier = false;
    for (int k = slice * per; k < min(slice * per + per, tile); k++) {
        const bool same = labels[k] == mine;
        sum += same ? changes[k] : 0.f;
        earlier = earlier || (same && k < r);
    }
    sums[tid] = sum;
    before[tid] = earlier;
    __syncthreads();
    if (label < 0) return;
    for (int s = 1; s < slices; s++) {
        sum += sums[s * tile + r];
        earlier = earlier || before[s * tile + r];
    }
    if (!earlier) *sum_to = old + (float)sum;
}

// The weights' gradient of few bf16 rows, a stream of results: a wave keeps the features
// of 64 columns (16 rows a matrix instruction) and walks over the classes.  g comes with
// 16 rows of a class together, rounded, and then what the rounding left: the same
// instruction adds both, so dw has no error of g's rounding.  Block b's row 4 g + r stands
// for column 32 (b / 2) + 8 g + 4 (b % 2) + r, so that a lane stores eight neighbours.
// Bound by its stores: 32000 classes of 2048 in 29.6 us = 4.4 TB/s with up to 16 rows, 38.6 up to
// 32 and 57.4 up to 64, where g's share of the loads doubles and doubles again.  (With more than
// 16 rows the scalars that the compiler spills are the conditions of the features' loads, before
// the loop; none is read in it.)
template <typename W, int KB>
__global__ __launch_bounds__(kThreads) void k_ce_outer(CeGemm p, int chunk)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane % 16, g = lane / 16, count = *p.count;
    const int blocks = (p.c + 255) / 256, j0 = (int)(blockIdx.x % blocks) * 256 + wave * 64;
    const int v0 = (int)(blockIdx.x / blocks) * chunk, v1 = min(v0 + chunk, p.classes);
    if (j0 >= p.c) return;
    const bf16_t *h = (const bf16_t *)p.i;
    bf16x8 f[KB][4];
    #pragma unroll
    for (int k = 0; k < KB; k++)
        #pragma unroll
        for (int b = 0; b < 4; b++) {
            const int j = j0 + 32 * (b / 2) + 8 * (q / 4) + 4 * (b % 2) + q % 4;
            #pragma unroll
            for (int e = 0; e < 8; e++) {
                const int row = 16 * k + (8 * g + e) % 16;
                const bool in = row < count && j < p.c;
                const bf16_t u = h[in ? (int64_t)row * p.c + j : 0];
                f[k][b][e] = __builtin_bit_cast(__bf16, in ? u : (bf16_t)0);
            }
        }
    const float factor = *p.factor;
    const char *gt = (const char *)p.gt + (int64_t)q * p.gt_rows * 64 + g * 16;
    // kSteps steps of 16 classes at a time, loaded a turn ahead (one step ahead: 80 us for
    // 65536 classes of 2048, the time of a load each)
    constexpr int kSteps = 8 / KB;
    bf16x8 now[kSteps][KB], next[kSteps][KB];
    auto load = [&](int v, bf16x8 (&to)[kSteps][KB]) __attribute__((always_inline)) {
        #pragma unroll
        for (int u = 0; u < kSteps; u++) {
            const int at = v + 16 * u < v1 ? v + 16 * u : v0;
            #pragma unroll
            for (int k = 0; k < KB; k++)         // (past the rows that count g is not written)
                to[u][k] = __builtin_bit_cast(bf16x8, k * 16 < count ? ldg16(gt + ((int64_t)at * p.gt_rows + k) * 64) : zero16());
        }
    };
    load(v0, now);
    for (int v = v0; v < v1; v += 16 * kSteps) {
        load(v + 16 * kSteps, next);
        #pragma unroll
        for (int u = 0; u < kSteps; u++) {
            f32x4 acc[4];
            #pragma unroll
            for (int b = 0; b < 4; b++) {
                acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
                #pragma unroll
                for (int k = 0; k < KB; k++) ce_mma(acc[b], f[k][b], now[u][k]);
            }
            if (v + 16 * u + q < v1) {
                W *o = (W *)p.out + (int64_t)(v + 16 * u + q) * p.out_ld + j0 + 8 * g;
                #pragma unroll
                for (int s = 0; s < 2; s++) {
                    float r[8];
                    #pragma unroll
                    for (int e = 0; e < 8; e++) r[e] = acc[2 * s + e / 4][e % 4] * factor;
                    if (j0 + 32 * s + 8 * g < p.c) ce_store8(o + 32 * s, r);
                }
            }
        }
        #pragma unroll
        for (int u = 0; u < kSteps; u++)
            #pragma unroll
            for (int k = 0; k < KB; k++) now[u][k] = next[u][k];
    }
}

// ---- rows' losses ------------------------------------------------------------
constexpr int kLossRows = 16;              // rows a workgroup takes, 16 threads each
// or 8 threads each: one workgroup of 1024, no launch for the mean.  Two launches are 1 to 3 us longer
// up to 63 tiles of classes (128 x 1024 x 1000 float32 16.5 us and 14.6, 40 x 1024 x 2500 22.3 and
// 21.8; 17 rows of 4000 classes alone 16.0 and 17.0), as long at 125 (128 x 1024 x 16000 bf16 34.9
// and 36.0, 40 x 1024 x 8000 16.5 and 15.8) and shorter from there on.
constexpr int kLossWide = 128;

__device__ __forceinline__ void ce_join(float &mx, double &sum, float mx2, double sum2)
{
    const float top = fmaxf(mx, mx2), base = top == -INFINITY ? 0.f : top;
    sum = sum * ce_exp(mx - base) + sum2 * ce_exp(mx2 - base);
    mx = top;
}

// The rows' losses and log sums from the tiles' maxima and sums (in float64), and the
// sum of the workgroup's losses.  R rows a workgroup of NT threads; a row's threads leave
// their part in kParts places (a wave each, or a thread each from 64 rows on).
template <int R, int NT>
__global__ __launch_bounds__(NT) void k_ce_rows(CeLoss p)
{
    constexpr int kParts = R < 64 ? NT / 64 : NT / R, kWaves = R < 64 ? 1 : R / 64;
    __shared__ float rm[kParts][R];
    __shared__ double rs[kParts][R], ra[kParts][R], red[kWaves];
    __shared__ int red_n[kWaves];
    const int tid = threadIdx.x, r = tid % R, slice = tid / R, place = R < 64 ? tid >> 6 : slice, count = p.rows ? *p.count : (int)p.m;
    const int i = blockIdx.x * R + r;
    if (blockIdx.x && (int)blockIdx.x * R >= count) return;
    float mx = -INFINITY;
    double sum = 0.0, all = 0.0;
    if (i < count) {
        #pragma unroll 4
        for (int t = slice; t < p.tiles; t += NT / R) {
            const float2 v = p.stats[(int64_t)t * p.m + i];
            if (p.sums) all += (double)p.sums[(int64_t)t * p.m + i];
            ce_join(mx, sum, v.x, (double)v.y);
        }
    }
    #pragma unroll
    for (int o = R; o < 64; o *= 2) {
        ce_join(mx, sum, __shfl_xor(mx, o, 64), __shfl_xor(sum, o, 64));
        all += __shfl_xor(all, o, 64);
    }
    if ((tid & 63) < R) { rm[place][r] = mx; rs[place][r] = sum; ra[place][r] = all; }
    __syncthreads();
    if (R < 64 && tid >= R) return;
    double loss = 0.0;
    int counted = 0;
    if (i < count && tid < R) {
        for (int w = 1; w < kParts; w++) {
            ce_join(mx, sum, rm[w][r], rs[w][r]);
            all += ra[w][r];
        }
        const int row = p.rows ? p.rows[i].row : i, label = p.rows ? p.rows[i].label : p.labels[i];
        double lse = 0.0;
        counted = label != p.ignore;
        if (counted) {
            lse = (double)mx + log(sum);
            loss = NAN;
            if ((uint32_t)label < (uint32_t)p.classes) {
                loss = lse - p.hit * (double)p.picked[i] + p.z * lse * lse;
                if (p.sums) loss -= p.flat * all;
            }
        }
        p.lse[1 + row] = (float)lse;
        p.loss[1 + row] = (float)loss;
    }
    #pragma unroll
    for (int o = 1; o < (R < 64 ? R : 64); o *= 2) {
        loss += __shfl_xor(loss, o, 64);
        counted += __shfl_xor(counted, o, 64);
    }
    if constexpr (kWaves > 1) {
        if (tid < R && (tid & 63) == 0) { red[tid >> 6] = loss; red_n[tid >> 6] = counted; }
        __syncthreads();
        if (tid) return;
        for (int w = 1; w < kWaves; w++) { loss += red[w]; counted += red_n[w]; }
    }
    if (tid) return;
    if (p.groups == 1) {
        p.loss[0] = counted ? (float)(loss / counted) : 0.f;
        p.lse[0] = (float)counted;
    } else {
        p.part[blockIdx.x] = double2{loss, (double)counted};
    }
}

__global__ __launch_bounds__(1024) void k_ce_mean(CeLoss p)
{
    __shared__ double red[16], red_n[16];
    const int tid = threadIdx.x, count = p.rows ? *p.count : (int)p.m, groups = (count + kLossRows - 1) / kLossRows;
    double v = 0.0, n = 0.0;
    for (int b = tid; b < groups; b += 1024) {
        const double2 u = p.part[b];
        v += u.x;
        n += u.y;
    }
    for (int o = 32; o > 0; o >>= 1) {
        v += __shfl_xor(v, o, 64);
        n += __shfl_xor(n, o, 64);
    }
    if ((tid & 63) == 0) { red[tid >> 6] = v; red_n[tid >> 6] = n; }
    __syncthreads();
    if (tid) return;
    v = n = 0.0;
    for (int w = 0; w < 16; w++) { v += red[w]; n += red_n[w]; }
    p.loss[0] = n > 0.0 ? (float)(v / n) : 0.f;
    p.lse[0] = (float)n;
}

// ---- sums over parts -----------------------------------------------------------
__device__ __forceinline__ void ce_bias(const CeBias &p, int block)
{
    const int j = block * kThreads + threadIdx.x, tiles = (*p.count + p.tile - 1) / p.tile;
    if (j >= p.classes) return;
    double v = 0.0;
    #pragma unroll 4
    for (int t = 0; t < tiles; t++) v += (double)p.colsum[(int64_t)t * p.ld + j];
    p.out[j] = (float)(v * *p.factor);
}
__global__ __launch_bounds__(kThreads) void k_ce_bias(CeBias p) { ce_bias(p, blockIdx.x); }

// out[row][j .. j + 3] = the sum of the parts' float32 results, in order.
// SL threads share a vector's parts (few results of many parts), joined in order.  The
// workgroups behind the first `first` add up dbias: a launch less (128 x 1024 x 1000 float32
// 38.3 us -> 36.4).
template <typename T, int SL>
__global__ __launch_bounds__(kThreads) void k_ce_sum(CeSum p, CeBias bias, int first)
{
    const int64_t block = wide_block();
    if (block >= first) {
        if (bias.out) ce_bias(bias, (int)(block - first));
        return;
    }
    __shared__ float red[SL > 1 ? SL : 1][SL > 1 ? kThreads / SL : 1][4];
    const int vecs = p.c / 4, tid = threadIdx.x, slice = tid / (kThreads / SL), at = tid % (kThreads / SL);
    const int64_t id = block * (kThreads / SL) + at, i = id / vecs;
    const int j = (int)(id - i * vecs) * 4;
    const int64_t n = p.rows ? *p.count : p.n;
    const bool mine = i < n;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
        for (int t = 0; t <= p.twice; t++) {     // (few bf16 rows: those of what g's rounding left)
            const float *src = p.part + (i + t * n) * p.c + j;
            #pragma unroll 4
            for (int s = slice; s < p.parts; s += SL) {
                const f32x4 u = *reinterpret_cast<const f32x4 *>(src + s * p.part_stride);
                #pragma unroll
                for (int r = 0; r < 4; r++) v[r] += u[r];
            }
        }
    }
    if constexpr (SL > 1) {
        #pragma unroll
        for (int r = 0; r < 4; r++) red[slice][at][r] = v[r];
        __syncthreads();
        if (slice) return;
        #pragma unroll
        for (int s = 1; s < SL; s++)
            #pragma unroll
            for (int r = 0; r < 4; r++) v[r] += red[s][at][r];
    }
    if (!mine) return;
    const int64_t row = p.rows ? p.rows[i].row : i;
    const float factor = *p.factor;
    #pragma unroll
    for (int r = 0; r < 4; r++) v[r] *= factor;
    ce_store4((T *)p.out + row * p.out_ld + j, v);
}

// ---- how a call runs -------------------------------------------------------------
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }

// How a product's tiles run: bf16 in 256 x 256 (one workgroup of eight waves a CU) where
// they fill the chip, else in 128 x 128 (two workgroups of four waves a CU), float32 in 64 x
// 128 (three of four; against two of 128 x 128: 128 x 1024 x 1000 backward 32.9 us and 36.5,
// 4907 x 1832 x 7449 1.61 ms and 1.72, 299 x 976 x 102340 forward 519 us and 637); logits of
// few rows or of too few tiles for that run as k_ce_small, 16 x i by 16 x j.
// Up to kFewRows bf16 rows g is kept in two parts, rounded and the rest, in separate rows
// (their products cost next to nothing beside reading the weights): with few rows the
// rounding of one label's g is no longer one of many.  Beyond, g is one bf16 operand, where
// float32 products would take ten times as long: dw of 1001 x 776 x 40961 is off float64 by 1.85e-3
// of its norm, where the result's own rounding alone is 1.65e-3, and by up to sqrt(2) times that
// where one label's entry makes up a row of dw.
constexpr int kFewRows = 64;
// The labels' entries of g are formed a second time (k_ce_own) where one piece holds all
// classes (kFewClasses always fit), so that the others' sum is whole before the products.  Not
// so beyond kFewClasses
//   with smoothing from kOwnSmoothing on: the entry is at least s then, which hides the
//     roundings (128 x 1024 x 1000 float32, s = 0.1: 32.7 us, with the launch 39.3), and
//   in bf16 past kFewRows: g is rounded to 8 bits, beside which the roundings of l and lse show
//     from 1 - p = 5e-4 down (1001 x 776 x 40961: 233 us, with sums and launch 247).
// It costs 128 x 1024 x 513 float32 3 to 5 us of 28, 1000 x 512 x 4000 3 of 129, 16 x 2048 x
// 65536 bf16 5 of 198, 20001 x 256 x 3 float32 6 of 90.
constexpr float kOwnSmoothing = 1.f / 64;
constexpr int kFewClasses = 512;
struct CeTile { int bi, bj; bool small; };
inline CeTile ce_tile(int dtype, int64_t ni, int64_t nj)
{
    if (dtype == DT_F32) return CeTile{64, 128, false};
    const int b = cdiv(ni, 256) * cdiv(nj, 256) >= 192 ? 256 : 128;
    return CeTile{b, b, false};
}
inline CeTile ce_logit_tile(int dtype, int64_t m, int64_t classes)
{
    const CeTile t = ce_tile(dtype, m, classes);
    if (m > kFewRows && cdiv(m, 128) * cdiv(classes, 128) >= 128) return t;
    const int mi = m > 16 ? 2 : 1;
    int nj = 4;
    while (nj > 1 && cdiv(m, 16 * mi) * cdiv(classes, 16 * nj) < 192) nj /= 2;
    return CeTile{16 * mi, 16 * nj, true};
}

// k ranges a product is cut into where its tiles would leave the chip idle
inline int ce_parts(const CeTile &t, int64_t ni, int64_t nj, int64_t steps, int least)
{
    const int64_t slots = t.bi == 256 ? 256 : 512, tiles = cdiv(ni, t.bi) * cdiv(nj, t.bj);
    const int64_t want = slots / tiles, most = steps / least;   // least: stages of a range
    const int64_t n = want < most ? want : most;
    return n < 1 ? 1 : (n > 64 ? 64 : (int)n);
}

template <typename T, int MODE>
void go(const CeGemm &p, const CeTile &t, int64_t grid, hipStream_t s)
{
    const dim3 g = wide_grid(grid);
    if constexpr (MODE == CE_STATS || MODE == CE_GRAD) {
        if (t.small) {
            const auto at = [&](auto mi) {
                constexpr int MI = decltype(mi)::value;
                if (t.bj == 64) hipLaunchKernelGGL((k_ce_small<T, MI, 4, MODE>), g, dim3(kThreads), 0, s, p);
                else if (t.bj == 32) hipLaunchKernelGGL((k_ce_small<T, MI, 2, MODE>), g, dim3(kThreads), 0, s, p);
                else hipLaunchKernelGGL((k_ce_small<T, MI, 1, MODE>), g, dim3(kThreads), 0, s, p);
            };
            if (t.bi == 16) at(std::integral_constant<int, 1>{});
            else at(std::integral_constant<int, 2>{});
            return;
        }
    }
    if constexpr (MODE == CE_DH) {
        if (t.bi == 32) {
            if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((k_ce_gemm<T, 32, 256, 1, 4, MODE>), g, dim3(256), 0, s, p);
            else hipLaunchKernelGGL((k_ce_gemm<T, 32, 128, 1, 2, MODE>), g, dim3(128), 0, s, p);
            return;
        }
    }
    if constexpr (sizeof(T) == 2) {
        if (t.bi == 256) {
            hipLaunchKernelGGL((k_ce_gemm<T, 256, 256, 2, 4, MODE>), g, dim3(512), 0, s, p);
            return;
        }
    }
    hipLaunchKernelGGL((k_ce_gemm<T, sizeof(T) == 2 ? 128 : 64, 128, 2, 2, MODE>), g, dim3(256), 0, s, p);
}

template <int MODE>
hipError_t gemm(const CeCall &a, const CeGemm &p, const CeTile &t, int64_t ni, int64_t nj, int64_t k, hipStream_t s)
{
    const double es = a.dtype == DT_BF16 ? 2 : 4;
    TraceScope tr(KC_CONV, KID_LINEAR_CE, s, es * ((double)ni * k + (double)nj * k + (double)ni * nj), 2.0 * ni * nj * k);
    const int64_t grid = cdiv(ni, t.bi) * cdiv(nj, t.bj) * p.parts;
    if (a.dtype == DT_BF16) go<bf16_t, MODE>(p, t, grid, s);
    else go<float, MODE>(p, t, grid, s);
    return hipGetLastError();
}

// tile: rows of a partial row of dbias; parts: column parts of the others' sums
hipError_t launch_own(const CeCall &a, const CeGemm &p, int tile, int parts, hipStream_t s)
{
    TraceScope tr(KC_SMALL, KID_LINEAR_CE, s, 4.0 * a.m * (parts + 8), 0.0);
    const dim3 g((unsigned)cdiv(a.m, tile));
    const auto at = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        if (a.dtype == DT_BF16) hipLaunchKernelGGL((k_ce_own<bf16_t, NT>), g, dim3(NT), 0, s, p, tile, parts);
        else hipLaunchKernelGGL((k_ce_own<float, NT>), g, dim3(NT), 0, s, p, tile, parts);
    };
    if (parts >= 64) at(std::integral_constant<int, 1024>{});
    else at(std::integral_constant<int, kThreads>{});
    return hipGetLastError();
}

// both products of g (dh has dh_rows results a column, dw `wide`)
hipError_t pair(const CeCall &a, const CeGemm &dh, const CeGemm &dw, const CeTile &t, int64_t dh_rows, int64_t wide, hipStream_t s)
{
    const double es = a.dtype == DT_BF16 ? 2 : 4;
    TraceScope tr(KC_CONV, KID_LINEAR_CE, s, es * ((double)a.m * wide + (2.0 * a.m + 2.0 * wide) * a.c), 4.0 * a.m * wide * a.c);
    const int64_t cols = cdiv(a.c, t.bj), first = cdiv(cdiv(dh_rows, t.bi) * cols * dh.parts, 8) * 8;
    const dim3 g = wide_grid(first + cdiv(wide, t.bi) * cols * dw.parts);
    if (a.dtype != DT_BF16) hipLaunchKernelGGL((k_ce_pair<float, 64, 128, 2, 2>), g, dim3(256), 0, s, dh, dw, (int)first);
    else if (t.bi == 256) hipLaunchKernelGGL((k_ce_pair<bf16_t, 256, 256, 2, 4>), g, dim3(512), 0, s, dh, dw, (int)first);
    else hipLaunchKernelGGL((k_ce_pair<bf16_t, 128, 128, 2, 2>), g, dim3(256), 0, s, dh, dw, (int)first);
    return hipGetLastError();
}

// What both directions keep in the workspace: the count, the list and the rows' copy.
struct CeHead {
    int64_t counts, rows, copy, end;
    explicit CeHead(const CeCall &a)
    {
        const int64_t es = a.dtype == DT_BF16 ? 2 : 4;
        counts = 256;
        rows = up256(counts + (a.m > 4 * kCountRows ? cdiv(a.m, kCountRows) * 4 : 0));
        copy = up256(rows + a.m * (int64_t)sizeof(CeRow));
        end = up256(copy + a.m * (int64_t)a.c * es);
    }
};

hipError_t launch_list(const CeCall &a, const CeHead &w, char *ws, hipStream_t s)
{
    const int es = a.dtype == DT_BF16 ? 2 : 4;
    CeList p{};
    p.m = a.m; p.classes = a.classes; p.ignore = a.ignore;
    p.labels = a.labels;
    p.count = (int *)ws;
    p.factor = (float *)(ws + 8);
    p.counts = a.m > 4 * kCountRows ? (int *)(ws + w.counts) : nullptr;
    p.rows = (CeRow *)(ws + w.rows);
    p.h = a.h; p.h_ld = a.h_ld * es;
    p.copy = ws + w.copy; p.row_bytes = a.c * es;
    if (a.loss) { p.zero_loss = a.loss; p.zero_lse = a.lse; }
    else { p.lse = a.lse; p.dloss = a.dloss; p.zero = a.dh; p.zero_ld = a.dh_ld * es; }
    TraceScope tr(KC_SMALL, KID_LINEAR_CE, s, 2.0 * a.m * p.row_bytes, 0.0);
    if (p.counts) hipLaunchKernelGGL(k_ce_count, dim3((unsigned)cdiv(a.m, kCountRows)), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL(k_ce_list, dim3((unsigned)cdiv(a.m, kListRows)), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

struct CeFwdPlan {
    CeHead head;
    CeTile tile;
    int64_t tiles, loss_rows, groups, stats, sums, picked, part, end;
    explicit CeFwdPlan(const CeCall &a) : head(a)
    {
        tile = ce_logit_tile(a.dtype, a.m, a.classes);
        tiles = cdiv(a.classes, tile.bj);
        loss_rows = a.m > kLossRows && a.m <= kLossWide && tiles < 64 ? kLossWide : kLossRows;
        groups = cdiv(a.m, loss_rows);
        stats = tile.small ? 0 : head.end;       // (few rows are taken as they are)
        sums = up256(stats + tiles * a.m * 8);
        picked = up256(sums + (a.smoothing > 0.f ? tiles * a.m * 4 : 0));
        part = up256(picked + a.m * 4);
        end = up256(part + groups * 16);
    }
};

// The widest piece of the classes whose g takes at most kPieceBytes, or kFewClasses of them (8192 x 4096 x 131072:
// 18.8 ms with 256 MiB and with 512, 18.5 with 1 GiB).
constexpr int64_t kPieceBytes = (int64_t)256 << 20;
constexpr int64_t kPieceWidth = kCeMaxLd;
struct CeBwdPlan {
    bool gather() const { return pieces > 1 || dh_parts > 1 || few; }      // dh leaves the products as parts
    CeHead head;
    int64_t pieces, width;                 // classes of a piece, a multiple of 256
    CeTile grad_tile, dh_tile, dw_tile;
    int grad_rows, dh_parts, dw_parts;     // grad_rows: of a partial row of dbias
    int few;                               // groups of 16 rows of g's second form (0: many rows)
    int own_parts;                         // column parts of the others' sums (0: the labels' entries stay as they are)
    int64_t g, gt, dh, dw, colsum, others, prob, end;
    explicit CeBwdPlan(const CeCall &a) : head(a)
    {
        const int64_t es = a.dtype == DT_BF16 ? 2 : 4, bk = 128 / es;
        int64_t most = kPieceBytes / (a.m * es) / 256 * 256;
        most = most < kFewClasses ? kFewClasses : (most > kPieceWidth ? kPieceWidth : most);
        pieces = cdiv(a.classes, most);
        width = cdiv(cdiv(a.classes, pieces), 256) * 256;
        pieces = cdiv(a.classes, width);
        const int64_t wide = width < a.classes ? width : a.classes;
        grad_tile = ce_logit_tile(a.dtype, a.m, wide);
        grad_rows = grad_tile.small ? grad_tile.bi : grad_tile.bi / 2;
        few = a.dtype == DT_BF16 && a.m <= kFewRows ? (a.m <= 16 ? 1 : (a.m <= 32 ? 2 : 4)) : 0;   // (tiles of k_ce_small: 32 rows past 16)
        const int64_t rows = few ? 2 * a.m : a.m;
        // few rows: dh streams the weights past them, dw writes more than it multiplies
        dh_tile = rows <= 32 ? CeTile{32, a.dtype == DT_BF16 ? 256 : 128, false} : ce_tile(a.dtype, rows, a.c);
        dw_tile = a.dtype == DT_BF16 && a.m <= 128 ? CeTile{128, 128, false} : ce_tile(a.dtype, wide, a.c);
        // one launch for both, which is shorter than two (5037 x 792 x 101207: 3301 us apart): a dw of
        // few stages in the smaller tiles, else a dh in the larger.  Measured in the smaller and the
        // larger, the crossing lies between 300 and 400 rows of 2048 channels (32768 classes: 178 us
        // and 192 with 300 rows, 391 and 378 with 1001, 1774 and 1601 with 5037), between 300 and 1001
        // of 792 (101207 classes: 283 and 321, 674 and 661, 2880 and 2788) and of 4096 (16384: 183 and
        // 200, 382 and 369), and past 5037 of 776 (40961: 131 and 149, 256 and 267, 1130 and 1214).
        if (dw_tile.bi == 256 && dh_tile.bi == 128) (a.m < 1024 ? dw_tile : dh_tile) = a.m < 1024 ? dh_tile : dw_tile;
        dh_parts = ce_parts(dh_tile, rows, a.c, cdiv(wide, bk), 2);
        dw_parts = few ? 1 : ce_parts(dw_tile, wide, a.c, cdiv(a.m, bk), 4);
        g = head.end;
        gt = up256(g + rows * width * es);
        dh = up256(gt + few * width * 64);
        dw = up256(dh + (a.dh && gather() ? dh_parts * rows * a.c * 4 : 0));
        colsum = up256(dw + (a.dw && dw_parts > 1 ? dw_parts * wide * a.c * 4 : 0));
        // (its place does not depend on smoothing, which the size query does not know)
        const bool shows = a.classes <= kFewClasses || a.dtype == DT_F32 || few;
        const int64_t parts = pieces == 1 && shows ? cdiv(a.classes, grad_tile.bj) : 0;
        own_parts = a.smoothing >= kOwnSmoothing && a.classes > kFewClasses ? 0 : (int)parts;
        others = up256(colsum + (a.dbias ? cdiv(a.m, grad_tile.bi) * (grad_tile.bi / grad_rows) * wide * 4 : 0));   // (of a piece)
        prob = up256(others + parts * a.m * 4);
        end = up256(prob + (parts ? a.m * 4 : 0));
    }
};

// (with dbias's workgroups behind it where `bias` asks for them)
hipError_t sum_parts(const CeSum &p, const CeBias &bias, int dtype, int64_t rows, hipStream_t s)
{
    TraceScope tr(KC_SMALL, KID_LINEAR_CE, s, ((double)p.parts * 4 + (dtype == DT_BF16 ? 2 : 4)) * rows * p.c, 0.0);
    const int64_t vecs = rows * (p.c / 4);
    const bool shared = vecs < 512 * kThreads && p.parts >= 8;   // (16 x 2048 of 64 parts: 13 us one thread a vector)
    const int first = (int)cdiv(vecs, shared ? kThreads / 8 : kThreads);
    const dim3 grid = wide_grid(first + (bias.out ? cdiv(bias.classes, kThreads) : 0)), block(kThreads);
    if (dtype == DT_BF16) {
        if (shared) hipLaunchKernelGGL((k_ce_sum<bf16_t, 8>), grid, block, 0, s, p, bias, first);
        else hipLaunchKernelGGL((k_ce_sum<bf16_t, 1>), grid, block, 0, s, p, bias, first);
    } else {
        if (shared) hipLaunchKernelGGL((k_ce_sum<float, 8>), grid, block, 0, s, p, bias, first);
        else hipLaunchKernelGGL((k_ce_sum<float, 1>), grid, block, 0, s, p, bias, first);
    }
    return hipGetLastError();
}

// classes in ranges that give the chip four workgroups a CU
hipError_t launch_outer(const CeCall &a, const CeGemm &p, int few, hipStream_t s)
{
    const int64_t blocks = cdiv(a.c, 256), ranges = cdiv(1024, blocks);
    const int chunk = (int)(cdiv(cdiv(p.classes, ranges), 16) * 16);
    const dim3 grid((unsigned)(blocks * cdiv(p.classes, chunk)));
    TraceScope tr(KC_CONV, KID_LINEAR_CE, s, (double)p.classes * a.c * (a.dw_dtype == DT_BF16 ? 2 : 4), 2.0 * a.m * p.classes * a.c);
    const auto at = [&](auto w, auto kb) {
        hipLaunchKernelGGL((k_ce_outer<decltype(w), decltype(kb)::value>), grid, dim3(kThreads), 0, s, p, chunk);
    };
    const auto of = [&](auto w) {
        if (few == 1) at(w, std::integral_constant<int, 1>{});
        else if (few == 2) at(w, std::integral_constant<int, 2>{});
        else at(w, std::integral_constant<int, 4>{});
    };
    if (a.dw_dtype == DT_BF16) of(bf16_t{});
    else of(float{});
    return hipGetLastError();
}

#define CE_TRY(e)                            \
    do {                                     \
        const hipError_t _e = (e);           \
        if (_e != hipSuccess) return _e;     \
    } while (0)

}  // namespace

size_t ce_fwd_bytes(const CeCall &a) { return (size_t)CeFwdPlan(a).end; }
size_t ce_bwd_bytes(const CeCall &a) { return (size_t)CeBwdPlan(a).end; }

hipError_t launch_ce_fwd(const CeCall &a, void *ws_, hipStream_t s)
{
    char *ws = (char *)ws_;
    const CeFwdPlan w(a);
    const int es = a.dtype == DT_BF16 ? 2 : 4;
    CeGemm p{};
    p.c = a.c; p.classes = a.classes; p.m = a.m; p.parts = 1;
    if (w.tile.small) {
        p.i = a.h; p.i_ld = a.h_ld * es;
        p.labels = a.labels;
    } else {
        CE_TRY(launch_list(a, w.head, ws, s));
        p.count = (const int *)ws; p.rows = (const CeRow *)(ws + w.head.rows);
        p.i = ws + w.head.copy; p.i_ld = (int64_t)a.c * es;
    }
    p.j = a.w; p.j_ld = a.w_ld * es;
    p.bias = a.bias;
    p.stats = (float2 *)(ws + w.stats);
    p.sums = a.smoothing > 0.f ? (float *)(ws + w.sums) : nullptr;
    p.picked = (float *)(ws + w.picked);
    CE_TRY(gemm<CE_STATS>(a, p, w.tile, a.m, a.classes, a.c, s));
    CeLoss l{};
    l.count = p.count; l.rows = p.rows; l.labels = a.labels; l.ignore = a.ignore;
    l.stats = p.stats; l.sums = p.sums; l.picked = p.picked;
    l.m = a.m; l.tiles = (int)w.tiles; l.groups = (int)w.groups; l.classes = a.classes;
    l.hit = 1.0 - (double)a.smoothing; l.flat = (double)a.smoothing / a.classes; l.z = a.z;
    l.loss = a.loss; l.lse = a.lse; l.part = (double2 *)(ws + w.part);
    TraceScope tr(KC_SMALL, KID_LINEAR_CE, s, 8.0 * a.m * w.tiles, 0.0);
    // (a single row takes all threads, and many tiles take 64 threads a row instead of 16)
    if (a.m == 1) hipLaunchKernelGGL((k_ce_rows<1, kThreads>), dim3(1), dim3(kThreads), 0, s, l);
    else if (w.loss_rows == kLossWide) hipLaunchKernelGGL((k_ce_rows<kLossWide, 1024>), dim3(1), dim3(1024), 0, s, l);
    else if (w.tiles >= 64) hipLaunchKernelGGL((k_ce_rows<kLossRows, 1024>), dim3((unsigned)w.groups), dim3(1024), 0, s, l);
    else hipLaunchKernelGGL((k_ce_rows<kLossRows, kThreads>), dim3((unsigned)w.groups), dim3(kThreads), 0, s, l);
    if (w.groups > 1) hipLaunchKernelGGL(k_ce_mean, dim3(1), dim3(1024), 0, s, l);
    return hipGetLastError();
}

hipError_t launch_ce_bwd(const CeCall &a, void *ws_, hipStream_t s)
{
    char *ws = (char *)ws_;
    const CeBwdPlan w(a);
    const int es = a.dtype == DT_BF16 ? 2 : 4;
    CE_TRY(launch_list(a, w.head, ws, s));
    CeGemm p{};
    p.count = (const int *)ws; p.rows = (const CeRow *)(ws + w.head.rows); p.factor = (const float *)(ws + 8);
    p.c = a.c; p.m = a.m;
    p.z = a.z; p.hit = 1.f - a.smoothing; p.flat = a.smoothing / (float)a.classes;
    p.g = ws + w.g; p.g_ld = w.width;
    p.colsum_ld = w.width < a.classes ? w.width : a.classes;
    const char *copy = ws + w.head.copy;
    const bool gather_dh = w.gather();
    const int64_t dh_rows = w.few ? 2 * a.m : a.m;
    if (w.few) { p.gt = ws + w.gt; p.gt_rows = w.few; }
    // dbias: of each piece, by the launch that adds up dh where that is behind all classes
    const bool bias_behind = w.pieces == 1 && a.dh && gather_dh;
    CeBias b{};
    b.count = p.count; b.tile = w.grad_rows; b.factor = p.factor;
    b.colsum = (const float *)(ws + w.colsum); b.ld = p.colsum_ld; b.out = a.dbias;
    for (int64_t n = 0; n < w.pieces; n++) {
        const int64_t first = n * w.width;
        const int64_t wide = a.classes - first < w.width ? a.classes - first : w.width;
        const char *weights = (const char *)a.w + first * a.w_ld * es;
        p.classes = (int)wide; p.first = (int)first;
        CeGemm q = p;
        q.parts = 1;
        q.i = copy; q.i_ld = (int64_t)a.c * es;
        q.j = weights; q.j_ld = a.w_ld * es;
        q.bias = a.bias ? a.bias + first : nullptr;
        q.colsum = a.dbias ? (float *)(ws + w.colsum) : nullptr;
        q.others = w.own_parts ? (float *)(ws + w.others) : nullptr;
        q.prob = (float *)(ws + w.prob);
        CE_TRY(gemm<CE_GRAD>(a, q, w.grad_tile, a.m, wide, a.c, s));
        if (w.own_parts) CE_TRY(launch_own(a, q, w.grad_rows, w.own_parts, s));
        b.classes = (int)wide;
        if (a.dbias && !bias_behind) {
            b.out = a.dbias + first;
            TraceScope tr(KC_SMALL, KID_LINEAR_CE, s, 4.0 * wide * (cdiv(a.m, w.grad_rows) + 1), 0.0);
            hipLaunchKernelGGL(k_ce_bias, dim3((unsigned)cdiv(wide, kThreads)), dim3(kThreads), 0, s, b);
        }
        CeGemm dh = p, dw = p;
        dh.i = dw.i = p.g; dh.i_ld = dw.i_ld = w.width * es;
        dh.j = weights; dh.j_ld = a.w_ld * es;
        dh.parts = w.dh_parts;
        dh.out = a.dh; dh.out_ld = a.dh_ld; dh.out_f32 = a.dtype == DT_F32;
        if (gather_dh) {
            dh.out = ws + w.dh; dh.out_ld = a.c; dh.out_f32 = 1;
            dh.part_stride = dh_rows * a.c; dh.add = n > 0;
        }
        dw.j = copy; dw.j_ld = (int64_t)a.c * es;
        dw.parts = w.dw_parts;
        dw.out = (char *)a.dw + first * a.dw_ld * (a.dw_dtype == DT_BF16 ? 2 : 4);
        dw.out_ld = a.dw_ld; dw.out_f32 = a.dw_dtype == DT_F32;
        CeSum t{};
        t.parts = w.dw_parts; t.c = a.c; t.n = wide; t.factor = p.factor;
        t.out = dw.out; t.out_ld = a.dw_ld;
        if (w.dw_parts > 1) {
            dw.out = ws + w.dw; dw.out_ld = a.c; dw.out_f32 = 1; dw.part_stride = wide * a.c;
            t.part = (const float *)dw.out; t.part_stride = dw.part_stride;
        }
        if (a.dh && a.dw && !w.few && w.dh_tile.bi == w.dw_tile.bi) {
            CE_TRY(pair(a, dh, dw, w.dh_tile, dh_rows, wide, s));
        } else {
            if (a.dh) CE_TRY(gemm<CE_DH>(a, dh, w.dh_tile, dh_rows, a.c, wide, s));
            if (a.dw && w.few) {
                dw.i = copy;
                CE_TRY(launch_outer(a, dw, w.few, s));
            } else if (a.dw) {
                CE_TRY(gemm<CE_DW>(a, dw, w.dw_tile, wide, a.c, a.m, s));
            }
        }
        if (a.dw && w.dw_parts > 1) CE_TRY(sum_parts(t, CeBias{}, a.dw_dtype, wide, s));
    }
    if (a.dh && gather_dh) {
        CeSum t{};
        t.part = (const float *)(ws + w.dh); t.part_stride = dh_rows * a.c; t.twice = w.few ? 1 : 0; t.parts = w.dh_parts; t.c = a.c;
        t.rows = p.rows; t.count = p.count; t.factor = p.factor;
        t.out = a.dh; t.out_ld = a.dh_ld;
        CE_TRY(sum_parts(t, bias_behind ? b : CeBias{}, a.dtype, a.m, s));
    }
    return hipGetLastError();
}

}  // namespace bnr
