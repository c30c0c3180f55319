// Orthogonalised updates: the matrices of a flat vector through Newton-Schulz products.
//
// A matrix is worked on as X [m, n], m <= n (transposed if it is tall).  Per step
//   G = X X' ;  B = b G + c G G ;  X <- a X + B X
// are three launches, each over the tiles of ALL matrices of the plan (a table in device memory says which tile a workgroup
// takes), so sixty layers of one model are three launches and not 180.  G and B are symmetric: only tiles on and below the
// diagonal are computed, the others are written as their transposes.
//
// Operands.  An fp32 value is held as hi + lo, two IEEE halves of 11 bits, hi = RN16(x), lo = RN16(x - hi), and a product of
// such operands is hi hi + hi lo + lo hi on the matrix cores with one fp32 sum: 22 bits, what is left out is 2^-22 of the
// product.  Half precision rather than bf16 because entries are bounded (|X| <= 1, singular values at most about 1.2): three
// more bits of significand per product for the same rate; the range is used by scaling with powers of two, X by 2^14, G by 2^13 and
// B by 2^12, the largest that their bounds allow.  Where lo falls below the smallest half, 2^-24, bits are lost: an entry of X is
// off by 2^-22 of itself or by 2^-39 of the norm, whichever is more, so rows and columns with entries below 2^-17 of the norm
// keep fewer than 22 bits.  (300 x 700, every other row times 1e-6: those rows are off by 3.6e-4 of themselves; by 1.1e-2 if X is
// scaled for entries near 16 in an orthogonal matrix, 2^9 here.)
// Roundings of X lie in all directions, and those of singular values near zero grow by a in every step, 3.44^5 = 485 times, while
// the strong ones stay near 1.  Where all are of one size the entries of X grow with the roundings; where a few
// fill the entries they do not.  768 x 2048, off by (relative to the whole, in fp32; rounding to bf16: 1.7e-3)
//                                    two halves   fp32 products   one half (DS_ORTHO_HALF)
//   noise                               2.3e-6        3.6e-6        1.1e-3
//   singular values 1 / k               4.6e-6        4.2e-6        4.0e-3
//   1 / k^1.5                           1.3e-5        1.6e-5        1.2e-2
//   rank 16                             5.7e-5        4.3e-5        4.6e-2
//   rank 2                              7.4e-5        8.5e-5        7.1e-2
//   rank 1                              1.4e-4        2.3e-4        1.5e-1
//
// Layout.  An operand lies in panels of 16 columns (32 with one half): row after row 64 bytes, 16 hi and 16 lo (32 halves).  A
// stage of a product, 16 (32) values of k, is then one contiguous piece of a tile's rows when k runs along the rows, and
// pieces of 1 KB (2 KB) when k runs across them.
//
// What bounds it.  One 4096 x 4096: the matrix cores and the power they draw: B X of 256 x 256 tiles runs at 1.1 to 1.3 PFLOP/s of
// half-precision products with the cores busy 75 % of the cycles at 1.65 GHz (the libraries' product of that size: 1.36).  G and
// B, 0.52 of the arithmetic each by symmetry, 1.1.  Many matrices of width 768: every tile is 48 (24) panels, and its first
// copies and results, 13 (7) us, come at the same time on all compute units: 0.9 (0.65) PFLOP/s.  Sums shorter still, or few
// tiles: the latency of 3 launches a step, 8 to 12 us each.
#include "ds_device.h"
#include "ds_internal.h"
#include "tails.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <vector>

using namespace ds;

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kRow = 64;                       // bytes of a row in a panel
constexpr float kOperandScale = 16384.0f;      // X is held times 2^14 (entries up to 4)
constexpr float kGramScale = 8192.0f;          // G is held times 2^13 (entries up to 8)
constexpr float kPolyScale = 4096.0f;          // B is held times 2^12 (entries up to 16)
constexpr int kTileSide = 64;
constexpr int kMaxParts = 512;                 // partial sums of a matrix's norm
constexpr int64_t kPartElements = 16384;
// A workspace beyond this, all of the card's memory, is refused before its tables are made, which would be gigabytes; one that
// is more than what is free is refused by its allocation.
constexpr int64_t kMostBytes = 288000000000;

struct Mat {
    int64_t offset, ld;          // in the vector
    int64_t x[2], g, b;          // byte offsets in the workspace
    int32_t rows, cols;          // as stored
    int32_t m, n, mp, np;        // as worked on: m <= n, and rounded up to tiles
    int32_t panel;               // bytes of a panel: mp rows
    int32_t flip;                // stored transposed
    int32_t part0, parts;        // partial sums of the norm
    float scale;                 // X is held times this
    float factor;
};

// What a workgroup of a product takes: tile (i, j) of a matrix, panels [k0, k1) of its sum.  slot < 0: the whole sum; else this
// part goes to that slot of the parts' buffer and a launch behind the product puts the parts together.
// The matrix stands in it: a number of one would cost a second trip to memory before the first copy.
struct Tile {
    int32_t mat, i, j, k0, k1, slot;
    Mat m;
};

struct Cut {                     // a tile in parts
    int32_t mat, i, j, slot, n, pad_[3];
};

template <bool SPLIT>
constexpr int kPanel = SPLIT ? 16 : 32;        // columns of a panel

// Byte of element (row, col) of an operand, of its hi where there are two.
template <bool SPLIT>
__device__ __forceinline__ int64_t element_at(int64_t panel, int row, int col)
{
    constexpr int W = kPanel<SPLIT>;
    return (col / W) * panel + row * kRow + (col % W) * 2;
}

constexpr int kToLo = kRow / 2;                // from hi to lo

template <bool SPLIT>
__device__ __forceinline__ void store8(char *p, const float *v)
{
    half8 hi, lo;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        hi[t] = static_cast<_Float16>(v[t]);
        lo[t] = static_cast<_Float16>(v[t] - static_cast<float>(hi[t]));
    }
    *reinterpret_cast<half8 *>(p) = hi;
    if (SPLIT) *reinterpret_cast<half8 *>(p + kToLo) = lo;
}

template <bool SPLIT>
__device__ __forceinline__ void store1(char *p, float v)
{
    const _Float16 hi = static_cast<_Float16>(v);
    *reinterpret_cast<_Float16 *>(p) = hi;
    if (SPLIT) *reinterpret_cast<_Float16 *>(p + kToLo) = static_cast<_Float16>(v - static_cast<float>(hi));
}

// Eight elements of a row as they lie in memory.
template <bool SPLIT>
struct Eight {
    half8 hi, lo;
    __device__ __forceinline__ void load(const char *p)
    {
        hi = *reinterpret_cast<const half8 *>(p);
        if (SPLIT) lo = *reinterpret_cast<const half8 *>(p + kToLo);
    }
    __device__ __forceinline__ void values(float *v) const
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = static_cast<float>(hi[t]) + (SPLIT ? static_cast<float>(lo[t]) : 0.f);
    }
};

template <bool BF16>
__device__ __forceinline__ float load_flat(const void *p, int64_t at)
{
    return BF16 ? bf16_widen(static_cast<const uint16_t *>(p)[at]) : static_cast<const float *>(p)[at];
}

__device__ __forceinline__ uint16_t bf16_round(float x)      // to nearest, ties to even; NaN stays NaN
{
    const uint32_t u = __float_as_uint(x);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return static_cast<uint16_t>((u >> 16) | 0x40u);
    return static_cast<uint16_t>((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

// Eight elements, the first n of them.
__device__ __forceinline__ void store_bf16(uint16_t *p, int n, const float *v)
{
    typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
    if (n >= 8) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = bf16_round(v[2 * e]) | (static_cast<uint32_t>(bf16_round(v[2 * e + 1])) << 16);
        __builtin_nontemporal_store(static_cast<u32x4_any>(w), reinterpret_cast<u32x4_any *>(p));
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = bf16_round(v[e]);
}

// ---------------------------------------------------------------------------------------
// norms and operands
// ---------------------------------------------------------------------------------------
// Four elements from `at` on, zero past `lim`; any alignment.
template <bool BF16>
__device__ __forceinline__ f32x4 load_flat4(const void *p, int64_t at, int64_t lim)
{
    if (!BF16) return ld4(static_cast<const float *>(p), at, lim);
    return ld4_bf16(static_cast<const uint16_t *>(p), at, lim);
}

// Partial sums of squares in fp64: part p of a matrix is a run of its elements.  Bound by the reads of U (sixty matrices, 85 M
// elements: 340 MB).
template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_ortho_norm(const Mat *__restrict__ mats, const int2 *__restrict__ parts, const void *src,
                                                       double *__restrict__ partial)
{
    __shared__ double lds[kWaves];
    const int2 pt = parts[blockIdx.x];
    const Mat M = mats[pt.x];
    const int64_t total = static_cast<int64_t>(M.rows) * M.cols;
    const int64_t each = ((total + M.parts - 1) / M.parts + 3) & ~static_cast<int64_t>(3);
    const int64_t lo = each * pt.y, hi = lo + each < total ? lo + each : total;
    double s = 0.0;
    if (M.ld == M.cols) {
#pragma unroll 8
        for (int64_t t = lo + threadIdx.x * 4; t < hi; t += kBlock * 4) {
            const f32x4 v = load_flat4<BF16>(src, M.offset + t, M.offset + hi);
            const double a = v.x, b = v.y, c = v.z, d = v.w;
            s = fma(a, a, s);
            s = fma(b, b, s);
            s = fma(c, c, s);
            s = fma(d, d, s);
        }
    } else {
        // column blocks: batches of eight elements asked for together
        for (int64_t t0 = lo + threadIdx.x; t0 < hi; t0 += kBlock * 8) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t t = t0 + e * kBlock < hi ? t0 + e * kBlock : lo;     // no branch: one would wait for every load
                const uint32_t r = static_cast<uint32_t>(t) / static_cast<uint32_t>(M.cols);
                v[e] = load_flat<BF16>(src, M.offset + r * M.ld + (t - static_cast<int64_t>(r) * M.cols));
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (t0 + e * kBlock >= hi) v[e] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), s);
        }
    }
    s = block_sum(s, lds, false);
    if (threadIdx.x == 0) partial[M.part0 + pt.y] = s;
}

// X = U / (norm + eps), times M.scale, zero beyond the matrix.
template <bool SPLIT, bool BF16>
__global__ __launch_bounds__(kThreads) void k_ortho_operands(const Tile *__restrict__ tiles, const void *src,
                                                             const double *__restrict__ partial, float eps, char *ws)
{
    constexpr int T = 64;
    __shared__ float tile[T][T + 1];
    __shared__ double sums[kThreads / 64];
    const Tile &tl = tiles[blockIdx.x];
    const Mat &M = tl.m;
    const int i0 = tl.i * T, j0 = tl.j * T;
    // the stored rows: four elements of one a thread, four rows
    const int row0 = M.flip ? j0 : i0, col0 = M.flip ? i0 : j0;
    const int c4 = (threadIdx.x & 15) * 4, r4 = threadIdx.x >> 4;
    f32x4 v[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int rr = row0 + r4 + 16 * t, c = col0 + c4;
        const int64_t row = M.offset + static_cast<int64_t>(rr) * M.ld;
        v[t] = rr < M.rows && c < M.cols ? load_flat4<BF16>(src, row + c, row + M.cols) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    double s = 0.0;
    for (int p = threadIdx.x; p < M.parts; p += kThreads) s += partial[M.part0 + p];
    s = wave_sum(s);
    if (lane_id() == 0) sums[wave_id()] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) s += sums[w];
    const double norm = sqrt(s) + static_cast<double>(eps);
    const double inv = norm == 0.0 ? 0.0 : static_cast<double>(M.scale) / norm;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int rr = r4 + 16 * t, c = c4 + e;
            (M.flip ? tile[c][rr] : tile[rr][c]) = static_cast<float>(static_cast<double>(v[t][e]) * inv);
        }
    __syncthreads();
    for (int t = threadIdx.x; t < T * T / 8; t += kThreads) {
        const int a = t / (T / 8), c = (t % (T / 8)) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[a][c + e];
        store8<SPLIT>(ws + M.x[0] + element_at<SPLIT>(M.panel, i0 + a, j0 + c), v);
    }
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
enum Stage { kGram, kPoly, kApply, kLast };    // G = X X' ; B = b G + c G G ; X <- a X + B X ; the same into the vector

constexpr int kStages = 4;                     // of a product's copies in LDS

// Whether sums may be cut into parts.  Tiles of 64 x 64 are for few or small ones, and then only G's sums, as long as the longer
// side, are worth a second launch: of 15,000 plans of 1 to 120 matrices up to 3000 x 3000, 769 cut G on such tiles and none B or X.
template <int SIDE, int STAGE>
constexpr bool kCanCut = SIDE != kTileSide || STAGE == kGram;

struct Step {
    float a, b, c;
    int from;                  // which of the two X the step starts from
};

// Where the last product goes.
struct Out {
    void *dst;                 // orthogonalised vector, or
    float *x;                  // the model: x <- keep x - gamma factor O
    float keep, gamma;
};

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Direct copy of 16 bytes per lane, from `base` + `offset` into LDS at `lds` + 16 l for lane l; `base` and `lds` are the same for
// the wavefront.  It has no output register.  Written as an instruction because the compiler waits for every
// outstanding copy of its own builtin before the next read of LDS, also of another stage; the wait that is needed
// stands in front of the barrier of that stage.  m0 is reserved (named as clobbered the compiler warns of it): nothing is allocated to
// it, the compiler sets it right before an instruction of its own that reads it, and in these kernels there is none.
__device__ __forceinline__ void copy_to_lds(const char *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(lds) : "memory");
}

// The same address in every lane, as a scalar.
__device__ __forceinline__ const char *uniform(const char *p)
{
    const uint64_t b = reinterpret_cast<uint64_t>(p);
    const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b)));
    const uint64_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b >> 32)));
    return reinterpret_cast<const char *>(lo | (hi << 32));
}

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)p));
}

__device__ __forceinline__ f32x16 mfma(half8 a, half8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Factors of the product and of the old value: the operands' scales away, the result's scale on.
template <int STAGE>
__device__ __forceinline__ float product_scale(const Mat &M, const Step &step)
{
    return STAGE == kGram ? kGramScale / (M.scale * M.scale)
           : STAGE == kPoly ? step.c * (kPolyScale / (kGramScale * kGramScale)) : 1.0f / kPolyScale;
}

template <int STAGE>
__device__ __forceinline__ float old_scale(const Step &step)
{
    return STAGE == kPoly ? step.b * (kPolyScale / kGramScale) : 0.f;
}

// a lies on B's diagonal, rounded as B is, so the last product does not read X a second time (124 M elements in fp32 3.79 ms, 3.94
// with a applied to X).  Its rounding is 2^-22 or 2^-11 of a row at most, as X's own is; but the sums hold a x from that
// panel on, and each of their roundings is relative to it: with two halves a rank of 16 comes out twice as far off as with a applied to X
// in fp32 (by an emulation), 1.3 times as far as by fp32 products (measured), matrices without strong directions nearer
// than those.  With one half results in bf16 of noise lie 1.9e-3 from those in 64 bits with it and 2.0e-3 without.
template <int STAGE>
constexpr bool kReadsOld = STAGE == kPoly;

// One element of a result from its product and the old value.
template <int STAGE>
__device__ __forceinline__ float result(float alpha, float beta, const Step &step, float product, float old, bool diagonal)
{
    float v = kReadsOld<STAGE> ? __fmaf_rn(beta, old, product * alpha) : product * alpha;
    if (STAGE == kPoly && diagonal) v = __fmaf_rn(step.a, kPolyScale, v);
    return v;
}

// Of a 32 x 32 part a lane holds row l % 32 and columns 8 t + 4 (l / 32) .. + 3, t = 0 .. 3; here the wavefront's halves
// exchange, and the lane has the eight columns from 16 g + 8 (l / 32) on.
struct EightColumns {
    float v[8];
    __device__ __forceinline__ EightColumns(const f32x16 &acc, int g)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * g + e]), __float_as_uint(acc[8 * g + 4 + e]), false, false);
            v[e] = __uint_as_float(w[0]);
            v[4 + e] = __uint_as_float(w[1]);
        }
    }
};

template <int N>
__device__ __forceinline__ void wait_copies()       // at most N copies of this wavefront under way, and its reads of LDS are done
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}

// One tile of TM x TN of C = P Q, by wavefronts of WM x WN.  P is read by rows of k.  Q = X' or G (symmetric) is read by rows
// of k as well; Q = X, in the last product, lies with k across the rows: its tile is transposed on the way from LDS to the
// registers.
//
// Pipeline.  LDS holds kStages stages of G panels, of 16 (32) values of k each.  While a panel is multiplied from registers, the
// fragments of the next are read from LDS and the copies of the stages behind, which pass no registers, are under way; one
// barrier a stage.  (Small tiles, whose panels are a few instructions, take two panels a stage.)
//
// LDS has 64 banks, 256 bytes.  A copy fills it linearly, so what a lane copies is chosen such that the 16-byte chunk c of
// row r lies at c ^ f(r), and 16 lanes that read 16 rows of one chunk (or, transposing, 32 lanes 4 rows of 4 chunks) meet
// different banks: 267 and 228 bytes a clock measured, 43 and 80 without.
//
// The wavefront multiplies Q' P': a lane then holds a row i of C and four consecutive j at a time.
template <int TM, int TN, int WM, int WN, int G, bool SPLIT, int STAGE, int OUT>      // OUT: 0 fp32, 1 bf16, 2 the model
__global__ __launch_bounds__((TM / WM) * (TN / WN) * 64) void k_ortho_product(const Tile *__restrict__ tiles, char *ws,
                                                                             float *parts, Step step, Out out)
{
    constexpr int S = kStages, WAVES_N = TN / WN, WAVES = (TM / WM) * WAVES_N, FM = WM / 32, FN = WN / 32;
    constexpr bool ACROSS = STAGE >= kApply;                   // Q is X
    constexpr int K = kPanel<SPLIT>, PIECE = K * kRow;         // values of k in a stage; a panel's part of a stage of X
    constexpr int PBYTES = TM * kRow, QBYTES = TN * kRow, PANEL_BYTES = PBYTES + QBYTES, STAGE_BYTES = G * PANEL_BYTES;
    constexpr int PCOPIES = PBYTES / (WAVES * 1024), QCOPIES = QBYTES / (WAVES * 1024), COPIES = G * (PCOPIES + QCOPIES);
    static_assert(PCOPIES * WAVES * 1024 == PBYTES && QCOPIES * WAVES * 1024 == QBYTES && (G == 1 || G == 2), "tile");
    __shared__ __attribute__((aligned(256))) char lds[S * STAGE_BYTES];
    const Tile &tl = tiles[blockIdx.x];
    const Mat &M = tl.m;
    const int i0 = tl.i * TM, j0 = tl.j * TN, mp = M.mp, np = M.np;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int wi = (wave / WAVES_N) * WM, wj = (wave % WAVES_N) * WN;
    const int64_t panel = M.panel;
    const int stages = (tl.k1 - tl.k0) / G;                    // panels come in even numbers: rounded sizes are multiples of 64
    const char *X = ws + M.x[step.from];
    const char *P = STAGE == kGram ? X : ws + (STAGE == kPoly ? M.g : M.b);
    const char *Q = ACROSS ? X : P;
    // what this lane copies; a tile may reach past the rounded matrix, whose last rows then stand in for what is not there
    uint32_t pa[PCOPIES], qa[QCOPIES];
    const char *p_base = P, *q_base = ACROSS ? Q + (j0 / K) * panel : Q;
#pragma unroll
    for (int t = 0; t < PCOPIES; ++t) {
        const int at = (t * WAVES + wave) * 1024 + lane * 16, r = at / kRow, c = ((at % kRow) / 16) ^ ((r >> 2) & 3);
        pa[t] = (i0 + r < mp ? i0 + r : mp - 1) * kRow + c * 16;
    }
#pragma unroll
    for (int t = 0; t < QCOPIES; ++t) {
        const int at = (t * WAVES + wave) * 1024 + lane * 16;
        if (ACROSS) {
            const int b = at / PIECE, r = (at % PIECE) / kRow, c = ((at % kRow) / 16) ^ (SPLIT ? 2 * (b & 1) : 0);
            const int last = (np - j0) / K - 1;
            qa[t] = static_cast<uint32_t>(b < last ? b : last) * M.panel + r * kRow + c * 16;
        } else {
            const int r = at / kRow, c = ((at % kRow) / 16) ^ ((r >> 2) & 3);
            qa[t] = (j0 + r < mp ? j0 + r : mp - 1) * kRow + c * 16;
        }
    }
    const int64_t q_step = ACROSS ? PIECE : panel;
    p_base = uniform(p_base + tl.k0 * panel);
    q_base = uniform(q_base + tl.k0 * q_step);
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane(lds_address(lds)) + wave * 1024;
    auto copy = [&](int buffer) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint32_t to = lds_at + buffer * STAGE_BYTES + g * PANEL_BYTES;
#pragma unroll
            for (int t = 0; t < PCOPIES; ++t) copy_to_lds(p_base, pa[t], to + t * WAVES * 1024);
#pragma unroll
            for (int t = 0; t < QCOPIES; ++t) copy_to_lds(q_base, qa[t], to + PBYTES + t * WAVES * 1024);
            p_base += panel;
            q_base += q_step;
        }
    };
    // Fragments of 32 rows by 16 values: lane l holds row l % 32, values 8 (l / 32) .. + 7.  Two of them in a stage, q: hi and
    // lo, or the two halves of k.
    struct Frags {
        half8 p[2][FM], q[2][FN];
    };
    const int r = lane & 31, h = lane >> 5;
    const int row_at[2] = {r * kRow + ((h ^ ((r >> 2) & 3)) * 16), r * kRow + (((2 + h) ^ ((r >> 2) & 3)) * 16)};
    int col_at[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int g = (lane >> 4) & 1, k = h * 8 + ((lane & 15) >> 2), byte = (lane & 3) * 8;
        // split: group g of 16 columns is a panel of its own, hi or lo a half of its rows; one half: a half of the panel's rows
        col_at[q] = SPLIT ? g * PIECE + k * kRow + ((q ^ g) * 32) + byte : (q * 16 + k) * kRow + g * 32 + byte;
    }
    auto read = [&](Frags &f, int buffer, int g) {
        const char *lp = lds + buffer * STAGE_BYTES + g * PANEL_BYTES + wi * kRow, *lq = lp + PBYTES + (wj - wi) * kRow;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int b = 0; b < FN; ++b) {
                if (ACROSS) {
                    union { half8 v; s16x4 part[2]; } u;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        u.part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lq + b * 32 * kRow + col_at[q] + e * 4 * kRow));
                    f.q[q][b] = u.v;
                } else {
                    f.q[q][b] = *reinterpret_cast<const half8 *>(lq + b * 32 * kRow + row_at[q]);
                }
            }
#pragma unroll
            for (int a = 0; a < FM; ++a) f.p[q][a] = *reinterpret_cast<const half8 *>(lp + a * 32 * kRow + row_at[q]);
        }
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.f;

    auto multiply = [&](const Frags &f) {
        auto one = [&](int qp, int qq) {
#pragma unroll
            for (int a = 0; a < FM; ++a)
#pragma unroll
                for (int b = 0; b < FN; ++b)
                    acc[a][b] = mfma(f.q[qq][b], f.p[qp][a], acc[a][b]);
        };
        if (SPLIT) {
            one(1, 0);
            one(0, 1);
            one(0, 0);
        } else {
            one(0, 0);
            one(1, 1);
        }
    };
    for (int k = 0; k < S && k < stages; ++k) copy(k);
    Frags f0, f1;
    if (stages >= S) wait_copies<(S - 1) * COPIES>();
    else wait_copies<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    read(f0, 0, 0);
    int here = 0;                                          // buffer of stage k
    // The next panel's fragments are read while this one's are multiplied: the reads are spread over the first products, and
    // nothing of it crosses a barrier.
    auto read_and_multiply = [&](const Frags &now, Frags &next, int g) {
        __builtin_amdgcn_sched_barrier(0);
        read(next, here, g);
        multiply(now);
#pragma unroll
        for (int t = 0; t < 2 * (FM + (ACROSS ? 2 : 1) * FN); ++t) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);     // one matrix instruction,
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);     // one read of LDS
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // The last panel of stage k from `now`, the first of stage k + 1 into `next`; steady: as many stages follow as there are
    // buffers.  The last panel of all stands by itself, so that on every way to a multiplication the reads of the next
    // fragments come after those of its own: where the two ways met, the compiler waited for all of them.
    auto cross = [&](auto steady, int k, const Frags &now, Frags &next) {
        const int under_way = stages - 2 - k;              // stages after the next that have been asked for
        if (decltype(steady)::value || under_way >= S - 2) wait_copies<(S - 2) * COPIES>();
        else if (under_way == S - 3) wait_copies<(S - 3) * COPIES>();
        else wait_copies<0>();
        // everybody's copies of stage k + 1 are there, and everybody holds the end of stage k in registers
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        if (decltype(steady)::value || k + S < stages) copy(here);
        here = here + 1 == S ? 0 : here + 1;
        read_and_multiply(now, next, 0);
    };
    int k = 0;
    if constexpr (G == 2) {
        for (; k + S < stages; ++k) {
            read_and_multiply(f0, f1, 1);
            cross(std::true_type{}, k, f1, f0);
        }
        for (; k + 1 < stages; ++k) {
            read_and_multiply(f0, f1, 1);
            cross(std::false_type{}, k, f1, f0);
        }
        read_and_multiply(f0, f1, 1);
    } else {
        for (; k + 1 + S < stages; k += 2) {
            cross(std::true_type{}, k, f0, f1);
            cross(std::true_type{}, k + 1, f1, f0);
        }
        for (; k + 2 < stages; k += 2) {
            cross(std::false_type{}, k, f0, f1);
            cross(std::false_type{}, k + 1, f1, f0);
        }
        cross(std::false_type{}, k, f0, f1);
    }
    multiply(f1);

    if (kCanCut<TM, STAGE> && tl.slot >= 0) {
        // eight columns of all rows behind each other: what 64 threads of the joining launch read lies together
        float *mine = parts + static_cast<int64_t>(tl.slot) * (TM * TN);
#pragma unroll
        for (int a = 0; a < FM; ++a)
#pragma unroll
            for (int b = 0; b < FN; ++b)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const EightColumns c(acc[a][b], g);
                    float *p = mine + (((wj + b * 32 + 16 * g) / 8 + h) * TM + wi + a * 32 + r) * 8;
                    *reinterpret_cast<f32x4 *>(p) = f32x4{c.v[0], c.v[1], c.v[2], c.v[3]};
                    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{c.v[4], c.v[5], c.v[6], c.v[7]};
                }
        return;
    }
    const float alpha = product_scale<STAGE>(M, step), beta = old_scale<STAGE>(step);
    const int j_end = ACROSS ? np : mp;
    char *to = ws + (STAGE == kGram ? M.g : STAGE == kPoly ? M.b : M.x[1 - step.from]);
    // the last product goes into the vector along its rows, through LDS: a region of its own for every wavefront
    constexpr int PITCH = WN + 1;
    float *mine = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
    static_assert(WAVES * 32 * PITCH * 4 <= S * STAGE_BYTES, "LDS");
    const float f = M.factor / M.scale;
    // Vector t of the 32 rows of part a that this lane writes: V elements along a row of the vector.
    constexpr int V = OUT == 1 ? 8 : 4, EACH = 32 * WN / (64 * V);
    auto place = [&](int a, int t, int &i, int &j, int &n) {   // its first element in the part, and how many there are
        if (M.flip) {
            i = (lane % (32 / V)) * V;
            j = t * (64 * V / 32) + lane / (32 / V);
        } else {
            i = t * (64 * V / WN) + lane / (WN / V);
            j = (lane % (WN / V)) * V;
        }
        const int64_t gi = i0 + wi + a * 32 + i, gj = j0 + wj + j;
        n = M.flip ? (gj < M.n ? M.m - static_cast<int>(gi) : 0) : (gi < M.m ? M.n - static_cast<int>(gj) : 0);
        return M.offset + (M.flip ? gj * M.ld + gi : gi * M.ld + gj);
    };
    if (STAGE == kLast) __syncthreads();                       // the stages' fragments have been read by everybody
#pragma unroll
    for (int a = 0; a < FM; ++a) {
        const int ib = i0 + wi + a * 32;
        if (ib >= mp) break;                                   // rounded sizes are multiples of 64: whole 32 x 32 parts
        f32x4 model[STAGE == kLast && OUT == 2 ? EACH : 1];
        if constexpr (STAGE == kLast && OUT == 2) {            // asked for early: they arrive while the part is put together
#pragma unroll
            for (int t = 0; t < EACH; ++t) {
                int i, j, n;
                const int64_t at = place(a, t, i, j, n);
                model[t] = n > 0 ? ld4_stream(out.x, at, at + n) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        Eight<SPLIT> was[FN][2];                               // asked for together
        if (kReadsOld<STAGE>) {
#pragma unroll
            for (int b = 0; b < FN; ++b)
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    if (j0 + wj + b * 32 < j_end) was[b][g].load(P + element_at<SPLIT>(panel, ib + r, j0 + wj + b * 32 + 16 * g + 8 * h));
        }
#pragma unroll
        for (int b = 0; b < FN; ++b) {
            const int jb = j0 + wj + b * 32;
            if (jb >= j_end) break;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const EightColumns c(acc[a][b], g);
                float v[8], x[8];
                const int i = ib + r, j = jb + 16 * g + 8 * h;
                const int64_t at = element_at<SPLIT>(panel, i, j);
                if (kReadsOld<STAGE>) was[b][g].values(x);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = result<STAGE>(alpha, beta, step, c.v[e], x[e], i == j + e);
                if constexpr (STAGE != kLast) {
                    store8<SPLIT>(to + at, v);
                    if (STAGE < kApply && tl.i != tl.j) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) store1<SPLIT>(to + element_at<SPLIT>(panel, j + e, i), v[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) mine[r * PITCH + b * 32 + 16 * g + 8 * h + e] = v[e];
                }
            }
        }
        if constexpr (STAGE == kLast) {
            // written and read by the same wavefront: its own accesses of LDS stay in order
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
#pragma unroll
            for (int t = 0; t < EACH; ++t) {
                int i, j, n;
                const int64_t at = place(a, t, i, j, n);
                if (n <= 0) continue;
                float o[V];
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = mine[M.flip ? (i + e) * PITCH + j : i * PITCH + j + e] * f;
                if constexpr (OUT == 1) {
                    store_bf16(static_cast<uint16_t *>(out.dst) + at, n, o);
                } else {
                    f32x4 v = {o[0], o[1], o[2], o[3]};
                    if (OUT == 2) v = fma4(-out.gamma, v, out.keep * model[t]);
                    st4_stream(OUT == 2 ? out.x : static_cast<float *>(out.dst), at, at + n, v);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        }
    }
}

// Columns j .. j + 7 of row i of the last X, into the vector.
template <int OUT>
__device__ __forceinline__ void eight_into_vector(const Mat &M, const Out &out, int i, int j, const float *v)
{
    if (i >= M.m) return;
    const float f = M.factor / M.scale;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (j + e >= M.n) return;
        const int64_t to = M.offset + (M.flip ? static_cast<int64_t>(j + e) * M.ld + i : static_cast<int64_t>(i) * M.ld + j + e);
        const float o = v[e] * f;
        if (OUT == 0) static_cast<float *>(out.dst)[to] = o;
        else if (OUT == 1) static_cast<uint16_t *>(out.dst)[to] = bf16_round(o);
        else out.x[to] = __fmaf_rn(-out.gamma, o, out.keep * out.x[to]);
    }
}

// Tiles whose sums were taken in parts: the parts in their order, then as a whole tile goes on.  A thread takes eight columns of
// a row, a wavefront 64 rows.
template <int SIDE, bool SPLIT, int STAGE, int OUT>
__global__ __launch_bounds__(kThreads) void k_ortho_join(const Mat *__restrict__ mats, const Cut *__restrict__ cuts, char *ws,
                                                         const float *__restrict__ parts, Step step, Out out)
{
    constexpr int PER_TILE = SIDE * SIDE / 8 / kThreads;
    const Cut cut = cuts[blockIdx.x / PER_TILE];
    const Mat M = mats[cut.mat];
    const int t = (blockIdx.x % PER_TILE) * kThreads + threadIdx.x, row = t % SIDE, col = t / SIDE * 8;
    const int i = cut.i * SIDE + row, j = cut.j * SIDE + col;
    if (i >= M.mp || j >= (STAGE >= kApply ? M.np : M.mp)) return;
    const float *from = parts + static_cast<int64_t>(cut.slot) * (SIDE * SIDE) + t * 8;
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll 4
    for (int p = 0; p < cut.n; ++p) {
        s0 += *reinterpret_cast<const f32x4 *>(from);
        s1 += *reinterpret_cast<const f32x4 *>(from + 4);
        from += SIDE * SIDE;
    }
    const float alpha = product_scale<STAGE>(M, step), beta = old_scale<STAGE>(step);
    const int64_t at = element_at<SPLIT>(M.panel, i, j);
    float v[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w}, x[8];
    if (kReadsOld<STAGE>) {
        Eight<SPLIT> was;
        was.load(ws + M.g + at);
        was.values(x);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = result<STAGE>(alpha, beta, step, v[e], x[e], i == j + e);
    if constexpr (STAGE != kLast) {
        char *to = ws + (STAGE == kGram ? M.g : STAGE == kPoly ? M.b : M.x[1 - step.from]);
        store8<SPLIT>(to + at, v);
        if (STAGE < kApply && cut.i != cut.j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) store1<SPLIT>(to + element_at<SPLIT>(M.panel, j + e, i), v[e]);
        }
    } else {
        eight_into_vector<OUT>(M, out, i, j, v);
    }
}

// ---------------------------------------------------------------------------------------
// small matrices: one workgroup and one launch for all of it
// ---------------------------------------------------------------------------------------
constexpr int kSmallBytes = 144 * 1024;        // X and G in LDS
constexpr int kSmallBytesMany = 40 * 1024;     // so that four of them share a compute unit

template <bool SPLIT>
int64_t small_bytes(int64_t mp, int64_t np) { return (mp * np + mp * mp) * (SPLIT ? 4 : 2); }

// Norm, operands, all steps and the result of one matrix, X [MP, np] and G (B in its place) in LDS.  Chains of small
// dependent products are bound by latency: five steps on 96 x 64 took 17 launches and 54 us, 25 us so.  Of 4.5 us a step the 60
// dependent matrix instructions take 0.9; the rest is trips through LDS, transposes two bytes at a time and barriers, with
// one wavefront per SIMD.
//
// Panels as in the large form; chunk c of row r of panel p lies at c ^ f(r, p), f = (r / 4) % 4, and with two halves the
// panels take turns with hi and lo: 16 lanes that read rows, and 32 lanes that read transposing, meet different banks.
template <int MP, int CAP, bool SPLIT, bool BF16, int OUT>
__global__ __launch_bounds__(kThreads) void k_ortho_small(const Mat *__restrict__ mats, const int32_t *__restrict__ list, const void *src,
                                                          const float *__restrict__ coef, int steps, float eps, Out out)
{
    constexpr int K = kPanel<SPLIT>, PANEL = MP * kRow, NB = MP / 32, WAVES = kThreads / 64, GBYTES = MP / K * PANEL;
    constexpr int SQUARE = NB * (NB + 1) / 2, PER_WAVE = (SQUARE + WAVES - 1) / WAVES;
    __shared__ __attribute__((aligned(256))) char lds[CAP];
    __shared__ double sums[WAVES];
    const Mat M = mats[list[blockIdx.x]];
    const int np = M.np, lane = lane_id(), wave = wave_id(), r = lane & 31, h = lane >> 5;
    char *G = lds, *X = lds + GBYTES;
    auto chunk = [&](char *base, int row, int panel, int c) {
        return base + panel * PANEL + row * kRow + ((c ^ ((row >> 2) & 3) ^ (SPLIT ? 2 * (panel & 1) : 0)) * 16);
    };
    auto put8 = [&](char *base, int row, int col, const float *v) {
        half8 hi, lo;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            hi[t] = static_cast<_Float16>(v[t]);
            lo[t] = static_cast<_Float16>(v[t] - static_cast<float>(hi[t]));
        }
        *reinterpret_cast<half8 *>(chunk(base, row, col / K, (col % K) / 8)) = hi;
        if (SPLIT) *reinterpret_cast<half8 *>(chunk(base, row, col / K, 2 + (col % K) / 8)) = lo;
    };
    auto put1 = [&](char *base, int row, int col, float v) {
        const _Float16 hi = static_cast<_Float16>(v);
        *reinterpret_cast<_Float16 *>(chunk(base, row, col / K, (col % K) / 8) + (col & 7) * 2) = hi;
        if (SPLIT)
            *reinterpret_cast<_Float16 *>(chunk(base, row, col / K, 2 + (col % K) / 8) + (col & 7) * 2) =
                static_cast<_Float16>(v - static_cast<float>(hi));
    };
    auto get8 = [&](char *base, int row, int col, float *v) {
        const half8 hi = *reinterpret_cast<const half8 *>(chunk(base, row, col / K, (col % K) / 8));
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = static_cast<float>(hi[t]);
        if (SPLIT) {
            const half8 lo = *reinterpret_cast<const half8 *>(chunk(base, row, col / K, 2 + (col % K) / 8));
#pragma unroll
            for (int t = 0; t < 8; ++t) v[t] += static_cast<float>(lo[t]);
        }
    };
    // fragments of a panel's values of k: q = hi and lo, or the panel's two halves of k
    auto rows = [&](char *base, int row0, int panel, int q) {
        return *reinterpret_cast<const half8 *>(chunk(base, row0 + r, panel, q * 2 + h));
    };
    auto columns = [&](int col0, int k0, int q) {
        union { half8 v; s16x4 part[2]; } u;
        const int g = (lane >> 4) & 1;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int k = k0 + (SPLIT ? 0 : q * 16) + h * 8 + e * 4 + ((lane & 15) >> 2);
            const char *p = SPLIT ? chunk(X, k, col0 / K + g, q * 2 + ((lane & 3) >> 1)) : chunk(X, k, col0 / K, g * 2 + ((lane & 3) >> 1));
            u.part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + (lane & 1) * 8));
        }
        return u.v;
    };
    auto multiply = [&](const half8 *p, const half8 *q, f32x16 acc) {
        if (SPLIT) {
            acc = mfma(q[0], p[1], acc);
            acc = mfma(q[1], p[0], acc);
            return mfma(q[0], p[0], acc);
        }
        acc = mfma(q[0], p[0], acc);
        return mfma(q[1], p[1], acc);
    };

    double s = 0.0;
    const uint32_t total = static_cast<uint32_t>(M.rows) * M.cols, cols = M.cols;
    for (uint32_t t0 = threadIdx.x; t0 < total; t0 += kThreads * 16) {       // sixteen elements asked for together
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t t = t0 + e * kThreads < total ? t0 + e * kThreads : 0u, row = t / cols;     // no branch: one would wait
            v[e] = load_flat<BF16>(src, M.offset + row * M.ld + (t - row * cols));
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (t0 + e * kThreads >= total) v[e] = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) s = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), s);
    }
    s = wave_sum(s);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += sums[w];
    const double norm = sqrt(s) + static_cast<double>(eps);
    const double inv = norm == 0.0 ? 0.0 : static_cast<double>(M.scale) / norm;
#pragma unroll 4
    for (int t = threadIdx.x; t < MP * np / 8; t += kThreads) {
        const int i = M.flip ? t % MP : t / (np / 8), j = (M.flip ? t / MP : t % (np / 8)) * 8;
        float v[8];
        const int64_t row = M.offset + (M.flip ? i : i * M.ld), step = M.flip ? M.ld : 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {                          // no branch here either
            const int64_t at = row + (j + e) * step;
            v[e] = load_flat<BF16>(src, i < M.m & j + e < M.n ? at : M.offset);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = i < M.m & j + e < M.n ? static_cast<float>(static_cast<double>(v[e]) * inv) : 0.f;
        put8(X, i, j, v);
    }
    __syncthreads();

    for (int k = 0; k < steps; ++k) {
        const Step step{coef[3 * k], coef[3 * k + 1], coef[3 * k + 2], 0};
        auto square = [&](auto stage) {
            constexpr int STAGE = decltype(stage)::value;
            const float alpha = product_scale<STAGE>(M, step), beta = old_scale<STAGE>(step);
            f32x16 acc[PER_WAVE];
#pragma unroll
            for (int u = 0; u < PER_WAVE; ++u) {
                const int t = u * WAVES + wave;
                if (t >= SQUARE) break;
                const int bi = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, bj = t - bi * (bi + 1) / 2;
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[u][e] = 0.f;
                char *from = STAGE == kGram ? X : G;
                const int panels = (STAGE == kGram ? np : MP) / K;
#pragma unroll 4
                for (int p = 0; p < panels; ++p) {
                    const half8 fp[2] = {rows(from, bi * 32, p, 0), rows(from, bi * 32, p, 1)};
                    const half8 fq[2] = {rows(from, bj * 32, p, 0), rows(from, bj * 32, p, 1)};
                    acc[u] = multiply(fp, fq, acc[u]);
                }
            }
            if (STAGE == kPoly) __syncthreads();               // everybody has read G, B takes its place
#pragma unroll
            for (int u = 0; u < PER_WAVE; ++u) {
                const int t = u * WAVES + wave;
                if (t >= SQUARE) break;
                const int bi = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, bj = t - bi * (bi + 1) / 2;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const EightColumns c(acc[u], g);
                    const int i = bi * 32 + r, j = bj * 32 + 16 * g + 8 * h;
                    float v[8];
                    if (STAGE == kPoly) get8(G, i, j, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = result<STAGE>(alpha, beta, step, c.v[e], v[e], i == j + e);
                    put8(G, i, j, v);
                    if (bi != bj)
#pragma unroll
                        for (int e = 0; e < 8; ++e) put1(G, j + e, i, v[e]);
                }
            }
            __syncthreads();
        };
        square(std::integral_constant<int, kGram>{});
        square(std::integral_constant<int, kPoly>{});
        // X <- a X + B X: a wavefront's columns are its own, so X changes in place
        const float alpha = product_scale<kApply>(M, step);
        for (int bj = wave; bj < np / 32; bj += WAVES) {
            f32x16 acc[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[b][e] = 0.f;
            for (int p = 0; p < MP / K; ++p) {
                const half8 fq[2] = {columns(bj * 32, p * K, 0), columns(bj * 32, p * K, 1)};
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const half8 fp[2] = {rows(G, b * 32, p, 0), rows(G, b * 32, p, 1)};
                    acc[b] = multiply(fp, fq, acc[b]);
                }
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const EightColumns c(acc[b], g);
                    const int i = b * 32 + r, j = bj * 32 + 16 * g + 8 * h;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = c.v[e] * alpha;
                    if (k + 1 < steps) put8(X, i, j, v);
                    else eight_into_vector<OUT>(M, out, i, j, v);
                }
        }
        __syncthreads();
    }
}

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace

struct ds_ortho {
    ds_ortho_config_t cfg;                 // its HOST pointers are cleared
    int device;
    bool split;
    std::vector<float> coef;
    void *mem;                             // one allocation behind everything below
    const Mat *mats;
    struct Launch {                        // a product of all matrices
        const Tile *tiles;
        const Cut *cuts;
        unsigned n_tiles, n_cuts;
        int side;
    };
    Launch gram, poly, wide;               // X X' ; G G ; B X
    const Tile *operands;
    const int2 *parts;
    int64_t n_operands, n_parts;
    float *sums;                           // parts of sums
    // every matrix fits one workgroup's LDS: their numbers by class (64 rows many to a compute unit, 64 rows, 128 rows), one
    // launch each, and nothing of the above but `mats`
    const int32_t *small[3];
    unsigned n_small[3];
    const float *small_coef;
    double *partial;
    uint64_t *inside;                      // plane of bits: the elements of the matrices
    const int32_t *vector_tiles[2];        // 2048-element tiles of the vector with an element outside, inside the matrices
    int32_t n_vector_tiles[2];
    float *u;                              // [d] what is orthogonalised, where it is not m
    char *ws;
};

namespace {

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Marks a run of elements; false if one of them was marked before.
bool mark(std::vector<uint64_t> &plane, int64_t lo, int64_t hi)
{
    while (lo < hi) {
        const int64_t end = std::min(hi, (lo | 63) + 1);
        const uint64_t bits = (end - lo == 64 ? ~0ull : ((1ull << (end - lo)) - 1)) << (lo & 63);
        uint64_t &w = plane[static_cast<size_t>(lo >> 6)];
        if (w & bits) return false;
        w |= bits;
        lo = end;
    }
    return true;
}

// The tiles of a product in the order in which they are given out.
struct Work {
    std::vector<Tile> tiles;
    std::vector<Cut> cuts;
    int32_t slots = 0;                     // of the parts' buffer
    int side = 64;
};

// Tables of the plan; the matrices were checked.
struct Tables {
    std::vector<Mat> mats;
    Work gram, poly, wide;
    std::vector<Tile> operands;
    std::vector<int2> parts;
    int64_t n_partial = 0, ws_bytes = 0;
    std::vector<int32_t> small[3];
};

// Which of the small classes takes a matrix, or -1.
int small_class(const Mat &M, bool split)
{
    if (M.mp > 128) return -1;
    const int64_t bytes = split ? small_bytes<true>(M.mp, M.np) : small_bytes<false>(M.mp, M.np);
    if (bytes > kSmallBytes) return -1;
    return M.mp == 128 ? 2 : bytes > kSmallBytesMany ? 1 : 0;
}

// All tiles of a product: long sums first, so that the launch ends with short ones; within a matrix strips of rows, so that
// tiles near each other in time share rows and columns.
std::vector<Tile> list_tiles(const std::vector<Mat> &mats, int side, int stage, int panel)
{
    std::vector<int32_t> order(mats.size());
    for (size_t k = 0; k < mats.size(); ++k) order[k] = static_cast<int32_t>(k);
    auto length = [&](int32_t k) { return stage == kGram ? mats[k].np : mats[k].mp; };
    std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return length(a) > length(b); });
    std::vector<Tile> list;
    const int32_t strip = 1024 / side;
    const bool square = stage != kApply;
    for (int32_t k : order) {
        const int32_t ti = (mats[k].mp + side - 1) / side, tj = square ? ti : (mats[k].np + side - 1) / side;
        for (int32_t i0 = 0; i0 < ti; i0 += strip)
            for (int32_t j = 0; j < tj; ++j)
                for (int32_t i = i0; i < std::min(i0 + strip, ti); ++i)
                    if (!square || j <= i) list.push_back(Tile{k, i, j, 0, length(k) / panel, -1, mats[static_cast<size_t>(k)]});
    }
    return list;
}

// Runs of kRun tiles to one XCD (workgroup p runs on XCD p % 8, each with an L2 of its own).
std::vector<Tile> by_xcd(const std::vector<Tile> &list)
{
    constexpr size_t kRun = 32;
    std::vector<Tile> out;
    out.reserve(list.size());
    size_t next[8], xcd = 0;
    for (size_t q = 0; q < 8; ++q) next[q] = q * kRun;
    while (out.size() < list.size()) {
        size_t from = xcd;
        if (next[from] >= list.size()) {
            // nothing is left for this XCD: its turn goes to the one that has most left
            from = 8;
            for (size_t q = 0; q < 8; ++q)
                if (next[q] < list.size() && (from == 8 || next[q] < next[from])) from = q;
        }
        out.push_back(list[next[from]]);
        if (++next[from] % kRun == 0) next[from] += 7 * kRun;
        xcd = (xcd + 1) % 8;
    }
    return out;
}

// What a launch of these tiles takes, in microseconds, from times measured with 1 to 4096 tiles of 8 to 512 panels.  A
// workgroup takes `base` (addresses, first copies, results) and a time per panel, which grow with the workgroups per compute
// unit (c): alone and with the device full a panel of a 256 x 256 tile takes 0.75 and 1.25 us (0.55 and 0.95 with one half;
// 32 values of k then), of a 128 x 128 tile 0.25 and, two per compute unit, 0.68 (0.19, 0.53), of a 64 x 64 tile 0.11 and,
// two, 0.25 (0.09, 0.22).
int tiles_at_once(int side) { return side == 256 ? 256 : 512; }

double launch_time(const std::vector<Tile> &tiles, int side, bool split)
{
    const size_t at_once = static_cast<size_t>(tiles_at_once(side));
    double time = 0.0;
    for (size_t first = 0; first < tiles.size(); first += at_once) {
        const size_t end = std::min(first + at_once, tiles.size());
        const double c = static_cast<double>(end - first) / 256.0;
        int64_t longest = 0, sum = 0;
        for (size_t k = first; k < end; ++k) {
            longest = std::max<int64_t>(longest, tiles[k].k1 - tiles[k].k0);
            sum += tiles[k].k1 - tiles[k].k0;
        }
        const double more = std::max(c - 1.0, 0.0), one = std::min(c, 1.0);
        const double stage = side == 256   ? (split ? 0.75 + 0.5 * c : 0.55 + 0.4 * c)
                             : side == 128 ? (split ? 0.25 + 0.06 * one + 0.37 * more : 0.19 + 0.06 * one + 0.28 * more)
                                           : (split ? 0.10 + 0.035 * one + 0.11 * more : 0.09 + 0.02 * one + 0.11 * more);
        const double base = side == 256 ? (split ? 13.0 : 7.0) : side == 128 ? 4.5 + (split ? 7.5 : 3.5) * more : 2.8;
        // rounds run into each other: only the last one's longest sum counts in full
        time += base + stage * (end == tiles.size() ? static_cast<double>(longest) : static_cast<double>(sum) / static_cast<double>(end - first));
    }
    return time;
}

// A product by tiles of `side`.  The device takes `at_once` workgroups; a workgroup's share of all panels is what it would have
// if they were dealt out evenly.  Tiles that fit into the shares stay whole; the others (those of a last round that would
// leave most of the device idle, or sums longer than a share) are cut into parts that do, if `cutting`.  The parts are for all that
// the device takes at once, two workgroups per compute unit below 256 x 256; parts for one per unit were not tried.
void deal_out(const std::vector<Tile> &list, int side, bool cutting, Work &w)
{
    constexpr int kLeast = 8;              // panels of a part: below, filling the pipeline costs more than it saves
    const int at_once = tiles_at_once(side);
    w.side = side;
    std::vector<Tile> whole, cut, pieces;
    int64_t total = 0, cut_panels = 0;
    for (const Tile &t : list) total += t.k1;
    const int64_t share = std::max<int64_t>((total + at_once - 1) / at_once, kLeast);
    // the launch as the device would deal it out: every tile to the workgroup that is free first
    std::vector<int64_t> free_at(static_cast<size_t>(at_once), 0);
    auto later = [](int64_t a, int64_t b) { return a > b; };
    for (const Tile &t : list) {
        if (cutting && free_at.front() + t.k1 > share + share / 16 && t.k1 >= 2 * kLeast) {
            cut.push_back(t);
            cut_panels += t.k1;
        } else {
            std::pop_heap(free_at.begin(), free_at.end(), later);
            free_at.back() += t.k1;
            std::push_heap(free_at.begin(), free_at.end(), later);
            whole.push_back(t);
        }
    }
    const int64_t part = std::max<int64_t>(kLeast, (cut_panels + at_once - 1) / at_once);
    for (const Tile &t : cut) {
        const int32_t n = static_cast<int32_t>((t.k1 + part / 2) / part);
        if (n < 2) {
            pieces.push_back(t);
            continue;
        }
        w.cuts.push_back(Cut{t.mat, t.i, t.j, w.slots, n, {0, 0, 0}});
        for (int32_t p = 0; p < n; ++p) {
            Tile q = t;
            q.k0 = static_cast<int32_t>(static_cast<int64_t>(t.k1 / 2) * p / n) * 2;           // even numbers of panels
            q.k1 = static_cast<int32_t>(static_cast<int64_t>(t.k1 / 2) * (p + 1) / n) * 2;
            q.slot = w.slots++;
            pieces.push_back(q);
        }
    }
    w.tiles = by_xcd(whole);
    const std::vector<Tile> rest = by_xcd(pieces);
    w.tiles.insert(w.tiles.end(), rest.begin(), rest.end());
}

// The best of the sides, with and without cutting.
void plan_product(const std::vector<Mat> &mats, int stage, bool split, Work &best)
{
    double least = 0.0;
    for (int side : {64, 128, 256}) {
        const std::vector<Tile> list = list_tiles(mats, side, stage, split ? kPanel<true> : kPanel<false>);
        for (bool cutting : {false, true}) {
            if (cutting && side == kTileSide && stage != kGram) continue;      // kCanCut
            Work w;
            deal_out(list, side, cutting, w);
            if (cutting && w.cuts.empty()) continue;
            double t = launch_time(w.tiles, side, split);
            // the joining launch: itself, the parts' bytes, what it writes (the transposes two bytes at a time)
            const double area = static_cast<double>(side) * side;
            if (cutting) t += 5.5 + w.slots * area * 4.0 / 6e6 + static_cast<double>(w.cuts.size()) * area * 2.5e-6;
            if (best.tiles.empty() || t < least) {
                least = t;
                best = std::move(w);
            }
        }
    }
}

void make_tables(const ds_ortho_config_t &cfg, bool split, Tables &t)
{
    bool all_small = true;
    for (int32_t k = 0; k < cfg.n_mats; ++k) {
        const ds_matrix_t &in = cfg.mats[k];
        Mat M{};
        M.offset = in.offset;
        M.ld = in.ld ? in.ld : in.cols;
        M.rows = in.rows;
        M.cols = in.cols;
        M.flip = in.rows > in.cols;
        M.m = std::min(in.rows, in.cols);
        M.n = std::max(in.rows, in.cols);
        M.mp = static_cast<int32_t>(round_up(M.m, kTileSide));
        M.np = static_cast<int32_t>(round_up(M.n, kTileSide));
        M.panel = M.mp * kRow;
        M.scale = kOperandScale;
        const double aspect = static_cast<double>(in.rows) / in.cols;
        M.factor = cfg.factor == DS_ORTHO_FACTOR_ASPECT ? static_cast<float>(sqrt(std::max(1.0, aspect)))
                   : cfg.factor == DS_ORTHO_FACTOR_RMS ? static_cast<float>(0.2 * sqrt(static_cast<double>(M.n))) : 1.0f;
        all_small = all_small && small_class(M, split) >= 0;
        t.mats.push_back(M);
    }
    // Small matrices among large ones go with them: there they cost a tile, here a launch.
    if (all_small) {
        for (int32_t k = 0; k < cfg.n_mats; ++k) t.small[small_class(t.mats[static_cast<size_t>(k)], split)].push_back(k);
        return;
    }
    auto take = [&](int64_t bytes) {
        const int64_t at = t.ws_bytes;
        t.ws_bytes += round_up(bytes, 256);
        return at;
    };
    for (int32_t k = 0; k < cfg.n_mats; ++k) {
        if (t.ws_bytes > kMostBytes) return;         // will be refused; thin matrices can be 64 times what they hold
        Mat &M = t.mats[static_cast<size_t>(k)];
        const int64_t each = split ? 4 : 2;
        M.x[0] = take(static_cast<int64_t>(M.mp) * M.np * each);
        M.x[1] = take(static_cast<int64_t>(M.mp) * M.np * each);
        M.g = take(static_cast<int64_t>(M.mp) * M.mp * each);
        M.b = take(static_cast<int64_t>(M.mp) * M.mp * each);
        const int64_t elements = static_cast<int64_t>(M.m) * M.n;
        M.parts = static_cast<int32_t>(std::min<int64_t>(kMaxParts, (elements + kPartElements - 1) / kPartElements));
        M.part0 = static_cast<int32_t>(t.n_partial);
        t.n_partial += M.parts;
        for (int32_t p = 0; p < M.parts; ++p) t.parts.push_back(int2{k, p});
    }
    if (t.ws_bytes > kMostBytes) return;
    plan_product(t.mats, kGram, split, t.gram);
    plan_product(t.mats, kPoly, split, t.poly);
    plan_product(t.mats, kApply, split, t.wide);
    t.operands = by_xcd(list_tiles(t.mats, 64, kApply, kPanel<true>));
}

template <int SIDE, bool SPLIT, int STAGE, int OUT>
void product_of(const ds_ortho *o, const ds_ortho::Launch &l, const Step &s, const Out &out, hipStream_t st)
{
    constexpr int WM = SIDE == 64 ? 32 : SIDE == 128 ? 64 : 128, WN = SIDE == 64 ? 32 : 64, THREADS = (SIDE / WM) * (SIDE / WN) * 64;
    k_ortho_product<SIDE, SIDE, WM, WN, SIDE == 64 ? 2 : 1, SPLIT, STAGE, OUT><<<l.n_tiles, THREADS, 0, st>>>(l.tiles, o->ws, o->sums, s, out);
    if constexpr (kCanCut<SIDE, STAGE>) {
        if (l.n_cuts)
            k_ortho_join<SIDE, SPLIT, STAGE, OUT><<<l.n_cuts * (SIDE * SIDE / 8 / kThreads), kThreads, 0, st>>>(o->mats, l.cuts, o->ws, o->sums,
                                                                                                             s, out);
    }
}

template <bool SPLIT, int STAGE, int OUT>
void product(const ds_ortho *o, const Step &s, const Out &out, hipStream_t st)
{
    const ds_ortho::Launch &l = STAGE == kGram ? o->gram : STAGE == kPoly ? o->poly : o->wide;
    switch (l.side) {
    case 256: return product_of<256, SPLIT, STAGE, OUT>(o, l, s, out, st);
    case 128: return product_of<128, SPLIT, STAGE, OUT>(o, l, s, out, st);
    default: return product_of<64, SPLIT, STAGE, OUT>(o, l, s, out, st);
    }
}

// The matrices through the plan's steps; `src` holds U, where the last product goes is `out`.
template <bool SPLIT, bool SRC_BF16, int OUT>
ds_status_t run(const ds_ortho *o, const void *src, const Out &out, hipStream_t st)
{
    if (o->n_small[0] + o->n_small[1] + o->n_small[2]) {
        auto go = [&](auto mp, auto cap, int c) {
            if (o->n_small[c])
                k_ortho_small<decltype(mp)::value, decltype(cap)::value, SPLIT, SRC_BF16, OUT><<<o->n_small[c], kThreads, 0, st>>>(
                    o->mats, o->small[c], src, o->small_coef, o->cfg.steps, o->cfg.eps, out);
        };
        go(std::integral_constant<int, 64>{}, std::integral_constant<int, kSmallBytesMany>{}, 0);
        go(std::integral_constant<int, 64>{}, std::integral_constant<int, kSmallBytes>{}, 1);
        go(std::integral_constant<int, 128>{}, std::integral_constant<int, kSmallBytes>{}, 2);
        return ds_launch_status();
    }
    auto grid = [](int64_t n) { return static_cast<unsigned>(n); };
    k_ortho_norm<SRC_BF16><<<grid(o->n_parts), kBlock, 0, st>>>(o->mats, o->parts, src, o->partial);
    k_ortho_operands<SPLIT, SRC_BF16><<<grid(o->n_operands), kThreads, 0, st>>>(o->operands, src, o->partial, o->cfg.eps, o->ws);
    for (int32_t k = 0; k < o->cfg.steps; ++k) {
        const Step s{o->coef[3 * k], o->coef[3 * k + 1], o->coef[3 * k + 2], k & 1};
        product<SPLIT, kGram, 0>(o, s, out, st);
        product<SPLIT, kPoly, 0>(o, s, out, st);
        if (k + 1 < o->cfg.steps) product<SPLIT, kApply, 0>(o, s, out, st);
        else product<SPLIT, kLast, OUT>(o, s, out, st);
    }
    return ds_launch_status();
}

template <bool SRC_BF16, int OUT>
ds_status_t run(const ds_ortho *o, const void *src, const Out &out, hipStream_t st)
{
    return o->split ? run<true, SRC_BF16, OUT>(o, src, out, st) : run<false, SRC_BF16, OUT>(o, src, out, st);
}

// Whether every operand of a list of steps stays in the range in which it is held.  h bounds the singular values of the X that a
// step reads: 1 at the start (the norm is Frobenius'), then the largest |p(s)|, p(s) = a s + b s^3 + c s^5, on [0, h] of the
// step before.  Entries of a matrix do not exceed its largest singular value, so with t = s^2 those of G stay below h^2, which
// times kGramScale has to be a half (65,504 at most: h <= 2.8), and those of B, a on its diagonal, below the largest
// |a + b t + c t^2| on [0, h^2], times kPolyScale: 16; 15 leaves room for roundings, and holds for b t + c t^2 as well.
// Rounding an operand moves its singular values by u of the largest one, 2^-11 with one half; with two, 2^-20 counts the sums in
// fp32 too.  A list that comes back from near 2 lies on so steep a part of its polynomials that this decides: one half may
// leave the range where two do not.
bool coefficients_fit(const float *coef, int32_t steps, bool split)
{
    const double u = split ? 0x1p-20 : 0x1p-11;
    double h = 1.0;
    for (int32_t k = 0; k < steps; ++k) {
        const double a = coef[3 * k], b = coef[3 * k + 1], c = coef[3 * k + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        h *= 1.0 + u;
        if (!(h <= 2.8)) return false;
        const double top = h * h;
        // extremes of b t + c t^2 and of p: at the ends and where the derivatives b + 2 c t and a + 3 b t + 5 c t^2 vanish
        double at[5] = {0.0, top, 0.0, 0.0, 0.0};
        if (c != 0.0) at[2] = -b / (2.0 * c);
        const double q = 9.0 * b * b - 20.0 * a * c;
        if (c == 0.0 && b != 0.0) at[3] = -a / (3.0 * b);
        if (c != 0.0 && q >= 0.0) {
            // the root without cancellation, and the other from their product a / (5 c)
            const double r = -0.5 * (3.0 * b + std::copysign(std::sqrt(q), b));
            at[3] = r / (5.0 * c);
            if (r != 0.0) at[4] = a / r;
        }
        double poly = 0.0, next = 0.0;
        for (double t : at) {
            if (!(t >= 0.0 && t <= top)) continue;
            const double v = b * t + c * t * t;
            if (std::fabs(v) > 15.0 || std::fabs(a + v) > 15.0) return false;
            poly = std::max(poly, std::fabs(a + v));
            next = std::max(next, std::sqrt(t) * std::fabs(a + v));
        }
        // G off by u h^2 moves B by the steepest b + 2 c t times that
        h = next + h * u * (top * std::max(std::fabs(b), std::fabs(b + 2.0 * c * top)) + poly);
    }
    return true;
}

}  // namespace

const uint64_t *ds_ortho_inside(const ds_ortho *o) { return o->inside; }
const int32_t *ds_ortho_tiles(const ds_ortho *o, bool inside, int32_t *n)
{
    *n = o->n_vector_tiles[inside];
    return o->vector_tiles[inside];
}
int64_t ds_ortho_elements(const ds_ortho *o) { return o->cfg.d; }
int ds_ortho_device(const ds_ortho *o) { return o->device; }
bool ds_ortho_nesterov(const ds_ortho *o) { return (o->cfg.flags & DS_ORTHO_NESTEROV) != 0; }
float *ds_ortho_buffer(const ds_ortho *o) { return o->u; }

ds_status_t ds_ortho_update(const ds_ortho *o, const float *u, float *x, float gamma, float decay, hipStream_t st)
{
    const Out out{nullptr, x, static_cast<float>(1.0 - static_cast<double>(gamma) * static_cast<double>(decay)), gamma};
    return run<false, 2>(o, u, out, st);
}

extern "C" {

ds_status_t ds_ortho_create(const ds_ortho_config_t *cfg, ds_ortho_t **out)
{
    if (!cfg || !out) return DS_ERR_NULL;
    *out = nullptr;
    if (!cfg->mats) return DS_ERR_NULL;
    if (cfg->d < 1 || cfg->d > 0x7FFFFFFFLL || cfg->n_mats < 1 || cfg->n_mats > (1 << 20)) return DS_ERR_SHAPE;
    if (cfg->steps < 1 || cfg->steps > 32) return DS_ERR_SHAPE;
    if (!(cfg->eps >= 0.f) || !std::isfinite(cfg->eps)) return DS_ERR_CONFIG;
    if (cfg->factor < DS_ORTHO_FACTOR_NONE || cfg->factor > DS_ORTHO_FACTOR_RMS) return DS_ERR_CONFIG;
    if (cfg->flags & ~(DS_ORTHO_NESTEROV | DS_ORTHO_HALF)) return DS_ERR_CONFIG;
    if (cfg->coef && !coefficients_fit(cfg->coef, cfg->steps, !(cfg->flags & DS_ORTHO_HALF))) return DS_ERR_CONFIG;
    for (int32_t k = 0; k < cfg->n_mats; ++k) {
        const ds_matrix_t &M = cfg->mats[k];
        if (M.rows < 1 || M.cols < 1 || M.offset < 0 || std::min(M.rows, M.cols) > 32768 || std::max(M.rows, M.cols) > (1 << 24)) return DS_ERR_SHAPE;
        const int64_t ld = M.ld ? M.ld : M.cols;
        if (ld < M.cols || ld > cfg->d || M.offset > cfg->d) return DS_ERR_SHAPE;
        if (M.offset + (static_cast<int64_t>(M.rows) - 1) * ld + M.cols > cfg->d) return DS_ERR_SHAPE;
    }
    ds_ortho *o = nullptr;
    // the tables are the host's memory, which may run out; no exception leaves a C function
    try {
        std::vector<uint64_t> plane(static_cast<size_t>((cfg->d + 63) / 64), 0);
        for (int32_t k = 0; k < cfg->n_mats; ++k) {
            const ds_matrix_t &M = cfg->mats[k];
            const int64_t ld = M.ld ? M.ld : M.cols;
            for (int64_t r = 0; r < M.rows; ++r)
                if (!mark(plane, M.offset + r * ld, M.offset + r * ld + M.cols)) return DS_ERR_CONFIG;
        }
        std::vector<int32_t> vector_tiles[2];
        for (int64_t first = 0; first < cfg->d; first += kTile) {
            uint64_t any = 0, all = ~0ull;
            for (int64_t e = first; e < std::min(first + kTile, cfg->d); e += 64) {
                const uint64_t w = plane[static_cast<size_t>(e >> 6)];
                any |= w;
                all &= cfg->d - e >= 64 ? w : w | (~0ull << (cfg->d - e));
            }
            if (any) vector_tiles[1].push_back(static_cast<int32_t>(first / kTile));
            if (~all) vector_tiles[0].push_back(static_cast<int32_t>(first / kTile));
        }
        o = new ds_ortho();
        o->cfg = *cfg;
        o->cfg.mats = nullptr;
        o->cfg.coef = nullptr;
        o->mem = nullptr;
        o->split = (cfg->flags & DS_ORTHO_HALF) == 0;
        static const float standard[3] = {3.4445f, -4.7750f, 2.0315f};
        for (int32_t k = 0; k < 3 * cfg->steps; ++k) o->coef.push_back(cfg->coef ? cfg->coef[k] : standard[k % 3]);
        Tables t;
        make_tables(*cfg, o->split, t);
        if (t.ws_bytes > kMostBytes) {
            delete o;
            return DS_ERR_DEVICE;
        }
        o->n_operands = static_cast<int64_t>(t.operands.size());
        o->n_parts = static_cast<int64_t>(t.parts.size());
        int64_t bytes = 0;
        auto take = [&](int64_t b) {
            const int64_t at = bytes;
            bytes += round_up(b, 256);
            return at;
        };
        auto size_of = [](const auto &v) { return static_cast<int64_t>(v.size() * sizeof(v[0])); };
        Work *const works[3] = {&t.gram, &t.poly, &t.wide};
        ds_ortho::Launch *const launches[3] = {&o->gram, &o->poly, &o->wide};
        int64_t at_tiles[3], at_cuts[3], sum_bytes = 0;
        for (int k = 0; k < 3; ++k) {
            at_tiles[k] = take(size_of(works[k]->tiles));
            at_cuts[k] = take(size_of(works[k]->cuts));
            sum_bytes = std::max<int64_t>(sum_bytes, static_cast<int64_t>(works[k]->slots) * works[k]->side * works[k]->side * 4);
        }
        const int64_t at_mats = take(size_of(t.mats)), at_operands = take(size_of(t.operands)), at_parts = take(size_of(t.parts)),
                      at_inside = take(size_of(plane));
        int64_t at_small[3];
        for (int k = 0; k < 3; ++k) at_small[k] = take(size_of(t.small[k]));
        const int64_t at_outside = take(size_of(vector_tiles[0])), at_within = take(size_of(vector_tiles[1]));
        const int64_t at_coef = take(size_of(o->coef));
        const int64_t at_partial = take(t.n_partial * 8), at_u = take(cfg->d * 4), at_sums = take(sum_bytes), at_ws = take(t.ws_bytes);
        ds_status_t rc = hipGetDevice(&o->device) == hipSuccess ? DS_OK : DS_ERR_DEVICE;
        if (rc == DS_OK && hipMalloc(&o->mem, static_cast<size_t>(bytes)) != hipSuccess) {
            o->mem = nullptr;
            (void)hipGetLastError();       // a failed allocation is this call's result and nobody else's
            rc = DS_ERR_DEVICE;
        }
        char *base = static_cast<char *>(o->mem);
        auto put = [&](int64_t at, const auto &v) {
            if (rc == DS_OK && !v.empty() && hipMemcpy(base + at, v.data(), v.size() * sizeof(v[0]), hipMemcpyHostToDevice) != hipSuccess) rc = DS_ERR_DEVICE;
        };
        for (int k = 0; k < 3; ++k) {
            put(at_small[k], t.small[k]);
            o->small[k] = reinterpret_cast<const int32_t *>(base + at_small[k]);
            o->n_small[k] = static_cast<unsigned>(t.small[k].size());
        }
        put(at_outside, vector_tiles[0]);
        put(at_within, vector_tiles[1]);
        for (int k = 0; k < 2; ++k) {
            o->vector_tiles[k] = reinterpret_cast<const int32_t *>(base + (k ? at_within : at_outside));
            o->n_vector_tiles[k] = static_cast<int32_t>(vector_tiles[k].size());
        }
        put(at_coef, o->coef);
        o->small_coef = reinterpret_cast<const float *>(base + at_coef);
        put(at_mats, t.mats);
        for (int k = 0; k < 3; ++k) {
            put(at_tiles[k], works[k]->tiles);
            put(at_cuts[k], works[k]->cuts);
            *launches[k] = {reinterpret_cast<const Tile *>(base + at_tiles[k]), reinterpret_cast<const Cut *>(base + at_cuts[k]),
                            static_cast<unsigned>(works[k]->tiles.size()), static_cast<unsigned>(works[k]->cuts.size()), works[k]->side};
        }
        put(at_operands, t.operands);
        put(at_parts, t.parts);
        put(at_inside, plane);
        if (rc == DS_OK && hipStreamSynchronize(nullptr) != hipSuccess) rc = DS_ERR_DEVICE;
        if (rc != DS_OK) {
            ds_ortho_destroy(o);
            return rc;
        }
        o->mats = reinterpret_cast<const Mat *>(base + at_mats);
        o->operands = reinterpret_cast<const Tile *>(base + at_operands);
        o->parts = reinterpret_cast<const int2 *>(base + at_parts);
        o->inside = reinterpret_cast<uint64_t *>(base + at_inside);
        o->partial = reinterpret_cast<double *>(base + at_partial);
        o->u = reinterpret_cast<float *>(base + at_u);
        o->sums = reinterpret_cast<float *>(base + at_sums);
        o->ws = base + at_ws;
    } catch (...) {
        ds_ortho_destroy(o);
        return DS_ERR_DEVICE;
    }
    *out = o;
    return DS_OK;
}

ds_status_t ds_ortho_destroy(ds_ortho_t *o)
{
    if (!o) return DS_OK;
    DeviceGuard guard(o->device);
    if (o->mem) (void)hipFree(o->mem);
    delete o;
    return DS_OK;
}

ds_status_t ds_orthogonalize(ds_ortho_t *o, const void *src, int32_t src_dtype, void *dst, int32_t dst_dtype, void *hip_stream)
{
    if (!o || !src || !dst) return DS_ERR_NULL;
    if ((src_dtype != DS_F32 && src_dtype != DS_BF16) || (dst_dtype != DS_F32 && dst_dtype != DS_BF16)) return DS_ERR_CONFIG;
    if (src == dst && src_dtype != dst_dtype) return DS_ERR_CONFIG;
    if (misaligned(src) || misaligned(dst)) return DS_ERR_ALIGN;
    DeviceGuard guard(o->device);
    if (!guard.ok) return DS_ERR_DEVICE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const Out out{dst, nullptr, 0.f, 0.f};
    if (src_dtype == DS_BF16) return dst_dtype == DS_BF16 ? run<true, 1>(o, src, out, st) : run<true, 0>(o, src, out, st);
    return dst_dtype == DS_BF16 ? run<false, 1>(o, src, out, st) : run<false, 0>(o, src, out, st);
}

}  // extern "C"
