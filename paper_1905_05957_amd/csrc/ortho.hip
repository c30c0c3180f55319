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
// more bits of significand per product for the same rate; the range is used by scaling with powers of two: X by 2^s with
// entries near 16 for an orthogonal matrix, G by 2^13 and B by 2^12, which leaves entries of lo 2^-20 below those of X.
// With one half (DS_ORTHO_HALF) a rounding is 2^-11 at most; it grows with the smallest singular values at most, 3.44^5 = 485 times
// while an entry of X grows as much or reaches 1 / sqrt(n), so it ends below a rounding to bf16.
//
// Layout.  A row of an operand is a sequence of 128-byte blocks: 32 values as 32 hi and 32 lo, or 64 values with one half.
#include "ds_device.h"
#include "ds_internal.h"
#include "tails.h"

#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

using namespace ds;

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kRowBlock = 128;                 // bytes of one block of a row
constexpr float kGramScale = 8192.0f;          // G is held times 2^13 (entries up to 8)
constexpr float kPolyScale = 4096.0f;          // B is held times 2^12 (entries up to 16)
constexpr int kTileSide = 64;
constexpr int kMaxParts = 256;                 // partial sums of a matrix's norm
constexpr int64_t kPartElements = 16384;

struct Mat {
    int64_t offset, ld;          // in the vector
    int64_t x[2], g, b;          // byte offsets in the workspace
    int32_t rows, cols;          // as stored
    int32_t m, n, mp, np;        // as worked on: m <= n, and rounded up to tiles
    int32_t row_n, row_m;        // bytes of a row of np and of mp values
    int32_t flip;                // stored transposed
    int32_t part0, parts;        // partial sums of the norm
    float scale;                 // X is held times this
    float factor;
    int32_t pad_;
};

struct Tile {
    int32_t mat, i, j, pad_;
};

template <bool SPLIT>
__device__ __forceinline__ int64_t chunk_at(int64_t row_bytes, int row, int k)     // k a multiple of 4
{
    return row * row_bytes + (SPLIT ? (k >> 5) * kRowBlock + (k & 31) * 2 : k * 2);
}

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
    if (SPLIT) *reinterpret_cast<half8 *>(p + kRowBlock / 2) = lo;
}

template <bool SPLIT>
__device__ __forceinline__ void store4(char *p, const float *v)
{
    half4 hi, lo;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        hi[t] = static_cast<_Float16>(v[t]);
        lo[t] = static_cast<_Float16>(v[t] - static_cast<float>(hi[t]));
    }
    *reinterpret_cast<half4 *>(p) = hi;
    if (SPLIT) *reinterpret_cast<half4 *>(p + kRowBlock / 2) = lo;
}

template <bool SPLIT>
__device__ __forceinline__ void store1(char *p, float v)
{
    const _Float16 hi = static_cast<_Float16>(v);
    *reinterpret_cast<_Float16 *>(p) = hi;
    if (SPLIT) *reinterpret_cast<_Float16 *>(p + kRowBlock / 2) = static_cast<_Float16>(v - static_cast<float>(hi));
}

template <bool SPLIT>
__device__ __forceinline__ void load4(const char *p, float *v)
{
    const half4 hi = *reinterpret_cast<const half4 *>(p);
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = static_cast<float>(hi[t]);
    if (SPLIT) {
        const half4 lo = *reinterpret_cast<const half4 *>(p + kRowBlock / 2);
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] += static_cast<float>(lo[t]);
    }
}

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

// ---------------------------------------------------------------------------------------
// norms and operands
// ---------------------------------------------------------------------------------------
// Partial sums of squares in fp64: part p of a matrix is a run of its rows' elements.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_ortho_norm(const Mat *__restrict__ mats, const int2 *__restrict__ parts, const void *src,
                                                       double *__restrict__ partial)
{
    __shared__ double lds[kWaves];
    const int2 pt = parts[blockIdx.x];
    const Mat &M = mats[pt.x];
    const int64_t total = static_cast<int64_t>(M.rows) * M.cols;
    const int64_t each = ((total + M.parts - 1) / M.parts + 3) & ~static_cast<int64_t>(3);
    const int64_t lo = each * pt.y, hi = lo + each < total ? lo + each : total;
    double s = 0.0;
    for (int64_t t = lo + threadIdx.x; t < hi; t += kBlock) {
        const uint32_t r = static_cast<uint32_t>(t) / static_cast<uint32_t>(M.cols);
        const double v = load_flat<BF16>(src, M.offset + r * M.ld + (t - static_cast<int64_t>(r) * M.cols));
        s += v * v;
    }
    s = block_sum(s, lds, false);
    if (threadIdx.x == 0) partial[M.part0 + pt.y] = s;
}

// X = U / (norm + eps), times 2^s, zero beyond the matrix.
template <bool SPLIT, bool BF16>
__global__ __launch_bounds__(kThreads) void k_ortho_operands(const Mat *__restrict__ mats, const Tile *__restrict__ tiles,
                                                             const void *src, const double *__restrict__ partial, float eps, char *ws)
{
    constexpr int T = 64;
    __shared__ float tile[T][T + 1];
    __shared__ double sums[kThreads / 64];
    const Tile tl = tiles[blockIdx.x];
    const Mat &M = mats[tl.mat];
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
    const int i0 = tl.i * T, j0 = tl.j * T;
    for (int t = threadIdx.x; t < T * T; t += kThreads) {
        const int fast = t & (T - 1), slow = t / T;
        const int i = M.flip ? fast : slow, j = M.flip ? slow : fast;
        float v = 0.f;
        if (i0 + i < M.m && j0 + j < M.n) {
            const int64_t r = M.flip ? j0 + j : i0 + i, c = M.flip ? i0 + i : j0 + j;
            v = static_cast<float>(static_cast<double>(load_flat<BF16>(src, M.offset + r * M.ld + c)) * inv);
        }
        tile[i][j] = v;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < T * T / 8; t += kThreads) {
        const int a = t / (T / 8), c = (t % (T / 8)) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[a][c + e];
        store8<SPLIT>(ws + M.x[0] + chunk_at<SPLIT>(M.row_n, i0 + a, j0 + c), v);
    }
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
enum Stage { kGram, kPoly, kApply, kLast };    // G = X X' ; B = b G + c G G ; X <- a X + B X ; the same into the vector

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

// Direct copy of 16 bytes per lane into LDS, lane l to `lds` + 16 l; `lds` is the same for the wavefront.  It has no output
// register.  Written as an instruction because the compiler waits for every outstanding copy of its own builtin before
// the next read of LDS, also of the other stage; the wait that is needed stands in front of the barrier of that stage.
__device__ __forceinline__ void copy_to_lds(const char *from, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(lds) : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)p));
}

__device__ __forceinline__ f32x16 mfma(half8 a, half8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// One tile of TM x TN of C = P Q, by wavefronts of WM x WN.  P is read by rows of k (blocks of 128 bytes).  Q = X' or G
// (symmetric) is read by rows of k as well; Q = X, in the last product, lies as rows of j under each other, k = row: its tile
// is transposed on the way from LDS to the registers.
//
// LDS: two stages; while one is multiplied, the next is copied in without passing the registers.  LDS has 64 banks, 256
// bytes; a copy fills it linearly, so what a lane copies is chosen such that the 16-byte chunk c of row r lies at c ^ f(r),
// and 16 lanes that read 16 rows of one chunk (or, transposing, 32 lanes 4 rows of 4 chunks) meet different banks: 267 and 228
// bytes a clock measured, 43 and 80 without.
//
// The wavefront multiplies Q' P': a lane then holds a row i of C and four consecutive j at a time.
template <int TM, int TN, int WM, int WN, bool SPLIT, int STAGE, int OUT>      // OUT: 0 fp32, 1 bf16, 2 the model
__global__ __launch_bounds__((TM / WM) * (TN / WN) * 64) void k_ortho_product(const Mat *__restrict__ mats, const Tile *__restrict__ tiles,
                                                                             char *ws, Step step, Out out)
{
    constexpr int WAVES_N = TN / WN, WAVES = (TM / WM) * WAVES_N, FM = WM / 32, FN = WN / 32;
    constexpr bool ROWS = STAGE >= kApply;                     // Q is X
    constexpr int KROWS = SPLIT ? 32 : 64;                     // values of k in a stage
    constexpr int QROW = SPLIT ? TN * 4 : TN * 2;              // bytes of one of its rows in LDS
    constexpr int PBYTES = TM * kRowBlock, QBYTES = TN * kRowBlock, STAGE_BYTES = PBYTES + QBYTES;
    constexpr int PCOPIES = PBYTES / (WAVES * 1024), QCOPIES = QBYTES / (WAVES * 1024);
    static_assert(PCOPIES * WAVES * 1024 == PBYTES && QCOPIES * WAVES * 1024 == QBYTES && QROW * KROWS == QBYTES, "tile");
    __shared__ __attribute__((aligned(256))) char lds[2 * STAGE_BYTES];
    const Tile tl = tiles[blockIdx.x];
    const Mat &M = mats[tl.mat];
    const int i0 = tl.i * TM, j0 = tl.j * TN;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int wi = (wave / WAVES_N) * WM, wj = (wave % WAVES_N) * WN;
    const int64_t row_k = STAGE == kGram ? M.row_n : M.row_m;
    const int steps_k = static_cast<int>(row_k / kRowBlock);
    const char *X = ws + M.x[step.from];
    const char *P = STAGE == kGram ? X : ws + (STAGE == kPoly ? M.g : M.b);
    const char *Q = ROWS ? X : P;
    // what this lane copies; a tile may reach past the rounded matrix, whose last rows then stand in for what is not there
    const char *pa[PCOPIES], *qa[QCOPIES];
#pragma unroll
    for (int t = 0; t < PCOPIES; ++t) {
        const int at = (t * WAVES + wave) * 1024 + lane * 16, r = at / kRowBlock, c = ((at % kRowBlock) / 16) ^ ((r >> 1) & 7);
        const int row = i0 + r < M.mp ? i0 + r : M.mp - 1;
        pa[t] = P + row * row_k + c * 16;
    }
#pragma unroll
    for (int t = 0; t < QCOPIES; ++t) {
        const int at = (t * WAVES + wave) * 1024 + lane * 16;
        if (ROWS) {
            const int r = at / QROW, f = QROW == 128 ? 4 * ((r >> 1) & 1) : 4 * (r & 3);
            const int byte = static_cast<int>(j0 * (SPLIT ? 4 : 2)) + ((((at % QROW) / 16) ^ f) * 16);
            qa[t] = Q + r * static_cast<int64_t>(M.row_n) + (byte < M.row_n ? byte : M.row_n - 16);
        } else {
            const int r = at / kRowBlock, c = ((at % kRowBlock) / 16) ^ ((r >> 1) & 7);
            const int row = j0 + r < M.mp ? j0 + r : M.mp - 1;
            qa[t] = Q + row * row_k + c * 16;
        }
    }
    const int64_t q_step = ROWS ? static_cast<int64_t>(M.row_n) * KROWS : kRowBlock;
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane(lds_address(lds));
    auto copy = [&](int stage) {
        const uint32_t to = lds_at + stage * STAGE_BYTES + wave * 1024;
#pragma unroll
        for (int t = 0; t < PCOPIES; ++t) {
            copy_to_lds(pa[t], to + t * WAVES * 1024);
            pa[t] += kRowBlock;
        }
#pragma unroll
        for (int t = 0; t < QCOPIES; ++t) {
            copy_to_lds(qa[t], to + PBYTES + t * WAVES * 1024);
            qa[t] += q_step;
        }
    };
    // fragments: row r of 32, values 8 h .. 8 h + 7 of the 16 of step s, plane lo or hi
    const int r = lane & 31, h = lane >> 5;
    auto by_rows = [&](const char *tile, int row, int s, int plane) {
        const int c = SPLIT ? plane * 4 + s * 2 + h : s * 2 + h;
        return *reinterpret_cast<const half8 *>(tile + (row + r) * kRowBlock + ((c ^ (((row + r) >> 1) & 7)) * 16));
    };
    auto by_columns = [&](const char *tile, int col0, int s, int plane) {
        union { half8 v; s16x4 part[2]; } u;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int k = s * 16 + h * 8 + q * 4 + ((lane & 15) >> 2), col = col0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
            const int c = SPLIT ? (col >> 5) * 8 + plane * 4 + ((col & 31) >> 3) : col >> 3;
            const int f = QROW == 128 ? 4 * ((k >> 1) & 1) : 4 * (k & 3);
            u.part[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + k * QROW + ((c ^ f) * 16) + (col & 7) * 2));
        }
        return u.v;
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.f;
    copy(0);
    for (int k = 0; k < steps_k; ++k) {
        const int stage = k & 1;
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");     // this wavefront's copies into `stage` are there
        __syncthreads();                                       // everybody's, and nobody reads the other stage any more
        if (k + 1 < steps_k) copy(1 - stage);
        const char *lp = lds + stage * STAGE_BYTES, *lq = lp + PBYTES;
#pragma unroll
        for (int s = 0; s < KROWS / 16; ++s) {
            half8 ph[FM], pl[FM], qh[FN], ql[FN];
#pragma unroll
            for (int a = 0; a < FM; ++a) {
                ph[a] = by_rows(lp, wi + a * 32, s, 0);
                if (SPLIT) pl[a] = by_rows(lp, wi + a * 32, s, 1);
            }
#pragma unroll
            for (int b = 0; b < FN; ++b) {
                qh[b] = ROWS ? by_columns(lq, wj + b * 32, s, 0) : by_rows(lq, wj + b * 32, s, 0);
                if (SPLIT) ql[b] = ROWS ? by_columns(lq, wj + b * 32, s, 1) : by_rows(lq, wj + b * 32, s, 1);
            }
#pragma unroll
            for (int a = 0; a < FM; ++a)
#pragma unroll
                for (int b = 0; b < FN; ++b) {
                    if (SPLIT) {
                        acc[a][b] = mfma(qh[b], pl[a], acc[a][b]);
                        acc[a][b] = mfma(ql[b], ph[a], acc[a][b]);
                    }
                    acc[a][b] = mfma(qh[b], ph[a], acc[a][b]);
                }
        }
    }
    // the product's scale away, the stage's scale on
    const float alpha = STAGE == kGram ? kGramScale / (M.scale * M.scale)
                        : STAGE == kPoly ? step.c * (kPolyScale / (kGramScale * kGramScale)) : 1.0f / kPolyScale;
    const float beta = STAGE == kGram ? 0.f : STAGE == kPoly ? step.b * (kPolyScale / kGramScale) : step.a;
    const int64_t row_c = ROWS ? M.row_n : M.row_m;
    const int j_end = ROWS ? M.np : M.mp;
    const char *old = STAGE == kPoly ? P : X;
    char *to = ws + (STAGE == kGram ? M.g : STAGE == kPoly ? M.b : M.x[1 - step.from]);
    const float f = M.factor / M.scale;
#pragma unroll
    for (int a = 0; a < FM; ++a) {
        const int i = i0 + wi + a * 32 + r;
        if (i0 + wi + a * 32 >= M.mp) break;                   // rounded sizes are multiples of 64: whole 32 x 32 parts
#pragma unroll
        for (int b = 0; b < FN; ++b) {
            const int jb = j0 + wj + b * 32;
            if (jb >= j_end) break;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int j = jb + 8 * g + 4 * h;
                const int64_t at = chunk_at<SPLIT>(row_c, i, j);
                float v[4];
                if (STAGE != kGram) load4<SPLIT>(old + at, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = acc[a][b][4 * g + e] * alpha;
                    v[e] = STAGE == kGram ? p : __fmaf_rn(beta, v[e], p);
                }
                if constexpr (STAGE != kLast) {
                    store4<SPLIT>(to + at, v);
                    if (STAGE < kApply && tl.i != tl.j) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) store1<SPLIT>(to + chunk_at<SPLIT>(row_c, j + e, i & ~7) + (i & 7) * 2, v[e]);
                    }
                } else if (i < M.m) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (j + e >= M.n) break;
                        const int64_t o_at = M.offset + (M.flip ? (j + e) * M.ld + i : i * M.ld + j + e);
                        const float o = v[e] * f;
                        if (OUT == 0) static_cast<float *>(out.dst)[o_at] = o;
                        else if (OUT == 1) static_cast<uint16_t *>(out.dst)[o_at] = bf16_round(o);
                        else out.x[o_at] = __fmaf_rn(-out.gamma, o, out.keep * out.x[o_at]);
                    }
                }
            }
        }
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
    const Tile *square, *wide, *operands;  // tiles of G and B, of X, and of the operands' pass
    const int2 *parts;
    int64_t n_square, n_wide, n_operands, n_parts;
    int square_side, wide_side;
    double *partial;
    uint64_t *inside;                      // plane of bits: the elements of the matrices
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

// Tables of the plan; the matrices were checked.
struct Tables {
    std::vector<Mat> mats;
    std::vector<Tile> square, wide, operands;
    std::vector<int2> parts;
    int64_t n_partial = 0, ws_bytes = 0;
    int square_side = 64, wide_side = 64;
};

// Tiles of `side` in the order in which they are given out: long sums first, so that the launch ends with short ones; within a
// matrix strips of rows, so that tiles near each other in time share rows and columns; runs of kRun tiles to one XCD
// (workgroup p runs on XCD p % 8, each with an L2 of its own).
std::vector<Tile> make_tiles(const std::vector<Mat> &mats, int side, bool square)
{
    constexpr size_t kRun = 32;
    std::vector<int32_t> order(mats.size());
    for (size_t k = 0; k < mats.size(); ++k) order[k] = static_cast<int32_t>(k);
    auto length = [&](int32_t k) { return square ? mats[k].np : mats[k].mp; };
    std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return length(a) > length(b); });
    std::vector<Tile> list;
    const int32_t strip = 1024 / side;
    for (int32_t k : order) {
        const int32_t ti = (mats[k].mp + side - 1) / side, tj = square ? ti : (mats[k].np + side - 1) / side;
        for (int32_t i0 = 0; i0 < ti; i0 += strip)
            for (int32_t j = 0; j < tj; ++j)
                for (int32_t i = i0; i < std::min(i0 + strip, ti); ++i)
                    if (!square || j <= i) list.push_back(Tile{k, i, j, 0});
    }
    std::vector<Tile> out;
    out.reserve(list.size());
    size_t next[8], xcd = 0;
    for (size_t q = 0; q < 8; ++q) next[q] = q * kRun;
    while (out.size() < list.size()) {
        if (next[xcd] < list.size()) {
            out.push_back(list[next[xcd]]);
            if (++next[xcd] % kRun == 0) next[xcd] += 7 * kRun;
        } else {
            // nothing is left for this XCD: its turn goes to the one that has most left
            size_t far = 8;
            for (size_t q = 0; q < 8; ++q)
                if (next[q] < list.size() && (far == 8 || next[q] < next[far])) far = q;
            out.push_back(list[next[far]]);
            if (++next[far] % kRun == 0) next[far] += 7 * kRun;
        }
        xcd = (xcd + 1) % 8;
    }
    return out;
}

int64_t count_tiles(const std::vector<Mat> &mats, int side, bool square)
{
    int64_t n = 0;
    for (const Mat &M : mats) {
        const int64_t ti = (M.mp + side - 1) / side, tj = (M.np + side - 1) / side;
        n += square ? ti * (ti + 1) / 2 : ti * tj;
    }
    return n;
}

// Side of the tiles: rounds of the device's 256 compute units times the time of a tile.
int tile_side(const std::vector<Mat> &mats, bool square)
{
    auto rounds = [&](int side, int64_t at_once) { return static_cast<double>((count_tiles(mats, side, square) + at_once - 1) / at_once); };
    const double t256 = rounds(256, 256) * 1.0, t128 = rounds(128, 512) * 0.55, t64 = rounds(64, 1024) * 0.35;
    return t64 < t128 && t64 < t256 ? 64 : t128 < t256 ? 128 : 256;
}

void make_tables(const ds_ortho_config_t &cfg, bool split, Tables &t)
{
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
        M.row_n = M.np * (split ? 4 : 2);
        M.row_m = M.mp * (split ? 4 : 2);
        // entries of an orthogonal [m, n] matrix are about 1 / sqrt(n); 16 there leaves 2^-25 of an entry to lo, and
        // 2^14 keeps the largest possible one, singular value 2, below the largest half
        int s = 4;
        while (s < 14 && (1ll << (2 * (s - 4))) < M.n) ++s;
        M.scale = static_cast<float>(1 << s);
        const double aspect = static_cast<double>(in.rows) / in.cols;
        M.factor = cfg.factor == DS_ORTHO_FACTOR_ASPECT ? static_cast<float>(sqrt(std::max(1.0, aspect)))
                   : cfg.factor == DS_ORTHO_FACTOR_RMS ? static_cast<float>(0.2 * sqrt(static_cast<double>(M.n))) : 1.0f;
        auto take = [&](int64_t bytes) {
            const int64_t at = t.ws_bytes;
            t.ws_bytes += round_up(bytes, 256);
            return at;
        };
        M.x[0] = take(static_cast<int64_t>(M.mp) * M.row_n);
        M.x[1] = take(static_cast<int64_t>(M.mp) * M.row_n);
        M.g = take(static_cast<int64_t>(M.mp) * M.row_m);
        M.b = take(static_cast<int64_t>(M.mp) * M.row_m);
        const int64_t elements = static_cast<int64_t>(M.m) * M.n;
        M.parts = static_cast<int32_t>(std::min<int64_t>(kMaxParts, (elements + kPartElements - 1) / kPartElements));
        M.part0 = static_cast<int32_t>(t.n_partial);
        t.n_partial += M.parts;
        for (int32_t p = 0; p < M.parts; ++p) t.parts.push_back(int2{k, p});
        t.mats.push_back(M);
    }
    t.square_side = tile_side(t.mats, true);
    t.wide_side = tile_side(t.mats, false);
    t.square = make_tiles(t.mats, t.square_side, true);
    t.wide = make_tiles(t.mats, t.wide_side, false);
    t.operands = make_tiles(t.mats, 64, false);
}

template <bool SPLIT, int STAGE, int OUT>
void product(const ds_ortho *o, const Step &s, const Out &out, hipStream_t st)
{
    constexpr bool WIDE = STAGE >= kApply;
    const Tile *tiles = WIDE ? o->wide : o->square;
    const unsigned n = static_cast<unsigned>(WIDE ? o->n_wide : o->n_square);
    switch (WIDE ? o->wide_side : o->square_side) {
    case 256: k_ortho_product<256, 256, 128, 64, SPLIT, STAGE, OUT><<<n, 512, 0, st>>>(o->mats, tiles, o->ws, s, out); break;
    case 128: k_ortho_product<128, 128, 64, 64, SPLIT, STAGE, OUT><<<n, 256, 0, st>>>(o->mats, tiles, o->ws, s, out); break;
    default: k_ortho_product<64, 64, 32, 32, SPLIT, STAGE, OUT><<<n, 256, 0, st>>>(o->mats, tiles, o->ws, s, out); break;
    }
}

// The matrices through the plan's steps; `src` holds U, where the last product goes is `out`.
template <bool SPLIT, bool SRC_BF16, int OUT>
ds_status_t run(const ds_ortho *o, const void *src, const Out &out, hipStream_t st)
{
    auto grid = [](int64_t n) { return static_cast<unsigned>(n); };
    k_ortho_norm<SRC_BF16><<<grid(o->n_parts), kBlock, 0, st>>>(o->mats, o->parts, src, o->partial);
    k_ortho_operands<SPLIT, SRC_BF16><<<grid(o->n_operands), kThreads, 0, st>>>(o->mats, o->operands, src, o->partial, o->cfg.eps, o->ws);
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

}  // namespace

const uint64_t *ds_ortho_inside(const ds_ortho *o) { return o->inside; }
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
    if (cfg->coef)
        for (int32_t k = 0; k < 3 * cfg->steps; ++k)
            if (!std::isfinite(cfg->coef[k])) return DS_ERR_CONFIG;
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
        o->n_square = static_cast<int64_t>(t.square.size());
        o->n_wide = static_cast<int64_t>(t.wide.size());
        o->n_operands = static_cast<int64_t>(t.operands.size());
        o->n_parts = static_cast<int64_t>(t.parts.size());
        o->square_side = t.square_side;
        o->wide_side = t.wide_side;
        int64_t bytes = 0;
        auto take = [&](int64_t b) {
            const int64_t at = bytes;
            bytes += round_up(b, 256);
            return at;
        };
        auto size_of = [](const auto &v) { return static_cast<int64_t>(v.size() * sizeof(v[0])); };
        const int64_t at_mats = take(size_of(t.mats)), at_square = take(size_of(t.square)), at_wide = take(size_of(t.wide)),
                      at_operands = take(size_of(t.operands)), at_parts = take(size_of(t.parts)), at_inside = take(size_of(plane));
        const int64_t at_partial = take(t.n_partial * 8), at_u = take(cfg->d * 4), at_ws = take(t.ws_bytes);
        ds_status_t rc = hipGetDevice(&o->device) == hipSuccess ? DS_OK : DS_ERR_DEVICE;
        if (rc == DS_OK && hipMalloc(&o->mem, static_cast<size_t>(bytes)) != hipSuccess) {
            o->mem = nullptr;
            (void)hipGetLastError();       // a failed allocation is this call's result and nobody else's
            rc = DS_ERR_DEVICE;
        }
        char *base = static_cast<char *>(o->mem);
        auto put = [&](int64_t at, const auto &v) {
            if (rc == DS_OK && hipMemcpy(base + at, v.data(), v.size() * sizeof(v[0]), hipMemcpyHostToDevice) != hipSuccess) rc = DS_ERR_DEVICE;
        };
        put(at_mats, t.mats);
        put(at_square, t.square);
        put(at_wide, t.wide);
        put(at_operands, t.operands);
        put(at_parts, t.parts);
        put(at_inside, plane);
        if (rc == DS_OK && hipStreamSynchronize(nullptr) != hipSuccess) rc = DS_ERR_DEVICE;
        if (rc != DS_OK) {
            ds_ortho_destroy(o);
            return rc;
        }
        o->mats = reinterpret_cast<const Mat *>(base + at_mats);
        o->square = reinterpret_cast<const Tile *>(base + at_square);
        o->wide = reinterpret_cast<const Tile *>(base + at_wide);
        o->operands = reinterpret_cast<const Tile *>(base + at_operands);
        o->parts = reinterpret_cast<const int2 *>(base + at_parts);
        o->inside = reinterpret_cast<uint64_t *>(base + at_inside);
        o->partial = reinterpret_cast<double *>(base + at_partial);
        o->u = reinterpret_cast<float *>(base + at_u);
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
