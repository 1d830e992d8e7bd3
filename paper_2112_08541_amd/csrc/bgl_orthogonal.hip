// Orthogonalised updates: X = U / (|U| + eps), then so many steps of  P = X X',  Q = a I + b P + c P P,  X <- Q X,  which move every
// singular value towards 1 and leave the singular vectors alone.  The shorter side is made the rows (the steps on X' give the same
// result transposed), so P and Q have the shorter side squared.
//
// All three products run on the matrix units in fp16 with every value split in two: v = hi + lo, hi the nearest half, lo the nearest
// half of the rest, together 22 bits; hi hi + hi lo + lo hi leaves out lo lo (2^-22 of the product at most).  Three fp16 products of 16x16x32 take
// 48 cycles, the fp32 instructions for the same tile 256.  One half alone (2^-11) will not do: the steps enlarge what lies in the
// directions of small singular values by up to a^steps (485 for the usual coefficients), rounding errors included.  Values are kept near the upper
// end of fp16's range by powers of two, known beforehand because the singular values are: |X| <= 1 to begin with, so the coefficients alone
// say how large X, P and Q can become.  Sums are fp32, the norm is fp64.
//
// A split row holds for each 32 values 32 hi, then 32 lo: 128 bytes, what a tile takes of a row.  X X' and P P read two operands along their rows;
// Q X reads X across them, by the transposing LDS read.  P and Q are symmetric: tiles on and below the diagonal are
// computed, and stored twice.
#include "bgl_internal.h"
#include "bgl_tile.h"

#include <cmath>
#include <type_traits>

namespace bgl {
namespace {

using namespace tile;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kNormParts = 256;

struct OrthoArgs {
    const void *update;
    void *out;
    int64_t in_matrix, in_row, out_matrix, out_row;  // strides in values
    int64_t batch;
    int m, n, mp, np;           // m <= n; padded to whole blocks of 32
    int lm, ln;                 // dwords from one split row to the next, of P and Q and of X
    bool tall;                  // the update has n rows and m columns
    float a, b, c, eps;
    float sx, sp, sq;           // what X, P and Q are scaled by
    double *norms;              // [batch][kNormParts]
    uint32_t *x[2], *p, *q;     // split rows: [m][ln], [m][lm], [m][lm] per matrix
};

__device__ __forceinline__ void split(float v, uint16_t &hi, uint16_t &lo)
{
    const _Float16 h = (_Float16)v;
    hi = __builtin_bit_cast(uint16_t, h);
    lo = __builtin_bit_cast(uint16_t, (_Float16)(v - (float)h));
}
// four neighbouring values of a split row, from column c (a multiple of 4)
__device__ __forceinline__ void joined4(const uint32_t *row, int c, float (&v)[4])
{
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    const uint16_t *at = reinterpret_cast<const uint16_t *>(row) + (c >> 5) * 64 + (c & 31);
    const f16x4 hi = *reinterpret_cast<const f16x4 *>(at), lo = *reinterpret_cast<const f16x4 *>(at + 32);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)hi[e] + (float)lo[e];
}
// TT neighbouring values of a split row, from column c (a multiple of TT)
template <int TT>
__device__ __forceinline__ void store_split(uint32_t *row, int c, const float (&v)[TT])
{
    struct __attribute__((aligned(2 * TT))) Pack { uint16_t e[TT]; } hi, lo;
#pragma unroll
    for (int i = 0; i < TT; ++i) split(v[i], hi.e[i], lo.e[i]);
    uint16_t *at = reinterpret_cast<uint16_t *>(row) + (c >> 5) * 64 + (c & 31);
    *reinterpret_cast<Pack *>(at) = hi;
    *reinterpret_cast<Pack *>(at + 32) = lo;
}

// In 64 bits: the norm of fp32 values may lie beyond fp32's largest, and without eps among its subnormal ones.
__device__ __forceinline__ double inverse_norm(double sum, float eps) { return 1.0 / (sqrt(sum) + (double)eps); }

// Sums of squares of equal shares of a matrix, for the norm: one pass in 256 workgroups a matrix, bound by its launch and a few dependent loads (24 of
// 256 x 512 bf16 5.2 us, 2 of 2048 x 1024 f32 4.4).
template <class T>
__global__ __launch_bounds__(kThreads) void k_ortho_norm(OrthoArgs a)
{
    __shared__ double sums[kThreads / kWave];
    const int rows = a.tall ? a.n : a.m, cols = a.tall ? a.m : a.n;
    const typename T::elem *u = (const typename T::elem *)a.update + (int64_t)blockIdx.y * a.in_matrix;
    double sum = 0.0;
    for (int c = threadIdx.x * T::VEC; c < cols; c += kThreads * T::VEC)
#pragma unroll 4
        for (int r = blockIdx.x; r < rows; r += kNormParts) {
            struct Piece { typename T::elem e[T::VEC]; } piece;
            const typename T::elem *from = u + (int64_t)r * a.in_row + c;
            if (c + T::VEC <= cols) {
                piece = load_any<Piece>(from);
            } else {
#pragma unroll
                for (int e = 0; e < T::VEC; ++e) piece.e[e] = c + e < cols ? from[e] : (typename T::elem)0;
            }
#pragma unroll
            for (int e = 0; e < T::VEC; ++e) {
                const double v = (double)T::get(piece.e[e]);
                sum += v * v;
            }
        }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.norms[(int64_t)blockIdx.y * kNormParts + blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// X of one 64 x 64 tile: the update over its norm, turned where it is tall (through LDS, so that both sides are read and written along rows), scaled and
// split.  Once a call; 2 of 2048 x 1024 f32 12.4 us (33 MB, 2.7 TB/s), 24 of 256 x 512 bf16 11.8: bound by its two chains of loads, norms and values.
template <class T>
__global__ __launch_bounds__(kThreads) void k_ortho_start(OrthoArgs a)
{
    __shared__ float tile[64][65];
    const int64_t matrix = blockIdx.z;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kNormParts / 64; ++i) sum += a.norms[matrix * kNormParts + i * 64 + (threadIdx.x & 63)];
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    const double inverse = inverse_norm(sum, a.eps);
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    const typename T::elem *u = (const typename T::elem *)a.update + matrix * a.in_matrix;
    for (int i = threadIdx.x; i < 64 * 64; i += kThreads) {
        const int slow = i / 64, fast = i % 64;
        const int r = a.tall ? fast : slow, c = a.tall ? slow : fast;
        float v = 0.0f;
        if (r0 + r < a.m && c0 + c < a.n)
            v = (float)(T::get(u[a.tall ? (int64_t)(c0 + c) * a.in_row + r0 + r : (int64_t)(r0 + r) * a.in_row + c0 + c]) * inverse);
        tile[r][c] = v * a.sx;
    }
    __syncthreads();
    uint32_t *x = a.x[0] + matrix * a.m * a.ln;
    for (int i = threadIdx.x; i < 64 * 16; i += kThreads) {
        const int s = i / 16, f = i % 16 * 4;
        if (r0 + s < a.m && c0 + f < a.np) store_split<4>(x + (int64_t)(r0 + s) * a.ln, c0 + f, {tile[s][f], tile[s][f + 1], tile[s][f + 2], tile[s][f + 3]});
    }
}

// acc += (ah + al) (bh + bl) without al bl
template <int FA, int FB>
__device__ __forceinline__ void add_split(const uint32_t (&ah)[FA][4], const uint32_t (&al)[FA][4], const uint32_t (&bh)[FB][4], const uint32_t (&bl)[FB][4], f32x4 (&acc)[FA][FB])
{
    const auto products = [&](const uint32_t(&x)[FA][4], const uint32_t(&y)[FB][4]) {
#pragma unroll
        for (int s = 0; s < FA; ++s)
#pragma unroll
            for (int u = 0; u < FB; ++u)
                acc[s][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x[s]), __builtin_bit_cast(f16x8, y[u]), acc[s][u], 0, 0, 0);
    };
    products(ah, bh);
    products(ah, bl);
    products(al, bh);
}

// The operand X of Q X: 32 of its rows (the summed index) by BO columns, [32][BO hi and lo].  Rows from m on, which meet zeros of Q, repeat the
// last.  In LDS the 32-byte units of a row (16 hi or 16 lo) are moved about so that four rows' equal units lie in different banks.
template <int BO>
struct SplitColumns {
    static constexpr int LDS = BO * kDwords, PER_ROW = BO / 4, ROWS = kThreads / PER_ROW, PASSES = 32 / ROWS, UNITS = BO / 8;
    const uint32_t *base;
    int stride, rows;
    uint4 reg[PASSES];
    __device__ __forceinline__ void init(const uint32_t *x, int np, int ld, int m, int c0)
    {
        const int c = c0 + team_thread() % PER_ROW * 4;
        base = x + (c < np ? c : 0);  // (a dword of a split row for each column)
        stride = ld;
        rows = m;
    }
    __device__ __forceinline__ void load_whole(int tile)
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int k = tile * 32 + team_thread() / PER_ROW + ROWS * p;
            reg[p] = *reinterpret_cast<const uint4 *>(base + (int64_t)(k < rows ? k : rows - 1) * stride);
        }
    }
    static __device__ __forceinline__ int place(int k, int h)  // half h of row k
    {
        constexpr int MASK = UNITS - 1;
        return k * 2 * BO + ((((h >> 4) ^ (((k & 3) | (k >> 3 & 1) << 2) & MASK)) << 4) | (h & 15));
    }
    __device__ __forceinline__ void store(uint32_t *lds) const
    {
        uint16_t *to = reinterpret_cast<uint16_t *>(lds);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) *reinterpret_cast<uint4 *>(to + place(team_thread() / PER_ROW + ROWS * p, team_thread() % PER_ROW * 8)) = reg[p];
    }
    template <int F>
    static __device__ __forceinline__ void read(const uint32_t *lds, int off, int lo, uint32_t (&f)[F][4])
    {
        const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
#pragma unroll
        for (int t = 0; t < F; ++t) {
            const int c = off + 16 * t;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t *from = reinterpret_cast<const uint16_t *>(lds) + place(8 * g + 4 * h + (i >> 2), (c >> 5) * 64 + (c & 31) + 32 * lo + 4 * (i & 3));
                const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uint16_t *)from));
                f[t][2 * h] = v.x, f[t][2 * h + 1] = v.y;
            }
        }
    }
};

enum { GRAM, POLY, APPLY, LAST };  // P = X X', Q from P P, X <- Q X, the same into the caller's memory

// One tile of one matrix's product; `from` says which of the two copies of X is read.  TEAMS of 256 threads take the summed index's tiles in
// turn and add up in LDS: where there are few tiles of the result, that many times the loads are on their way.
//
// 2 of 1024 x 2048 f32, a step: X X' 38.5 us (9.1 GFLOP on and below the diagonal, 237 TFLOP/s, as three fp16 products 710), P P 24, Q X 34 (253; 758 of
// 1,161 that a large fp16 product reaches).  24 of 256 x 512 bf16: 11, 9.2, 11.4.  The symmetric products are bound by loads: 136 tiles of 64 x 64 a matrix
// read 32 KB for 3 x 0.5 MFLOP, from L2 and the caches beyond it; the smaller ones by the launch and the first tile's loads, 4 to 5 us.  Two tiles ahead in
// registers instead of one: 477 us for all five steps instead of 468.
template <int TT, int STAGE, class T, int TEAMS>
__global__ __launch_bounds__(kThreads * TEAMS, 2) void k_ortho_product(OrthoArgs a, int from, int row_tiles, int col_tiles)
{
    constexpr int BO = 32 * TT;
    using C = Cut<2, 2, TT, TT>;
    __shared__ __attribute__((aligned(16))) uint32_t lds[BO * BO > TEAMS * 2 * KcOperand<F32, BO>::LDS ? BO * BO : TEAMS * 2 * KcOperand<F32, BO>::LDS];  // the operands; the sums afterwards
    constexpr bool SYMMETRIC = STAGE == GRAM || STAGE == POLY;
    const int tiles = SYMMETRIC ? row_tiles * (row_tiles + 1) / 2 : row_tiles * col_tiles;
    // each XCD (workgroup numbers go round them) has its eighth of all matrices' tiles in a row: few rows and columns meet in its L2
    const int64_t all = a.batch * tiles, eighth = (all + 7) / 8, at = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
    if (at >= all) return;
    const int64_t matrix = at / tiles;
    const int t = (int)(at % tiles);
    int rt, ct;
    if constexpr (SYMMETRIC) {
        rt = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (rt * (rt + 1) / 2 > t) --rt;
        while ((rt + 1) * (rt + 2) / 2 <= t) ++rt;
        ct = t - rt * (rt + 1) / 2;
    } else {
        ct = t / row_tiles, rt = t % row_tiles;
    }
    const int64_t mm = matrix * a.m * a.lm, mn = matrix * a.m * a.ln;
    const uint32_t *left = STAGE == GRAM ? a.x[from] + mn : STAGE == POLY ? a.p + mm : a.q + mm;
    const uint32_t *right = STAGE == GRAM ? left : STAGE == POLY ? left : a.x[from] + mn;
    const int K = STAGE == GRAM ? a.np : a.mp, ld = STAGE == GRAM ? a.ln : a.lm, cols = SYMMETRIC ? a.m : a.n;
    const int r0 = rt * BO, c0 = ct * BO;
    using Op = KcOperand<F32, BO>;  // (its 32 dwords are 32 pairs of halves here)
    using Right = std::conditional_t<SYMMETRIC, Op, SplitColumns<BO>>;
    Op l;
    Right r;
    l.init([&](int i) { return reinterpret_cast<const float *>(left) + (int64_t)(r0 + i < a.m ? r0 + i : a.m - 1) * ld; });
    if constexpr (SYMMETRIC) r.init([&](int i) { return reinterpret_cast<const float *>(right) + (int64_t)(c0 + i < cols ? c0 + i : cols - 1) * ld; });
    else r.init(right, a.np, a.ln, a.m, c0);
    f32x4 acc[TT][TT] = {};
    const int team = threadIdx.x / kThreads, depth = K / kDwords;
    uint32_t *mine = lds + team * 2 * Op::LDS;
    pipeline(
        (depth + TEAMS - 1) / TEAMS,
        [&](int i) {  // the team's i-th tile; behind the last one nothing is read and nothing added
            if (i * TEAMS + team < depth) {
                l.load_whole(i * TEAMS + team);
                r.load_whole(i * TEAMS + team);
            }
        },
        [&](int) {
            l.store(mine);
            r.store(mine + Op::LDS);
        },
        [&](int i) {
            if (TEAMS > 1 && i * TEAMS + team >= depth) return;
            uint32_t ah[TT][4], al[TT][4], bh[TT][4], bl[TT][4];
            Op::read(mine, C::a_off(), 0, ah);
            Right::read(mine + Op::LDS, C::b_off(), 0, bh);
            Op::read(mine, C::a_off(), 1, al);
            Right::read(mine + Op::LDS, C::b_off(), 1, bl);
            add_split<TT, TT>(ah, al, bh, bl, acc);
        });
    const float scale = STAGE == GRAM ? 1.0f / (a.sx * a.sx) : STAGE == POLY ? 1.0f / (a.sp * a.sp) : 1.0f / (a.sq * a.sx);
    float *sums = reinterpret_cast<float *>(lds);
    for (int t = 0; t < TEAMS; ++t) {
        if (t == team) Result<C, BO * BO>::put(sums, 0, acc, t > 0);
        __syncthreads();
    }
    constexpr int THREADS = kThreads * TEAMS;
    // four columns of a row, then (for the copies in the other order) four rows of a column
    constexpr int FOURS = BO / 4;
    if constexpr (SYMMETRIC) {
        uint32_t *to = (STAGE == GRAM ? a.p : a.q) + mm;
        for (int i = threadIdx.x; i < BO * FOURS; i += THREADS) {
            const int r = i / FOURS, c = i % FOURS * 4;
            if (r0 + r >= a.m || c0 + c >= a.mp) continue;
            f32x4 *at = reinterpret_cast<f32x4 *>(sums + result_place<BO>(r, c));
            f32x4 v = *at;
            float w[4];
            float p[4] = {};
            if (STAGE == POLY) joined4(a.p + mm + (int64_t)(r0 + r) * a.lm, c0 + c, p);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] *= scale;
                if (STAGE == POLY) v[e] = (r0 + r == c0 + c + e ? a.a : 0.0f) + a.b * (p[e] / a.sp) + a.c * v[e];
                v[e] = w[e] = c0 + c + e < a.m ? v[e] * (STAGE == GRAM ? a.sp : a.sq) : 0.0f;
            }
            if (rt != ct) *at = v;
            store_split<4>(to + (int64_t)(r0 + r) * a.lm, c0 + c, w);
        }
        if (rt == ct) return;
        __syncthreads();
        for (int i = threadIdx.x; i < BO * FOURS; i += THREADS) {  // (the columns are whole here: ct < rt)
            const int c = i % BO, r = i / BO * 4;
            if (r0 + r >= a.mp) continue;
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = r0 + r + e < a.m ? sums[result_place<BO>(r + e, c)] : 0.0f;
            store_split<4>(to + (int64_t)(c0 + c) * a.lm, r0 + r, w);
        }
    } else if constexpr (STAGE == APPLY) {
        for (int i = threadIdx.x; i < BO * FOURS; i += THREADS) {
            const int r = i / FOURS, c = i % FOURS * 4;
            if (r0 + r >= a.m || c0 + c >= a.np) continue;
            const f32x4 v = *reinterpret_cast<const f32x4 *>(sums + result_place<BO>(r, c));
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = c0 + c + e < a.n ? v[e] * scale * a.sx : 0.0f;
            store_split<4>(a.x[from ^ 1] + mn + (int64_t)(r0 + r) * a.ln, c0 + c, w);
        }
    } else {
        typename T::elem *out = (typename T::elem *)a.out + matrix * a.out_matrix;
        for (int i = threadIdx.x; i < BO * BO; i += THREADS) {
            const int r = a.tall ? i % BO : i / BO, c = a.tall ? i / BO : i % BO;
            if (r0 + r < a.m && c0 + c < a.n)
                out[a.tall ? (int64_t)(c0 + c) * a.out_row + r0 + r : (int64_t)(r0 + r) * a.out_row + c0 + c] = T::put(sums[result_place<BO>(r, c)] * scale);
        }
    }
}

// A whole update by one workgroup, X and P (then Q, in its place) in LDS: one launch instead of two and three for each step, which for
// small matrices are 4 to 7 us each (32 x 32 19 us instead of 69, 4 of 128 x 100 63 instead of 100, 128 x 128 62 instead of 100).  Split rows as in
// global memory, the 16-byte chunks of a block of 32 values moved about so that eight rows' equal chunks, and four rows' equal pairs of chunks, lie in
// different banks; X is read along its rows (X X') and across them (Q X; the transposing LDS read).  Bound by the one CU: a step of 128 x 100 is 12 us, of
// which the vector units, which split every value, are busy 70 %, the LDS 39 %, the matrix units 22 %.  A wavefront makes blocks of 32 x 32 of a product; X's new blocks wait in
// registers until all have been made.
constexpr int kWholeThreads = 1024, kWholeWaves = kWholeThreads / kWave, kWholeRounds = 2;

__device__ __forceinline__ int whole_place(int ld, int r, int c, int lo)  // in halves
{
    return r * 2 * ld + (c >> 5) * 64 + (((lo * 4 + (c >> 3 & 3)) ^ ((r & 3) << 1 | (r >> 2 & 1))) << 3 | (c & 7));
}
__device__ __forceinline__ void whole_put(uint16_t *to, int ld, int r, int c, float v)
{
    uint16_t hi, lo;
    split(v, hi, lo);
    to[whole_place(ld, r, c, 0)] = hi;
    to[whole_place(ld, r, c, 1)] = lo;
}
// Four neighbouring values of a row, from column c (a multiple of 4).
__device__ __forceinline__ void whole_put4(uint16_t *to, int ld, int r, int c, const float (&v)[4])
{
    struct __attribute__((aligned(8))) Four { uint16_t e[4]; } hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) split(v[i], hi.e[i], lo.e[i]);
    *reinterpret_cast<Four *>(to + whole_place(ld, r, c, 0)) = hi;
    *reinterpret_cast<Four *>(to + whole_place(ld, r, c, 1)) = lo;
}
// Four lanes of four rows by one column each: four columns of one row each.
__device__ __forceinline__ void turn4(int l, float (&v)[4])
{
    const auto swap = [&](float &x, float &y, bool upper, auto move) {  // the lower lane's y for the upper lane's x
        const float got = move(upper ? x : y);
        (upper ? x : y) = got;
    };
    const auto near = [](float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, true)); };  // lanes 1 0 3 2
    const auto far = [](float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, true)); };   // lanes 2 3 0 1
    swap(v[0], v[1], l & 1, near);
    swap(v[2], v[3], l & 1, near);
    swap(v[0], v[2], l & 2, far);
    swap(v[1], v[3], l & 2, far);
}
// A fragment's values to rows r0 .. r0 + 15 and columns c0 .. c0 + 15, and with `mirror` to the transposed place too.
__device__ __forceinline__ void whole_put_fragment(uint16_t *to, int ld, int l, int r0, int c0, float (&v)[4], bool mirror)
{
    if (mirror) whole_put4(to, ld, c0 + (l & 15), r0 + 4 * (l >> 4), v);
    turn4(l, v);
    whole_put4(to, ld, r0 + 4 * (l >> 4) + (l & 3), c0 + (l & 12), v);
}
// Two fragments along rows r0 .. r0 + 31 (Kc), 32 values of the summed index from k0.
__device__ __forceinline__ void whole_rows(const uint16_t *m, int ld, int l, int r0, int k0, int lo, uint32_t (&f)[2][4])
{
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint4 v = *reinterpret_cast<const uint4 *>(m + whole_place(ld, r0 + 16 * t + (l & 15), k0 + 8 * (l >> 4), lo));
        f[t][0] = v.x, f[t][1] = v.y, f[t][2] = v.z, f[t][3] = v.w;
    }
}
// Two fragments of columns c0 .. c0 + 31 (Oc): the summed index runs over rows k0 .. k0 + 31.
__device__ __forceinline__ void whole_columns(const uint16_t *m, int ld, int l, int c0, int k0, int lo, uint32_t (&f)[2][4])
{
    const int i = l & 15;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint16_t *from = m + whole_place(ld, k0 + 8 * (l >> 4) + 4 * h + (i >> 2), c0 + 16 * t + 4 * (i & 3), lo);
            const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uint16_t *)from));
            f[t][2 * h] = v.x, f[t][2 * h + 1] = v.y;
        }
}

template <class T>
__global__ __launch_bounds__(kWholeThreads) void k_ortho_whole(OrthoArgs a, int steps)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t whole[];
    __shared__ double partial[kWholeWaves];
    uint16_t *x = reinterpret_cast<uint16_t *>(whole), *p = reinterpret_cast<uint16_t *>(whole + a.mp * a.np);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), l = threadIdx.x & 63, bm = a.mp / 32, bn = a.np / 32;
    const int rows = a.tall ? a.n : a.m, cols = a.tall ? a.m : a.n;
    const typename T::elem *u = (const typename T::elem *)a.update + (int64_t)blockIdx.x * a.in_matrix;
    double sum = 0.0;
    for (int i = threadIdx.x; i < rows * cols; i += kWholeThreads) {
        const double v = (double)T::get(u[(int64_t)(i / cols) * a.in_row + i % cols]);
        sum += v * v;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (l == 0) partial[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kWholeWaves; ++w) sum += partial[w];
    const double inverse = inverse_norm(sum, a.eps);
    const int pad_rows = a.tall ? a.np : a.mp, pad_cols = a.tall ? a.mp : a.np;
    for (int i = threadIdx.x; i < pad_rows * pad_cols; i += kWholeThreads) {
        const int r = i / pad_cols, c = i % pad_cols;
        const float v = r < rows && c < cols ? (float)(T::get(u[(int64_t)r * a.in_row + c]) * inverse) * a.sx : 0.0f;
        whole_put(x, a.np, a.tall ? c : r, a.tall ? r : c, v);
    }
    __syncthreads();

    const int triangle = bm * (bm + 1) / 2;
    // the wavefront's block of P and Q: on or below the diagonal
    int br = 0;
    while ((br + 1) * (br + 2) / 2 <= wave) ++br;
    const int r0 = br * 32, c0 = (wave - br * (br + 1) / 2) * 32;
    // (the lane's number is made anew for each phase: else the addresses of all phases are kept in registers through all steps)
    const auto lane = [] {
        int l = threadIdx.x & 63;
        asm volatile("" : "+v"(l));
        return l;
    };
    const auto product = [&](const uint16_t *left, int ld, int lr, const uint16_t *right, int rd, int rc, auto across, int K, f32x4(&acc)[2][2]) {
        const int l = lane();
        for (int k = 0; k < K; k += 32) {
            uint32_t ah[2][4], al[2][4], bh[2][4], bl[2][4];
            whole_rows(left, ld, l, lr, k, 0, ah);
            whole_rows(left, ld, l, lr, k, 1, al);
            if constexpr (decltype(across)::value) {
                whole_columns(right, rd, l, rc, k, 0, bh);
                whole_columns(right, rd, l, rc, k, 1, bl);
            } else {
                whole_rows(right, rd, l, rc, k, 0, bh);
                whole_rows(right, rd, l, rc, k, 1, bl);
            }
            add_split<2, 2>(ah, al, bh, bl, acc);
        }
    };
    const std::false_type along{};
    const std::true_type across{};
    for (int step = 0; step < steps; ++step) {
        float own[2][2][4];  // the block's values of P
        if (wave < triangle) {
            f32x4 acc[2][2] = {};
            product(x, a.np, r0, x, a.np, c0, along, a.np, acc);
            const float scale = 1.0f / (a.sx * a.sx);
            const int l = lane();
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        own[s][t][j] = acc[s][t][j] * scale;
                        v[j] = own[s][t][j] * a.sp;
                    }
                    whole_put_fragment(p, a.mp, l, r0 + 16 * s, c0 + 16 * t, v, r0 != c0);
                }
        }
        __syncthreads();
        f32x4 square[2][2] = {};
        if (wave < triangle) product(p, a.mp, r0, p, a.mp, c0, along, a.mp, square);
        __syncthreads();
        if (wave < triangle) {
            const float scale = 1.0f / (a.sp * a.sp);
            const int l = lane();
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = r0 + 16 * s + 4 * (l >> 4) + j, c = c0 + 16 * t + (l & 15);
                        v[j] = ((r == c && r < a.m ? a.a : 0.0f) + a.b * own[s][t][j] + a.c * square[s][t][j] * scale) * a.sq;
                    }
                    whole_put_fragment(p, a.mp, l, r0 + 16 * s, c0 + 16 * t, v, r0 != c0);
                }
        }
        __syncthreads();
        f32x4 fresh[kWholeRounds][2][2] = {};
#pragma unroll
        for (int round = 0; round < kWholeRounds; ++round) {
            const int b = wave + round * kWholeWaves;
            if (b < bm * bn) product(p, a.mp, b / bn * 32, x, a.np, b % bn * 32, across, a.mp, fresh[round]);
        }
        __syncthreads();
        const bool last = step + 1 == steps;
        typename T::elem *out = (typename T::elem *)a.out + (int64_t)blockIdx.x * a.out_matrix;
        const float scale = 1.0f / (a.sq * a.sx);
        const int l = lane();
#pragma unroll
        for (int round = 0; round < kWholeRounds; ++round) {
            const int b = wave + round * kWholeWaves;
            if (b >= bm * bn) break;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int r = b / bn * 32 + 16 * s, c = b % bn * 32 + 16 * t;
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = fresh[round][s][t][j] * scale * (last ? 1.0f : a.sx);
                    if (!last) {
                        whole_put_fragment(x, a.np, l, r, c, v, false);
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int rr = r + 4 * (l >> 4) + j, cc = c + (l & 15);
                        if (rr < a.m && cc < a.n) out[a.tall ? (int64_t)cc * a.out_row + rr : (int64_t)rr * a.out_row + cc] = T::put(v[j]);
                    }
                }
        }
        __syncthreads();
    }
}

// Bytes of LDS, or 0 where a workgroup cannot have the whole of it.
size_t whole_bytes(int mp, int np)
{
    const size_t bytes = (size_t)mp * (np + mp) * 4;
    const int bm = mp / 32, bn = np / 32;
    return bm * (bm + 1) / 2 <= kWholeWaves && bm * bn <= kWholeWaves * kWholeRounds && bytes + 1024 <= 160 * 1024 ? bytes : 0;
}

// The largest |a s + b s^3 + c s^5| and |a + b s^2 + c s^4| for s in [0, most]: at the ends or where the slope is 0.
void largest(double a, double b, double c, double most, double &p, double &q)
{
    p = q = 0.0;
    const auto look = [&](double t) {  // t = s^2
        if (!(t >= 0.0 && t <= most * most)) return;
        const double v = std::fabs(a + b * t + c * t * t);
        q = std::fmax(q, v);
        p = std::fmax(p, v * std::sqrt(t));
    };
    look(0.0);
    look(most * most);
    look(-b / (2.0 * c));                                // of q
    const double root = std::sqrt(9.0 * b * b - 20.0 * a * c);  // of p: a + 3 b t + 5 c t^2 = 0 (none: NaN, which look() leaves out)
    look((-3.0 * b + root) / (10.0 * c));
    look((-3.0 * b - root) / (10.0 * c));
    look(-a / (3.0 * b));  // c = 0
}

// Powers of two that keep X, P and Q below a quarter of fp16's largest value.  False: with these coefficients the steps may lead out of bounds.
bool scales(double a, double b, double c, int steps, OrthoArgs &o)
{
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    double now = 1.0, most_x = 1.0, most_q = 0.0;
    for (int k = 0; k < steps; ++k) {
        double p, q;
        largest(a, b, c, now, p, q);
        if (!(p < 64.0) || !(q < 4096.0)) return false;
        now = p;
        most_x = std::fmax(most_x, p);
        most_q = std::fmax(most_q, q);
    }
    const auto power = [](double most) { return (float)std::exp2(std::floor(std::log2(16384.0 / most))); };
    o.sx = power(most_x);
    o.sp = power(most_x * most_x);
    o.sq = power(std::fmax(most_q, 1e-3));
    return true;
}

struct OrthoSizes {
    int m, n, mp, np, lm, ln;
    size_t norms, x, p, total;
};

OrthoSizes ortho_sizes(int64_t batch, int32_t rows, int32_t cols)
{
    OrthoSizes s;
    s.m = rows < cols ? rows : cols;
    s.n = rows < cols ? cols : rows;
    s.mp = (int)round_up(s.m, 32);
    s.np = (int)round_up(s.n, 32);
    s.norms = round_up((size_t)batch * kNormParts * sizeof(double), 256);
    // Rows an odd number of 256 bytes apart, so that the 128 bytes a tile reads of each of its rows lie in different channels of the L2 (1 of 1280 x
    // 1280: rows 5,120 bytes apart 345 us, 5,376 apart 319; 20 of 160 x 640 166 and 154; others within 2 %).
    s.lm = (int)round_up(s.mp + 64, 128) - 64;
    s.ln = (int)round_up(s.np + 64, 128) - 64;
    s.x = round_up((size_t)batch * s.m * s.ln * 4, 256);
    s.p = round_up((size_t)batch * s.m * s.lm * 4, 256);
    s.total = s.norms + 2 * (s.x + s.p);
    return s;
}

int check_matrices(int64_t batch, int32_t rows, int32_t cols, int32_t dtype)
{
    if (dtype != BGL_F32 && dtype != BGL_BF16) BGL_FAIL(BGL_EINVAL, "unknown dtype %d", dtype);
    if (batch < 0 || rows < 1 || cols < 1) BGL_FAIL(BGL_EINVAL, "batch, rows and cols must be positive (got %lld, %d, %d)", (long long)batch, rows, cols);
    if (rows > BGL_MAX_DIM || cols > BGL_MAX_DIM || batch > 65535)
        BGL_FAIL(BGL_EUNSUPPORTED, "rows and cols must be at most %d and batch at most 65535 (got %d, %d, %lld)", BGL_MAX_DIM, rows, cols, (long long)batch);
    return BGL_OK;
}

// 128 x 128 tiles (half the reads), where the sums are long enough to pay for the larger tile's ends (512), where the tiles are one for most CUs or
// more than three for two (257 to 384 leave half of the CUs idle for the second), and where they cover the result with no more than a 16th of it for nothing
// beyond what tiles of 64 do.  All five steps, us, with the larger tiles and without: Q X of 2 of 1024 x 2048 (256 tiles) 468 and 500, 1 of 3200 x 3200
// (625) 2,834 and 3,150, 24 of 256 x 512 (256 long) 185 and 176, 3 of 1280 x 1280 (300) 734 and 668, 4 of 1000 x 1300 (352) 642 and 615, 14 of 520 x 900 (a
// fifth for nothing) 593 and 528; X X' and P P of 7 of 1024 x 1024 (252) 734 and 745, 3 of 1536 x 1536 (234) 952 and 1,001, 1 of 2560 x 2560 (210) 1,381 and
// 1,593, 2 of 2560 x 2560 (420) 2,711 and 2,867, 1 of 3500 x 3500 (406) 3,524 and 3,927, 8 of 1024 x 1024 (288) 968 and 832, 2 of 2048 x 2048 (272) 1,725
// and 1,489, 13 of 640 x 640 (an 11th for nothing) 525 and 468, 20 of 520 x 700 (a third) 729 and 577.
//
// Else 64 x 64; two teams to a tile, four where the CUs have one tile at most and the sums are long.  Four teams instead of two: 1 of 1024 x 1024 232 us
// instead of 254, 4 of 400 x 800 (shorter sums) 214 instead of 195, 24 of 256 x 512 206 instead of 176, 2 of 1024 x 2048 (272 tiles) 541 instead of 498, 5 of
// 640 x 640 (275 tiles) 298 instead of 265.
template <int STAGE, class T>
void launch_product(const OrthoArgs &a, int from, hipStream_t st)
{
    constexpr bool SYMMETRIC = STAGE == GRAM || STAGE == POLY;
    const auto tiles = [&](int bo, int &rt, int &ct) {
        rt = (int)ceil_div(a.m, bo);
        ct = SYMMETRIC ? rt : (int)ceil_div(a.n, bo);
        return a.batch * (SYMMETRIC ? (int64_t)rt * (rt + 1) / 2 : (int64_t)rt * ct);
    };
    int rt, ct;
    const int64_t small = tiles(64, rt, ct), large = tiles(128, rt, ct);
    const int depth = STAGE == GRAM ? a.np : a.mp;
    const bool filled = large >= 192 && (large <= 256 || large > 384), covers = 64 * large <= 17 * small;
    if (filled && covers && depth >= 512) {
        k_ortho_product<4, STAGE, T, 2><<<dim3((unsigned)((large + 7) / 8 * 8)), dim3(2 * kThreads), 0, st>>>(a, from, rt, ct);
        return;
    }
    tiles(64, rt, ct);
    const dim3 grid((unsigned)((small + 7) / 8 * 8));
    if (small <= 256 && depth >= 640) k_ortho_product<2, STAGE, T, 4><<<grid, dim3(4 * kThreads), 0, st>>>(a, from, rt, ct);
    else k_ortho_product<2, STAGE, T, 2><<<grid, dim3(2 * kThreads), 0, st>>>(a, from, rt, ct);
}

template <class T>
int orthogonalize(const OrthoArgs &a, int steps, hipStream_t st)
{
    if (const size_t bytes = whole_bytes(a.mp, a.np)) {
        k_ortho_whole<T><<<dim3((unsigned)a.batch), dim3(kWholeThreads), bytes, st>>>(a, steps);
        BGL_HIP(hipGetLastError());
        return BGL_OK;
    }
    if (a.batch * ceil_div(a.m, 64) * ceil_div(a.n, 64) > INT32_MAX / 2)
        BGL_FAIL(BGL_EUNSUPPORTED, "%lld matrices of %d x %d need too many workgroups", (long long)a.batch, a.m, a.n);
    k_ortho_norm<T><<<dim3(kNormParts, (unsigned)a.batch), dim3(kThreads), 0, st>>>(a);
    k_ortho_start<T><<<dim3((unsigned)ceil_div(a.np, 64), (unsigned)ceil_div(a.mp, 64), (unsigned)a.batch), dim3(kThreads), 0, st>>>(a);
    for (int k = 0; k < steps; ++k) {
        launch_product<GRAM, T>(a, k & 1, st);
        launch_product<POLY, T>(a, k & 1, st);
        if (k + 1 < steps) launch_product<APPLY, T>(a, k & 1, st);
        else launch_product<LAST, T>(a, k & 1, st);
    }
    BGL_HIP(hipGetLastError());
    return BGL_OK;
}

}  // namespace
}  // namespace bgl

using namespace bgl;

extern "C" int bgl_orthogonalize_workspace_bytes(int64_t batch, int32_t rows, int32_t cols, int32_t dtype, size_t *bytes)
try {
    if (!bytes) BGL_FAIL(BGL_EINVAL, "bytes is null");
    const int rc = check_matrices(batch, rows, cols, dtype);
    if (rc != BGL_OK) return rc;
    *bytes = ortho_sizes(batch, rows, cols).total;
    return BGL_OK;
} BGL_NOTHROW_END

extern "C" int bgl_orthogonalize(const void *update, int64_t update_matrix_stride, int64_t update_row_stride, int64_t batch, int32_t rows, int32_t cols,
                                 int32_t dtype, int32_t steps, const float *coefficients, float eps, void *out, int64_t out_matrix_stride,
                                 int64_t out_row_stride, void *workspace, size_t workspace_bytes, void *stream)
try {
    const int rc = check_matrices(batch, rows, cols, dtype);
    if (rc != BGL_OK) return rc;
    if (!coefficients) BGL_FAIL(BGL_EINVAL, "coefficients is null");
    if (steps < 1 || steps > 64) BGL_FAIL(BGL_EINVAL, "steps must be in [1, 64] (got %d)", steps);
    if (!(eps >= 0.0f)) BGL_FAIL(BGL_EINVAL, "eps is negative");
    if (batch == 0) return BGL_OK;
    const size_t es = dtype == BGL_F32 ? 4 : 2;
    if (!update || !out || !aligned(update, es) || !aligned(out, es)) BGL_FAIL(BGL_EINVAL, "update or out is null or misaligned");
    if (update_row_stride < cols || out_row_stride < cols) BGL_FAIL(BGL_EINVAL, "a row stride is less than the row's %d values", cols);
    if (batch > 1 && (update_matrix_stride < (rows - 1) * update_row_stride + cols || out_matrix_stride < (rows - 1) * out_row_stride + cols))
        BGL_FAIL(BGL_EINVAL, "matrices overlap: a matrix stride is less than a matrix");
    const OrthoSizes s = ortho_sizes(batch, rows, cols);
    if (!workspace || !aligned(workspace, 256)) BGL_FAIL(BGL_EINVAL, "workspace is null or not 256-byte aligned");
    if (workspace_bytes < s.total) BGL_FAIL(BGL_ECAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, s.total);
    OrthoArgs a{};
    a.a = coefficients[0], a.b = coefficients[1], a.c = coefficients[2], a.eps = eps;
    if (!scales(a.a, a.b, a.c, steps, a)) BGL_FAIL(BGL_EUNSUPPORTED, "with coefficients %g, %g, %g the singular values grow out of bounds", a.a, a.b, a.c);
    a.update = update, a.out = out;
    a.in_matrix = update_matrix_stride, a.in_row = update_row_stride, a.out_matrix = out_matrix_stride, a.out_row = out_row_stride;
    a.batch = batch, a.m = s.m, a.n = s.n, a.mp = s.mp, a.np = s.np, a.lm = s.lm, a.ln = s.ln, a.tall = rows > cols;
    char *at = (char *)workspace;
    a.norms = (double *)at, at += s.norms;
    for (int i = 0; i < 2; ++i) a.x[i] = (uint32_t *)at, at += s.x;
    a.p = (uint32_t *)at, at += s.p;
    a.q = (uint32_t *)at;
    return dtype == BGL_F32 ? orthogonalize<tile::F32>(a, steps, (hipStream_t)stream) : orthogonalize<tile::BF16>(a, steps, (hipStream_t)stream);
} BGL_NOTHROW_END
