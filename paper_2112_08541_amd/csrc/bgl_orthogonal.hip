// Orthogonalised updates: X = U / (|U| + eps), then so many steps of  P = X X',  Q = a I + b P + c P P,  X <- Q X,  which move every
// singular value towards 1 and leave the singular vectors alone.  The shorter side is made the rows (the steps on X' give the same
// result transposed), so P and Q have the shorter side squared.
//
// All three products run on the matrix units in fp16 with every value split in two: v = hi + lo, hi the nearest half, lo the nearest
// half of the rest, together 22 bits; hi hi + hi lo + lo hi leaves out lo lo (2^-22 of the product at most).  Three fp16 products of 16x16x32 take
// 48 cycles, the fp32 instructions for the same tile 256.  One half alone (2^-11) will not do: the steps enlarge what lies in the
// directions of small singular values by up to a^steps (485 for the usual coefficients), rounding errors included.  Values are kept near the upper
// end of fp16's range by powers of two, known beforehand because the singular values are: |X| <= 1 to begin with, so the coefficients alone
// say how large X, P and Q can become.  Sums are fp32, the norm is summed in fp64.
//
// X is kept in both orders, so that in each product both operands have the summed index contiguous.  A split row holds for each 32
// values 32 hi, then 32 lo: 128 bytes, what a tile takes of a row.  P and Q are symmetric: tiles on and below the diagonal are
// computed, and stored twice.
#include "bgl_internal.h"
#include "bgl_tile.h"

#include <cmath>

namespace bgl {
namespace {

using namespace tile;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kNormParts = 64;

struct OrthoArgs {
    const void *update;
    void *out;
    int64_t in_matrix, in_row, out_matrix, out_row;  // strides in values
    int64_t batch;
    int m, n, mp, np;           // m <= n; padded to whole blocks of 32
    bool tall;                  // the update has n rows and m columns
    float a, b, c, eps;
    float sx, sp, sq;           // what X, P and Q are scaled by
    double *norms;              // [batch][kNormParts]
    uint32_t *x[2], *xt[2], *p, *q;  // split rows: [m][np], [n][mp], [m][mp], [m][mp] per matrix
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

// Sums of squares of equal shares of a matrix.
template <class T>
__global__ __launch_bounds__(kThreads) void k_ortho_norm(OrthoArgs a)
{
    __shared__ double sums[kThreads / kWave];
    const int rows = a.tall ? a.n : a.m, cols = a.tall ? a.m : a.n;
    const typename T::elem *u = (const typename T::elem *)a.update + (int64_t)blockIdx.y * a.in_matrix;
    double sum = 0.0;
    for (int r = blockIdx.x; r < rows; r += kNormParts)
        for (int c = threadIdx.x; c < cols; c += kThreads) {
            const double v = (double)T::get(u[(int64_t)r * a.in_row + c]);
            sum += v * v;
        }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.norms[(int64_t)blockIdx.y * kNormParts + blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// X, in both orders, of one 64 x 64 tile.
template <class T>
__global__ __launch_bounds__(kThreads) void k_ortho_start(OrthoArgs a)
{
    __shared__ float tile[64][65];
    const int64_t matrix = blockIdx.z;
    double sum = a.norms[matrix * kNormParts + (threadIdx.x & 63)];
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    const float norm = (float)sqrt(sum) + a.eps;
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    const typename T::elem *u = (const typename T::elem *)a.update + matrix * a.in_matrix;
    for (int i = threadIdx.x; i < 64 * 64; i += kThreads) {
        const int slow = i / 64, fast = i % 64;
        const int r = a.tall ? fast : slow, c = a.tall ? slow : fast;
        float v = 0.0f;
        if (r0 + r < a.m && c0 + c < a.n)
            v = T::get(u[a.tall ? (int64_t)(c0 + c) * a.in_row + r0 + r : (int64_t)(r0 + r) * a.in_row + c0 + c]) / norm;
        tile[r][c] = v * a.sx;
    }
    __syncthreads();
    uint32_t *x = a.x[0] + matrix * a.m * a.np, *xt = a.xt[0] + matrix * a.n * a.mp;
    for (int i = threadIdx.x; i < 64 * 16; i += kThreads) {
        const int s = i / 16, f = i % 16 * 4;
        if (r0 + s < a.m && c0 + f < a.np) store_split<4>(x + (int64_t)(r0 + s) * a.np, c0 + f, {tile[s][f], tile[s][f + 1], tile[s][f + 2], tile[s][f + 3]});
        if (c0 + s < a.n && r0 + f < a.mp) store_split<4>(xt + (int64_t)(c0 + s) * a.mp, r0 + f, {tile[f][s], tile[f + 1][s], tile[f + 2][s], tile[f + 3][s]});
    }
}

enum { GRAM, POLY, APPLY, LAST };  // P = X X', Q from P P, X <- Q X, the same into the caller's memory

// One tile of one matrix's product; `from` says which of the two copies of X is read.
template <int TT, int STAGE, class T>
__global__ __launch_bounds__(kThreads, 2) void k_ortho_product(OrthoArgs a, int from, int row_tiles, int col_tiles)
{
    constexpr int BO = 32 * TT;
    using C = Cut<2, 2, TT, TT>;
    __shared__ __attribute__((aligned(16))) uint32_t lds[BO * BO > 2 * KcOperand<F32, BO>::LDS ? BO * BO : 2 * KcOperand<F32, BO>::LDS];  // both operands; the sums afterwards
    constexpr bool SYMMETRIC = STAGE == GRAM || STAGE == POLY;
    const int tiles = SYMMETRIC ? row_tiles * (row_tiles + 1) / 2 : row_tiles * col_tiles;
    int64_t matrix;
    int t;
    if (a.batch >= 8) {  // a matrix's tiles on one XCD
        if (!tile_of(blockIdx.x, a.batch, tiles, matrix, t)) return;
    } else {
        matrix = blockIdx.x / tiles, t = blockIdx.x % tiles;
    }
    int rt, ct;
    if constexpr (SYMMETRIC) {
        rt = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (rt * (rt + 1) / 2 > t) --rt;
        while ((rt + 1) * (rt + 2) / 2 <= t) ++rt;
        ct = t - rt * (rt + 1) / 2;
    } else {
        rt = t / col_tiles, ct = t % col_tiles;
    }
    const int64_t mm = matrix * a.m * a.mp, mn = matrix * a.m * a.np, nm = matrix * a.n * a.mp;
    const uint32_t *left = STAGE == GRAM ? a.x[from] + mn : STAGE == POLY ? a.p + mm : a.q + mm;
    const uint32_t *right = STAGE == GRAM ? a.x[from] + mn : STAGE == POLY ? a.p + mm : a.xt[from] + nm;
    const int K = STAGE == GRAM ? a.np : a.mp, cols = SYMMETRIC ? a.m : a.n;
    const int r0 = rt * BO, c0 = ct * BO;
    KcOperand<F32, BO> l, r;  // (its 32 dwords are 32 pairs of halves here)
    l.init([&](int i) { return reinterpret_cast<const float *>(left) + (int64_t)(r0 + i < a.m ? r0 + i : a.m - 1) * K; });
    r.init([&](int i) { return reinterpret_cast<const float *>(right) + (int64_t)(c0 + i < cols ? c0 + i : cols - 1) * K; });
    f32x4 acc[TT][TT] = {};
    using Op = KcOperand<F32, BO>;
    pipeline(
        K / kDwords,
        [&](int i) {
            l.load_whole(i);
            r.load_whole(i);
        },
        [&] {
            l.store(lds);
            r.store(lds + Op::LDS);
        },
        [&](int) {
            uint32_t ah[TT][4], al[TT][4], bh[TT][4], bl[TT][4];
            Op::read(lds, C::a_off(), 0, ah);
            Op::read(lds + Op::LDS, C::b_off(), 0, bh);
            Op::read(lds, C::a_off(), 1, al);
            Op::read(lds + Op::LDS, C::b_off(), 1, bl);
            const auto mma = [&](uint32_t(&x)[TT][4], uint32_t(&y)[TT][4]) {
#pragma unroll
                for (int s = 0; s < TT; ++s)
#pragma unroll
                    for (int u = 0; u < TT; ++u)
                        acc[s][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x[s]), __builtin_bit_cast(f16x8, y[u]), acc[s][u], 0, 0, 0);
            };
            mma(ah, bh);
            mma(ah, bl);
            mma(al, bh);
        });
    const float scale = STAGE == GRAM ? 1.0f / (a.sx * a.sx) : STAGE == POLY ? 1.0f / (a.sp * a.sp) : 1.0f / (a.sq * a.sx);
    float *sums = reinterpret_cast<float *>(lds);
    Result<C, BO * BO>::put(sums, 0, acc);
    __syncthreads();
    // four columns of a row, then (for the copies in the other order) four rows of a column
    constexpr int FOURS = BO / 4;
    if constexpr (SYMMETRIC) {
        uint32_t *to = (STAGE == GRAM ? a.p : a.q) + mm;
        for (int i = threadIdx.x; i < BO * FOURS; i += kThreads) {
            const int r = i / FOURS, c = i % FOURS * 4;
            if (r0 + r >= a.m || c0 + c >= a.mp) continue;
            f32x4 *at = reinterpret_cast<f32x4 *>(sums + result_place<BO>(r, c));
            f32x4 v = *at;
            float w[4];
            float p[4] = {};
            if (STAGE == POLY) joined4(a.p + mm + (int64_t)(r0 + r) * a.mp, c0 + c, p);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] *= scale;
                if (STAGE == POLY) v[e] = (r0 + r == c0 + c + e ? a.a : 0.0f) + a.b * (p[e] / a.sp) + a.c * v[e];
                v[e] = w[e] = c0 + c + e < a.m ? v[e] * (STAGE == GRAM ? a.sp : a.sq) : 0.0f;
            }
            if (rt != ct) *at = v;
            store_split<4>(to + (int64_t)(r0 + r) * a.mp, c0 + c, w);
        }
        if (rt == ct) return;
        __syncthreads();
        for (int i = threadIdx.x; i < BO * FOURS; i += kThreads) {  // (the columns are whole here: ct < rt)
            const int c = i % BO, r = i / BO * 4;
            if (r0 + r >= a.mp) continue;
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = r0 + r + e < a.m ? sums[result_place<BO>(r + e, c)] : 0.0f;
            store_split<4>(to + (int64_t)(c0 + c) * a.mp, r0 + r, w);
        }
    } else if constexpr (STAGE == APPLY) {
        for (int i = threadIdx.x; i < BO * FOURS; i += kThreads) {
            const int r = i / FOURS, c = i % FOURS * 4;
            if (r0 + r >= a.m || c0 + c >= a.np) continue;
            const f32x4 v = *reinterpret_cast<const f32x4 *>(sums + result_place<BO>(r, c));
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = c0 + c + e < a.n ? v[e] * scale * a.sx : 0.0f;
            store_split<4>(a.x[from ^ 1] + mn + (int64_t)(r0 + r) * a.np, c0 + c, w);
        }
        for (int i = threadIdx.x; i < BO * FOURS; i += kThreads) {
            const int c = i % BO, r = i / BO * 4;
            if (c0 + c >= a.n || r0 + r >= a.mp) continue;
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = r0 + r + e < a.m ? sums[result_place<BO>(r + e, c)] * scale * a.sx : 0.0f;
            store_split<4>(a.xt[from ^ 1] + nm + (int64_t)(c0 + c) * a.mp, r0 + r, w);
        }
    } else {
        typename T::elem *out = (typename T::elem *)a.out + matrix * a.out_matrix;
        for (int i = threadIdx.x; i < BO * BO; i += kThreads) {
            const int r = a.tall ? i % BO : i / BO, c = a.tall ? i / BO : i % BO;
            if (r0 + r < a.m && c0 + c < a.n)
                out[a.tall ? (int64_t)(c0 + c) * a.out_row + r0 + r : (int64_t)(r0 + r) * a.out_row + c0 + c] = T::put(sums[result_place<BO>(r, c)] * scale);
        }
    }
}

// Powers of two that keep X, P and Q below a quarter of fp16's largest value.  False: with these coefficients the steps lead out of bounds.
bool scales(float a, float b, float c, int steps, OrthoArgs &o)
{
    double most_x = 1.0, most_q = 0.0;
    for (int i = 0; i <= 4096; ++i) {
        double s = i / 4096.0;
        for (int k = 0; k < steps; ++k) {
            const double q = a + b * s * s + c * s * s * s * s;
            s *= q;
            if (!(std::fabs(s) < 64.0) || !(std::fabs(q) < 4096.0)) return false;
            most_x = std::fmax(most_x, std::fabs(s));
            most_q = std::fmax(most_q, std::fabs(q));
        }
    }
    const auto power = [](double most) { return (float)std::exp2(std::floor(std::log2(16384.0 / most))); };
    o.sx = power(most_x);
    o.sp = power(most_x * most_x);
    o.sq = power(std::fmax(most_q, 1e-3));
    return true;
}

struct OrthoSizes {
    int m, n, mp, np;
    size_t norms, x, xt, p, total;
};

OrthoSizes ortho_sizes(int64_t batch, int32_t rows, int32_t cols)
{
    OrthoSizes s;
    s.m = rows < cols ? rows : cols;
    s.n = rows < cols ? cols : rows;
    s.mp = (int)round_up(s.m, 32);
    s.np = (int)round_up(s.n, 32);
    s.norms = round_up((size_t)batch * kNormParts * sizeof(double), 256);
    s.x = round_up((size_t)batch * s.m * s.np * 4, 256);
    s.xt = round_up((size_t)batch * s.n * s.mp * 4, 256);
    s.p = round_up((size_t)batch * s.m * s.mp * 4, 256);
    s.total = s.norms + 2 * (s.x + s.xt + s.p);
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

template <int TT, class T>
int launch_steps(const OrthoArgs &a, int steps, hipStream_t st)
{
    const int bo = 32 * TT, rt = (int)ceil_div(a.m, bo), ct = (int)ceil_div(a.n, bo);
    const auto grid = [&](int64_t tiles) { return a.batch >= 8 ? tile_count(a.batch, (int)tiles) : a.batch * tiles; };
    const int64_t half = grid((int64_t)rt * (rt + 1) / 2), full = grid((int64_t)rt * ct);
    if (half > INT32_MAX || full > INT32_MAX) BGL_FAIL(BGL_EUNSUPPORTED, "%lld matrices of %d x %d need too many workgroups", (long long)a.batch, a.m, a.n);
    const dim3 block(kThreads);
    for (int k = 0; k < steps; ++k) {
        k_ortho_product<TT, GRAM, T><<<dim3((unsigned)half), block, 0, st>>>(a, k & 1, rt, rt);
        k_ortho_product<TT, POLY, T><<<dim3((unsigned)half), block, 0, st>>>(a, k & 1, rt, rt);
        if (k + 1 < steps) k_ortho_product<TT, APPLY, T><<<dim3((unsigned)full), block, 0, st>>>(a, k & 1, rt, ct);
        else k_ortho_product<TT, LAST, T><<<dim3((unsigned)full), block, 0, st>>>(a, k & 1, rt, ct);
    }
    BGL_HIP(hipGetLastError());
    return BGL_OK;
}

template <class T>
int orthogonalize(const OrthoArgs &a, int steps, hipStream_t st)
{
    k_ortho_norm<T><<<dim3(kNormParts, (unsigned)a.batch), dim3(kThreads), 0, st>>>(a);
    k_ortho_start<T><<<dim3((unsigned)ceil_div(a.np, 64), (unsigned)ceil_div(a.mp, 64), (unsigned)a.batch), dim3(kThreads), 0, st>>>(a);
    BGL_HIP(hipGetLastError());
    // 128 x 128 tiles once the symmetric products have one for each CU
    const int64_t rt = ceil_div(a.m, 128);
    return a.batch * (rt * (rt + 1) / 2) >= 256 ? launch_steps<4, T>(a, steps, st) : launch_steps<2, T>(a, steps, st);
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
    a.batch = batch, a.m = s.m, a.n = s.n, a.mp = s.mp, a.np = s.np, a.tall = rows > cols;
    char *at = (char *)workspace;
    a.norms = (double *)at, at += s.norms;
    for (int i = 0; i < 2; ++i) a.x[i] = (uint32_t *)at, at += s.x;
    for (int i = 0; i < 2; ++i) a.xt[i] = (uint32_t *)at, at += s.xt;
    a.p = (uint32_t *)at, at += s.p;
    a.q = (uint32_t *)at;
    return dtype == BGL_F32 ? orthogonalize<tile::F32>(a, steps, (hipStream_t)stream) : orthogonalize<tile::BF16>(a, steps, (hipStream_t)stream);
} BGL_NOTHROW_END
