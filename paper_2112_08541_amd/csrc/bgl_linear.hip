// A layer over the rows of a batch: product with the weight, bias, residual and activation, and its gradients; with one weight for
// all rows or one per group of rows (nodes by type), and the grouping itself.
//
//   z = x W' + b (+ r)      y = act(z) (+ r)                      k_linear_forward
//   dz = dy act'(z)                                               k_linear_dz
//   dx = dz W                                                     k_linear_dx
//   dW = dz' x, db = sum dz                                       k_linear_dw (by ranges of rows), k_linear_reduce
//
// Sums are kept in fp32 whatever the type, and every result is rounded once.  What is rounded besides, in bf16 layers: z where it is kept for the gradient
// (gelu and silu: to a half, 2^-11; relu: to bf16, of which only the sign counts) and the dz of gelu and silu, because the matrix units read it in the type
// (2^-8 of itself at most, as the rows and weights that it meets are; without an activation and with relu it is dy or 0).  dx and dW are then some 1.4 times
// as far off as with dz in 32 bits; db is summed before.
#include "bgl_internal.h"
#include "bgl_tile.h"

#include <type_traits>

namespace bgl {
namespace {

using namespace tile;

constexpr int kMaxGroups = BGL_MAX_GROUPS;
constexpr int kGroupThreads = 512;   // of the grouping kernels
constexpr int kGroupTiles = 256;     // workgroups of one grouping pass at most
constexpr int kGroupTileRows = 2048; // rows a workgroup takes at least

// ----------------------------------------------------------------- activations
// The library's erff and expf are 30 to 50 instructions, which made the epilogue of 428,377 x 256 gelu values longer than their stores.  The forms here are
// as near in the tails as elsewhere, relative to the value: fp32 layers to some units of the last place, bf16 layers to 2^-15 or nearer, which rounding
// to the type outweighs a hundred times.
constexpr float kLog2e = 1.44269504088896341f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.693147180559945309f;

// exp(x + rest) for |x| <= 150 or so, |rest| small.  fp32: the hardware's 2^x of the rounded argument, times what rounding it left out; bf16 without that,
// which is |x| 2^-24 of the value.
template <class T>
__device__ __forceinline__ float exp_near(float x, float rest)
{
    const float whole = x * kLog2e, power = __builtin_amdgcn_exp2f(whole);
    if constexpr (T::PER == 2) return power;
    const float left = fmaf(rest, kLog2e, fmaf(x, kLog2eRest, fmaf(x, kLog2e, -whole)));
    return power * fmaf(left, kLn2, 1.0f);
}

// Phi(z) and, in `bell`, exp(-z^2 / 2) = phi(z) sqrt(2 pi).  Phi(-a) = bell R(a) for a >= 0, where R(a) = erfc(a / sqrt 2) exp(a^2 / 2) / 2 falls slowly: a
// rational function with positive coefficients (nothing cancels), fitted to the least relative error on [0, 14], beyond which bell is 0: 5.5e-9 with
// five and six coefficients, 3.8e-7 with four and five.
template <class T>
__device__ __forceinline__ float normal_cdf(float z, float &bell)
{
    const float a = fminf(fabsf(z), 16.0f), square = -0.5f * a * a;  // (NaN: 16, and z makes the result NaN)
    float above, below;
    if constexpr (T::PER == 2) {
        above = fmaf(a, fmaf(a, fmaf(a, 0.0170477093f, 0.119531738f), 0.361971406f), 0.49999981f);
        below = fmaf(a, fmaf(a, fmaf(a, fmaf(a, 0.0427372715f, 0.299418992f), 0.953440215f), 1.52180854f), 1.0f);
    } else {
        above = fmaf(a, fmaf(a, fmaf(a, fmaf(a, 0.00407761085f, 0.040372551f), 0.182461808f), 0.437250858f), 0.5f);
        below = fmaf(a, fmaf(a, fmaf(a, fmaf(a, fmaf(a, 0.0102209259f, 0.101205788f), 0.467429045f), 1.1992906f), 1.67238667f), 1.0f);
    }
    bell = exp_near<T>(square, fmaf(-0.5f * a, a, -square));
    const float tail = bell * above * __builtin_amdgcn_rcpf(below);
    return z < 0.0f ? tail : 1.0f - tail;
}
template <class T>
__device__ __forceinline__ float logistic(float z)
{
    if constexpr (T::PER == 1) z = __builtin_amdgcn_fmed3f(z, -150.0f, 150.0f);  // (past fp32's largest exp, and what rounding leaves out is finite)
    return __builtin_amdgcn_rcpf(1.0f + exp_near<T>(-z, 0.0f));
}

template <class T, int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == BGL_ACT_RELU) return z < 0.0f ? 0.0f : z;  // (NaN stays)
    if constexpr (ACT == BGL_ACT_GELU) {
        float bell;
        return z * normal_cdf<T>(z, bell);
    }
    if constexpr (ACT == BGL_ACT_SILU) return z * logistic<T>(z);
    return z;
}
template <class T, int ACT>
__device__ __forceinline__ float slope(float z)
{
    if constexpr (ACT == BGL_ACT_GELU) {
        float bell;
        const float p = normal_cdf<T>(z, bell);
        return fmaf(z * bell, 0.39894228040143268f, p);
    }
    if constexpr (ACT == BGL_ACT_SILU) {
        const float p = logistic<T>(z);
        return p * fmaf(z, 1.0f - p, 1.0f);
    }
    return 1.0f;
}
// z as it is kept for the backward call, in the layer's width.  bf16 layers keep the z of gelu and silu as a half: three bits more, so that the slope
// adds nothing to what rounding dz costs; beyond its range, where the slope is 0 or 1, the end of it.  relu's z stays bf16: only its sign counts, and
// no z > 0 may become 0.
template <class T>
__device__ __forceinline__ typename T::elem keep(int act, float z)
{
    if constexpr (T::PER == 2) {
        if (act == BGL_ACT_GELU || act == BGL_ACT_SILU) return __builtin_bit_cast(uint16_t, (_Float16)(z > 65504.0f ? 65504.0f : z < -65504.0f ? -65504.0f : z));
    }
    return T::put(z);
}
template <class T>
__device__ __forceinline__ float kept(int act, typename T::elem v)
{
    if constexpr (T::PER == 2) {
        if (act == BGL_ACT_GELU || act == BGL_ACT_SILU) return (float)__builtin_bit_cast(_Float16, v);
    }
    return T::get(v);
}
// One choice for several values: one for each kept their chains apart.
template <class T, int V>
__device__ __forceinline__ void activate_all(int act, float (&v)[V])
{
    const auto all = [&](auto which) {
#pragma unroll
        for (int u = 0; u < V; ++u) v[u] = activate<T, decltype(which)::value>(v[u]);
    };
    if (act == BGL_ACT_RELU) all(std::integral_constant<int, BGL_ACT_RELU>{});
    else if (act == BGL_ACT_GELU) all(std::integral_constant<int, BGL_ACT_GELU>{});
    else if (act == BGL_ACT_SILU) all(std::integral_constant<int, BGL_ACT_SILU>{});
}
template <class T, int V>
__device__ __forceinline__ void times_slope(int act, const float (&z)[V], float (&d)[V])
{
    const auto all = [&](auto which) {
#pragma unroll
        for (int u = 0; u < V; ++u) d[u] *= slope<T, decltype(which)::value>(z[u]);
    };
    if (act == BGL_ACT_RELU) {  // (no product: a dy that is not finite leaves nothing where z <= 0)
#pragma unroll
        for (int u = 0; u < V; ++u) d[u] = z[u] > 0.0f ? d[u] : 0.0f;
    } else if (act == BGL_ACT_GELU) {
        all(std::integral_constant<int, BGL_ACT_GELU>{});
    } else if (act == BGL_ACT_SILU) {
        all(std::integral_constant<int, BGL_ACT_SILU>{});
    }
}

// ----------------------------------------------------------------- groups
// Rows in group order: sorted position s is row index[s] (index null: s itself); group g has positions offsets[g] .. offsets[g+1]; what
// is behind the last group's belongs to none and counts as group `groups`.
struct Groups {
    const int32_t *offsets, *index;
    int32_t groups;  // 0: all rows in group 0, offsets unused
};

__device__ __forceinline__ void group_range(const Groups &q, int64_t n, int g, int64_t &lo, int64_t &hi)
{
    lo = q.offsets[g < q.groups ? g : q.groups];
    hi = g < q.groups ? q.offsets[g + 1] : n;
    lo = lo < 0 ? 0 : lo > n ? n : lo;  // (offsets are device data: no value of theirs leads outside)
    hi = hi < lo ? lo : hi > n ? n : hi;
}

// A value that is the same in all lanes, said so: loops and branches that depend on it then need no lane masks.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct Span {
    int group;      // -1: there is no such tile
    int64_t start;  // sorted position
    int count;
};

// Tile number `t` of the list that cuts each of the first `classes` groups into tiles of tile_rows.  Same in every lane of the workgroup.
__device__ __forceinline__ Span find_span(const Groups &q, int64_t n, int classes, int tile_rows, int64_t t)
{
    Span s{-1, 0, 0};
    if (q.groups == 0) {
        s.start = t * tile_rows;
        if (s.start < n) s.group = 0, s.count = (int)(n - s.start < tile_rows ? n - s.start : tile_rows);
        return s;
    }
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int g0 = 0; g0 < classes; g0 += 64) {
        const int g = g0 + lane;
        int64_t lo = 0, hi = 0;
        if (g < classes) group_range(q, n, g, lo, hi);
        const int tiles = (int)((hi - lo + tile_rows - 1) / tile_rows);
        const int upto = wave_incl_scan(tiles);
        const uint64_t past = __ballot(before + upto > t);
        if (past) {
            const int k = __ffsll((unsigned long long)past) - 1;
            const int64_t first = before + uniform(__shfl(upto - tiles, k));
            s.group = g0 + k;
            s.start = uniform(__shfl((int)lo, k)) + (t - first) * tile_rows;
            const int64_t left = uniform(__shfl((int)hi, k)) - s.start;
            s.count = (int)(left < tile_rows ? left : tile_rows);
            return s;
        }
        before += uniform(__shfl(upto, 63));
    }
    return s;
}

// The rows of the first `classes` groups in units of unit_rows (a group's last may be short): those of the groups before g, g's own, all.
__device__ __forceinline__ void count_units(const Groups &q, int64_t n, int classes, int unit_rows, int g, int64_t &before, int &own, int64_t &all)
{
    if (q.groups == 0) {
        before = 0;
        all = own = (int)((n + unit_rows - 1) / unit_rows);
        return;
    }
    const int lane = threadIdx.x & 63;
    before = all = 0;
    own = 0;
    for (int g0 = 0; g0 < classes; g0 += 64) {
        int64_t lo = 0, hi = 0;
        if (g0 + lane < classes) group_range(q, n, g0 + lane, lo, hi);
        const int units = (int)((hi - lo + unit_rows - 1) / unit_rows);
        const int upto = wave_incl_scan(units);
        if (g >= g0 && g < g0 + 64) {
            own = uniform(__shfl(units, g - g0));
            before = all + uniform(__shfl(upto, g - g0)) - own;
        }
        all += uniform(__shfl(upto, 63));
    }
}

__device__ __forceinline__ int32_t row_at(const Groups &q, int64_t n, int64_t position)
{
    const int32_t r = q.index ? q.index[position] : (int32_t)position;
    return (uint32_t)r < (uint64_t)n ? r : -1;
}

// ----------------------------------------------------------------- columns of a row
template <class T, int TT>
struct Cols {
    typename T::elem e[TT];
};
template <class T, int TT>
__device__ __forceinline__ Cols<T, TT> load_cols_upto(const typename T::elem *p, int left)
{
    Cols<T, TT> pack;
    if (left >= TT) return load_any<Cols<T, TT>>(p);
#pragma unroll
    for (int i = 0; i < TT; ++i) pack.e[i] = i < left ? p[i] : (typename T::elem)0;
    return pack;
}
template <class T, int TT>
__device__ __forceinline__ void load_cols(const typename T::elem *p, int left, float (&v)[TT])
{
    const Cols<T, TT> pack = load_cols_upto<T, TT>(p, left);
#pragma unroll
    for (int i = 0; i < TT; ++i) v[i] = T::get(pack.e[i]);
}
template <class T, int TT>
__device__ __forceinline__ void store_piece(typename T::elem *p, int left, const Cols<T, TT> &pack)
{
    if (left >= TT) {
        __builtin_memcpy(p, &pack, sizeof(pack));
    } else {
#pragma unroll
        for (int i = 0; i < TT; ++i)
            if (i < left) p[i] = pack.e[i];
    }
}
template <class T, int TT>
__device__ __forceinline__ void store_cols(typename T::elem *p, int left, const float (&v)[TT])
{
    Cols<T, TT> pack;
#pragma unroll
    for (int i = 0; i < TT; ++i) pack.e[i] = T::put(v[i]);
    store_piece<T, TT>(p, left, pack);
}

// ----------------------------------------------------------------- forward, and dx
// One kernel for both: rows (n x K) times a weight whose summed index is contiguous (forward: out_dim x in_dim, B_OC false) or is
// not (dx: the summed index is out_dim, B_OC true).
//
// A workgroup makes one tile of the result from operands staged through 32 KB of LDS, one tile of both ahead in registers; three workgroups a CU (two
// with dz), each of which fills the waits of the others, do more than a second buffer would.  Tiles of one block of rows go to one XCD, whose L2 then has the rows.
//
//   f32 100 -> 256, 428,377 rows, gelu, y and z written   414 us: 1.05 GB at 2.5 TB/s, 53 TFLOP/s; matrix units busy 44 % of the time: reading,
//                                                   multiplying (157 us) and writing follow each other in a workgroup, and three overlap in part
//   f32 dx and dz of it                             445 us: 1.49 GB at 3.3 TB/s, 49 TFLOP/s; matrix units 42 %; dz made on the way takes the registers of
//                                                   the third workgroup
//   bf16 512 -> 256, 302,709 rows, residual, z      179 us: 775 MB at 4.3 TB/s, 443 TFLOP/s
//   bf16 dx of it                                   161 us: 465 MB, 493 TFLOP/s, matrix units 23 %
//   bf16 512 -> 512, 302,709 rows, residual         280 us: 930 MB, 567 TFLOP/s: a tile's loads, its 96 KB through LDS (a fragment is read for each of
//                                                   its users), its products and its epilogue take about equally long
//   one row of 512 -> 512 bf16                      4.9 us, f32 100 -> 128 of 5,485 rows 7.2: one tile's loads, products and stores, one after the other
template <class T>
struct RowsArgs {
    const typename T::elem *x, *w, *bias, *residual;
    typename T::elem *y, *saved;
    int64_t n, x_stride, y_stride, residual_stride, saved_stride, row_tiles;
    int K, N, col_tiles;  // summed and kept width
    int residual_mode, activation;
    Groups q;
    // dx from dy: z as kept by the forward call, and where dz goes (null: nowhere)
    const typename T::elem *z;
    typename T::elem *dz;
    int64_t z_stride, dz_stride;
    int z_activation;
};

// The tile's sums, in LDS, to their rows: a thread has VEC neighbouring columns of every so many rows.  WHOLE: N is a multiple of VEC.
template <class T, class C, class R, bool WHOLE, int TEAMS>
__device__ __forceinline__ void finish_rows(const RowsArgs<T> &a, const float *sums, const int32_t *row_of, int part, int group, int n0)
{
    constexpr int W = R::W, V = T::VEC, PER_ROW = W / V, ROWS = kThreads * TEAMS / PER_ROW, PASSES = R::ROWS > ROWS ? R::ROWS / ROWS : 1;
    constexpr int BATCH = PASSES < 8 ? PASSES : 8;
    using Piece = Cols<T, V>;
    const int c = (int)(threadIdx.x % PER_ROW) * V, r0 = threadIdx.x / PER_ROW, left = a.N - n0 - c;
    if (left <= 0 || c >= C::BB || r0 >= R::ROWS) return;
    float bias[V] = {};
    if (a.bias && group >= 0) load_cols<T, V>(a.bias + (int64_t)group * a.N + n0 + c, WHOLE ? V : left, bias);
#pragma unroll
    for (int p0 = 0; p0 < PASSES; p0 += BATCH) {
        int32_t row[BATCH];
        Piece res[BATCH];
#pragma unroll
        for (int p = 0; p < BATCH; ++p) row[p] = row_of[R::row(part, r0 + (p0 + p) * ROWS)];
        if (a.residual_mode) {  // all asked for before the first is used: one after the other they took longer than the product
#pragma unroll
            for (int p = 0; p < BATCH; ++p) {
                const typename T::elem *from = a.residual + (row[p] < 0 ? 0 : row[p]) * a.residual_stride + n0 + c;
                res[p] = WHOLE ? load_any<Piece>(from) : load_cols_upto<T, V>(from, left);
            }
        }
#pragma unroll
        for (int p = 0; p < BATCH; ++p) {
            float v[V];
#pragma unroll
            for (int u = 0; u < V; u += 4) {
                f32x4 four = {};
#pragma unroll
                for (int t = 0; t < TEAMS; ++t) four += *reinterpret_cast<const f32x4 *>(sums + t * R::SIZE + result_place<W>(r0 + (p0 + p) * ROWS, c + u));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u + e] = four[e] + bias[u + e];
            }
            if (a.residual_mode == BGL_RESIDUAL_BEFORE) {
#pragma unroll
                for (int u = 0; u < V; ++u) v[u] += T::get(res[p].e[u]);
            }
            if (row[p] < 0) continue;
            if (a.saved) {
                Piece piece;
#pragma unroll
                for (int u = 0; u < V; ++u) piece.e[u] = keep<T>(a.activation, v[u]);
                store_piece<T, V>(a.saved + row[p] * a.saved_stride + n0 + c, WHOLE ? V : left, piece);
            }
            activate_all<T>(a.activation, v);
            if (a.residual_mode == BGL_RESIDUAL_AFTER) {
#pragma unroll
                for (int u = 0; u < V; ++u) v[u] += T::get(res[p].e[u]);
            }
            store_cols<T, V>(a.y + row[p] * a.y_stride + n0 + c, WHOLE ? V : left, v);
        }
    }
}

// The operand dz = dy act'(z) of dx, made on its way to LDS, and stored to `dz` unless that is null.
template <class T, int BO>
struct DzOperand : KcOperand<T, BO> {
    using Base = KcOperand<T, BO>;
    const typename T::elem *saved;
    typename T::elem *dz;
    int64_t saved_stride, dz_stride;
    int32_t row[Base::PASSES];
    uint4 z[Base::PASSES];
    int act, tile, K;

    template <class Row>
    __device__ __forceinline__ void rows(Row row_of)
    {
#pragma unroll
        for (int p = 0; p < Base::PASSES; ++p) row[p] = row_of((team_thread() >> 3) + 32 * p);
    }
    __device__ __forceinline__ void load(int t, int width)
    {
        tile = t;
        Base::load(t, width);
        const int first = t * Base::BK + (team_thread() & 7) * T::VEC, left = width - first;
#pragma unroll
        for (int p = 0; p < Base::PASSES; ++p) {
            const typename T::elem *from = saved + (row[p] < 0 ? 0 : row[p]) * saved_stride + first;
            z[p] = (t + 1) * Base::BK <= width ? load_any<uint4>(from) : load_end<T>(from, left, width);
        }
    }
    __device__ __forceinline__ void store(uint32_t *lds)
    {
        const int first = tile * Base::BK + (team_thread() & 7) * T::VEC, left = K - first;
#pragma unroll
        for (int p = 0; p < Base::PASSES; ++p) {
            auto d = __builtin_bit_cast(Cols<T, T::VEC>, Base::reg[p]);
            const auto s = __builtin_bit_cast(Cols<T, T::VEC>, z[p]);
            float dv[T::VEC], zv[T::VEC];
#pragma unroll
            for (int e = 0; e < T::VEC; ++e) dv[e] = T::get(d.e[e]), zv[e] = kept<T>(act, s.e[e]);
            times_slope<T>(act, zv, dv);
#pragma unroll
            for (int e = 0; e < T::VEC; ++e) d.e[e] = T::put(dv[e]);
            Base::reg[p] = __builtin_bit_cast(uint4, d);
            if (dz && row[p] >= 0) store_piece<T, T::VEC>(dz + row[p] * dz_stride + first, left, d);
        }
        Base::store(lds);
    }
};

// DZ: x is dy, and dz is made from it and from z on the way (dx of few tiles of columns, each of which makes it again).  TEAMS of 256 threads take the summed
// index's tiles in turn; their sums meet when the rows are finished.
template <class T, bool B_OC, class C, bool NARROW, int TEAMS, bool DZ>
__global__ __launch_bounds__(kThreads * TEAMS, 2) void k_linear_rows(RowsArgs<T> a)
{
    using A = std::conditional_t<DZ, DzOperand<T, C::BA>, KcOperand<T, C::BA>>;
    using B = std::conditional_t<B_OC, OcOperand<T, C::BB, false, NARROW>, KcOperand<T, C::BB>>;
    constexpr int OPERANDS = A::LDS + B::LDS;
    using R = Result<C, OPERANDS>;
    constexpr int LDS = TEAMS * (OPERANDS > R::SIZE ? OPERANDS : R::SIZE);
    __shared__ __attribute__((aligned(16))) uint32_t lds[LDS];
    __shared__ int32_t row_of[C::BA];
    int64_t rt;
    int ct;
    if (!tile_of(blockIdx.x, a.row_tiles, a.col_tiles, rt, ct)) return;
    const Span s = find_span(a.q, a.n, a.q.groups + (a.q.groups > 0), C::BA, rt);
    if (s.group < 0) return;
    const bool none = a.q.groups > 0 && s.group == a.q.groups;
    const int n0 = ct * C::BB, K = none && !DZ ? 0 : a.K;  // (rows of no group have a dz too)
    const typename T::elem *w = a.w + (none ? 0 : (int64_t)s.group * a.N * a.K);

    if ((int)threadIdx.x < C::BA) row_of[threadIdx.x] = (int)threadIdx.x < s.count ? row_at(a.q, a.n, s.start + threadIdx.x) : -1;
    __syncthreads();
    f32x4 acc[C::FA][C::FB] = {};
    if (K > 0) {
        A rows;
        B weight;
        rows.init([&](int i) {
            const int32_t r = row_of[i];
            return a.x + (r < 0 ? 0 : r) * a.x_stride;
        });
        if constexpr (DZ) {
            rows.rows([&](int i) { return row_of[i]; });
            rows.saved = a.z, rows.saved_stride = a.z_stride, rows.dz = ct == 0 ? a.dz : nullptr, rows.dz_stride = a.dz_stride;
            rows.act = a.z_activation, rows.K = K;
        }
        if constexpr (B_OC) {
            weight.init(w, a.N, K, n0, a.N);
            weight.range(nullptr, 0, K);
        } else {
            weight.init([&](int i) { return w + (int64_t)(n0 + i < a.N ? n0 + i : a.N - 1) * a.K; });
        }
        const int team = TEAMS > 1 ? uniform(threadIdx.x / kThreads) : 0, tiles = (K + A::BK - 1) / A::BK;
        uint32_t *mine = lds + team * OPERANDS;
        pipeline(
            (tiles + TEAMS - 1) / TEAMS,
            [&](int i) {
                if (TEAMS > 1 && i * TEAMS + team >= tiles) return;
                rows.load(i * TEAMS + team, K);
                if constexpr (B_OC) weight.load(i * TEAMS + team);
                else weight.load(i * TEAMS + team, K);
            },
            [&](int i) {
                if (TEAMS > 1 && i * TEAMS + team >= tiles) return;
                rows.store(mine);
                if constexpr (B_OC) weight.settle();
                weight.store(mine + A::LDS);
            },
            [&](int i) {
                if (TEAMS > 1 && i * TEAMS + team >= tiles) return;
                const int steps = (K - (i * TEAMS + team) * A::BK + 16 * T::PER - 1) / (16 * T::PER);
                multiply<T, A, B, C>(mine, mine + A::LDS, steps, acc, [](const auto &, const auto &) {});
            });
        if (DZ && none) {
#pragma unroll
            for (auto &line : acc)
#pragma unroll
                for (auto &f : line) f = f32x4{};
        }
    }
    float *sums = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int part = 0; part < R::PARTS; ++part) {
        if (part) __syncthreads();
        R::put(sums + (TEAMS > 1 ? threadIdx.x / kThreads : 0) * R::SIZE, part, acc);
        __syncthreads();
        if (a.N % T::VEC == 0) finish_rows<T, C, R, true, TEAMS>(a, sums, row_of, part, none ? -1 : s.group, n0);
        else finish_rows<T, C, R, false, TEAMS>(a, sums, row_of, part, none ? -1 : s.group, n0);
    }
}

// ----------------------------------------------------------------- dz
constexpr int kUnit = 64;

// No share is empty (rows of no group make units fewer than the host can know), so every slot between a group's first and last is written.
__device__ __forceinline__ int64_t shares_of(int64_t units, int planned) { return units < planned ? units : planned; }

// dz of all rows, in group order, and the sums of its columns before they are rounded (bf16: sums of rounded values would be off by as much again as
// the result's own rounding).  The rows, in units of kUnit, are dealt evenly to `shares` workgroups; share w leaves its sums for group g in slot
// w + g of `part`.  A thread has VEC neighbouring columns, kDzColumns of a workgroup's rows at a time at most (blockIdx.y: which).  Bound by its bytes:
// bf16 256 columns, 302,709 rows, relu (no sums) 90 us, 465 MB at 5.2 TB/s; gelu with the sums of 24 groups 122 us, 3.8 TB/s: 69 % of the time has vector
// instructions in flight (the slope is some 30 of them a value) and rows are reached through the group order.
constexpr int kDzColumns = 2048;

template <class T>
struct DzArgs {
    const typename T::elem *dy, *saved;
    typename T::elem *dz;
    float *part;  // null: no sums
    int64_t n, dy_stride, saved_stride, dz_stride;
    int N, act, shares, classes;
    Groups q;
};

template <class T>
__global__ __launch_bounds__(kThreads) void k_linear_dz(DzArgs<T> a)
{
    constexpr int V = T::VEC;
    constexpr int COLUMNS = kThreads * V < kDzColumns ? kThreads * V : kDzColumns;
    __shared__ float sums[kThreads * V];
    const int first = blockIdx.y * COLUMNS, width = a.N - first < COLUMNS ? a.N - first : COLUMNS, per_row = (width + V - 1) / V, rows = kThreads / per_row;
    const int lane_row = threadIdx.x / per_row, c = first + (int)(threadIdx.x % per_row) * V, left = a.N - c;
    const bool idle = lane_row >= rows;
    int64_t before, units;
    int own;
    count_units(a.q, a.n, a.classes, kUnit, 0, before, own, units);
    const int64_t shares = shares_of(units, a.shares), share = blockIdx.x;
    if (share >= shares) return;
    const int64_t last = (share + 1) * units / shares;
    for (int64_t unit = share * units / shares; unit < last;) {
        const Span s = find_span(a.q, a.n, a.classes, kUnit, unit);
        int64_t lo = 0, hi = a.n;
        if (a.q.groups > 0) group_range(a.q, a.n, s.group, lo, hi);
        hi = uniform((int)hi);
        const int64_t room = (last - unit) * kUnit, end = hi - s.start < room ? hi : s.start + room;
        unit += (end - s.start + kUnit - 1) / kUnit;
        float sum[V] = {};
        const auto all = [&](auto whole) {  // whole: N is a multiple of VEC
            constexpr int BATCH = 4;        // rows whose loads are on their way together
            using Piece = Cols<T, V>;
            for (int64_t at = s.start + lane_row; at < end; at += BATCH * rows) {
                int32_t r[BATCH];
                Piece d[BATCH], z[BATCH];
#pragma unroll
                for (int p = 0; p < BATCH; ++p) {
                    const int64_t here = at + p * rows;
                    r[p] = row_at(a.q, a.n, here < end ? here : end - 1);
                    if (here >= end) r[p] = -1;
                }
#pragma unroll
                for (int p = 0; p < BATCH; ++p) {
                    const int64_t from = r[p] < 0 ? 0 : r[p];
                    d[p] = decltype(whole)::value ? load_any<Piece>(a.dy + from * a.dy_stride + c) : load_cols_upto<T, V>(a.dy + from * a.dy_stride + c, left);
                    if (a.act) z[p] = decltype(whole)::value ? load_any<Piece>(a.saved + from * a.saved_stride + c) : load_cols_upto<T, V>(a.saved + from * a.saved_stride + c, left);
                }
#pragma unroll
                for (int p = 0; p < BATCH; ++p) {
                    float dv[V], zv[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) dv[e] = T::get(d[p].e[e]), zv[e] = a.act ? kept<T>(a.act, z[p].e[e]) : 0.0f;
                    times_slope<T>(a.act, zv, dv);
                    if (r[p] < 0) continue;
#pragma unroll
                    for (int e = 0; e < V; ++e) sum[e] += dv[e];
                    store_cols<T, V>(a.dz + r[p] * a.dz_stride + c, decltype(whole)::value ? V : left, dv);
                }
            }
        };
        if (!idle) {
            if (a.N % V == 0) all(std::true_type{});
            else all(std::false_type{});
        }
        if (a.part && s.group < (a.q.groups ? a.q.groups : 1)) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) sums[threadIdx.x * V + e] = sum[e];
            __syncthreads();
            for (int i = threadIdx.x; i < width; i += kThreads) {
                float v = 0.0f;
                for (int r = 0; r < rows; ++r) v += sums[r * per_row * V + i];
                a.part[(share + s.group) * a.N + first + i] = v;
            }
        }
    }
}

// ----------------------------------------------------------------- dW, db
// The rows of all groups are cut into units of 64 and dealt evenly to `shares` workgroups for each tile of dW: a share may end one group
// and begin the next, so that no workgroup has more than its part however the sizes fall.  Share w leaves its sums for group g in slot w + g
// of `part` (both grow along the rows, so no two meet in a slot): A_dim * B_dim of the matrix, then out_dim of db.
// Side A is the wider of dz and x, side B the narrower; the matrix is laid out [A][B].
//
// f32 100 x 256, 428,377 rows 251 us: 610 MB at 2.4 TB/s, 87 TFLOP/s of 154 that a large product reaches, matrix units busy 75 % of the time (7 of 8 blocks
// of columns hold something).  bf16 512 x 256, 302,709 rows 141 us, 24 groups 143: 465 MB at 3.3 TB/s, 562 TFLOP/s: the transposing LDS reads bring
// half as much a cycle as plain ones.
template <class T>
struct WeightArgs {
    const typename T::elem *a, *b;
    float *part;
    int64_t n, a_stride, b_stride;
    int a_dim, b_dim, N, shares, a_tiles, b_tiles;
    int bias;  // which side is dz, if db is asked for: 1 A, 2 B, else 0
    Groups q;
};

template <class T, bool LIST, class C, bool NARROW>
__global__ __launch_bounds__(kThreads, 2) void k_linear_dw(WeightArgs<T> a)
{
    using A = OcOperand<T, C::BA, LIST, NARROW>;
    using B = OcOperand<T, C::BB, LIST, NARROW>;
    using R = Result<C, A::LDS + B::LDS>;
    constexpr int LDS = A::LDS + B::LDS > R::SIZE ? A::LDS + B::LDS : R::SIZE, SUMS = C::FA > C::FB ? C::FA : C::FB;
    __shared__ __attribute__((aligned(16))) uint32_t lds[LDS];
    int64_t share;
    int tile;
    if (!tile_of(blockIdx.x, a.shares, a.a_tiles * a.b_tiles, share, tile)) return;
    const int a0 = tile / a.b_tiles * C::BA, b0 = tile % a.b_tiles * C::BB;
    int64_t before, units;
    int own;
    count_units(a.q, a.n, a.q.groups, kUnit, 0, before, own, units);
    const int64_t shares = shares_of(units, a.shares);
    if (share >= shares) return;
    const int64_t last = (share + 1) * units / shares;
    A left;
    B right;
    left.init(a.a, a.a_stride, a.n, a0, a.a_dim);
    right.init(a.b, a.b_stride, a.n, b0, a.b_dim);
    // dz's columns are summed from the fragments, by the wavefronts whose tiles are the first of their rows or columns
    const bool bias_a = a.bias == 1 && b0 == 0 && uniform(C::b_off()) == 0, bias_b = a.bias == 2 && a0 == 0 && uniform(C::a_off()) == 0;
    const int64_t len = (int64_t)a.a_dim * a.b_dim + a.N;
    for (int64_t unit = share * units / shares; unit < last;) {
        const Span s = find_span(a.q, a.n, a.q.groups, kUnit, unit);
        int64_t lo = 0, hi = a.n;
        if (a.q.groups > 0) group_range(a.q, a.n, s.group, lo, hi);
        hi = uniform((int)hi);
        const int64_t room = (last - unit) * kUnit;
        const int count = (int)(hi - s.start < room ? hi - s.start : room);
        unit += (count + kUnit - 1) / kUnit;
        left.range(a.q.index, s.start, count);
        right.range(a.q.index, s.start, count);
        f32x4 acc[C::FA][C::FB] = {};
        float sum[SUMS] = {};
        pipeline(
            (count + A::BK - 1) / A::BK,
            [&](int i) {
                left.load(i);
                right.load(i);
            },
            [&](int) {
                left.settle();
                right.settle();
                left.store(lds);
                right.store(lds + A::LDS);
            },
            [&](int i) {
                const int steps = (count - i * A::BK + 16 * T::PER - 1) / (16 * T::PER);
                multiply<T, A, B, C>(lds, lds + A::LDS, steps, acc, [&](const auto &l, const auto &r) {
                    if (bias_a) {
#pragma unroll
                        for (int f = 0; f < C::FA; ++f) sum[f] = T::sum(l[f], sum[f]);
                    } else if (bias_b) {
#pragma unroll
                        for (int f = 0; f < C::FB; ++f) sum[f] = T::sum(r[f], sum[f]);
                    }
                });
            });
        float *part = a.part + (share + s.group) * len;
        float *sums = reinterpret_cast<float *>(lds);
#pragma unroll
        for (int half = 0; half < R::PARTS; ++half) {
            if (half) __syncthreads();
            R::put(sums, half, acc);
            __syncthreads();
            constexpr int PER_ROW = R::W / 4, ROWS = kThreads / PER_ROW;
            const int c = (int)(threadIdx.x % PER_ROW) * 4, columns = a.b_dim - b0 - c;
#pragma unroll 1  // (unrolled, its addresses were kept in registers through the products: 256 of them, and memory)
            for (int i = threadIdx.x / PER_ROW; i < R::ROWS; i += ROWS) {
                const int r = a0 + R::row(half, i);
                if (r >= a.a_dim || columns <= 0 || c >= C::BB) continue;
                const f32x4 four = *reinterpret_cast<const f32x4 *>(sums + result_place<R::W>(i, c));
                float *to = part + (int64_t)r * a.b_dim + b0 + c;
                if (columns >= 4) __builtin_memcpy(to, &four, 16);
                else
                    for (int e = 0; e < columns; ++e) to[e] = four[e];
            }
        }
        if (bias_a || bias_b) {  // a lane has the sum over its lane group's part of the rows
            const int lane = threadIdx.x & 63;
            const int o0 = (bias_a ? a0 + C::a_off() : b0 + C::b_off()) + lane, O = bias_a ? a.a_dim : a.b_dim, frags = bias_a ? C::FA : C::FB;
            float *to = part + (int64_t)a.a_dim * a.b_dim;
#pragma unroll
            for (int f = 0; f < SUMS; ++f) {
                sum[f] += __shfl_xor(sum[f], 16);
                sum[f] += __shfl_xor(sum[f], 32);
                if (f < frags && lane < 16 && o0 + 16 * f < O) to[o0 + 16 * f] = sum[f];
            }
        }
        __syncthreads();  // (the next group's first tile goes where these were read)
    }
}

// dW and db of group blockIdx.y: what the shares left of it, added in a fixed order (atomics would add in another one each time).  Bound by its loads: 512
// shares of f32 100 x 256 (53 MB, much of it still in L2) 8.2 us; bf16 512 x 256 for 24 groups, 64 shares and a group's sums of dz 29 us.
template <class T>
struct ReduceArgs {
    const float *part;
    typename T::elem *dw, *db;
    const float *dz_part;  // db's parts, if the dz kernel made them: [slot][N]
    int64_t n;
    int N, K, shares, dz_shares, dz_classes, matrix_blocks;
    bool swapped;  // the parts' matrix is [K][N]
    Groups q;
};

// SPLIT: the four wavefronts take the shares of 256 values in turn; else (many groups, a few shares each) 256 values each.  With the gradients of a
// layer of 100 -> 256 f32 in one group 1,025 to 1,035 us with SPLIT, 1,040 without; of 512 -> 256 bf16 in 24 groups 691 to 693 without, 701 with.
template <class T, bool SPLIT>
__global__ __launch_bounds__(kThreads) void k_linear_reduce(ReduceArgs<T> a)
{
    __shared__ float4 sums[kThreads];
    const int g = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x / kWave;
    int64_t before, units;
    int own;
    if ((int)blockIdx.x >= a.matrix_blocks) {  // db
        count_units(a.q, a.n, a.dz_classes, kUnit, g, before, own, units);
        constexpr int STRIPES = kThreads / 16;  // 16 columns to a workgroup: a large group's hundreds of shares are read 16 at a time
        const int stripe = threadIdx.x / 16, c = ((int)blockIdx.x - a.matrix_blocks) * 16 + (threadIdx.x & 15);
        float v = 0.0f;
        if (c < a.N && own > 0) {
            const int64_t shares = shares_of(units, a.dz_shares), first = ((before + 1) * shares - 1) / units, last = ((before + own) * shares - 1) / units;
#pragma unroll 8
            for (int64_t w = first + stripe; w <= last; w += STRIPES) v += a.dz_part[(w + g) * a.N + c];
        }
        float *column = reinterpret_cast<float *>(sums);
        column[threadIdx.x] = v;
        __syncthreads();
        if (stripe || c >= a.N) return;
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < STRIPES; ++i) v += column[i * 16 + threadIdx.x];
        a.db[(int64_t)g * a.N + c] = T::put(v);
        return;
    }
    count_units(a.q, a.n, a.q.groups, kUnit, g, before, own, units);
    const int64_t NK = (int64_t)a.N * a.K, len = NK + a.N, e = ((SPLIT ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave) * 64 + lane) * 4;
    const int left = len - e < 4 ? (int)(len - e) : 4;
    float v[4] = {};
    if (left > 0 && own > 0) {
        const int64_t shares = shares_of(units, a.shares), first = ((before + 1) * shares - 1) / units, last = ((before + own) * shares - 1) / units;
        constexpr int STEP = SPLIT ? kThreads / kWave : 1;
        const auto add = [&](auto whole) {
#pragma unroll 8
            for (int64_t w = first + (SPLIT ? wave : 0); w <= last; w += STEP) {
                const float *from = a.part + (w + g) * len + e;
                const auto p = decltype(whole)::value ? load_any<Cols<F32, 4>>(from) : load_cols_upto<F32, 4>(from, left);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] += p.e[u];
            }
        };
        if (left == 4) add(std::true_type{});
        else add(std::false_type{});
    }
    if constexpr (SPLIT) {
        sums[threadIdx.x] = float4{v[0], v[1], v[2], v[3]};
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < kThreads / kWave; ++w) {
            const float4 o = sums[w * 64 + lane];
            v[0] += o.x, v[1] += o.y, v[2] += o.z, v[3] += o.w;
        }
    }
    for (int u = 0; u < left; ++u) {
        const int64_t at = e + u;
        if (at >= NK) {
            if (a.db && !a.dz_part) a.db[(int64_t)g * a.N + at - NK] = T::put(v[u]);
        } else {
            a.dw[g * NK + (a.swapped ? at % a.N * a.K + at / a.N : at)] = T::put(v[u]);
        }
    }
}

// ----------------------------------------------------------------- grouping
// A stable counting sort by group in two passes over the group numbers: rows per tile and group, then each row's place.  Both are bound by their
// dependent steps (group number, LDS counter, store), not by bytes: 428,377 rows of 8 groups 8.4 and 7.7 us, 302,709 of 24 groups 7.2 and 9.3
// (2.5 MB).  One tile's rows (2,048) need one launch: 37 rows 2.6 us.
struct GroupArgs {
    const int32_t *group_of, *ids;
    int64_t num_nodes, n;
    int32_t groups, tile_rows;  // tile_rows: a multiple of 64 rows for each of the workgroup's wavefronts
    int32_t *rows, *offsets, *counts;  // counts: [tiles][groups + 1]
    uint16_t *group;                   // of each row; groups for none
};

__device__ __forceinline__ int group_of_row(const GroupArgs &a, int64_t i)
{
    int64_t v = i;
    if (a.ids) {
        v = a.ids[i];
        if (v < 0 || v >= a.num_nodes) return a.groups;
    }
    const int32_t g = a.group_of[v];
    return (uint32_t)g < (uint32_t)a.groups ? g : a.groups;
}

// Rows per group of each tile, and each row's group for the second pass.
__global__ __launch_bounds__(kGroupThreads) void k_group_count(GroupArgs a)
{
    extern __shared__ int32_t hist[];
    const int classes = a.groups + 1;
    for (int g = threadIdx.x; g < classes; g += kGroupThreads) hist[g] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.tile_rows;
    const int64_t last = first + a.tile_rows < a.n ? first + a.tile_rows : a.n;
    for (int64_t i = first + threadIdx.x; i < last; i += kGroupThreads) {
        const int g = group_of_row(a, i);
        a.group[i] = (uint16_t)g;
        atomicAdd(&hist[g], 1);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < classes; g += kGroupThreads) a.counts[(int64_t)blockIdx.x * classes + g] = hist[g];
}

// Rows of each tile to their places: behind all rows of smaller groups, the tiles before, the wavefronts before (a wavefront has a
// contiguous piece of the tile) and the rows before in the wavefront, so that a group's rows keep their order.
// SINGLE: one workgroup has all rows and no first pass ran.
template <bool SINGLE>
__global__ __launch_bounds__(kGroupThreads) void k_group_place(GroupArgs a)
{
    constexpr int WAVES = kGroupThreads / kWave;
    extern __shared__ int32_t sh[];
    __shared__ int32_t scan[WAVES];
    const int classes = a.groups + 1, lane = threadIdx.x & 63, wave = threadIdx.x / kWave;
    int32_t *next = sh + wave * classes;  // [WAVES][classes]: the wavefront's next place in each group
    int32_t *base = sh + WAVES * classes;  // [classes]
    for (int g = lane; g < classes; g += 64) next[g] = 0;
    __syncthreads();
    const int piece = a.tile_rows / WAVES;
    const int64_t first = (int64_t)blockIdx.x * a.tile_rows + (int64_t)wave * piece;
    const int64_t last = first + piece < a.n ? first + piece : a.n;
    for (int64_t i = first + lane; i < last; i += 64) {
        int g;
        if (SINGLE) {
            g = group_of_row(a, i);
            a.group[i] = (uint16_t)g;
        } else {
            g = a.group[i];
        }
        atomicAdd(&next[g], 1);
    }
    __syncthreads();
    // the groups' totals over all tiles, and what the tiles before this one have of each
    int32_t *total = base + classes;  // [classes]
    if (!SINGLE) {
        for (int g = threadIdx.x; g < classes; g += kGroupThreads) total[g] = base[g] = 0;
        __syncthreads();
        const int all = (int)gridDim.x * classes, mine = (int)blockIdx.x * classes;
        for (int i = threadIdx.x; i < all; i += kGroupThreads) {  // (whole numbers: any order gives the same sum)
            const int g = i % classes, c = a.counts[i];
            if (c) atomicAdd(&total[g], c);
            if (c && i < mine) atomicAdd(&base[g], c);
        }
        __syncthreads();
    }
    int carry = 0;
    for (int g0 = 0; g0 < classes; g0 += kGroupThreads) {
        const int g = g0 + threadIdx.x;
        int count = 0;
        if (g < classes) {
            if (SINGLE)
                for (int w = 0; w < WAVES; ++w) count += sh[w * classes + g];
            else
                count = total[g];
        }
        int all;
        const int before = block_excl_scan<kGroupThreads>(count, scan, all);
        if (g < classes) {
            base[g] = carry + before + (SINGLE ? 0 : base[g]);
            if (blockIdx.x == 0) a.offsets[g] = carry + before;  // offsets[groups]: the end of the last group
        }
        carry += all;
    }
    __syncthreads();
    for (int g = threadIdx.x; g < classes; g += kGroupThreads) {
        int at = base[g];
        for (int w = 0; w < WAVES; ++w) {
            const int c = sh[w * classes + g];
            sh[w * classes + g] = at;
            at += c;
        }
    }
    __syncthreads();
    for (int64_t i0 = first; i0 < last; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool live = i < last;
        const int g = live ? a.group[i] : classes;
        uint64_t same = __ballot(live);
        for (int bit = 1; bit <= a.groups; bit <<= 1) {
            const uint64_t set = __ballot(g & bit);
            same &= g & bit ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        int at = 0;
        if (live) at = next[g];
        __builtin_amdgcn_wave_barrier();
        if (live && rank == 0) next[g] = at + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (live) a.rows[at + rank] = (int32_t)i;
    }
}

// ----------------------------------------------------------------- host side
int check_layer(const bgl_linear_t *l, int64_t n)
{
    if (!l) BGL_FAIL(BGL_EINVAL, "layer is null");
    if (l->dtype != BGL_F32 && l->dtype != BGL_BF16) BGL_FAIL(BGL_EINVAL, "unknown dtype %d", l->dtype);
    if (l->activation < BGL_ACT_NONE || l->activation > BGL_ACT_SILU) BGL_FAIL(BGL_EINVAL, "unknown activation %d", l->activation);
    if (l->residual < BGL_RESIDUAL_NONE || l->residual > BGL_RESIDUAL_AFTER) BGL_FAIL(BGL_EINVAL, "unknown residual %d", l->residual);
    if (l->in_dim < 1 || l->out_dim < 1) BGL_FAIL(BGL_EINVAL, "in_dim and out_dim must be positive (got %d, %d)", l->in_dim, l->out_dim);
    if (l->in_dim > BGL_MAX_DIM || l->out_dim > BGL_MAX_DIM)
        BGL_FAIL(BGL_EUNSUPPORTED, "in_dim and out_dim must be at most %d (got %d, %d)", BGL_MAX_DIM, l->in_dim, l->out_dim);
    if (l->num_groups < 0) BGL_FAIL(BGL_EINVAL, "num_groups is negative");
    if (l->num_groups > kMaxGroups) BGL_FAIL(BGL_EUNSUPPORTED, "num_groups must be at most %d (got %d)", kMaxGroups, l->num_groups);
    if (n < 0 || n > INT32_MAX) BGL_FAIL(BGL_EINVAL, "n must be in [0, 2^31) (got %lld)", (long long)n);
    return BGL_OK;
}

int check_groups(const bgl_linear_t *l, const int32_t *rows, const int32_t *offsets)
{
    if (l->num_groups == 0 && (rows || offsets)) BGL_FAIL(BGL_EINVAL, "rows and offsets belong to a layer with groups");
    if (l->num_groups > 0 && !offsets) BGL_FAIL(BGL_EINVAL, "offsets is null");
    if (!aligned(rows, 4) || !aligned(offsets, 4)) BGL_FAIL(BGL_EINVAL, "rows and offsets must be 4-byte aligned");
    return BGL_OK;
}

int elem_bytes(const bgl_linear_t *l) { return l->dtype == BGL_F32 ? 4 : 2; }

// Cuts of a product into workgroup tiles.  Wide results take 128 x 128; one that fits into fewer than 8 fragments of 16 columns takes as many as
// it has (100 columns: 7), the four wavefronts one above the other.  us so and with 128 columns (large tiles) or 64 (small ones), 100,000 rows of 512, then
// dW over 100,000 rows:
//   columns                 16           32           48           64           80           96           112
//   forward f32         41 and 146   48 and 147   66 and 146   83 and 146  104 and 147  117 and 147  136 and 148
//   forward bf16        21 and 30    21 and 30    24 and 29    24 and 29    26 and 30    28 and 30    29 and 30
//   dW f32              40 and 123   48 and 122   62 and 122   74 and 123   89 and 124  102 and 125  117 and 126
//   dW bf16             25 and 31    26 and 31    28 and 32    29 and 31    32 and 33    33 and 33    34 and 34.5
//   5,485 rows, forward f32  7.6 and 14  9.3 and 14  12 and 14  (bf16: 6.0 either way, the call's host time)
//   5,485 rows, dW f32       12 and 22   15 and 23   18 and 24; bf16 11 and 14, 12 and 15, 14 and 16
// dx as forward.  f32 100 -> 256 with its gradients, 428,377 rows 1,030 and 1,060; f32 100 -> 64, 5,485 rows of 4 types, 42 and 46.
// Wavefronts with 128 x 64 or 96 x 64 sums each, instead of 64 x 64, take the registers of the third workgroup of a CU (bf16 512 -> 512, 302,709 rows: 316 to 326 us instead of 297), and 64 x 128 tiles read more (354 instead of 325).
using Large = Cut<2, 2, 4, 4>;
using Small = Cut<2, 2, 2, 2>;
template <int F>
using Narrow = Cut<4, 1, 2, F>;
template <int F>
using SmallNarrow = Cut<4, 1, 1, F>;

// call(cut, narrow): narrow where a row may be shorter than `vec` values.
template <class Do>
void with_cut(bool large, int cols, int vec, Do call)
{
    const int f = (cols + 15) / 16;
    const std::true_type yes{};
    const std::false_type no{};
    if (large) {
        switch (f) {
        case 1: return cols < vec ? call(Narrow<1>{}, yes) : call(Narrow<1>{}, no);
        case 2: return call(Narrow<2>{}, no);
        case 3: return call(Narrow<3>{}, no);
        case 4: return call(Narrow<4>{}, no);
        case 5: return call(Narrow<5>{}, no);
        case 6: return call(Narrow<6>{}, no);
        case 7: return call(Narrow<7>{}, no);
        default: return call(Large{}, no);
        }
    }
    switch (f) {
    case 1: return cols < vec ? call(SmallNarrow<1>{}, yes) : call(SmallNarrow<1>{}, no);
    case 2: return call(SmallNarrow<2>{}, no);
    case 3: return call(SmallNarrow<3>{}, no);
    default: return call(Small{}, no);
    }
}

// How the backward pass cuts a layer's rows: some 512 workgroups (two on each CU), each with one tile of dW and an equal share of the rows.  More leave
// more sums to add up, fewer leave loads unhidden; with 256, 512 and 1,024, us of a training call: f32 100 -> 256, 428,377 rows 1,054, 1,030, 1,051;
// bf16 512 -> 256, 302,709 rows 629, 583, 619; the same in 24 groups 749, 692, 714.
struct WeightPlan {
    bool swapped, large;
    int a_dim, b_dim, a_tiles, b_tiles, shares;
    int64_t slots;
    bool sums_with_dz;  // db comes from the dz kernel
    int dz_shares;
    size_t dz_bytes, dz_stride, part_bytes, dz_part_bytes, bytes;
};

WeightPlan plan_weight(const bgl_linear_t *l, int64_t n)
{
    WeightPlan p;
    p.swapped = l->in_dim > l->out_dim;
    p.a_dim = p.swapped ? l->in_dim : l->out_dim;
    p.b_dim = p.swapped ? l->out_dim : l->in_dim;
    p.large = p.a_dim > 64;
    with_cut(p.large, p.b_dim, 0, [&](auto cut, auto) {
        p.a_tiles = (int)ceil_div(p.a_dim, decltype(cut)::BA);
        p.b_tiles = (int)ceil_div(p.b_dim, decltype(cut)::BB);
    });
    const int64_t most = ceil_div(n > 0 ? n : 1, kUnit), want = 512 / ((int64_t)p.a_tiles * p.b_tiles);
    p.shares = (int)(want < 1 ? 1 : want < most ? want : most);
    p.slots = p.shares + (l->num_groups > 1 ? l->num_groups - 1 : 0);
    const int per = 16 / elem_bytes(l);
    p.dz_stride = round_up(l->out_dim, per);
    p.dz_bytes = l->activation == BGL_ACT_NONE ? 0 : round_up((size_t)n * p.dz_stride * elem_bytes(l), 256);
    p.part_bytes = round_up((size_t)p.slots * ((size_t)l->out_dim * l->in_dim + l->out_dim) * sizeof(float), 256);
    // eight workgroups on each CU for dz with its sums, fewer where rows are so wide that the sums would count, more without sums (gradients of bf16
    // 512 -> 256 gelu, 302,709 rows of 24 groups: 692 us with 2,048 workgroups, 710 with 512, 703 with 8,192)
    p.sums_with_dz = l->dtype == BGL_BF16 && (l->activation == BGL_ACT_GELU || l->activation == BGL_ACT_SILU);
    const int64_t dz_most = !p.sums_with_dz ? 8192 : l->out_dim > 512 ? (1 << 20) / l->out_dim : 2048;
    p.dz_shares = (int)(most < dz_most ? most : dz_most);
    p.dz_part_bytes = p.sums_with_dz ? (size_t)(p.dz_shares + l->num_groups) * l->out_dim * sizeof(float) : 0;
    p.bytes = p.dz_bytes + p.part_bytes + p.dz_part_bytes;
    return p;
}

// 128 rows to a tile where that leaves the 256 CUs some three workgroups for two, else 64.  us with 64 and with 128 rows: f32 100 -> 128, 5,485 rows (43
// tiles of 128) 8 and 19, 40,000 (313) 22 and 28, 45,000 (352) 24 and 28, 60,000 (469) 30 and 30; bf16 512 -> 128, 40,000 16 and 19; 512 -> 256, 30,000
// (470) 20.5 and 19.3; f32 100 -> 256, 428,377 rows, with 64: 1.3 times the time.
bool large_tiles(int64_t n, int64_t cols) { return ceil_div(n, 128) * ceil_div(cols, 128) >= 384; }

template <class T, bool B_OC, bool DZ>
int launch_rows(RowsArgs<T> &a, hipStream_t st)
{
    const int64_t extra = a.q.groups > 0 ? (a.q.groups + 1 < a.n ? a.q.groups + 1 : a.n) : 1;
    const bool large = large_tiles(a.n, a.N);
    int64_t blocks = 0;
    with_cut(large, a.N, T::VEC, [&](auto cut, auto narrow) {
        using C = decltype(cut);
        constexpr bool NARROW = B_OC && decltype(narrow)::value;
        a.row_tiles = a.n / C::BA + extra;
        a.col_tiles = (int)ceil_div(a.N, C::BB);
        blocks = tile_count(a.row_tiles, a.col_tiles);
        if (blocks > INT32_MAX) return;
        // Four teams where no CU has a second workgroup: they wait for their loads once instead of once for each tile of the summed index.  us with
        // four and with one: f32 100 -> 128, 1,000 rows (32 workgroups) 7.7 and 8.5, 8,000 (250) 8.3 and 9.3, 12,000 (376) 13.2 and 11.3.
        if constexpr (C::BA == 64) {
            if (blocks <= 256) {
                k_linear_rows<T, B_OC, C, NARROW, 4, DZ><<<dim3((unsigned)blocks), dim3(4 * kThreads), 0, st>>>(a);
                return;
            }
        }
        k_linear_rows<T, B_OC, C, NARROW, 1, DZ><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a);
    });
    if (blocks > INT32_MAX) BGL_FAIL(BGL_EUNSUPPORTED, "%lld rows of width %d need too many workgroups", (long long)a.n, a.N);
    BGL_HIP(hipGetLastError());
    return BGL_OK;
}

template <class T>
int forward(const bgl_linear_t *l, int64_t n, const Groups &q, const void *x, int64_t x_stride, const void *weight, const void *bias, const void *residual,
            int64_t residual_stride, void *y, int64_t y_stride, void *saved, int64_t saved_stride, hipStream_t st)
{
    using E = typename T::elem;
    RowsArgs<T> a{};
    a.x = (const E *)x, a.w = (const E *)weight, a.bias = (const E *)bias, a.residual = (const E *)residual;
    a.y = (E *)y, a.saved = (E *)saved;
    a.n = n, a.x_stride = x_stride, a.y_stride = y_stride, a.residual_stride = residual_stride, a.saved_stride = saved_stride;
    a.K = l->in_dim, a.N = l->out_dim;
    a.residual_mode = l->residual, a.activation = l->activation;
    a.q = q;
    return launch_rows<T, false, false>(a, st);
}

template <class T>
int backward(const bgl_linear_t *l, int64_t n, const Groups &q, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *weight,
             const void *saved, int64_t saved_stride, void *dx, int64_t dx_stride, void *dweight, void *dbias, void *dresidual,
             int64_t dresidual_stride, void *workspace, hipStream_t st)
{
    using E = typename T::elem;
    const WeightPlan p = plan_weight(l, n);
    const int classes = l->num_groups > 0 ? l->num_groups : 1, dz_classes = l->num_groups > 0 ? l->num_groups + 1 : 0;
    const void *dz = dy;
    int64_t dz_stride = dy_stride;
    float *dz_part = p.sums_with_dz && dbias ? reinterpret_cast<float *>((char *)workspace + p.dz_bytes + p.part_bytes) : nullptr;
    // dz is made where dx first needs it if few tiles of columns make it again, or few rows make a launch count: us of a training call so and with dz
    // apart, f32 gelu 100 -> 256, 428,377 rows 1,030 and 1,153, 256 -> 256, 100,000 rows 489 and 497, 512 -> 256 848 and 809; bf16 relu 256 -> 256 168
    // and 171, 512 -> 256 239 and 225; 512 -> 128, 5,485 rows f32 57 and 60, bf16 36 and 41.  Not where dz takes dy's place and dx has several tiles of
    // columns: one may still be reading the dy that the first replaces.
    const bool large = large_tiles(n, l->in_dim), alone = l->in_dim <= (large ? Large::BB : Small::BB);
    const bool act = l->activation != BGL_ACT_NONE;
    const bool together = act && dx && n > 0 && l->in_dim <= (large ? 256 : 512) && !dz_part && (alone || dresidual != dy);
    if (n > 0 && (dresidual || act)) {
        void *to = dresidual ? dresidual : workspace;
        dz_stride = dresidual ? dresidual_stride : (int64_t)p.dz_stride;
        if (!together) {
            DzArgs<T> a{};
            a.dy = (const E *)dy, a.saved = (const E *)saved, a.dz = (E *)to, a.part = dz_part;
            a.n = n, a.dy_stride = dy_stride, a.saved_stride = saved_stride, a.dz_stride = dz_stride;
            a.N = l->out_dim, a.act = l->activation, a.shares = p.dz_shares, a.classes = dz_classes;
            a.q = q;
            const int columns = kThreads * T::VEC < kDzColumns ? kThreads * T::VEC : kDzColumns;
            k_linear_dz<T><<<dim3((unsigned)p.dz_shares, (unsigned)ceil_div(l->out_dim, columns)), dim3(kThreads), 0, st>>>(a);
            BGL_HIP(hipGetLastError());
        }
        dz = to;
    }
    if (dx && n > 0) {
        RowsArgs<T> a{};
        a.x = (const E *)(together ? dy : dz), a.w = (const E *)weight, a.y = (E *)dx;
        a.n = n, a.x_stride = together ? dy_stride : dz_stride, a.y_stride = dx_stride;
        a.K = l->out_dim, a.N = l->in_dim;
        a.q = q;
        if (together) {
            a.z = (const E *)saved, a.z_stride = saved_stride, a.z_activation = l->activation;
            a.dz = dresidual || dweight ? (E *)dz : nullptr, a.dz_stride = dz_stride;
            BGL_TRY((launch_rows<T, true, true>(a, st)));
        } else {
            BGL_TRY((launch_rows<T, true, false>(a, st)));
        }
    }
    if (dweight) {
        float *part = reinterpret_cast<float *>((char *)workspace + p.dz_bytes);
        if (n > 0) {
            WeightArgs<T> a{};
            a.a = (const E *)(p.swapped ? x : dz), a.b = (const E *)(p.swapped ? dz : x);
            a.a_stride = p.swapped ? x_stride : dz_stride, a.b_stride = p.swapped ? dz_stride : x_stride;
            a.part = part, a.n = n, a.a_dim = p.a_dim, a.b_dim = p.b_dim, a.N = l->out_dim, a.shares = p.shares, a.a_tiles = p.a_tiles, a.b_tiles = p.b_tiles;
            a.bias = dz_part || !dbias ? 0 : p.swapped ? 2 : 1;
            a.q = q;
            const dim3 grid((unsigned)tile_count(p.shares, p.a_tiles * p.b_tiles)), block(kThreads);
            with_cut(p.large, p.b_dim, T::VEC, [&](auto cut, auto narrow) {
                if (q.index) k_linear_dw<T, true, decltype(cut), decltype(narrow)::value><<<grid, block, 0, st>>>(a);
                else k_linear_dw<T, false, decltype(cut), decltype(narrow)::value><<<grid, block, 0, st>>>(a);
            });
            BGL_HIP(hipGetLastError());
        }
        ReduceArgs<T> r{};
        r.part = part, r.dw = (E *)dweight, r.db = (E *)dbias, r.n = n, r.N = l->out_dim, r.K = l->in_dim, r.shares = p.shares, r.swapped = p.swapped;
        r.q = q;
        r.dz_part = dz_part, r.dz_shares = p.dz_shares, r.dz_classes = dz_classes;
        const bool split = p.shares > 8 * classes;  // more than two shares for each wavefront
        r.matrix_blocks = (int)ceil_div((int64_t)l->out_dim * l->in_dim + l->out_dim, split ? 256 : 1024);
        const dim3 grid((unsigned)(r.matrix_blocks + (dz_part ? (int)ceil_div(l->out_dim, 16) : 0)), (unsigned)classes);
        if (split) k_linear_reduce<T, true><<<grid, dim3(kThreads), 0, st>>>(r);
        else k_linear_reduce<T, false><<<grid, dim3(kThreads), 0, st>>>(r);
        BGL_HIP(hipGetLastError());
    }
    return BGL_OK;
}

int group_tiles(int64_t n, int64_t &tile_rows)
{
    tile_rows = ceil_div(n, kGroupTiles);
    tile_rows = (int64_t)round_up((size_t)(tile_rows < kGroupTileRows ? kGroupTileRows : tile_rows), kGroupThreads);
    return (int)ceil_div(n, tile_rows);
}

// Room for as many tiles as group_tiles() may cut n rows or fewer into: a longer batch's tiles are rounded up to more rows, so it can have fewer.
size_t group_bytes(int64_t n, int groups)
{
    const int64_t tiles = ceil_div(n, kGroupTileRows);
    return round_up((size_t)n * sizeof(uint16_t), 256) + (size_t)(tiles < 1 ? 1 : tiles < kGroupTiles ? tiles : kGroupTiles) * (groups + 1) * sizeof(int32_t);
}

int check_group_sizes(int64_t n, int32_t num_groups)
{
    if (n < 0 || n > INT32_MAX) BGL_FAIL(BGL_EINVAL, "n must be in [0, 2^31) (got %lld)", (long long)n);
    if (num_groups < 1) BGL_FAIL(BGL_EINVAL, "num_groups must be positive (got %d)", num_groups);
    if (num_groups > kMaxGroups) BGL_FAIL(BGL_EUNSUPPORTED, "num_groups must be at most %d (got %d)", kMaxGroups, num_groups);
    return BGL_OK;
}

}  // namespace
}  // namespace bgl

using namespace bgl;

extern "C" int bgl_linear_workspace_bytes(const bgl_linear_t *layer, int64_t n, size_t *bytes)
try {
    if (!bytes) BGL_FAIL(BGL_EINVAL, "bytes is null");
    BGL_TRY(check_layer(layer, n));
    const WeightPlan p = plan_weight(layer, n);
    *bytes = p.bytes;
    return BGL_OK;
} BGL_NOTHROW_END

extern "C" int bgl_linear_forward(const bgl_linear_t *layer, int64_t n, const int32_t *rows, const int32_t *offsets, const void *x, int64_t x_stride,
                                  const void *weight, const void *bias, const void *residual, int64_t residual_stride, void *y, int64_t y_stride,
                                  void *saved, int64_t saved_stride, void *stream)
try {
    BGL_TRY(check_layer(layer, n));
    BGL_TRY(check_groups(layer, rows, offsets));
    const int es = elem_bytes(layer);
    BGL_TRY(check_rows("x", x, x_stride, layer->in_dim, es, n > 0));
    BGL_TRY(check_rows("y", y, y_stride, layer->out_dim, es, n > 0));
    BGL_TRY(check_rows("residual", residual, residual_stride, layer->out_dim, es, n > 0 && layer->residual != BGL_RESIDUAL_NONE));
    BGL_TRY(check_rows("saved", saved, saved_stride, layer->out_dim, es, false));
    if (residual && layer->residual == BGL_RESIDUAL_NONE) BGL_FAIL(BGL_EINVAL, "the layer has no residual");
    if (!weight || !aligned(weight, es) || !aligned(bias, es)) BGL_FAIL(BGL_EINVAL, "weight is null, or weight or bias is misaligned");
    if (n == 0) return BGL_OK;
    const Groups q{offsets, rows, layer->num_groups};
    return layer->dtype == BGL_F32 ? forward<tile::F32>(layer, n, q, x, x_stride, weight, bias, residual, residual_stride, y, y_stride, saved, saved_stride, (hipStream_t)stream)
                                   : forward<tile::BF16>(layer, n, q, x, x_stride, weight, bias, residual, residual_stride, y, y_stride, saved, saved_stride, (hipStream_t)stream);
} BGL_NOTHROW_END

extern "C" int bgl_linear_backward(const bgl_linear_t *layer, int64_t n, const int32_t *rows, const int32_t *offsets, const void *dy, int64_t dy_stride,
                                   const void *x, int64_t x_stride, const void *weight, const void *saved, int64_t saved_stride, void *dx,
                                   int64_t dx_stride, void *dweight, void *dbias, void *dresidual, int64_t dresidual_stride, void *workspace,
                                   size_t workspace_bytes, void *stream)
try {
    BGL_TRY(check_layer(layer, n));
    BGL_TRY(check_groups(layer, rows, offsets));
    const int es = elem_bytes(layer);
    BGL_TRY(check_rows("dy", dy, dy_stride, layer->out_dim, es, n > 0));
    BGL_TRY(check_rows("x", x, x_stride, layer->in_dim, es, n > 0 && dweight));
    BGL_TRY(check_rows("saved", saved, saved_stride, layer->out_dim, es, n > 0 && layer->activation != BGL_ACT_NONE));
    BGL_TRY(check_rows("dx", dx, dx_stride, layer->in_dim, es, false));
    BGL_TRY(check_rows("dresidual", dresidual, dresidual_stride, layer->out_dim, es, false));
    if (dresidual && layer->residual != BGL_RESIDUAL_BEFORE)
        BGL_FAIL(BGL_EINVAL, "dresidual belongs to a residual before the activation (behind it the residual's gradient is dy)");
    if (dx && (!weight || !aligned(weight, es))) BGL_FAIL(BGL_EINVAL, "weight is null or misaligned");
    if (dbias && !dweight) BGL_FAIL(BGL_EINVAL, "dbias without dweight");
    if (!aligned(dweight, es) || !aligned(dbias, es)) BGL_FAIL(BGL_EINVAL, "dweight or dbias is misaligned");
    const WeightPlan p = plan_weight(layer, n);
    if (p.bytes > 0) {
        if (!workspace || !aligned(workspace, 256)) BGL_FAIL(BGL_EINVAL, "workspace is null or not 256-byte aligned");
        if (workspace_bytes < p.bytes) BGL_FAIL(BGL_ECAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
    }
    const Groups q{offsets, rows, layer->num_groups};
    return layer->dtype == BGL_F32 ? backward<tile::F32>(layer, n, q, dy, dy_stride, x, x_stride, weight, saved, saved_stride, dx, dx_stride, dweight, dbias, dresidual, dresidual_stride, workspace, (hipStream_t)stream)
                                   : backward<tile::BF16>(layer, n, q, dy, dy_stride, x, x_stride, weight, saved, saved_stride, dx, dx_stride, dweight, dbias, dresidual, dresidual_stride, workspace, (hipStream_t)stream);
} BGL_NOTHROW_END

extern "C" int bgl_group_rows_workspace_bytes(int64_t n, int32_t num_groups, size_t *bytes)
try {
    if (!bytes) BGL_FAIL(BGL_EINVAL, "bytes is null");
    BGL_TRY(check_group_sizes(n, num_groups));
    *bytes = group_bytes(n, num_groups);
    return BGL_OK;
} BGL_NOTHROW_END

extern "C" int bgl_group_rows(const int32_t *group_of, int64_t num_nodes, const int32_t *ids, int64_t n, int32_t num_groups, int32_t *rows,
                              int32_t *offsets, void *workspace, size_t workspace_bytes, void *stream)
try {
    BGL_TRY(check_group_sizes(n, num_groups));
    if (!offsets || !aligned(offsets, 4)) BGL_FAIL(BGL_EINVAL, "offsets is null or misaligned");
    if (n > 0 && (!group_of || !rows)) BGL_FAIL(BGL_EINVAL, "group_of or rows is null");
    if (!aligned(group_of, 4) || !aligned(ids, 4) || !aligned(rows, 4)) BGL_FAIL(BGL_EINVAL, "group_of, ids or rows is misaligned");
    if (num_nodes < 0 || (!ids && num_nodes < n)) BGL_FAIL(BGL_EINVAL, "group_of has %lld entries, %lld rows ask for one each", (long long)num_nodes, (long long)n);
    if (!workspace || !aligned(workspace, 256)) BGL_FAIL(BGL_EINVAL, "workspace is null or not 256-byte aligned");
    if (workspace_bytes < group_bytes(n, num_groups)) BGL_FAIL(BGL_ECAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, group_bytes(n, num_groups));
    GroupArgs a{};
    a.group_of = group_of, a.ids = ids, a.num_nodes = num_nodes, a.n = n, a.groups = num_groups;
    int64_t tile_rows;
    int tiles = group_tiles(n, tile_rows);
    a.tile_rows = (int32_t)tile_rows;
    a.rows = rows, a.offsets = offsets;
    a.group = (uint16_t *)workspace;
    a.counts = (int32_t *)((char *)workspace + round_up((size_t)n * sizeof(uint16_t), 256));
    const hipStream_t st = (hipStream_t)stream;
    const size_t classes = (size_t)num_groups + 1, place = (kGroupThreads / kWave + 2) * classes * sizeof(int32_t);
    if (tiles <= 1) {
        k_group_place<true><<<dim3(1), dim3(kGroupThreads), place, st>>>(a);
    } else {
        k_group_count<<<dim3((unsigned)tiles), dim3(kGroupThreads), classes * sizeof(int32_t), st>>>(a);
        k_group_place<false><<<dim3((unsigned)tiles), dim3(kGroupThreads), place, st>>>(a);
    }
    BGL_HIP(hipGetLastError());
    return BGL_OK;
} BGL_NOTHROW_END
