// Losses over class scores z = x W' + b that are not kept, and their gradients.
//
//   labels     loss = lse(z) - z_label                               dz = s (exp(z - lse(z)) - onehot)
//   teacher    t^2 sum p (log p - log q), p = softmax(score / t)     dz = s' t (q - p), q = softmax(z / t) = exp(z / t - lse(z / t))
//
// The products bound them: 2 n V D operations forward, 6 backward, where the scores are made again, a piece of rows x classes at a time, so that what is kept does not
// grow with n V.  One row is bound by the weight's bytes, few rows and classes by their launches.
//
//   k_class_scores            z tile by tile; forward: every tile's largest value and sums of exp, per row; backward: dz of a piece (rows x classes)
//   k_class_top               forward: the scores of the teacher's classes
//   k_class_merge, _finish    forward: the parts of a row with many, the losses from all of that
//   k_class_fix               backward: dz of the teacher's classes, over what the scores' kernel left there
//   k_class_products          backward: dx = dz W and dW = dz' x of a piece, db = the sum of dz's rows
//   k_class_reduce            backward: what pieces or ranges of a sum share a result
//   k_class_zero              backward: the gradients of no rows
// and for large calls, whose operands are laid out for bgl_stage.h first,
//   k_class_scores_stage, k_class_products_stage
//   k_class_split             fp32 operands as three bf16
//   k_class_lay               bf16 operands in whole steps, forward; k_class_largest, k_class_halves: as halves, backward
#include "bgl_internal.h"
#include "bgl_reduce.h"
#include "bgl_stage.h"
#include "bgl_tile.h"

#include <cmath>
#include <type_traits>

namespace bgl {
namespace {

using namespace tile;

#pragma clang fp contract(off)  // (a base has to be the same number wherever it is used)

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr int64_t kPieceRows = 16384;
constexpr int64_t kPieceClasses = 256;                 // pieces of some classes only are multiples
constexpr int64_t kPartialBytes = (int64_t)64 << 20;   // of a forward call's tiles' maxima and sums
constexpr int kCus = 256;
constexpr int kStoredBeside = 512;                     // bytes of classes' rows that storing a tile's row in LDS takes as long as
constexpr int64_t kMostThreads = (int64_t)1 << 31;     // of a launch, which has room for 2^32 - 1
// Calls that are laid out for large tiles have more rows than one of these has, more classes than one of the small ones has, and many products.  us, forward + backward, in
// small tiles and so: bf16, rows x 512 x 65,536: 128 rows 29 + 111 and 31 + 122, 160 39 + 172 and 40 + 140; 50,000 x 512 x classes: 128 classes 17 + 84 and 18 + 104, 160
// 31 + 135 and 19 + 108; f32: 85 + 259 and 145 + 322, 197 + 471 and 172 + 388; 73 + 219 and 103 + 256, 149 + 355 and 107 + 271.  2e9 products: 512 x 256 x 16,384 bf16 19 + 59
// and 19 + 50, f32 47 + 129 and 54 + 131; 10,000 x 256 x 1,001 bf16 17 + 70 and 16 + 60, f32 61 + 188 and 52 + 186.
constexpr int kLargeRows = 129, kLargeClasses = 129;
constexpr double kLargeProducts = 2e9;

// Exponentials are powers of two: exp(k v) / 2^base with k = log2(e) or that over the temperature, as 2^(k v - base) with one rounding.  A sum of them is taken to
// the base of its largest value, k most, rounded: what rounding leaves of it is the same for all of a sum, and sums of two bases meet exactly, as the bases' difference has no
// rounding to speak of.  From `far` (2^24 / k) on it leaves more than 1, in the end more than a power's range: of such rows the largest value itself is taken from the others
// first (`shift`), which is exact for those near it, and the base is 0.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
struct Base {
    float shift, base, base_t;  // at the temperature: base_t
};
template <class A>
__device__ __forceinline__ Base base_of(const A &a, float most)
{
    const bool near = fabsf(most) < a.far, nothing = most == -INFINITY;  // (nothing there: the sum is 0)
    return Base{near || nothing ? 0.0f : most, near ? most * a.k : 0.0f, near ? most * a.k_t : 0.0f};
}
__device__ __forceinline__ float power_to(float v, float k, float base) { return __builtin_amdgcn_exp2f(fmaf(v, k, -base)); }
__device__ __forceinline__ float max3(float a, float b, float c)  // (of fmaxf the compiler makes two instructions more, for signalling NaN)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// What a row keeps for its gradients, from which q is as near as its power and its sum (with the sum's logarithm in 32 bits it was off by up to that much of its last place:
// gradients of few classes were 2e-6 off, now 3e-7).  sum_t: of scores over the temperature, +inf where the teacher names no class; behind it its classes' scores.
__device__ __forceinline__ void keep(float *to, int width, float most, float sum, float sum_t)
{
    to[0] = most, to[1] = sum;
    if (width > 2) to[2] = sum_t;
}
// The logarithm of the sum less the score, both to the sum's base (what they have in common goes before they meet), in natural units.
template <class A>
__device__ __forceinline__ float loss_of(const A &a, float log_sum, float score, const Base &b) { return kLn2 * (log_sum - fmaf(score - b.shift, a.k, -b.base)); }
// What a sum to the base of `most` is to be multiplied by to be to the base `to`, that of no smaller a value.  A sum of nothing has no base (base_of's 0 for it may be far
// above `to`: 0 times 2^(0 - to) was NaN for rows whose scores are all below -88): 0, which leaves a NaN one.  rebase_t: of sums at the temperature.
template <class A>
__device__ __forceinline__ float rebase(const A &a, float most, const Base &to)
{
    const Base from = base_of(a, most);
    const float power = __builtin_amdgcn_exp2f(fmaf(from.shift - to.shift, a.k, from.base - to.base));
    return most == -INFINITY ? 0.0f : power;
}
template <class A>
__device__ __forceinline__ float rebase_t(const A &a, float most, const Base &to)
{
    const Base from = base_of(a, most);
    const float power = __builtin_amdgcn_exp2f(fmaf(from.shift - to.shift, a.k_t, from.base_t - to.base_t));
    return most == -INFINITY ? 0.0f : power;
}

// The other lanes with the same lane % 16.
template <class F>
__device__ __forceinline__ float down_column(float v, F both)
{
    const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t a = s[0], b = s[1];
    v = both(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    const auto t = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t c = t[0], d = t[1];
    return both(__builtin_bit_cast(float, c), __builtin_bit_cast(float, d));
}

// Large calls keep dz in blocks of 16 rows x 32 classes (bgl_stage.h), plane by plane within a block.
constexpr int kPad = 64;                           // values that laid out rows are padded to
// Tiles of classes that an XCD has in hand while it goes through the rows (512 values each: 3 MB beside the rows', of its L2's 4): 4,096 x 512 x 65,536 took 298 us
// with the rows' 4 MB read again for every tile or two of classes, 255 with 16 (the products alone, with their exponentials).
constexpr int kClassGroup = 8;
using StageCut = stage::Cut<6, 4>;                 // scores: 192 classes x 128 rows
using ProductCut = stage::Cut<8, 4>;               // dW: 256 classes, dx: 256 rows; x 128 columns
constexpr int kBlockRows = 16, kBlockClasses = 32, kBlockValues = kBlockRows * kBlockClasses;
__device__ __forceinline__ int64_t dz_block(int64_t r, int c, int stride, int planes)
{
    return ((r / kBlockRows * (stride / kBlockClasses) + c / kBlockClasses) * planes) * kBlockValues + r % kBlockRows * kBlockClasses + c % kBlockClasses;
}

// A fp32 value as three of bf16 (bgl_stage.h).  One that is not finite, or rounds to infinity, is in the first alone.
__device__ __forceinline__ void split(float v, uint16_t (&e)[3])
{
    e[0] = BF16::put(v);
    if (fabsf(v) < INFINITY && (e[0] & 0x7fff) == 0x7f80) e[0] -= 1;  // (a value that rounds up to infinity: the largest there is)
    const float rest = fabsf(v) < INFINITY ? v - BF16::get(e[0]) : 0.0f;
    e[1] = BF16::put(rest);
    e[2] = BF16::put(rest - BF16::get(e[1]));
}

// dz as large calls keep it: three bf16 of fp32 layers; of bf16 ones a half, or (`whole`, see k_class_halves) two bf16.
template <class T>
__device__ __forceinline__ void parts(float d, bool whole, uint16_t (&e)[3])
{
    if constexpr (T::PER == 1) split(d, e);
    else if (whole) e[0] = BF16::put(d), e[1] = BF16::put(d - BF16::get(e[0]));
    else e[0] = __builtin_bit_cast(uint16_t, (_Float16)d);
}
template <class T>
__device__ __forceinline__ int dz_planes(bool whole) { return T::PER == 1 ? 3 : whole ? 2 : 1; }

template <class T>
struct ScoreArgs {
    const typename T::elem *x, *w, *bias;
    const int32_t *labels;
    int64_t x_stride, n;      // rows of the call
    int64_t row0, rows;       // those of this launch
    int64_t row_tiles;
    int class0, classes;      // this launch's classes: from class0 up to `classes`
    int all_classes;
    bool by_rows;             // tiles of one block of rows, not of classes, follow one another on an XCD
    int class_tiles, D;
    float k, k_t, far;        // log2(e), and over the temperature; see base_of()
    // forward: {largest, sum} of part t of the classes and row r at part[t * rows + r], the sum at the temperature at part_t[t * rows + r]
    float2 *part;
    float *part_t, *label_score;
    float *loss, *kept;       // one tile has all classes and there is no teacher: the losses and what is saved (or null) instead
    bool whole;
    bool two;                 // labels, and a teacher at a temperature that is not 1: two sums (of a teacher alone, k is k_t)
    // backward
    const float *saved;       // n x width, see keep()
    int saved_width;
    float scale, teacher_scale;
    typename T::elem *dz;     // rows x dz_stride
    typename T::elem *dz_rest;  // bf16: what rounding dz left, laid out the same
    int dz_stride;
    int32_t *listed;          // null, or the row's number among this launch's for rows with a gradient, else -1
};

// The row's values of a lane's fragments less the largest, where scores are far from 0.
template <class C>
__device__ __forceinline__ void take_shift(f32x4 (&acc)[C::FA][C::FB], int t, float shift)
{
#pragma unroll
    for (int i = 0; i < C::FA; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][t][j] -= shift;
}

// One tile of classes x rows: a lane holds, of one row, 4 neighbouring classes of every 16, so that a row's maximum and sum meet in 4 lanes.  One row of 512 and 65,536
// classes, bf16: 13.1 us, 5.1 TB/s of the weight.  1,024 x 128 x 50 f32: 5.1 us.
template <class T, class C, bool DZ>
__global__ void __launch_bounds__(kThreads, 2) k_class_scores(ScoreArgs<T> a)
{
    using A = KcOperand<T, C::BA>;
    using B = KcOperand<T, C::BB>;
    __shared__ __attribute__((aligned(16))) uint32_t lds[A::LDS + B::LDS];
    __shared__ float meet[DZ ? 1 : 3 * C::BA / 16 / C::FA * C::BB], own_score[DZ ? 1 : C::BB];
    int64_t ct, rt;
    int fast;
    const uint32_t slow_tiles = a.by_rows ? (uint32_t)a.row_tiles : a.class_tiles, fast_tiles = a.by_rows ? a.class_tiles : (uint32_t)a.row_tiles;
    if (!stage::tile_of(blockIdx.x, slow_tiles, fast_tiles, 1, a.by_rows ? rt : ct, fast)) return;
    (a.by_rows ? ct : rt) = fast;
    const int c0 = a.class0 + (int)ct * C::BA, last = a.classes - 1;
    const int64_t r0 = rt * C::BB;  // of this launch's rows
    f32x4 acc[C::FA][C::FB] = {};
    A weight;
    B rows;
    weight.init([&](int i) { return a.w + (int64_t)(c0 + i < last ? c0 + i : last) * a.D; });
    rows.init([&](int i) { return a.x + (a.row0 + (r0 + i < a.rows ? r0 + i : a.rows - 1)) * a.x_stride; });
    pipeline(
        (a.D + A::BK - 1) / A::BK,
        [&](int i) {
            weight.load(i, a.D);
            rows.load(i, a.D);
        },
        [&](int) {
            weight.store(lds);
            rows.store(lds + A::LDS);
        },
        [&](int i) {
            const int steps = (a.D - i * A::BK + 16 * T::PER - 1) / (16 * T::PER);
            multiply<T, A, B, C>(lds, lds + A::LDS, steps, acc, [](const auto &, const auto &) {});
        });
    const int l = threadIdx.x & 63, first = c0 + C::a_off() + 4 * (l >> 4);
#pragma unroll
    for (int i = 0; i < C::FA; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = first + 16 * i + j;
            const float b = a.bias ? T::get(a.bias[c < last ? c : last]) : 0.0f;
#pragma unroll
            for (int t = 0; t < C::FB; ++t) acc[i][t][j] = c <= last ? acc[i][t][j] + b : -INFINITY;
        }
#pragma unroll
    for (int t = 0; t < C::FB; ++t) {
        const int in_tile = C::b_off() + 16 * t + (l & 15);
        const int64_t r = r0 + in_tile;
        const bool live = r < a.rows;
        const int64_t row = a.row0 + (live ? r : a.rows - 1);
        int label = a.labels ? a.labels[row] : -1;
        if ((uint32_t)label >= (uint32_t)a.all_classes) label = -1;
        if constexpr (!DZ) {
            float most = -INFINITY, sum = 0.0f, sum_t = 0.0f;
#pragma unroll
            for (int i = 0; i < C::FA; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) most = fmaxf(most, acc[i][t][j]);
            most = down_column(most, [](float p, float q) { return fmaxf(p, q); });
            const Base to = base_of(a, most);
#pragma unroll
            for (int i = 0; i < C::FA; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (first + 16 * i + j == label && live) {
                        if (a.whole) own_score[in_tile] = acc[i][t][j];
                        else a.label_score[row] = acc[i][t][j];
                    }
            if (__any(to.shift != 0.0f)) take_shift<C>(acc, t, to.shift);
#pragma unroll
            for (int i = 0; i < C::FA; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = acc[i][t][j];
                    sum += power_to(v, a.k, to.base);
                    if (a.two) sum_t += power_to(v, a.k_t, to.base_t);
                }
            sum = down_column(sum, [](float p, float q) { return p + q; });
            if (a.two) sum_t = down_column(sum_t, [](float p, float q) { return p + q; });
            float *at = meet + (C::a_off() / C::FA / 16 * C::BB + in_tile) * 3;
            if (l < 16) at[0] = most, at[1] = sum, at[2] = sum_t;
        } else {
            const float *kept = a.saved + row * a.saved_width;
            const float sum_t = a.teacher_scale != 0.0f ? kept[2] : INFINITY;
            const Base to = base_of(a, kept[0]);
            if (__any(to.shift != 0.0f)) take_shift<C>(acc, t, to.shift);
            const float s = label >= 0 ? a.scale : 0.0f, st = sum_t != INFINITY ? a.teacher_scale : 0.0f;
            const float share = 1.0f / kept[1], share_t = st / sum_t;
            // (the products that sum over rows leave the others out, whatever x holds there)
            if (a.listed && ct == 0 && C::a_off() == 0 && l < 16 && live) a.listed[r] = s != 0.0f || st != 0.0f ? (int32_t)r : -1;
#pragma unroll
            for (int i = 0; i < C::FA; ++i) {
                typename T::elem e[4], rest[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = acc[i][t][j];
                    float d = 0.0f;
                    if (s != 0.0f) d = s * (power_to(v, a.k, to.base) * share - (first + 16 * i + j == label ? 1.0f : 0.0f));
                    if (st != 0.0f) d = fmaf(share_t, power_to(v, a.k_t, to.base_t), d);
                    e[j] = T::put(d);
                    rest[j] = T::put(d - T::get(e[j]));
                }
                const int c = first + 16 * i;
                const int64_t at = r * a.dz_stride + (c - a.class0);  // (dz_stride is a multiple of 4; what is behind the classes is not read)
                if (live && c - a.class0 < a.dz_stride) {
                    __builtin_memcpy(a.dz + at, e, sizeof(e));
                    if constexpr (T::PER == 2) __builtin_memcpy(a.dz_rest + at, rest, sizeof(rest));
                }
            }
        }
    }
    if constexpr (!DZ) {
        constexpr int WA = C::BA / 16 / C::FA;
        __syncthreads();
        for (int in_tile = threadIdx.x; in_tile < C::BB; in_tile += kThreads) {
            if (r0 + in_tile >= a.rows) break;
            float most = -INFINITY, sum = 0.0f, sum_t = 0.0f;
#pragma unroll
            for (int w = 0; w < WA; ++w) most = fmaxf(most, meet[(w * C::BB + in_tile) * 3]);
            const Base to = base_of(a, most);
#pragma unroll
            for (int w = 0; w < WA; ++w) {
                const float *from = meet + (w * C::BB + in_tile) * 3;
                sum += from[1] * rebase(a, from[0], to);
                if (a.two) sum_t += from[2] * rebase_t(a, from[0], to);
            }
            if (a.whole) {
                const int64_t row = a.row0 + r0 + in_tile;
                const float log_sum = log2f(sum);
                const bool has = (uint32_t)a.labels[row] < (uint32_t)a.all_classes;
                if (a.loss) a.loss[row] = has ? loss_of(a, log_sum, own_score[in_tile], to) : 0.0f;
                if (a.kept) keep(a.kept + row * a.saved_width, a.saved_width, most, sum, INFINITY);
                continue;
            }
            a.part[ct * a.rows + r0 + in_tile] = float2{most, sum};
            if (a.two) a.part_t[ct * a.rows + r0 + in_tile] = sum_t;
        }
    }
}

template <class T>
struct RowArgs {
    const typename T::elem *x, *w, *bias;
    const int32_t *labels, *top_class;
    const float *top_score;
    int64_t x_stride, n, row0, rows;
    int D, classes, top, class_parts, saved_width;
    float t, over_t, k, k_t, far, scale, teacher_scale;
    const float2 *part;
    const float *part_t, *label_score;
    float *loss, *teacher_loss;
    float *saved;  // forward: null, or what keep() keeps and the scores; backward: those
    float *z_top;  // forward: the scores of the teacher's classes, z_stride apart for each row
    int z_stride;
    bool two;
    // backward: the piece of dz
    typename T::elem *dz, *dz_rest;
    int class0, piece_classes, dz_stride;
    bool blocks;     // dz lies in blocks, as parts() makes them
    const int32_t *whole;
};

// The scores of the teacher's classes: 8 lanes for four of a row's, 128 bytes of x and of the classes' rows at a time.  4,096 rows of 512 bf16, 32 classes each: 20 us, 6.6
// TB/s of rows that the L2s mostly have.
// keep(k, z) for each, in the first lane.
constexpr int kTopLanes = 8, kTopEach = 4;
template <class T, class F>
__device__ __forceinline__ void top_scores(const RowArgs<T> a, int64_t row, int k0, F keep)
{
    constexpr int LANES = kTopLanes, EACH = kTopEach, AHEAD = 2, STEP = LANES * T::VEC;
    const int l = threadIdx.x % LANES;
    const typename T::elem *x = a.x + row * a.x_stride, *w[EACH];
    int c[EACH];
    float z[EACH] = {};
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        c[k] = k0 + k < a.top ? a.top_class[row * a.top + k0 + k] : -1;
        if ((uint32_t)c[k] >= (uint32_t)a.classes) c[k] = -1;
        w[k] = a.w + (int64_t)(c[k] < 0 ? 0 : c[k]) * a.D;  // (the first class's row stands in for none)
    }
    const auto add = [](const uint4 &p, const uint4 &q, float z) {
        const uint32_t u[4] = {p.x, p.y, p.z, p.w}, v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (T::PER == 1) {
                z = fmaf(__uint_as_float(u[i]), __uint_as_float(v[i]), z);
            } else {
                z = fmaf(__uint_as_float(u[i] << 16), __uint_as_float(v[i] << 16), z);
                z = fmaf(__uint_as_float(u[i] & 0xffff0000u), __uint_as_float(v[i] & 0xffff0000u), z);
            }
        }
        return z;
    };
    int d = l * T::VEC;
    for (; d + (AHEAD - 1) * STEP + T::VEC <= a.D; d += AHEAD * STEP) {
        uint4 p[AHEAD], q[AHEAD][EACH];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            p[u] = load_any<uint4>(x + d + u * STEP);
#pragma unroll
            for (int k = 0; k < EACH; ++k) q[u][k] = load_any<uint4>(w[k] + d + u * STEP);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int k = 0; k < EACH; ++k) z[k] = add(p[u], q[u][k], z[k]);
    }
    for (; d < a.D; d += STEP) {
        const uint4 p = load_end<T>(x + d, a.D - d, a.D);
#pragma unroll
        for (int k = 0; k < EACH; ++k) z[k] = add(p, load_end<T>(w[k] + d, a.D - d, a.D), z[k]);
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        z[k] = sum_across<LANES>(z[k]);
        if (l == 0 && k0 + k < a.top) keep(k0 + k, c[k] < 0 ? 0.0f : z[k] + (a.bias ? T::get(a.bias[c[k]]) : 0.0f));
    }
}
template <class T>
__global__ void __launch_bounds__(256) k_class_top(RowArgs<T> a)
{
    const uint32_t groups = ((uint32_t)a.top + kTopEach - 1) / kTopEach;
    const uint64_t task = (uint64_t)blockIdx.x * (256 / kTopLanes) + threadIdx.x / kTopLanes, r = task / groups;
    if (r >= (uint64_t)a.rows) return;
    const int64_t row = a.row0 + r;
    top_scores(a, row, (int)(task % groups) * kTopEach, [=](int k, float z) { a.z_top[row * a.z_stride + k] = z; });
}

// The teacher's distribution of a row, for LANES neighbours: largest score and the sum of exp((score - largest) / t); false where it names no class.  (Scores are taken from
// each other before they meet the temperature: their own quotients round as they are large.)
template <int LANES, class T>
__device__ __forceinline__ bool teacher_of(const RowArgs<T> &a, int64_t row, float &most, float &total)
{
    const int l = threadIdx.x % LANES;
    most = -INFINITY, total = 0.0f;
    float bad = 0.0f;
    for (int k = l; k < a.top; k += LANES)
        if ((uint32_t)a.top_class[row * a.top + k] < (uint32_t)a.classes) {
            const float v = a.top_score[row * a.top + k];
            most = fmaxf(most, v);
            if (v != v) bad = v;
        }
    most = max_across<LANES>(most);
    bad = sum_across<LANES>(bad);
    if (bad != bad) most = bad;
    if (most == -INFINITY) return false;
    for (int k = l; k < a.top; k += LANES)
        if ((uint32_t)a.top_class[row * a.top + k] < (uint32_t)a.classes) total += exp_of((a.top_score[row * a.top + k] - most) * a.over_t);
    total = sum_across<LANES>(total);
    return true;
}

// Many parts of many rows: added up by 16 lanes for each of 16 rows (whose parts are neighbours), into the first part's place.  4,096 rows of 684 parts: 11 us.
constexpr int kMergeRows = 16, kMergeLanes = 16;
template <class T>
__global__ void __launch_bounds__(kMergeRows *kMergeLanes) k_class_merge(RowArgs<T> a, float2 *part, float *part_t)
{
    constexpr int AHEAD = 8;
    __shared__ float largest[kMergeLanes][kMergeRows], sums[kMergeLanes][kMergeRows], sums_t[kMergeLanes][kMergeRows];
    const int i = threadIdx.x % kMergeRows, l = threadIdx.x / kMergeRows;
    const int64_t row = (int64_t)blockIdx.x * kMergeRows + i, r = row < a.rows ? row : a.rows - 1;
    float most = -INFINITY, sum = 0.0f, sum_t = 0.0f;
    const auto take = [&](const Base &to, float largest, float s, float t) {
        sum += s * rebase(a, largest, to);
        if (a.two) sum_t += t * rebase_t(a, largest, to);
    };
    for (int first = l; first < a.class_parts; first += kMergeLanes * AHEAD) {
        float2 from[AHEAD];
        float at_t[AHEAD], m = most;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int ct = first + u * kMergeLanes;
            const bool there = ct < a.class_parts;
            from[u] = there ? part[ct * a.rows + r] : float2{-INFINITY, 0.0f};
            at_t[u] = a.two && there ? part_t[ct * a.rows + r] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) m = fmaxf(m, from[u].x);
        const Base to = base_of(a, m);
        sum *= rebase(a, most, to);
        if (a.two) sum_t *= rebase_t(a, most, to);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) take(to, from[u].x, from[u].y, at_t[u]);
        most = m;
    }
    largest[l][i] = most, sums[l][i] = sum, sums_t[l][i] = sum_t;
    __syncthreads();
    if (l > 0 || row >= a.rows) return;
    most = -INFINITY, sum = sum_t = 0.0f;
#pragma unroll
    for (int u = 0; u < kMergeLanes; ++u) most = fmaxf(most, largest[u][i]);
    const Base to = base_of(a, most);
#pragma unroll
    for (int u = 0; u < kMergeLanes; ++u) take(to, largest[u][i], sums[u][i], sums_t[u][i]);
    part[row] = float2{most, sum};
    if (a.two) part_t[row] = sum_t;
}

// TOP: with the scores of the teacher's classes, kTopHere at most, of kTopRows rows (forward call of 512 x 100 x 150 with 8 classes: 16.5 us with a launch of k_class_top, 14.1 so;
// 20 rows with 64 classes 15 and 27; a row with 16 and 512 parts to add up 33 and 37; 100,000 rows with 4 64 and 76, as 16 lanes are many for a row).
constexpr int kTopHere = 8, kTopRows = 64 * kCus;
// LANES neighbours for each row: 4 for few parts and classes of the teacher (4,096 rows 4.6 us, a launch), 16, or a wavefront.
template <class T, int LANES, bool TOP = false>
__global__ void __launch_bounds__(256) k_class_finish(RowArgs<T> a)
{
    constexpr int ROWS = 256 / LANES;
    __shared__ float z_here[TOP ? ROWS : 1][TOP ? kTopHere + 1 : 1];
    const int64_t first_row = (int64_t)blockIdx.x * ROWS, r = first_row + threadIdx.x / LANES;
    if constexpr (TOP) {
        const uint32_t groups = ((uint32_t)a.top + kTopEach - 1) / kTopEach;
        for (uint32_t task = threadIdx.x / kTopLanes; task < ROWS * groups; task += 256 / kTopLanes) {
            const int at = (int)(task / groups);
            if (first_row + at >= a.rows) break;
            const int64_t row = a.row0 + first_row + at;
            top_scores(a, row, (int)(task % groups) * kTopEach, [&](int k, float z) { a.z_top[row * a.z_stride + k] = z_here[at][k] = z; });
        }
        __syncthreads();
    }
    if (r >= a.rows) return;
    const int64_t row = a.row0 + r;
    const int l = threadIdx.x % LANES;
    float most = -INFINITY, sum = 0.0f, sum_t = 0.0f;
    constexpr int AHEAD = LANES == 64 ? 8 : 2;  // (parts on their way at a time: one after the other, 512 of one row took 4.6 us)
    for (int first = l; first < a.class_parts; first += LANES * AHEAD) {
        float2 from[AHEAD];
        float at_t[AHEAD], m = most;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int ct = first + u * LANES;
            const bool there = ct < a.class_parts;
            from[u] = there ? a.part[ct * a.rows + r] : float2{-INFINITY, 0.0f};
            at_t[u] = a.two && there ? a.part_t[ct * a.rows + r] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) m = fmaxf(m, from[u].x);
        const Base to = base_of(a, m);
        sum *= rebase(a, most, to);
        if (a.two) sum_t *= rebase_t(a, most, to);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            sum += from[u].y * rebase(a, from[u].x, to);
            if (a.two) sum_t += at_t[u] * rebase_t(a, from[u].x, to);
        }
        most = m;
    }
    const float m = max_across<LANES>(most);
    const Base to = base_of(a, m);
    sum = sum_across<LANES>(sum * rebase(a, most, to));
    sum_t = a.two ? sum_across<LANES>(sum_t * rebase_t(a, most, to)) : sum;  // (if not, k and k_t are the same)
    const float log_sum = log2f(sum), log_sum_t = log2f(sum_t);
    if (a.labels) {
        const int label = a.labels[row];
        const bool has = (uint32_t)label < (uint32_t)a.classes;
        if (l == 0 && a.loss) a.loss[row] = has ? loss_of(a, log_sum, a.label_score[row], to) : 0.0f;
    }
    float kept_t = INFINITY;
    if (a.top_class) {
        float top_most, total, kl = 0.0f;
        const bool taught = teacher_of<LANES>(a, row, top_most, total);
        if (taught) {
            kept_t = sum_t;
            const float log_total = log2f(total);
            for (int k = l; k < a.top; k += LANES)
                if ((uint32_t)a.top_class[row * a.top + k] < (uint32_t)a.classes) {
                    const float v = (a.top_score[row * a.top + k] - top_most) * a.over_t;
                    const float p = exp_of(v) / total, z = TOP ? z_here[threadIdx.x / LANES][k] : a.z_top[row * a.z_stride + k];
                    if (p != 0.0f) kl = fmaf(p, (v * kLog2e - log_total) + (log_sum_t - fmaf(z - to.shift, a.k_t, -to.base_t)), kl);
                }
            kl = sum_across<LANES>(kl);
        }
        if (l == 0 && a.teacher_loss) a.teacher_loss[row] = taught ? a.t * a.t * kLn2 * kl : 0.0f;
    }
    if (l == 0 && a.saved) keep(a.saved + row * a.saved_width, a.saved_width, m, sum, kept_t);
}

// dz where the teacher names a class: LANES neighbours for each row, workgroups of them for each 64 classes.  A class named twice has the sum of its shares.
template <class T, int LANES>
__global__ void __launch_bounds__(256) k_class_fix(RowArgs<T> a)
{
    constexpr int AHEAD = 8;
    const int64_t r = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (r >= a.rows) return;
    const int64_t row = a.row0 + r;
    const int l = threadIdx.x % LANES;
    float most, total;
    if (!teacher_of<LANES>(a, row, most, total)) return;
    const float *kept = a.saved + row * a.saved_width;
    const Base to = base_of(a, kept[0]);
    int label = a.labels ? a.labels[row] : -1;
    if ((uint32_t)label >= (uint32_t)a.classes) label = -1;
    const int32_t *classes = a.top_class + row * a.top;
    const auto share = [&](int k) { return exp_of((a.top_score[row * a.top + k] - most) * a.over_t) / total; };
    for (int k = (int)blockIdx.y * LANES + l; k - l < a.top; k += (int)gridDim.y * LANES) {
        const int c = k < a.top ? classes[k] : -1;
        const bool here = c >= a.class0 && c < a.class0 + a.piece_classes;
        float p = 0.0f;
        bool before = false;  // an entry before this one names the class
        if constexpr (LANES == 64) {
            // (read by every lane from memory, 200 classes of 200 rows took 100 us)
            for (int o = 0; o < a.top; o += 64) {
                const int other = o + l < a.top ? classes[o + l] : -2;
                const float its = (uint32_t)other < (uint32_t)a.classes ? share(o + l) : 0.0f;
#pragma unroll 16
                for (int j = 0; j < 64; ++j) {
                    const float add = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(its), j));
                    if (__builtin_amdgcn_readlane(other, j) == c) p += add, before |= o + j < k;
                }
            }
        }
        if (!here) continue;
        for (int o = 0; LANES < 64 && o < a.top; o += AHEAD) {
            int other[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) other[u] = o + u < a.top ? classes[o + u] : -1;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (other[u] == c) p += share(o + u), before |= o + u < k;
        }
        const bool whole = T::PER == 2 && a.blocks && a.whole[0];
        const int planes = dz_planes<T>(whole);
        uint16_t *const block = reinterpret_cast<uint16_t *>(a.dz) + (a.blocks ? dz_block(r, c - a.class0, a.dz_stride, planes) : 0);
        typename T::elem *const value = a.dz + r * a.dz_stride + (c - a.class0);
        float d = 0.0f;
        if constexpr (T::PER == 1) {
            // of what the scores' kernel made of the very score that the sum has: with one made anew, q is not near 1 as exactly as the others are near 0 (gradients of 2 classes
            // were 2e-6 off, now 3e-7)
            if (before) continue;
            if (a.blocks) {
#pragma unroll
                for (int p = 0; p < 3; ++p) d += BF16::get(block[p * kBlockValues]);
            } else {
                d = *value;
            }
            d = fmaf(-a.teacher_scale, p, d);
        } else {
            // (there it has been rounded)
            const float z = kept[3 + k] - to.shift;
            if (label >= 0 && a.scale != 0.0f) d = a.scale * (power_to(z, a.k, to.base) / kept[1] - (c == label ? 1.0f : 0.0f));
            d = fmaf(a.teacher_scale, power_to(z, a.k_t, to.base_t) / kept[2] - p, d);
        }
        if (a.blocks) {
            uint16_t e[3];
            parts<T>(d, whole, e);
#pragma unroll
            for (int p = 0; p < 3; ++p)
                if (p < planes) block[p * kBlockValues] = e[p];
        } else {
            *value = T::put(d);
            if constexpr (T::PER == 2) a.dz_rest[value - a.dz] = T::put(d - T::get(*value));
        }
    }
}

// ----------------------------------------------------------------- products of a piece
template <class T>
struct PieceArgs {
    const typename T::elem *a, *a_rest, *b;  // dz, and (bf16) what rounding it left; W or x
    int64_t a_stride, b_stride;
    const int32_t *list;            // of the summed rows (dW): the row itself, or -1 for none
    int64_t M, K;                   // kept and summed index
    int N, a_width;                 // columns of the result; of dz that can be read
    int64_t row_tiles;
    int col_tiles, shares;
    uint32_t tiles;                 // of a share
    int64_t per_share;              // of the summed index
    typename T::elem *out, *sums;   // the result, if it is whole; M values of sums over the summed index
    int64_t out_stride;
    float *slots, *sum_slots;       // else shares x slot_rows x N, shares x slot_rows
    int64_t slot_rows;
    bool add;                       // to what is in the slots
};

// The first `left` of V neighbours of a row, on top of what is there if `add` says so.
template <int V, class E, class F>
__device__ __forceinline__ void write_row(E *to, const float (&v)[V], int left, bool add, F round)
{
    E e[V];
    if (left >= V) {
        if (add) __builtin_memcpy(e, to, sizeof(e));
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = round(add ? (float)e[i] + v[i] : v[i]);
        __builtin_memcpy(to, e, sizeof(e));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) to[i] = round(add ? (float)to[i] + v[i] : v[i]);
    }
}

// M x N = A B over the summed index, B's rows being that index.  OC: A's rows too (dW: they are batch rows), else A's rows are the result's (dx).
template <class T, class C, bool OC, bool NARROW>
struct Product {
    using A = std::conditional_t<OC, OcOperand<T, C::BA, false, false>, KcOperand<T, C::BA>>;
    using B = OcOperand<T, C::BB, OC, NARROW>;
    using R = Result<C, A::LDS + B::LDS>;
    static constexpr int LDS = A::LDS + B::LDS > R::SIZE ? A::LDS + B::LDS : R::SIZE;
    static __device__ __forceinline__ void make(const PieceArgs<T> &a, uint32_t id, uint32_t *lds);
};
template <class T, class C, bool OC, bool NARROW>
__device__ __forceinline__ void Product<T, C, OC, NARROW>::make(const PieceArgs<T> &a, uint32_t id, uint32_t *lds)
{
    const int share = (int)(id / a.tiles);
    int64_t rt;
    int ct;
    if (!stage::tile_of(id % a.tiles, (uint32_t)a.row_tiles, a.col_tiles, 1, rt, ct)) return;
    const int64_t m0 = rt * C::BA, k0 = share * a.per_share;
    const int n0 = ct * C::BB, K = (int)(a.K - k0 < a.per_share ? a.K - k0 : a.per_share);
    f32x4 acc[C::FA][C::FB] = {};
    float *slot = a.slots ? a.slots + share * a.slot_rows * a.N : nullptr;
    float sums[C::FA] = {};
    const bool summing = OC && (a.sums || a.sum_slots) && n0 == 0 && C::b_off() == 0;
    // bf16: the products of what rounding dz left come on top: with the rounded dz alone results were up to 1.4 times as far off as their own rounding is
    for (int part = 0; K > 0 && part < (T::PER == 2 ? 2 : 1); ++part) {
        const typename T::elem *dz = part ? a.a_rest : a.a;
        A left;
        B right;
        if constexpr (OC) {
            left.init(dz, a.a_stride, a.K, (int)m0, a.a_width);
            left.range(nullptr, k0, K);
        } else {
            left.init([&](int i) { return dz + (m0 + i < a.M ? m0 + i : a.M - 1) * a.a_stride + k0; });
        }
        right.init(a.b, a.b_stride, a.K, n0, a.N);
        right.range(a.list, k0, K);
        pipeline(
            (K + A::BK - 1) / A::BK,
            [&](int i) {
                if constexpr (OC) left.load(i);
                else left.load(i, K);
                right.load(i);
            },
            [&](int) {
                if constexpr (OC) left.settle();
                left.store(lds);
                right.settle();
                right.store(lds + A::LDS);
            },
            [&](int i) {
                const int steps = (K - i * A::BK + 16 * T::PER - 1) / (16 * T::PER);
                multiply<T, A, B, C>(lds, lds + A::LDS, steps, acc, [&](const auto &f, const auto &) {
                    if (summing) {
#pragma unroll
                        for (int t = 0; t < C::FA; ++t) sums[t] = T::sum(f[t], sums[t]);
                    }
                });
            });
    }
    const int l = threadIdx.x & 63;
    // through LDS to whole rows: value by value from the lanes that have them, 20 MB took 190 us
    float *result = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int part = 0; part < R::PARTS; ++part) {
        constexpr int W = R::W, V = T::VEC, PER_ROW = W / V, ROWS = kThreads / PER_ROW;
        if (part) __syncthreads();
        R::put(result, part, acc);
        __syncthreads();
        const int c = (int)(threadIdx.x % PER_ROW) * V, left = a.N - n0 - c;
        if (left > 0 && c < C::BB) {
            for (int r = threadIdx.x / PER_ROW; r < R::ROWS; r += ROWS) {
                const int64_t m = m0 + R::row(part, r);
                if (m >= a.M) continue;
                float v[V];
#pragma unroll
                for (int u = 0; u < V; u += 4) {
                    const f32x4 four = *reinterpret_cast<const f32x4 *>(result + result_place<W>(r, c + u));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[u + e] = four[e];
                }
                if (slot) write_row(slot + m * a.N + n0 + c, v, left, a.add, [](float x) { return x; });
                else write_row(a.out + m * a.out_stride + n0 + c, v, left, false, [](float x) { return T::put(x); });
            }
        }
    }
    if (summing) {
#pragma unroll
        for (int t = 0; t < C::FA; ++t) {
            const float v = down_column(sums[t], [](float p, float q) { return p + q; });
            const int64_t m = m0 + C::a_off() + 16 * t + (l & 15);
            if (l >= 16 || m >= a.M) continue;
            if (a.sum_slots) {
                float *to = a.sum_slots + share * a.slot_rows + m;
                *to = a.add ? *to + v : v;
            } else {
                a.sums[m] = T::put(v);
            }
        }
    }
}

// Both products of a piece in one launch, dW's workgroups first: they need nothing of each other, and each fills what the other leaves free at its end.
template <class T, class C, bool NARROW>
__global__ void __launch_bounds__(kThreads, 2) k_class_products(PieceArgs<T> dw, PieceArgs<T> dx, uint32_t dw_groups)
{
    using W = Product<T, C, true, NARROW>;
    using X = Product<T, C, false, NARROW>;
    __shared__ __attribute__((aligned(16))) uint32_t lds[W::LDS > X::LDS ? W::LDS : X::LDS];
    if (blockIdx.x < dw_groups) W::make(dw, blockIdx.x, lds);
    else X::make(dx, blockIdx.x - dw_groups, lds);
}

// Sums over ranges: of rows x width values, four of a row a thread, and of `rows` more (db).
template <class T>
struct ReduceArgs {
    const float *slots, *sum_slots;
    int64_t slot_rows, rows;       // of a slot (sum_slots: `rows`); of the result
    int slot_width, width, shares, sum_shares;
    typename T::elem *out, *sums;  // either may be null
    int64_t out_stride;
    const int32_t *exponent;       // null, or values times undo 2^exponent, sums times undo
    float undo;
};
// LANES neighbours share what there is to add: 1 for few ranges, 8 for many.
template <class T, int LANES>
__global__ void __launch_bounds__(256) k_class_reduce(ReduceArgs<T> one, ReduceArgs<T> two, uint32_t one_groups, uint32_t group0)
{
    constexpr int PER = 256 / LANES;
    __shared__ f32x4 meet[LANES > 1 ? LANES : 1][LANES > 1 ? PER : 1];
    const uint32_t group = group0 + blockIdx.x;
    const bool first = group < one_groups;
    const ReduceArgs<T> &a = first ? one : two;
    const int item = threadIdx.x % PER, lane = threadIdx.x / PER;
    const uint64_t i = (uint64_t)(first ? group : group - one_groups) * PER + item;
    const uint32_t fours = (uint32_t)(a.width + 3) / 4;
    const uint64_t values = a.out ? (uint64_t)a.rows * fours : 0;
    const bool value = i < values, sum = !value && a.sums && i - values < (uint64_t)a.rows;
    const uint64_t row = !value ? 0 : values >> 32 ? i / fours : (uint32_t)i / fours;
    const int c = value ? (int)(i - row * fours) * 4 : 0;
    f32x4 s = {};
    if (value) {
        const float *from = a.slots + row * a.slot_width + c;
        const int64_t step = a.slot_rows * a.slot_width;
        int p = lane;
        for (; p + 3 * LANES < a.shares; p += 4 * LANES) {  // (four on their way at a time)
            f32x4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = load_any<f32x4>(from + (p + u * LANES) * step);
#pragma unroll
            for (int u = 0; u < 4; ++u) s += v[u];
        }
        for (; p < a.shares; p += LANES) s += load_any<f32x4>(from + p * step);
    } else if (sum) {
        const float *from = a.sum_slots + (i - values);
        for (int p = lane; p < a.sum_shares; p += LANES) s[0] += from[p * a.rows];
    }
    if constexpr (LANES > 1) {
        meet[lane][item] = s;
        __syncthreads();
        if (lane > 0) return;
#pragma unroll
        for (int u = 1; u < LANES; ++u) s += meet[u][item];
    }
    if (value) {
        const float up = a.exponent ? ldexpf(a.undo, a.exponent[0]) : 1.0f;
        typename T::elem e[4], *to = a.out + row * a.out_stride + c;
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = T::put(s[j] * up);
        if (c + 4 <= a.width) {
            __builtin_memcpy(to, e, sizeof(e));
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (c + j < a.width) to[j] = e[j];
        }
    } else if (sum) {
        a.sums[i - values] = T::put(a.exponent ? s[0] * a.undo : s[0]);
    }
}
template <class T>
__global__ void __launch_bounds__(256) k_class_zero(typename T::elem *p, int64_t count)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) p[i] = T::put(0.0f);
}

// ----------------------------------------------------------------- large calls: operands laid out for bgl_stage.h
// Rows of D values as rows of planes, each `padded` wide, zeros behind D and in rows from `rows` to `all_rows`: of fp32 three planes of bf16, of bf16 as they are or halves.
template <class T>
struct LayArgs {
    const typename T::elem *from;
    int64_t stride, rows, all_rows;
    int D, padded;
    uint16_t *to;
    int32_t *exponent;  // backward, bf16: of halves; behind it `whole`
    // backward, x: rows without a gradient become zeros, whatever they hold
    bool select;
    const int32_t *labels;
    const float *saved;
    int saved_width, classes;
    bool by_label, by_teacher;
};
template <class T>
__device__ __forceinline__ bool lives(const LayArgs<T> &a, int64_t row)
{
    if (row >= a.rows) return false;
    if (!a.select) return true;
    return (a.by_label && (uint32_t)a.labels[row] < (uint32_t)a.classes) || (a.by_teacher && a.saved[row * a.saved_width + 2] != INFINITY);
}
__device__ __forceinline__ uint4 eight(const LayArgs<BF16> &a, int64_t row, int d)
{
    if (d >= a.D || !lives(a, row)) return uint4{0, 0, 0, 0};
    const uint16_t *from = a.from + row * a.stride + d;
    return d + 8 <= a.D ? load_any<uint4>(from) : load_end<BF16>(from, a.D - d, a.D);
}
template <class F>
__device__ __forceinline__ void each_eight(const LayArgs<BF16> &a, uint32_t group, uint32_t groups, F f)
{
    const uint64_t each = a.padded / 8, all = (uint64_t)a.all_rows * each;
    for (uint64_t i = (uint64_t)group * 256 + threadIdx.x; i < all; i += (uint64_t)groups * 256) {
        const uint64_t row = all >> 32 ? i / each : (uint32_t)i / (uint32_t)each;
        f((int64_t)row, (int)(i - row * each) * 8);
    }
}
__global__ void __launch_bounds__(256) k_class_lay(LayArgs<BF16> a)
{
    each_eight(a, blockIdx.x, gridDim.x, [&](int64_t row, int d) { *reinterpret_cast<uint4 *>(a.to + row * a.padded + d) = eight(a, row, d); });
}

// bf16 rows and weight as halves, for the backward call, whose dz is in halves: times 2^-exponent, one for all of x and one for all of W, so that the largest is
// in [2^14, 2^15) and a bf16's eight bits fit a half's from 2^-32 of it on; below, a value is off by 2^-39 of it at most.  That is as good as exact where no row (of x: with a
// gradient) is far smaller than another, and no score's products: where the rows' largest values are within 12 powers of two, and where what scores can be off by,
// 2^-38 D max|x| max|w| over the temperature, is below 2^-23.  Else (`whole`) x and W stay bf16 and dz is two of them, twice the products: of one row 2^32 above the others
// these lost everything (4,096 x 512 x 65,536 training: 1,305 us, so 1,951).  First the largest and smallest of kLayGroups groups of rows of each, then every workgroup finds
// exponent and choice from them.  65,536 and 4,096 rows of 512: 16 and 22 us.
constexpr int kLayGroups = 1024, kHalvesHead = 2 * kLayGroups * 4 + 256;
constexpr int kRowsApart = 12;             // powers of two
constexpr float kProductMost = 0x1p15f;    // D max|x| max|w|, at a temperature of 1
struct HalvesArgs {
    LayArgs<BF16> w, x;
    // of kLayGroups groups: of the rows' largest finite values the largest, and 0x7f80 less the smallest that is not 0 (as bits of a bf16)
    uint32_t *w_sizes, *x_sizes;
    float product_most;
};
__device__ __forceinline__ uint32_t largest_of(const uint4 &v)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = d[i] & 0x7fff, hi = d[i] >> 16 & 0x7fff;
        most = lo < 0x7f80 && lo > most ? lo : most;
        most = hi < 0x7f80 && hi > most ? hi : most;
    }
    return most;
}
// The largest over a workgroup, of COUNT numbers of up to 24 bits.
template <int COUNT>
__device__ __forceinline__ void group_largest(uint32_t (&v)[COUNT])
{
    __shared__ float all[COUNT][4];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const float w = max_across<64>((float)v[i]);
        if (threadIdx.x % 64 == 0) all[i][threadIdx.x / 64] = w;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = (uint32_t)fmaxf(fmaxf(all[i][0], all[i][1]), fmaxf(all[i][2], all[i][3]));
}
// TEAM lanes for a row, four rows on their way at a time.
template <int TEAM>
__global__ void __launch_bounds__(256) k_class_largest(HalvesArgs a)
{
    constexpr int TEAMS = 256 / TEAM, AHEAD = 4;
    const bool second = blockIdx.x >= kLayGroups;
    const LayArgs<BF16> &m = second ? a.x : a.w;
    const int group = blockIdx.x % kLayGroups, l = (int)threadIdx.x % TEAM;
    uint32_t v[2] = {};
    for (int64_t row = (int64_t)group * TEAMS + threadIdx.x / TEAM; row < m.rows; row += (int64_t)kLayGroups * TEAMS * AHEAD) {
        uint32_t most[AHEAD] = {};
        for (int d = l * 8; d < m.D; d += TEAM * 8) {
            uint4 u[AHEAD];
#pragma unroll
            for (int r = 0; r < AHEAD; ++r) u[r] = eight(m, row + (int64_t)r * kLayGroups * TEAMS, d);
#pragma unroll
            for (int r = 0; r < AHEAD; ++r) {
                const uint32_t of = largest_of(u[r]);
                most[r] = of > most[r] ? of : most[r];
            }
        }
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            const uint32_t of = (uint32_t)max_across<TEAM>((float)most[r]), under = of ? 0x7f80 - of : 0;
            v[0] = of > v[0] ? of : v[0], v[1] = under > v[1] ? under : v[1];
        }
    }
    group_largest(v);
    uint32_t *to = (second ? a.x_sizes : a.w_sizes) + group;
    if (threadIdx.x == 0) to[0] = v[0], to[kLayGroups] = v[1];
}
__global__ void __launch_bounds__(256) k_class_halves(HalvesArgs a, uint32_t w_groups)
{
    const bool second = blockIdx.x >= w_groups;
    const LayArgs<BF16> &m = second ? a.x : a.w;
    uint32_t v[4] = {};  // of w, of x
#pragma unroll
    for (int i = 0; i < kLayGroups / 256; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t of = (j < 2 ? a.w_sizes : a.x_sizes)[j % 2 * kLayGroups + i * 256 + threadIdx.x];
            v[j] = of > v[j] ? of : v[j];
        }
    group_largest(v);
    const auto value = [](uint32_t bits) { return __uint_as_float(bits << 16); };
    bool whole = !(value(v[0]) * value(v[2]) * (float)m.D <= a.product_most);
#pragma unroll
    for (int i = 0; i < 4; i += 2)  // (below 2^-101 exponents end)
        if (v[i] > 0) whole |= (int)(v[i] >> 7) - (int)((0x7f80 - v[i + 1]) >> 7) > kRowsApart || value(v[i]) < 0x1p-101f;
    const float most = value(v[second ? 2 : 0]);
    const int exponent = !whole && most > 0.0f ? ilogbf(most) - 14 : 0;
    const uint32_t group = second ? blockIdx.x - w_groups : blockIdx.x;
    if (group == 0 && threadIdx.x == 0) m.exponent[0] = exponent, m.exponent[1] = whole;
    const float scale = ldexpf(1.0f, -exponent);
    each_eight(m, group, second ? gridDim.x - w_groups : w_groups, [&](int64_t row, int d) {
        uint4 v = eight(m, row, d);
        if (!whole) {
            const uint32_t in[4] = {v.x, v.y, v.z, v.w};
            _Float16 h[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                h[2 * j] = (_Float16)(__uint_as_float(in[j] << 16) * scale);
                h[2 * j + 1] = (_Float16)(__uint_as_float(in[j] & 0xffff0000u) * scale);
            }
            v = __builtin_bit_cast(uint4, h);
        }
        *reinterpret_cast<uint4 *>(m.to + row * m.padded + d) = v;
    });
}
// A wavefront for a row.  50,001 x 256: 22 us (128 MB, 5.9 TB/s).
__global__ void __launch_bounds__(256) k_class_split(LayArgs<F32> a, int64_t row0)
{
    const int64_t row = row0 + (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    const int l = threadIdx.x & 63;
    if (row >= a.all_rows) return;
    const bool live = lives(a, row);
    const float *from = a.from + (live ? row : 0) * a.stride;
    for (int d = 4 * l; d < a.padded; d += 256) {
        f32x4 v = {};
        if (live && d < a.D) v = __builtin_bit_cast(f32x4, d + 4 <= a.D ? load_any<uint4>(from + d) : load_end<F32>(from + d, a.D - d, a.D));
        uint16_t e[3][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint16_t three[3];
            split(v[j], three);
#pragma unroll
            for (int p = 0; p < 3; ++p) e[p][j] = three[p];
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2 *>(a.to + (row * 3 + p) * a.padded + d) = __builtin_bit_cast(uint2, e[p]);
    }
}

// k_class_scores from laid out operands: 192 classes x 128 rows, the largest tile of which two workgroups fit a CU: one's exponentials beside the other's products (a training
// call of 4,096 x 512 x 65,536 bf16 took 1,278 us with 128 x 128, 1,227 so).  4,096 x 512 x 65,536 bf16: 334 us, 820 TFLOP/s with the exponentials (a plain library product
// of 4,096 x 512 x 16,384 makes 831); backward 193 us for half of the classes, 710 TFLOP/s and 268 MB of dz.  1,024 x 256 x 50,001 f32: 177 us, 890 TFLOP/s of its six
// products of bf16; backward 229, with 307 MB of dz.  (From two halves of a value scaled by its row's largest, three products, these took 103 and 162: 22 bits, and what was
// far below the row's largest lost all of them, so that a large column with small weights beside it made other columns' products wrong.)
template <class T>
struct StageScoreArgs {
    ScoreArgs<T> s;
    const char *x, *w;           // of the call's first row, of class 0: three planes of bf16, or bf16 or halves
    int64_t x_bytes, w_bytes;    // rows
    uint32_t plane;              // bytes
    const int32_t *x_exponent, *w_exponent;  // of halves, and `whole` behind each
    // forward, or null: the teacher's classes, n x top, whose scores go to z_top
    const int32_t *top_class;
    float *z_top;
    int top, z_stride;
};

template <class T, bool DZ>
__global__ void __launch_bounds__(stage::kThreads, 2) k_class_scores_stage(StageScoreArgs<T> q)
{
    using C = StageCut;
    using A = stage::Kc<C::BA, kPad>;
    using B = stage::Kc<C::BB, kPad>;
    constexpr bool CHOICE = T::PER == 2 && DZ;
    constexpr stage::Kind READ = T::PER == 1 ? stage::THREE_BF16 : DZ ? stage::ONE_HALF : stage::ONE_BF16;
    __shared__ __attribute__((aligned(1024))) char lds[stage::lds_bytes<A, B>()];
    const ScoreArgs<T> &a = q.s;
    int64_t ct, rt;
    int fast;
    const uint32_t slow_tiles = a.by_rows ? (uint32_t)a.row_tiles : a.class_tiles, fast_tiles = a.by_rows ? a.class_tiles : (uint32_t)a.row_tiles;
    if (!stage::tile_of(blockIdx.x, slow_tiles, fast_tiles, a.by_rows ? 1 : kClassGroup, a.by_rows ? rt : ct, fast)) return;
    (a.by_rows ? ct : rt) = fast;
    const int c0 = a.class0 + (int)ct * C::BA, last = a.classes - 1, l = threadIdx.x & 63;
    const int64_t r0 = rt * C::BB;
    A weight;
    B rows;
    weight.init(q.w + c0 * q.w_bytes, [&](int i) { return (uint32_t)((c0 + i < last ? i : last - c0) * q.w_bytes); });
    rows.init(q.x + (a.row0 + r0) * q.x_bytes, [&](int i) { return (uint32_t)((r0 + i < a.rows ? i : (int)(a.rows - 1 - r0)) * q.x_bytes); });
    // what the tile's classes and rows have of their own: a value for each thread, on its way during the products
    static_assert(C::BA <= stage::kThreads && C::BB <= stage::kThreads, "");
    float my_bias = 0.0f, my_most = INFINITY, my_sum = INFINITY, my_sum_t = INFINITY;  // (+inf: everything is 2^-inf of it, nothing has a share)
    int my_label = -1;
    if (a.bias && threadIdx.x < C::BA) my_bias = T::get(a.bias[c0 + (int)threadIdx.x < last ? c0 + (int)threadIdx.x : last]);
    if (threadIdx.x < C::BB && r0 + threadIdx.x < a.rows) {
        const int64_t row = a.row0 + r0 + threadIdx.x;
        if (a.labels) my_label = a.labels[row];
        if constexpr (DZ) {
            my_most = a.saved[row * a.saved_width];
            if (a.scale != 0.0f) my_sum = a.saved[row * a.saved_width + 1];
            if (a.teacher_scale != 0.0f) my_sum_t = a.saved[row * a.saved_width + 2];
        }
    }
    f32x4 acc[C::FA][C::FB] = {};
    const stage::Walk walk{2 * kPad, 2 * kPad, q.plane, q.plane, a.D, 0};
    const auto nothing = [](int, int, const auto &) {};
    const bool whole = CHOICE && q.w_exponent[1];
    if (CHOICE && whole) stage::multiply<stage::ONE_BF16, false, A, B, C>(lds, weight, rows, walk, acc, nothing);
    else stage::multiply<READ, false, A, B, C>(lds, weight, rows, walk, acc, nothing);

    if ((uint32_t)my_label >= (uint32_t)a.all_classes) my_label = -1, my_sum = INFINITY;
    if (my_sum == INFINITY && my_sum_t == INFINITY) my_most = INFINITY;  // (whatever such a row holds)
    struct Own {
        float bias[C::BA], shift[C::BB], base[C::BB], base_t[C::BB], share[C::BB], share_t[C::BB];
        int label[C::BB];
    };
    struct Meet {
        float own[C::BB], part[2][2][C::BB];  // the label's score; largest value and sum of both halves of the classes
    };
    static_assert(sizeof(Own) + sizeof(Meet) <= sizeof(lds), "");
    Own &own = *reinterpret_cast<Own *>(lds);
    Meet &meet = *reinterpret_cast<Meet *>(lds + sizeof(Own));
    if (threadIdx.x < C::BA) own.bias[threadIdx.x] = my_bias;
    if (threadIdx.x < C::BB) {
        own.label[threadIdx.x] = my_label;
        if constexpr (DZ) {
            const Base to = my_most == INFINITY ? Base{0.0f, INFINITY, INFINITY} : base_of(a, my_most);
            own.shift[threadIdx.x] = to.shift, own.base[threadIdx.x] = to.base, own.base_t[threadIdx.x] = to.base_t;
            own.share[threadIdx.x] = 1.0f / my_sum, own.share_t[threadIdx.x] = a.teacher_scale / my_sum_t;
        }
    }
    __syncthreads();
    const float all_up = READ == stage::ONE_HALF ? ldexpf(1.0f, q.w_exponent[0] + q.x_exponent[0]) : 1.0f;
    const int in_tile = C::a_off() + 4 * (l >> 4), first = c0 + in_tile;
#pragma unroll
    for (int i = 0; i < C::FA; ++i) {
        const f32x4 b = *reinterpret_cast<const f32x4 *>(own.bias + in_tile + 16 * i);
#pragma unroll
        for (int t = 0; t < C::FB; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (READ == stage::ONE_HALF) acc[i][t][j] = fmaf(acc[i][t][j], all_up, b[j]);
                else acc[i][t][j] += b[j];
            }
    }
    if (c0 + C::BA > a.classes) {
#pragma unroll
        for (int i = 0; i < C::FA; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (first + 16 * i + j > last) {
#pragma unroll
                    for (int t = 0; t < C::FB; ++t) acc[i][t][j] = -INFINITY;
                }
    }
    if constexpr (!DZ) {
        if (q.top_class) {
            // scores of the teacher's classes: 64 rows of the tile at a time in LDS, four threads for a row (50,000 x 256 x 1,001 bf16 with 16 classes and labels: 81 us; 92
            // with k_class_top, which reads their weights once more.  4,096 x 512 x 10,003 with 32: 79 and 80; x 40,003: 250 and 228)
            constexpr int WIDE = C::BA + 4, ROWS = C::BB / 2, EACH = stage::kThreads / ROWS, AHEAD = 4;
            static_assert(C::FB == 4 && sizeof(Own) + sizeof(Meet) + ROWS * WIDE * 4 <= sizeof(lds), "");
            float *z = reinterpret_cast<float *>(lds + sizeof(Own) + sizeof(Meet));
            const int at = threadIdx.x / EACH;
#pragma unroll
            for (int pass = 0; pass < 2; ++pass) {
                const int64_t r = r0 + at / 32 * 64 + pass * 32 + at % 32, row = a.row0 + r;
                const int k0 = threadIdx.x % EACH, mine = r < a.rows ? q.top : 0;
                const int32_t *classes = q.top_class + row * q.top;
                int c[AHEAD];
                const auto ask = [&](int k) {
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) c[u] = k + u * EACH < mine ? classes[k + u * EACH] : 0;
                };
                ask(k0);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < C::FA; ++i)
                        *reinterpret_cast<f32x4 *>(z + (C::b_off() / 2 + 16 * u + (l & 15)) * WIDE + in_tile + 16 * i) = acc[i][2 * pass + u];
                __syncthreads();
                for (int k = k0; k < mine; k += AHEAD * EACH) {
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        const bool there = (uint32_t)c[u] < (uint32_t)a.all_classes;
                        const bool here = there ? (uint32_t)(c[u] - c0) < (uint32_t)C::BA : ct == 0;
                        if (k + u * EACH < mine && here) q.z_top[row * q.z_stride + k + u * EACH] = there ? z[at * WIDE + c[u] - c0] : 0.0f;
                    }
                    ask(k + AHEAD * EACH);
                }
                __syncthreads();
            }
        }
    }
    const bool teachers = DZ && a.teacher_scale != 0.0f, labels = a.labels != nullptr && (!DZ || a.scale != 0.0f);
    const auto end = [&](auto form) {
#pragma unroll
    for (int t = 0; t < C::FB; ++t) {
        const int b = C::b_off() + 16 * t + (l & 15);
        const int64_t r = r0 + b;
        // the label's place among the lane's values; few tiles have one, and only these look for it
        const int at = labels ? own.label[b] - first : -1;
        const bool mine = at >= 0 && at < 16 * C::FA && (at & 15) < 4, any = __ballot(mine) != 0;
        const auto own_score = [&](int t) {
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < C::FA; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) v = at == 16 * i + j ? acc[i][t][j] : v;
            return v;
        };
        if constexpr (!DZ) {
            float most = -INFINITY, sum = 0.0f, sum_t = 0.0f;
#pragma unroll
            for (int i = 0; i < C::FA; ++i) most = max3(max3(most, acc[i][t][0], acc[i][t][1]), acc[i][t][2], acc[i][t][3]);
            most = down_column(most, [](float p, float q) { return fmaxf(p, q); });
            const Base to = base_of(a, most);
            if (any) {
                const float v = own_score(t);
                if (mine && a.whole) meet.own[b] = v;
                else if (mine && r < a.rows) a.label_score[a.row0 + r] = v;
            }
            if (__any(to.shift != 0.0f)) take_shift<C>(acc, t, to.shift);
#pragma unroll
            for (int i = 0; i < C::FA; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += power_to(acc[i][t][j], a.k, to.base);
            if (a.two) {
#pragma unroll
                for (int i = 0; i < C::FA; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum_t += power_to(acc[i][t][j], a.k_t, to.base_t);
            }
            sum = down_column(sum, [](float p, float q) { return p + q; });
            if (a.two) sum_t = down_column(sum_t, [](float p, float q) { return p + q; });
            const int half = C::a_off() / (16 * C::FA);
            if (a.whole) {
                if (l < 16) meet.part[0][half][b] = most, meet.part[1][half][b] = sum;
            } else if (l < 16 && r < a.rows) {
                const int64_t at = (ct * 2 + half) * a.rows + r;
                a.part[at] = float2{most, sum};
                if (a.two) a.part_t[at] = sum_t;
            }
        } else {
            constexpr bool WHOLE = decltype(form)::value;
            constexpr int planes = T::PER == 1 ? 3 : WHOLE ? 2 : 1;
            const float shift = own.shift[b], base = own.base[b], base_t = own.base_t[b], share = a.scale * own.share[b], share_t = own.share_t[b];
            if (__any(shift != 0.0f)) take_shift<C>(acc, t, shift);
#pragma unroll
            for (int i = 0; i < C::FA; ++i) {
                float d[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) d[j] = share * power_to(acc[i][t][j], a.k, base);
                if (teachers) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = fmaf(share_t, power_to(acc[i][t][j], a.k_t, base_t), d[j]);
                }
                uint16_t *to = reinterpret_cast<uint16_t *>(a.dz) + dz_block(r, first - a.class0 + 16 * i, a.dz_stride, planes);
                uint16_t e[planes][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint16_t one[3];
                    parts<T>(d[j], WHOLE, one);
#pragma unroll
                    for (int p = 0; p < planes; ++p) e[p][j] = one[p];
                }
#pragma unroll
                for (int p = 0; p < planes; ++p) __builtin_memcpy(to + p * kBlockValues, e[p], sizeof(e[p]));
            }
            if (any) {  // the label's class again, with the label
                const float v = own_score(t);
                float d = a.scale * (power_to(v, a.k, base) * own.share[b] - 1.0f);
                if (teachers) d = fmaf(share_t, power_to(v, a.k_t, base_t), d);
                uint16_t e[3], *to = reinterpret_cast<uint16_t *>(a.dz) + dz_block(r, first - a.class0 + (mine ? at : 0), a.dz_stride, planes);
                parts<T>(d, WHOLE, e);
                if (mine) {
#pragma unroll
                    for (int p = 0; p < planes; ++p) to[p * kBlockValues] = e[p];
                }
            }
        }
    }
    };
    if (CHOICE && whole) end(std::true_type{});
    else end(std::false_type{});
    if constexpr (!DZ) {
        // (204,800 x 256 x 150 bf16: 46 us with a launch of k_class_finish)
        if (!a.whole) return;
        __syncthreads();
        const int b = threadIdx.x;
        if (b >= C::BB || r0 + b >= a.rows) return;
        const int64_t row = a.row0 + r0 + b;
        const float most = fmaxf(meet.part[0][0][b], meet.part[0][1][b]);
        const Base to = base_of(a, most);
        float sum = 0.0f;
#pragma unroll
        for (int half = 0; half < 2; ++half) sum += meet.part[1][half][b] * rebase(a, meet.part[0][half][b], to);
        const float log_sum = log2f(sum);
        if (a.loss) a.loss[row] = my_label >= 0 ? loss_of(a, log_sum, meet.own[b], to) : 0.0f;
        if (a.kept) keep(a.kept + row * a.saved_width, a.saved_width, most, sum, INFINITY);
    }
}

// k_class_products from laid out operands: 256 x 128 (eight wavefronts with 256 x 256, one workgroup a CU, were slower).  OC: dW, else dx.  Both products of 4,096 rows, 512 columns and
// 32,768 classes, bf16: 300 us, 920 TFLOP/s; of 1,024, 256 and 50,001, f32: 398 us, 790 TFLOP/s of six bf16 products for one.
template <class T>
struct StagePieceArgs {
    const char *a, *b;                 // dz, in blocks; W or x
    int64_t b_bytes;                   // rows
    uint32_t b_plane;
    int64_t M, K;                      // (dW: rows up to a multiple of 32)
    int N, a_stride, b_width;          // columns of the result, of dz, and of the other that can be read
    int a_rows;                        // of dz, a multiple of 16
    int64_t row_tiles;
    int col_tiles, shares;
    int64_t per_share;                 // a multiple of 32
    typename T::elem *out;
    int64_t out_stride;
    const int32_t *exponent;           // bf16: of b, and `whole`
    float undo;                        // 1 over what dz was multiplied by: the result is the product times this and 2^exponent
    float *slots, *sum_slots;          // (both without that)  sums: shares x min(kSummers, column tiles) x 2 of them
    int64_t slot_rows;                 // of a slot, a multiple of the tiles' as slot_width is
    int slot_width;
    bool add;
};

// dz's sums over the rows are made by the tiles of the first columns and both halves of their wavefronts in turn, a stage each: made by one of them they took a
// seventh of the whole product's time.
constexpr int kSummers = 4;

template <stage::Kind KIND>
__device__ __forceinline__ float sum_of(const uint4 &v, float s)
{
    if constexpr (KIND == stage::ONE_HALF) {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        const f16x2 ones = {(_Float16)1.0f, (_Float16)1.0f};
        const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, d[i]), ones, s, false);
        return s;
    } else {
        return BF16::sum({v.x, v.y, v.z, v.w}, s);
    }
}

template <class T, bool OC>
struct StageProduct {
    using C = ProductCut;
    using A = std::conditional_t<OC, stage::OcBlocks<C::BA>, stage::Kc<C::BA, kBlockClasses>>;
    using B = stage::Oc<C::BB>;
    static constexpr int LDS = stage::lds_bytes<A, B>();
    template <stage::Kind KIND>
    static __device__ __forceinline__ void make(const StagePieceArgs<T> &a, uint32_t id, char *lds);
};
template <class T, bool OC>
template <stage::Kind KIND>
__device__ __forceinline__ void StageProduct<T, OC>::make(const StagePieceArgs<T> &a, uint32_t id, char *lds)
{
    constexpr int PLANES = stage::Pairs<KIND>::PLANES;
    const int share = (int)(id % (uint32_t)a.shares);
    int64_t rt;
    int ct;
    if (!stage::tile_of(id / (uint32_t)a.shares, (uint32_t)a.row_tiles, a.col_tiles, 1, rt, ct)) return;
    const int64_t m0 = rt * C::BA, k0 = share * a.per_share;
    const int n0 = ct * C::BB, K = (int)(a.K - k0 < a.per_share ? a.K - k0 : a.per_share);
    A left;
    B right;
    // dz's blocks: 16 rows of it, one block
    constexpr uint32_t BLOCK = kBlockValues * 2 * PLANES;
    const uint32_t down = a.a_stride / kBlockClasses * BLOCK;
    if constexpr (OC) {
        left.init(a.a + k0 / kBlockRows * down, down, BLOCK, (int)(m0 / kBlockClasses), a.a_stride / kBlockClasses);
    } else {
        left.init(a.a + m0 / kBlockRows * down + k0 / kBlockClasses * BLOCK, [&](int i) {
            const int most = (int)((a.a_rows - m0) / kBlockRows) - 1;
            return (uint32_t)((i / kBlockRows < most ? i / kBlockRows : most) * down + i % kBlockRows * kBlockClasses * 2);
        });
    }
    const uint32_t a_block = OC ? 2 * down : BLOCK;
    right.init(a.b + k0 * a.b_bytes, (uint32_t)a.b_bytes, n0, a.b_width);
    f32x4 acc[C::FA][C::FB] = {};
    const int l = threadIdx.x & 63;
    // slots are whole tiles: nothing of theirs is beyond an edge.  What is there already goes before the products.
    float *slot = a.slots ? a.slots + (share * a.slot_rows + m0 + C::a_off() + (l & 15)) * a.slot_width + n0 + C::b_off() + 4 * (l >> 4) : nullptr;
    if (slot && a.add) {
#pragma unroll
        for (int i = 0; i < C::FA; ++i)
#pragma unroll
            for (int t = 0; t < C::FB; ++t) acc[i][t] = *reinterpret_cast<const f32x4 *>(slot + 16 * i * (int64_t)a.slot_width + 16 * t);
    }
    float sums[C::FA] = {};
    const int summers = a.col_tiles < kSummers ? a.col_tiles : kSummers, summer = 2 * ct + (C::b_off() > 0);
    const bool summing = OC && a.sum_slots && ct < summers;
    const stage::Walk walk{a_block, (uint32_t)(A::STEP * a.b_bytes), kBlockValues * 2, a.b_plane, K, 0};
    stage::multiply<KIND, true, A, B, C>(lds, left, right, walk, acc, [&](int s, int b_plane, const auto &f) {
        if (summing && b_plane == 0 && s / stage::Pairs<KIND>::COUNT % (2 * summers) == summer) {
#pragma unroll
            for (int t = 0; t < C::FA; ++t) {
                const uint4 v = __builtin_bit_cast(uint4, f[t]);
                sums[t] = sum_of<KIND>(v, sums[t]);
            }
        }
    });
    const int64_t m1 = m0 + C::a_off() + (l & 15);
    const int c1 = n0 + C::b_off() + 4 * (l >> 4);
    if (slot) {
#pragma unroll
        for (int i = 0; i < C::FA; ++i)
#pragma unroll
            for (int t = 0; t < C::FB; ++t) *reinterpret_cast<f32x4 *>(slot + 16 * i * (int64_t)a.slot_width + 16 * t) = acc[i][t];
    } else {
        typename T::elem *to = a.out + m1 * a.out_stride + c1;
        const float up = a.exponent ? ldexpf(a.undo, a.exponent[0]) : 1.0f;
#pragma unroll
        for (int i = 0; i < C::FA; ++i) {
            if (m1 + 16 * i >= a.M) break;
#pragma unroll
            for (int t = 0; t < C::FB; ++t) {
                typename T::elem e[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) e[j] = T::put(acc[i][t][j] * up);
                if (c1 + 16 * t < a.N) __builtin_memcpy(to + 16 * t, e, sizeof(e));  // (N is a multiple of 4)
            }
            to += 16 * a.out_stride;
        }
    }
    if (summing) {
#pragma unroll
        for (int t = 0; t < C::FA; ++t) {
            const float v = down_column(sums[t], [](float p, float q) { return p + q; });
            const int64_t m = m0 + C::a_off() + 16 * t + (l & 15);
            if (l >= 16 || m >= a.M) continue;
            float *to = a.sum_slots + ((int64_t)share * 2 * summers + summer) * a.M + m;
            *to = a.add ? *to + v : v;
        }
    }
}

template <class T>
__global__ void __launch_bounds__(stage::kThreads, 2) k_class_products_stage(StagePieceArgs<T> dw, StagePieceArgs<T> dx, uint32_t dw_groups)
{
    using W = StageProduct<T, true>;
    using X = StageProduct<T, false>;
    __shared__ __attribute__((aligned(1024))) char lds[W::LDS > X::LDS ? W::LDS : X::LDS];
    if constexpr (T::PER == 1) {
        if (blockIdx.x < dw_groups) W::template make<stage::THREE_BF16>(dw, blockIdx.x, lds);
        else X::template make<stage::THREE_BF16>(dx, blockIdx.x - dw_groups, lds);
    } else if (blockIdx.x < dw_groups) {
        if (dw.exponent[1]) W::template make<stage::TWO_BF16>(dw, blockIdx.x, lds);
        else W::template make<stage::ONE_HALF>(dw, blockIdx.x, lds);
    } else {
        if (dx.exponent[1]) X::template make<stage::TWO_BF16>(dx, blockIdx.x - dw_groups, lds);
        else X::template make<stage::ONE_HALF>(dx, blockIdx.x - dw_groups, lds);
    }
}

// ----------------------------------------------------------------- plans
using Large = Cut<2, 2, 4, 4>;   // 128 x 128
using Middle = Cut<2, 2, 4, 2>;  // 128 x 64
using Low = Cut<4, 1, 2, 1>;     // 128 x 16
using Slim = Cut<4, 1, 1, 1>;    // 64 x 16
using Small = Cut<2, 2, 2, 2>;   // 64 x 64
using Flat = Cut<1, 4, 1, 2>;    // 16 x 128
using Flat2 = Cut<1, 4, 2, 2>;   // 32 x 128
using Flat4 = Cut<1, 4, 4, 2>;   // 64 x 128

uint32_t groups_for(int64_t groups) { return (uint32_t)(groups < kMostThreads / 256 ? groups : kMostThreads / 256); }  // (of kernels that go round)

struct Plan {
    // forward
    int64_t pass_rows;
    int class_parts;
    size_t part_bytes, label_bytes, top_bytes, forward_bytes;
    // backward
    int64_t piece_rows, row_pieces, dz_stride;
    int piece_classes, class_pieces, dx_shares, dx_tile, slot_width;
    size_t dz_bytes, list_bytes, dx_bytes, dw_bytes, db_bytes, backward_bytes;
    // large calls: laid out operands, forward (0: as they are) and backward
    int padded;
    size_t x_bytes, w_bytes, back_x_bytes, back_w_bytes;
};

// How a call is cut up.  Small ones: tiles of 128 x 128 straight from the operands.  Large ones: larger tiles of operands laid out for bgl_stage.h (bf16 whose rows
// are whole steps are laid out already).
struct Scheme {
    bool large;
    int score_classes, product_rows;  // of a tile
    int64_t values, round_classes, round_rows;
    int dz_value_bytes, planes;
    int slot_round;                   // rows of a slot
    int64_t fill, least;              // ranges of a product's summed index: workgroups they are to make together, of the index for each
};
Scheme scheme_of(const bgl_class_loss_t *l, bool large)
{
    const bool f32 = l->dtype == BGL_F32;
    const int64_t values = ((int64_t)1 << 27) + ((int64_t)1 << 23);
    if (large) return Scheme{true, StageCut::BA, ProductCut::BA, values, StageCut::BA, StageCut::BB, f32 ? 6 : 4, f32 ? 3 : 1, ProductCut::BA, 2 * kCus, 512};
    return Scheme{false, 128, 128, (int64_t)1 << 25, 8, 1, 4, 1, 1, kCus, 64};  // (pieces of 4 classes are stored, and 16 bytes of bf16 read)
}
bool large_call(const bgl_class_loss_t *l, int64_t n)
{
    return n >= kLargeRows && l->classes >= kLargeClasses && (double)n * l->classes * l->in_dim >= kLargeProducts;
}
bool laid_out(const bgl_class_loss_t *l) { return l->dtype == BGL_BF16 && l->in_dim % kPad == 0; }

// Ranges of the summed index that a product of rows x cols is made in, and the tiles' rows: small calls take tiles of 16 x 128 for up to 16 rows (in 128 x 128 the
// matrix units worked for nothing: a row of 133 and 37,570 classes 60 us) and of 64 x 64 where 128 x 128 do not fill the GPU.
int shares_for(const Scheme &s, int64_t rows, int64_t cols, int64_t summed, int &tile)
{
    const int64_t most = summed / s.least;
    const auto fit = [&](int64_t tiles) {
        const int64_t want = s.fill / (tiles < 1 ? 1 : tiles);
        return want < 1 || most < 1 ? 1 : want < most ? want : most;
    };
    tile = !s.large && rows <= Flat::BA ? Flat::BA : s.product_rows;
    int64_t tiles = ceil_div(rows, tile) * ceil_div(cols, 128);
    if (!s.large && tile != Flat::BA && tiles * fit(tiles) < s.fill / 2) tile = 64, tiles = ceil_div(rows, 64) * ceil_div(cols, 64);
    return (int)fit(tiles);
}

// (rows are read four values at a time)
size_t slot_bytes(int64_t shares, int64_t rows, int64_t width) { return round_up((size_t)(shares * rows * width) * 4 + 16, 256); }
int64_t per_share(int64_t summed, int shares) { return (int64_t)round_up((size_t)ceil_div(summed, shares), 64); }
int shares_used(int64_t summed, int shares) { return (int)ceil_div(summed, per_share(summed, shares)); }  // (none is empty)

// dW of a piece of classes.
struct WeightPlan {
    int shares, tile;
    bool slots;
};
WeightPlan weight_plan(const bgl_class_loss_t *l, const Scheme &s, int classes, int64_t piece_rows, int64_t row_pieces)
{
    WeightPlan w{};
    w.shares = shares_for(s, classes, l->in_dim, piece_rows, w.tile);
    w.shares = piece_rows > 0 ? shares_used(piece_rows, w.shares) : 1;
    w.slots = w.shares > 1 || row_pieces > 1 || (s.large && l->in_dim % 4);  // (large tiles are written four values of a row at a time)
    return w;
}
int summers_of(const bgl_class_loss_t *l, const Scheme &s)
{
    const int64_t tiles = ceil_div(l->in_dim, ProductCut::BB);
    return s.large ? 2 * (int)(tiles < kSummers ? tiles : kSummers) : 1;
}

Plan plan_of(const bgl_class_loss_t *l, int64_t n, const Scheme &s)
{
    Plan p{};
    p.class_parts = (int)ceil_div(l->classes, s.score_classes) * (s.large ? 2 : 1);  // (tiles of 64 classes: only where one has them all)
    p.pass_rows = kPartialBytes / (12 * (int64_t)p.class_parts);
    p.pass_rows = p.pass_rows < 1024 ? 1024 : p.pass_rows / 128 * 128;
    const int64_t top_rows = kMostThreads / (2 * l->top + 8) / 128 * 128;  // (k_class_top's)
    if (p.pass_rows > top_rows) p.pass_rows = top_rows;
    if (p.pass_rows > n) p.pass_rows = n;
    p.part_bytes = round_up((size_t)p.pass_rows * p.class_parts * 12, 256);
    p.label_bytes = round_up((size_t)n * 4, 256);
    p.top_bytes = round_up((size_t)n * l->top * 4, 256);
    if (s.large) {
        p.padded = (int)round_up(l->in_dim, kPad);
        const auto bytes = [&](int64_t rows, bool back) {  // as stage_args lays them
            return round_up((size_t)rows * p.padded * 2 * s.planes, 256) + (back && l->dtype == BGL_BF16 ? kHalvesHead : 0);
        };
        const int64_t rows = round_up(n, 32);
        p.back_x_bytes = bytes(rows, true), p.back_w_bytes = bytes(l->classes, true);
        if (!laid_out(l)) p.x_bytes = bytes(rows, false), p.w_bytes = bytes(l->classes, false);
    }
    p.forward_bytes = p.part_bytes + p.label_bytes + p.top_bytes + p.x_bytes + p.w_bytes;

    // one piece if it is small enough; else all classes of some rows (dx is then written once and dW added up), and with very many classes some
    // classes of all rows, or of kPieceRows (dW is then written once for each of these, and dx added up); about equal ones
    const int64_t stride = round_up(l->classes, s.round_classes);
    p.piece_rows = n, p.piece_classes = l->classes;
    if (n * stride > s.values) {
        if (l->classes <= kPieceRows) {
            p.piece_rows = (int64_t)round_up((size_t)ceil_div(n, ceil_div(n * stride, s.values)), 128);
            if (p.piece_rows > n) p.piece_rows = n;
        } else {
            if (n > kPieceRows) p.piece_rows = kPieceRows;
            // whole rounds of dW's workgroups, if one fits (of 4,096 x 512: two pieces of 129 x 4 tiles took a third longer than two of 128 x 4)
            const int64_t round = s.fill / ceil_div(l->in_dim, 128) * s.product_rows, most = s.values / p.piece_rows;
            int64_t fit = (int64_t)round_up((size_t)ceil_div(stride, ceil_div(p.piece_rows * stride, s.values)), kPieceClasses);
            if (round > 0 && most >= round) fit = most / round * round;
            if (fit < l->classes) p.piece_classes = (int)fit;
        }
    }
    p.class_pieces = (int)ceil_div(l->classes, p.piece_classes);
    p.row_pieces = p.piece_rows > 0 ? ceil_div(n, p.piece_rows) : 0;
    p.dz_stride = round_up(p.piece_classes, s.round_classes);
    p.dz_bytes = round_up(round_up(p.piece_rows, s.round_rows) * p.dz_stride * s.dz_value_bytes, 256);
    p.list_bytes = s.large ? 0 : round_up((size_t)n * 4, 256);
    p.slot_width = s.large ? (int)round_up(l->in_dim, ProductCut::BB) : l->in_dim;
    p.dx_shares = shares_for(s, p.piece_rows, l->in_dim, p.piece_classes, p.dx_tile);
    p.dx_shares = p.class_pieces > 1 && p.row_pieces > 1 ? 1 : shares_used(p.piece_classes, p.dx_shares);
    const bool dx_slots = p.dx_shares > 1 || p.class_pieces > 1 || (s.large && l->in_dim % 4);
    const int64_t dx_rows = round_up(p.class_pieces > 1 ? n : p.piece_rows, s.slot_round);
    p.dx_bytes = dx_slots ? slot_bytes(p.dx_shares, dx_rows, p.slot_width) : 0;
    const int last = l->classes - (p.class_pieces - 1) * p.piece_classes;
    for (const int classes : {p.piece_classes, last}) {
        const WeightPlan w = weight_plan(l, s, classes, p.piece_rows, p.row_pieces);
        const size_t dw = w.slots ? slot_bytes(w.shares, round_up(classes, s.slot_round), p.slot_width) : 0;
        const size_t db = w.slots || s.large ? round_up((size_t)w.shares * summers_of(l, s) * classes * 4, 256) : 0;
        if (dw > p.dw_bytes) p.dw_bytes = dw;
        if (db > p.db_bytes) p.db_bytes = db;
    }
    p.backward_bytes = p.dz_bytes + p.list_bytes + p.dx_bytes + p.dw_bytes + p.db_bytes + p.back_x_bytes + p.back_w_bytes;
    return p;
}

// What the backward calls of up to n rows need: no call of fewer rows needs more.  (Tiles in several ranges are s.fill at most.)
size_t backward_room(const bgl_class_loss_t *l, int64_t n, const Scheme &s)
{
    const int64_t V = l->classes, D = l->in_dim, stride = round_up(V, s.round_classes), shared = s.fill * s.product_rows;
    const bool many = V > kPieceRows;
    const auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    const auto most = [](int64_t a, int64_t b) { return a > b ? a : b; };
    const int64_t over = (many ? kPieceClasses * least(n, kPieceRows) : 128 * stride) + 128 * least(stride, s.values);
    const Plan p = plan_of(l, n, s);
    const int64_t dz_values = least(round_up(n, 128) * stride, s.values + over);
    size_t bytes = round_up((size_t)dz_values * s.dz_value_bytes, 256) + round_up((size_t)n * 4, 256) + p.back_x_bytes + p.back_w_bytes;
    // (ranges of the summed index leave s.fill tiles at most; a result of one range is rounded up to tiles)
    const int64_t width = s.large ? round_up(D, ProductCut::BB) : D, up = s.slot_round;
    const bool odd = s.large && D % 4;
    if (V >= 2 * s.least || (many && n > 0) || odd) {
        const int64_t dx_shares = least(shared, round_up(n, up) * (V / s.least)), dx_pieces = many || odd ? round_up(n, up) : 0;
        bytes += slot_bytes(1, most(dx_pieces, dx_shares), width);
    }
    const int64_t shares = n >= 2 * s.least ? least(shared, round_up(V, up) * (n / s.least)) : 0;
    const int64_t of_many = n > kPieceRows ? s.values / kPieceRows + kPieceClasses : 0, of_few = n * stride > s.values ? V : 0;
    const int64_t pieces = round_up(many ? of_many : of_few, up), odd_pieces = odd ? round_up(V, up) : 0;
    const int64_t sums = most(most(most(shares, pieces), odd_pieces), s.large ? least(V, s.values / 128) : 0) * summers_of(l, s);
    bytes += slot_bytes(1, most(most(shares, pieces), odd_pieces), width) + round_up((size_t)sums * 4, 256);
    return bytes > p.backward_bytes ? bytes : p.backward_bytes;
}

template <class T, bool DZ>
void launch_scores(ScoreArgs<T> &s, hipStream_t st)
{
    const auto go = [&](auto cut) {
        using C = decltype(cut);
        s.class_tiles = (int)ceil_div(s.classes - s.class0, C::BA);
        s.row_tiles = ceil_div(s.rows, C::BB);
        s.by_rows = s.row_tiles > s.class_tiles;
        const int64_t tiles = s.by_rows ? stage::tile_count(s.row_tiles, s.class_tiles) : stage::tile_count(s.class_tiles, s.row_tiles);
        k_class_scores<T, C, DZ><<<dim3((unsigned)tiles), dim3(kThreads), 0, st>>>(s);
    };
    // the largest tiles that the rows fill and that leave no CU without one: 1,024 x 128 x 50 f32 took 15 us in 8 tiles of 128 x 128
    const int64_t classes = s.classes - s.class0, across = ceil_div(classes, 128);
    // (13 classes of 32,780 rows of 266 f32 took 43 us in tiles of 128 classes)
    if (classes <= 64 && s.rows >= 128 * kCus / 4) {
        if (classes <= 16) go(Flat{});
        else if (classes <= 32) go(Flat2{});
        else go(Flat4{});
    } else if (s.rows > 64 && across * ceil_div(s.rows, 128) >= kCus) go(Large{});
    else if (s.rows > 16 && across * ceil_div(s.rows, 64) >= kCus) go(Middle{});
    else if (classes > 64) go(Low{});
    else go(Slim{});
}

struct Call {
    const bgl_class_loss_t *l;
    int64_t n;
    const void *x;
    int64_t x_stride;
    const void *weight, *bias;
    const int32_t *labels, *top_class;
    const float *top_score;
    char *workspace;
    hipStream_t stream;
};

float far_of(const bgl_class_loss_t *l) { return 0x1p24f / kLog2e * (l->temperature < 1.0f ? l->temperature : 1.0f); }  // (of the loss alone: both calls go by it)
int saved_width_of(const bgl_class_loss_t *l) { return l->top > 0 ? 3 + l->top : 2; }

template <class T>
RowArgs<T> row_args(const Call &c)
{
    using E = typename T::elem;
    RowArgs<T> r{};
    r.x = (const E *)c.x, r.w = (const E *)c.weight, r.bias = (const E *)c.bias, r.labels = c.labels, r.top_class = c.top_class, r.top_score = c.top_score;
    r.x_stride = c.x_stride, r.n = c.n, r.D = c.l->in_dim, r.classes = c.l->classes, r.top = c.l->top, r.saved_width = saved_width_of(c.l);
    r.t = c.l->temperature, r.over_t = 1.0f / c.l->temperature, r.k = kLog2e, r.k_t = (float)(1.4426950408889634 / c.l->temperature);
    r.far = far_of(c.l), r.two = c.top_class && c.l->temperature != 1.0f;
    return r;
}
template <class T>
ScoreArgs<T> score_args(const Call &c)
{
    using E = typename T::elem;
    ScoreArgs<T> s{};
    s.x = (const E *)c.x, s.w = (const E *)c.weight, s.bias = (const E *)c.bias, s.labels = c.labels, s.x_stride = c.x_stride, s.n = c.n;
    s.classes = s.all_classes = c.l->classes, s.D = c.l->in_dim, s.k = kLog2e, s.k_t = (float)(1.4426950408889634 / c.l->temperature);
    s.two = c.top_class && c.l->temperature != 1.0f;
    s.far = far_of(c.l), s.saved_width = saved_width_of(c.l);
    return s;
}

template <class T, bool DZ>
void launch_scores_stage(StageScoreArgs<T> &q, hipStream_t st)
{
    ScoreArgs<T> &s = q.s;
    s.class_tiles = (int)ceil_div(s.classes - s.class0, StageCut::BA);
    s.row_tiles = ceil_div(s.rows, StageCut::BB);
    s.by_rows = s.row_tiles > s.class_tiles;
    const int64_t tiles = s.by_rows ? stage::tile_count(s.row_tiles, s.class_tiles) : stage::tile_count(s.class_tiles, s.row_tiles);
    k_class_scores_stage<T, DZ><<<dim3((unsigned)tiles), dim3(stage::kThreads), 0, st>>>(q);
}

// rows of `all` rows, those behind `rows` zeros; select: rows without a gradient zeros too.
template <class T>
LayArgs<T> lay_args(const void *from, int64_t stride, int64_t rows, int64_t all, int D, int padded, const RowArgs<T> *select)
{
    LayArgs<T> a{};
    a.from = (const typename T::elem *)from, a.stride = stride, a.rows = rows, a.all_rows = all, a.D = D, a.padded = padded;
    if (select) {
        a.select = true, a.labels = select->labels, a.saved = select->saved, a.saved_width = select->saved_width, a.classes = select->classes;
        a.by_label = select->labels && select->scale != 0.0f, a.by_teacher = select->top_class && select->teacher_scale != 0.0f;
    }
    return a;
}

// Whether a call goes the large way: of what the forward call reads where it is, rows have to begin on multiples of 16 bytes.
bool goes_large(const Call &c, bool forward)
{
    if (!large_call(c.l, c.n)) return false;
    return !forward || !laid_out(c.l) || (aligned(c.weight, 16) && aligned(c.x, 16) && c.x_stride % 8 == 0 && c.x_stride < (int64_t)1 << 23);
}

// The laid out weight and rows, in the workspace from x and w on; what is laid out already is where it is.  select: the backward call's.
StageScoreArgs<F32> stage_args(const Call &c, const Plan &p, const ScoreArgs<F32> &s, char *x, char *w, const RowArgs<F32> *select)
{
    StageScoreArgs<F32> q{};
    q.s = s, q.plane = p.padded * 2, q.x_bytes = q.w_bytes = (int64_t)p.padded * 6;
    const auto lay = [&](LayArgs<F32> a, char *to) {
        a.to = (uint16_t *)to;
        const int64_t most = kMostThreads / 64;
        for (int64_t row0 = 0; row0 < a.all_rows; row0 += most) {
            const int64_t rows = a.all_rows - row0 < most ? a.all_rows - row0 : most;
            k_class_split<<<dim3((unsigned)ceil_div(rows, 4)), dim3(256), 0, c.stream>>>(a, row0);
        }
        return to;
    };
    q.w = lay(lay_args<F32>(s.w, s.D, s.classes, s.classes, s.D, p.padded, nullptr), w);
    q.x = lay(lay_args<F32>(s.x, s.x_stride, c.n, round_up(c.n, 32), s.D, p.padded, select), x);
    return q;
}
StageScoreArgs<BF16> stage_args(const Call &c, const Plan &p, const ScoreArgs<BF16> &s, char *x, char *w, const RowArgs<BF16> *select)
{
    StageScoreArgs<BF16> q{};
    q.s = s, q.plane = p.padded * 2;
    q.x_bytes = q.w_bytes = (int64_t)p.padded * 2;
    const LayArgs<BF16> lw = lay_args<BF16>(s.w, s.D, s.classes, s.classes, s.D, p.padded, nullptr);
    const LayArgs<BF16> lx = lay_args<BF16>(s.x, s.x_stride, c.n, round_up(c.n, 32), s.D, p.padded, select);
    if (select) {
        // shares of sizes, the exponent and the choice, the values
        HalvesArgs a{lw, lx, (uint32_t *)w, (uint32_t *)x, kProductMost * (c.l->temperature < 1.0f ? c.l->temperature : 1.0f)};
        const auto place = [&](LayArgs<BF16> &m, char *to, const char *&read, const int32_t *&exponent) {
            m.exponent = (int32_t *)(to + 2 * kLayGroups * 4), m.to = (uint16_t *)(to + kHalvesHead);
            read = to + kHalvesHead, exponent = m.exponent;
        };
        place(a.w, w, q.w, q.w_exponent), place(a.x, x, q.x, q.x_exponent);
        const auto groups = [&](const LayArgs<BF16> &m) {
            const int64_t all = ceil_div(m.all_rows * (p.padded / 8), 256);
            return (uint32_t)(all < 8 * kCus ? all : 8 * kCus);
        };
        if (s.D <= 64) k_class_largest<8><<<dim3(2 * kLayGroups), dim3(256), 0, c.stream>>>(a);
        else if (s.D <= 256) k_class_largest<32><<<dim3(2 * kLayGroups), dim3(256), 0, c.stream>>>(a);
        else k_class_largest<64><<<dim3(2 * kLayGroups), dim3(256), 0, c.stream>>>(a);
        k_class_halves<<<dim3(groups(a.w) + groups(a.x)), dim3(256), 0, c.stream>>>(a, groups(a.w));
        return q;
    }
    q.w = (const char *)s.w, q.x = (const char *)s.x;
    if (p.w_bytes) {
        const auto lay = [&](LayArgs<BF16> a, char *to) {
            a.to = (uint16_t *)to;
            k_class_lay<<<dim3(groups_for(ceil_div(a.all_rows * (p.padded / 8), 256))), dim3(256), 0, c.stream>>>(a);
            return to;
        };
        q.w = lay(lw, w), q.x = lay(lx, x);
    } else {
        q.w_bytes = (int64_t)s.D * 2, q.x_bytes = s.x_stride * 2;
    }
    return q;
}

template <class T>
int forward(const Call &c, float *loss, float *teacher_loss, float *saved)
{
    const Scheme h = scheme_of(c.l, goes_large(c, true));
    const Plan p = plan_of(c.l, c.n, h);
    ScoreArgs<T> s = score_args<T>(c);
    RowArgs<T> r = row_args<T>(c);
    char *ws = c.workspace;
    s.part = (float2 *)ws, s.part_t = (float *)(s.part + p.pass_rows * p.class_parts), s.label_score = (float *)(ws += p.part_bytes);
    char *top = ws += p.label_bytes, *x = ws += p.top_bytes, *w = ws += p.x_bytes;
    r.part = s.part, r.part_t = s.part_t, r.label_score = s.label_score;
    r.z_top = saved ? saved + 3 : (float *)top, r.z_stride = saved ? r.saved_width : r.top;
    r.loss = loss, r.teacher_loss = teacher_loss, r.saved = saved;
    if (!c.labels) s.k = r.k = s.k_t, s.two = r.two = false;  // (no sums but those at the temperature are asked for)
    StageScoreArgs<T> q{};
    if (h.large) {
        q = stage_args(c, p, s, x, w, nullptr);
        // (what the tiles would read of the teacher's classes and store, beside the classes' rows)
        const int64_t tiles = ceil_div(c.l->classes, StageCut::BA);
        if (c.top_class && tiles * (4 * r.top + kStoredBeside) < (int64_t)r.top * c.l->in_dim * (int64_t)sizeof(typename T::elem))
            q.top_class = c.top_class, q.top = r.top, q.z_top = r.z_top, q.z_stride = r.z_stride;
    }
    for (int64_t row0 = 0; row0 < c.n; row0 += p.pass_rows) {
        s.row0 = r.row0 = row0, s.rows = r.rows = c.n - row0 < p.pass_rows ? c.n - row0 : p.pass_rows;
        s.loss = loss, s.kept = saved, s.whole = !c.top_class && c.l->classes <= (h.large ? StageCut::BA : Large::BA);
        if (h.large) q.s = s, launch_scores_stage<T, false>(q, c.stream);
        else launch_scores<T, false>(s, c.stream);
        if (s.whole) continue;  // (every tile has all classes)
        const bool top_here = c.top_class && !q.top_class && r.top <= kTopHere && r.rows <= kTopRows && p.class_parts <= 32;
        if (c.top_class && !q.top_class && !top_here) k_class_top<T><<<dim3((unsigned)ceil_div(r.rows * ((r.top + 3) / 4), 32)), dim3(256), 0, c.stream>>>(r);
        r.class_parts = p.class_parts;
        if (r.class_parts > 32 && r.rows >= 64) {
            k_class_merge<T><<<dim3((unsigned)ceil_div(r.rows, kMergeRows)), dim3(kMergeRows * kMergeLanes), 0, c.stream>>>(r, s.part, s.part_t);
            r.class_parts = 1;
        }
        const int values = c.top_class && r.top > r.class_parts ? r.top : r.class_parts;
        if (top_here) k_class_finish<T, 16, true><<<dim3((unsigned)ceil_div(r.rows, 16)), dim3(256), 0, c.stream>>>(r);
        else if (values <= 8) k_class_finish<T, 4><<<dim3((unsigned)ceil_div(r.rows, 64)), dim3(256), 0, c.stream>>>(r);
        else if (values <= 32) k_class_finish<T, 16><<<dim3((unsigned)ceil_div(r.rows, 16)), dim3(256), 0, c.stream>>>(r);
        else k_class_finish<T, 64><<<dim3((unsigned)ceil_div(r.rows, 4)), dim3(256), 0, c.stream>>>(r);
    }
    BGL_HIP(hipGetLastError());
    return BGL_OK;
}

// dW of a piece, dx of it, or both; tile: its rows.
template <class T>
void launch_products(PieceArgs<T> *dw, PieceArgs<T> *dx, int tile, hipStream_t st)
{
    const auto go = [&](auto cut, auto narrow) {
        using C = decltype(cut);
        uint32_t groups[2] = {};
        for (int i = 0; i < 2; ++i)
            if (PieceArgs<T> *a = i ? dx : dw) {
                a->row_tiles = ceil_div(a->M, C::BA), a->col_tiles = (int)ceil_div(a->N, C::BB), a->tiles = (uint32_t)stage::tile_count(a->row_tiles, a->col_tiles);
                groups[i] = a->tiles * a->shares;
            }
        const PieceArgs<T> none{};
        k_class_products<T, C, decltype(narrow)::value><<<dim3(groups[0] + groups[1]), dim3(kThreads), 0, st>>>(dw ? *dw : none, dx ? *dx : none, groups[0]);
    };
    if ((dw ? dw : dx)->N < T::VEC) go(Small{}, std::true_type{});  // (one form of reading rows shorter than 16 bytes will do)
    else if (tile == Flat::BA) go(Flat{}, std::false_type{});
    else if (tile == Small::BA) go(Small{}, std::false_type{});
    else go(Large{}, std::false_type{});
}
template <class T>
void launch_products(StagePieceArgs<T> *dw, StagePieceArgs<T> *dx, hipStream_t st)
{
    uint32_t groups[2] = {};
    for (int i = 0; i < 2; ++i)
        if (StagePieceArgs<T> *a = i ? dx : dw) {
            a->row_tiles = ceil_div(a->M, ProductCut::BA), a->col_tiles = (int)ceil_div(a->N, ProductCut::BB);
            groups[i] = (uint32_t)(stage::tile_count(a->row_tiles, a->col_tiles) * a->shares);
        }
    const StagePieceArgs<T> none{};
    k_class_products_stage<T><<<dim3(groups[0] + groups[1]), dim3(stage::kThreads), 0, st>>>(dw ? *dw : none, dx ? *dx : none, groups[0]);
}
// Either may have nothing to do.
template <class T>
void launch_reduce(const ReduceArgs<T> &one, const ReduceArgs<T> &two, hipStream_t st)
{
    const bool many = (one.out && one.shares > 8) || (one.sums && one.sum_shares > 8) || (two.out && two.shares > 8);
    const auto groups = [&](const ReduceArgs<T> &a) {
        const int64_t items = (a.out ? a.rows * ceil_div(a.width, 4) : 0) + (a.sums ? a.rows : 0);
        return (uint32_t)ceil_div(items, many ? 32 : 256);
    };
    const uint32_t all = groups(one) + groups(two), most = kMostThreads / 256;
    for (uint32_t group0 = 0; group0 < all; group0 += most) {
        const uint32_t count = all - group0 < most ? all - group0 : most;
        if (many) k_class_reduce<T, 8><<<dim3(count), dim3(256), 0, st>>>(one, two, groups(one), group0);
        else k_class_reduce<T, 1><<<dim3(count), dim3(256), 0, st>>>(one, two, groups(one), group0);
    }
}

template <class T>
int backward(const Call &c, const float *saved, float scale, float teacher_scale, void *dx_, int64_t dx_stride, void *dweight_, void *dbias_)
{
    using E = typename T::elem;
    E *dx = (E *)dx_, *dweight = (E *)dweight_, *dbias = (E *)dbias_;
    const int D = c.l->in_dim, V = c.l->classes;
    if (c.n == 0) {
        const auto zero = [&](E *to, int64_t count) { k_class_zero<T><<<dim3(groups_for(ceil_div(count, 256))), dim3(256), 0, c.stream>>>(to, count); };
        if (dweight) zero(dweight, (int64_t)V * D);
        if (dbias) zero(dbias, V);
        BGL_HIP(hipGetLastError());
        return BGL_OK;
    }
    const Scheme h = scheme_of(c.l, goes_large(c, false));
    const Plan p = plan_of(c.l, c.n, h);
    char *ws = c.workspace;
    E *dz = (E *)ws;
    int32_t *listed = (int32_t *)(ws += p.dz_bytes);
    float *dx_slots = (float *)(ws += p.list_bytes), *dw_slots = (float *)(ws += p.dx_bytes), *db_slots = (float *)(ws += p.dw_bytes);
    char *x_laid = ws += p.db_bytes, *w_laid = ws += p.back_x_bytes;
    ScoreArgs<T> s = score_args<T>(c);
    RowArgs<T> r = row_args<T>(c);
    s.saved = saved, s.dz = dz, s.dz_stride = (int)p.dz_stride;
    s.scale = r.scale = c.labels ? scale : 0.0f;
    s.teacher_scale = r.teacher_scale = c.top_class ? teacher_scale * c.l->temperature : 0.0f;
    r.saved = const_cast<float *>(saved), r.dz = dz, r.dz_stride = (int)p.dz_stride, r.blocks = h.large;
    s.dz_rest = r.dz_rest = dz + p.piece_rows * p.dz_stride;  // (small calls of bf16)
    StageScoreArgs<T> q{};
    float undo = 1.0f;
    if (h.large) {
        q = stage_args(c, p, s, x_laid, w_laid, &r);
        r.whole = T::PER == 2 ? q.w_exponent + 1 : nullptr;
        if (T::PER == 2) {
            // dz in halves: a power of two takes what it can be at most, |scale| + |teacher_scale|, to [2^13, 2^14]; what is below 2^-28 of that has fewer than a half's
            // eleven bits, and below 2^-39 none
            const float most = fabsf(s.scale) + fabsf(s.teacher_scale);
            if (most > 0.0f && most < INFINITY) {
                const int up = 13 - ilogbf(most) < 100 ? 13 - ilogbf(most) : 100;
                undo = ldexpf(1.0f, -up);
                s.scale = r.scale = ldexpf(s.scale, up), s.teacher_scale = r.teacher_scale = ldexpf(s.teacher_scale, up);
            }
        }
    }
    const int32_t *const w_up = T::PER == 2 ? q.w_exponent : nullptr, *const x_up = T::PER == 2 ? q.x_exponent : nullptr;
    for (int cp = 0; cp < p.class_pieces; ++cp) {
        const int class0 = cp * p.piece_classes, classes = V - class0 < p.piece_classes ? V - class0 : p.piece_classes;
        const WeightPlan w = weight_plan(c.l, h, classes, p.piece_rows, p.row_pieces);
        const int dx_shares = shares_used(classes, p.dx_shares);  // (the first piece's are the most)
        ReduceArgs<T> x_sums{};
        for (int64_t rp = 0; rp < p.row_pieces; ++rp) {
            const int64_t row0 = rp * p.piece_rows, rows = c.n - row0 < p.piece_rows ? c.n - row0 : p.piece_rows;
            s.row0 = r.row0 = row0, s.rows = r.rows = rows, s.class0 = r.class0 = class0, r.piece_classes = classes, s.classes = class0 + classes;
            if (h.large) {
                q.s = s;
                launch_scores_stage<T, true>(q, c.stream);
            } else {
                s.listed = cp == 0 && dweight ? listed + row0 : nullptr;
                launch_scores<T, true>(s, c.stream);
            }
            if (r.teacher_scale != 0.0f) {
                // (20,000 rows of 8 classes, f32: backward 191 us with wavefronts, 175 with 8 lanes; a few rows leave the GPU to wavefronts)
                const dim3 wavefronts((unsigned)ceil_div(rows, 4), (unsigned)ceil_div(r.top, 64));
                if (rows < 4 * kCus || r.top > 32) k_class_fix<T, 64><<<wavefronts, dim3(256), 0, c.stream>>>(r);
                else if (r.top <= 8) k_class_fix<T, 8><<<dim3((unsigned)ceil_div(rows, 32)), dim3(256), 0, c.stream>>>(r);
                else k_class_fix<T, 16><<<dim3((unsigned)ceil_div(rows, 16)), dim3(256), 0, c.stream>>>(r);
            }
            float *slots = p.dx_bytes ? dx_slots + (p.class_pieces > 1 ? row0 * p.slot_width : 0) : nullptr;
            const int64_t slot_rows = round_up(p.class_pieces > 1 ? c.n : rows, h.slot_round);
            const auto fill_dx = [&](auto &a) {
                a.M = rows, a.K = classes, a.N = D, a.shares = dx_shares, a.per_share = per_share(classes, dx_shares);
                a.out = dx + row0 * dx_stride, a.out_stride = dx_stride, a.slots = slots, a.slot_rows = slot_rows, a.add = cp > 0;
            };
            const auto fill_dw = [&](auto &a) {
                a.M = classes, a.N = D, a.shares = shares_used(rows, w.shares), a.per_share = per_share(rows, a.shares);
                a.out = dweight + (int64_t)class0 * D, a.out_stride = D, a.slot_rows = round_up(classes, h.slot_round), a.add = rp > 0;
                if (w.slots) a.slots = dw_slots;
                if (dbias && (w.slots || h.large)) a.sum_slots = db_slots;
            };
            if (h.large) {
                StagePieceArgs<T> x{}, y{};
                fill_dx(x), fill_dw(y);
                x.b = q.w + class0 * q.w_bytes, x.b_bytes = q.w_bytes, x.exponent = w_up;
                y.b = q.x + row0 * q.x_bytes, y.b_bytes = q.x_bytes, y.exponent = x_up;
                y.K = round_up(rows, 32);  // (rows of zeros in both)
                for (StagePieceArgs<T> *a : {&x, &y}) {
                    a->a = (const char *)dz, a->a_rows = (int)round_up(rows, StageCut::BB), a->a_stride = (int)p.dz_stride;
                    a->b_width = p.padded, a->b_plane = q.plane, a->slot_width = p.slot_width, a->undo = undo;
                }
                launch_products<T>(dweight ? &y : nullptr, dx ? &x : nullptr, c.stream);
            } else {
                PieceArgs<T> x{}, y{};
                fill_dx(x), fill_dw(y);
                x.b = s.w + (int64_t)class0 * D, x.b_stride = D;
                y.b = s.x + row0 * c.x_stride, y.b_stride = c.x_stride, y.list = listed + row0, y.K = rows, y.sums = dbias ? dbias + class0 : nullptr;
                for (PieceArgs<T> *a : {&x, &y}) a->a = dz, a->a_rest = s.dz_rest, a->a_stride = p.dz_stride, a->a_width = (int)p.dz_stride;
                if (dx && dweight && w.tile == p.dx_tile) {
                    launch_products<T>(&y, &x, w.tile, c.stream);
                } else {
                    if (dweight) launch_products<T>(&y, nullptr, w.tile, c.stream);
                    if (dx) launch_products<T>(nullptr, &x, p.dx_tile, c.stream);
                }
            }
            // (where one piece has all classes; the last piece of rows leaves it to the launch that finishes dW too)
            x_sums = {};
            if (slots && dx && p.class_pieces == 1)
                x_sums = {slots, nullptr, slot_rows, rows, p.slot_width, D, dx_shares, 0, dx + row0 * dx_stride, nullptr, dx_stride, w_up, undo};
            if (x_sums.out && rp + 1 < p.row_pieces) launch_reduce<T>(x_sums, {}, c.stream);
        }
        // (small calls without slots have written both already, large ones dweight)
        E *dw_out = dweight && w.slots ? dweight + (int64_t)class0 * D : nullptr, *db_out = dbias && (w.slots || h.large) ? dbias + class0 : nullptr;
        ReduceArgs<T> w_sums{};
        const int64_t dw_rows = round_up(classes, h.slot_round), dx_rows = round_up(c.n, h.slot_round);
        if (dw_out || db_out) w_sums = {dw_slots, db_slots, dw_rows, classes, p.slot_width, D, w.shares, w.shares * summers_of(c.l, h), dw_out, db_out, D, x_up, undo};
        if (p.dx_bytes && dx && cp > 0 && cp + 1 == p.class_pieces)
            x_sums = {dx_slots, nullptr, dx_rows, c.n, p.slot_width, D, p.dx_shares, 0, dx, nullptr, dx_stride, w_up, undo};
        launch_reduce<T>(w_sums, x_sums, c.stream);
    }
    BGL_HIP(hipGetLastError());
    return BGL_OK;
}

// Both ways' needs: which one a call goes depends on where its operands lie.
void room_of(const bgl_class_loss_t *l, int64_t n, size_t &forward, size_t &backward)
{
    forward = backward = 0;
    for (const bool large : {false, true}) {
        if (large && !large_call(l, n)) continue;
        const Scheme h = scheme_of(l, large);
        const size_t f = plan_of(l, n, h).forward_bytes, b = backward_room(l, n, h);
        if (f > forward) forward = f;
        if (b > backward) backward = b;
    }
}

int check_loss(const bgl_class_loss_t *l, int64_t n)
{
    if (!l) BGL_FAIL(BGL_EINVAL, "loss is null");
    if (l->dtype != BGL_F32 && l->dtype != BGL_BF16) BGL_FAIL(BGL_EINVAL, "unknown dtype %d", l->dtype);
    if (l->in_dim < 1 || l->classes < 1 || l->top < 0) BGL_FAIL(BGL_EINVAL, "in_dim %d, classes %d, top %d", l->in_dim, l->classes, l->top);
    if (!(l->temperature >= 0x1p-10f && l->temperature <= 0x1p10f)) BGL_FAIL(BGL_EINVAL, "temperature %g is not in [2^-10, 2^10]", (double)l->temperature);
    if (l->in_dim > BGL_MAX_DIM) BGL_FAIL(BGL_EUNSUPPORTED, "in_dim %d is more than %d", l->in_dim, BGL_MAX_DIM);
    if (l->classes > BGL_MAX_CLASSES) BGL_FAIL(BGL_EUNSUPPORTED, "%d classes are more than %d", l->classes, BGL_MAX_CLASSES);
    if (l->top > BGL_MAX_TOP) BGL_FAIL(BGL_EUNSUPPORTED, "top %d is more than %d", l->top, BGL_MAX_TOP);
    if (n < 0 || n > INT32_MAX) BGL_FAIL(BGL_EINVAL, "%lld rows", (long long)n);
    return BGL_OK;
}
int check_call(const Call &c)
{
    BGL_TRY(check_loss(c.l, c.n));
    const int es = c.l->dtype == BGL_F32 ? 4 : 2;
    BGL_TRY(check_rows("x", c.x, c.x_stride, c.l->in_dim, es, c.n > 0));
    if ((c.n > 0 && !c.weight) || !aligned(c.weight, es) || !aligned(c.bias, es)) BGL_FAIL(BGL_EINVAL, "weight is null, or weight or bias is misaligned");
    if (!aligned(c.labels, 4) || !aligned(c.top_class, 4) || !aligned(c.top_score, 4))
        BGL_FAIL(BGL_EINVAL, "labels or the teacher's classes or scores are misaligned");
    if (!c.top_class != !c.top_score) BGL_FAIL(BGL_EINVAL, "the teacher's classes and scores come together");
    if (c.top_class && c.l->top == 0) BGL_FAIL(BGL_EINVAL, "the loss has no teacher (top is 0)");
    if (c.n > 0 && !c.labels && !c.top_class) BGL_FAIL(BGL_EINVAL, "neither labels nor a teacher");
    return BGL_OK;
}
int check_workspace(const void *workspace, size_t have, size_t need)
{
    if (need == 0) return BGL_OK;
    if (!workspace || !aligned(workspace, 256)) BGL_FAIL(BGL_EINVAL, "workspace is null or not 256-byte aligned");
    if (have < need) BGL_FAIL(BGL_ECAPACITY, "workspace of %zu bytes, %zu needed", have, need);
    return BGL_OK;
}

}  // namespace
}  // namespace bgl

using namespace bgl;

extern "C" int bgl_class_loss_workspace_bytes(const bgl_class_loss_t *loss, int64_t n, size_t *forward_bytes, size_t *backward_bytes)
try {
    if (!forward_bytes && !backward_bytes) BGL_FAIL(BGL_EINVAL, "forward_bytes and backward_bytes are null");
    BGL_TRY(check_loss(loss, n));
    size_t forward, backward;
    room_of(loss, n, forward, backward);
    if (forward_bytes) *forward_bytes = forward;
    if (backward_bytes) *backward_bytes = backward;
    return BGL_OK;
} BGL_NOTHROW_END

extern "C" int bgl_class_loss_forward(const bgl_class_loss_t *loss, int64_t n, const void *x, int64_t x_stride, const void *weight, const void *bias,
                                      const int32_t *labels, const int32_t *teacher_classes, const float *teacher_scores, float *label_loss,
                                      float *teacher_loss, float *saved, void *workspace, size_t workspace_bytes, void *stream)
try {
    const Call c{loss, n, x, x_stride, weight, bias, labels, teacher_classes, teacher_scores, (char *)workspace, (hipStream_t)stream};
    BGL_TRY(check_call(c));
    if (!aligned(label_loss, 4) || !aligned(teacher_loss, 4) || !aligned(saved, 4)) BGL_FAIL(BGL_EINVAL, "label_loss, teacher_loss or saved is misaligned");
    if ((label_loss && n > 0 && !labels) || (teacher_loss && n > 0 && !teacher_classes)) BGL_FAIL(BGL_EINVAL, "a loss without its labels or teacher");
    BGL_TRY(check_workspace(workspace, workspace_bytes, n > 0 ? plan_of(loss, n, scheme_of(loss, goes_large(c, true))).forward_bytes : 0));
    if (n == 0) return BGL_OK;
    return loss->dtype == BGL_F32 ? forward<tile::F32>(c, label_loss, teacher_loss, saved) : forward<tile::BF16>(c, label_loss, teacher_loss, saved);
} BGL_NOTHROW_END

extern "C" int bgl_class_loss_backward(const bgl_class_loss_t *loss, int64_t n, const void *x, int64_t x_stride, const void *weight, const void *bias,
                                       const int32_t *labels, const int32_t *teacher_classes, const float *teacher_scores, const float *saved, float scale,
                                       float teacher_scale, void *dx, int64_t dx_stride, void *dweight, void *dbias, void *workspace,
                                       size_t workspace_bytes, void *stream)
try {
    const Call c{loss, n, x, x_stride, weight, bias, labels, teacher_classes, teacher_scores, (char *)workspace, (hipStream_t)stream};
    BGL_TRY(check_call(c));
    const int es = loss->dtype == BGL_F32 ? 4 : 2;
    BGL_TRY(check_rows("dx", dx, dx_stride, loss->in_dim, es, false));
    if ((n > 0 && !saved) || !aligned(saved, 4)) BGL_FAIL(BGL_EINVAL, "saved is null or misaligned");
    if (!aligned(dweight, es) || !aligned(dbias, es)) BGL_FAIL(BGL_EINVAL, "dweight or dbias is misaligned");
    if (dbias && !dweight) BGL_FAIL(BGL_EINVAL, "dbias without dweight");
    if (!dx && !dweight) BGL_FAIL(BGL_EINVAL, "no gradient is asked for");
    BGL_TRY(check_workspace(workspace, workspace_bytes, n > 0 ? plan_of(loss, n, scheme_of(loss, goes_large(c, false))).backward_bytes : 0));
    return loss->dtype == BGL_F32 ? backward<tile::F32>(c, saved, scale, teacher_scale, dx, dx_stride, dweight, dbias)
                                  : backward<tile::BF16>(c, saved, scale, teacher_scale, dx, dx_stride, dweight, dbias);
} BGL_NOTHROW_END
