// A layer over the rows of a batch: product with the weight, bias, residual and activation, and its gradients; with one weight for
// all rows or one per group of rows (nodes by type), and the grouping itself.
//
//   z = x W' + b (+ r)      y = act(z) (+ r)                      k_linear_forward
//   dz = dy act'(z)                                               k_linear_dz
//   dx = dz W                                                     k_linear_dx
//   dW = dz' x, db = sum dz                                       k_linear_dw (by ranges of rows), k_linear_reduce
//
// Sums are kept in fp32 whatever the type; z is rounded to the type where it is kept for the gradient, dz because the matrix units
// read it in the type (bf16: off by 2^-8 of themselves at most, as the rows they meet are).
#include "bgl_internal.h"
#include "bgl_tile.h"

namespace bgl {
namespace {

using namespace tile;

constexpr int kMaxGroups = BGL_MAX_GROUPS;
constexpr int kGroupThreads = 512;   // of the grouping kernels
constexpr int kGroupTiles = 256;     // workgroups of one grouping pass at most
constexpr int kGroupTileRows = 2048; // rows a workgroup takes at least

// ----------------------------------------------------------------- activations
template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == BGL_ACT_RELU) return z < 0.0f ? 0.0f : z;  // (NaN stays)
    if constexpr (ACT == BGL_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    if constexpr (ACT == BGL_ACT_SILU) return z / (1.0f + expf(-z));
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope(float z)
{
    if constexpr (ACT == BGL_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == BGL_ACT_GELU) return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    if constexpr (ACT == BGL_ACT_SILU) {
        const float p = 1.0f / (1.0f + expf(-z));
        return p * (1.0f + z * (1.0f - p));
    }
    return 1.0f;
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
            const int64_t first = before + __shfl(upto - tiles, k);
            const int64_t from = __shfl((int)lo, k) + (t - first) * tile_rows;
            const int64_t left = __shfl((int)hi, k) - from;
            s.group = __builtin_amdgcn_readfirstlane(g0 + k);
            s.start = __builtin_amdgcn_readfirstlane((int)from);
            s.count = __builtin_amdgcn_readfirstlane((int)(left < tile_rows ? left : tile_rows));
            return s;
        }
        before += __shfl(upto, 63);
    }
    return s;
}

// Tiles of the groups before group g (g < 64 * passes), and g's own.
__device__ __forceinline__ void tiles_before(const Groups &q, int64_t n, int tile_rows, int g, int64_t &before, int &own)
{
    if (q.groups == 0) {
        before = 0;
        own = (int)((n + tile_rows - 1) / tile_rows);
        return;
    }
    const int lane = threadIdx.x & 63;
    before = 0;
    for (int g0 = 0;; g0 += 64) {
        int64_t lo = 0, hi = 0;
        if (g0 + lane < q.groups) group_range(q, n, g0 + lane, lo, hi);
        const int tiles = (int)((hi - lo + tile_rows - 1) / tile_rows);
        const int upto = wave_incl_scan(tiles);
        if (g < g0 + 64) {
            own = __shfl(tiles, g - g0);
            before += __shfl(upto, g - g0) - own;
            return;
        }
        before += __shfl(upto, 63);
    }
}

__device__ __forceinline__ int32_t row_at(const Groups &q, int64_t n, int64_t position)
{
    const int32_t r = q.index ? q.index[position] : (int32_t)position;
    return (uint32_t)r < (uint64_t)n ? r : -1;
}

// ----------------------------------------------------------------- columns of a row
template <class T, int TT>
__device__ __forceinline__ void load_cols(const typename T::elem *p, int left, float (&v)[TT])
{
    struct Pack { typename T::elem e[TT]; } pack;
    if (left >= TT) {
        pack = load_any<Pack>(p);
    } else {
#pragma unroll
        for (int i = 0; i < TT; ++i) pack.e[i] = i < left ? p[i] : (typename T::elem)0;
    }
#pragma unroll
    for (int i = 0; i < TT; ++i) v[i] = T::get(pack.e[i]);
}
template <class T, int TT>
__device__ __forceinline__ void store_cols(typename T::elem *p, int left, const float (&v)[TT])
{
    struct Pack { typename T::elem e[TT]; } pack;
#pragma unroll
    for (int i = 0; i < TT; ++i) pack.e[i] = T::put(v[i]);
    if (left >= TT) {
        __builtin_memcpy(p, &pack, sizeof(pack));
    } else {
#pragma unroll
        for (int i = 0; i < TT; ++i)
            if (i < left) p[i] = pack.e[i];
    }
}

// ----------------------------------------------------------------- forward, and dx
// One kernel for both: rows (n x K) times a weight whose summed index is contiguous (forward: out_dim x in_dim, B_OC false) or is
// not (dx: the summed index is out_dim, B_OC true).
template <class T>
struct RowsArgs {
    const typename T::elem *x, *w, *bias, *residual;
    typename T::elem *y, *saved;
    int64_t n, x_stride, y_stride, residual_stride, saved_stride, row_tiles;
    int K, N, col_tiles;  // summed and kept width
    int residual_mode;
    Groups q;
};

template <class T, bool B_OC, int TT, int ACT>
__global__ __launch_bounds__(kThreads, 2) void k_linear_rows(RowsArgs<T> a)
{
    constexpr int BO = 32 * TT;
    __shared__ __attribute__((aligned(16))) uint32_t lds[2][2][BO * kDwords];
    __shared__ int32_t row_of[BO];
    int64_t rt;
    int ct;
    if (!tile_of(blockIdx.x, a.row_tiles, a.col_tiles, rt, ct)) return;
    const Span s = find_span(a.q, a.n, a.q.groups + (a.q.groups > 0), BO, rt);
    if (s.group < 0) return;
    const bool grouped = a.q.groups > 0, none = grouped && s.group == a.q.groups;
    const int n0 = ct * BO, K = none ? 0 : a.K;
    const typename T::elem *w = a.w + (none ? 0 : (int64_t)s.group * a.N * a.K);

    if ((int)threadIdx.x < BO) row_of[threadIdx.x] = (int)threadIdx.x < s.count ? row_at(a.q, a.n, s.start + threadIdx.x) : -1;
    __syncthreads();
    KcOperand<T, BO, TT> rows;
    rows.init([&](int i) {
        const int32_t r = row_of[i];
        return a.x + (r < 0 ? 0 : r) * a.x_stride;
    });
    constexpr int BK = KcOperand<T, BO, TT>::BK;
    f32x4 acc[TT][TT] = {};
    const int wave = threadIdx.x / kWave, a_off = (wave >> 1) * 16 * TT, b_off = (wave & 1) * 16 * TT;
    const int tiles = (K + BK - 1) / BK;
    auto loop = [&](auto &weight, auto load) {
        if (tiles == 0) return;
        rows.load(0, K);
        load(0);
        for (int i = 0; i < tiles; ++i) {
            rows.store(lds[i & 1][0]);
            weight.store(lds[i & 1][1]);
            __syncthreads();
            if (i + 1 < tiles) {
                rows.load((i + 1) * BK, K);
                load((i + 1) * BK);
            }
            const int steps = (K - i * BK + 16 * T::PER - 1) / (16 * T::PER);
            multiply<T, false, B_OC, BO, TT>(lds[i & 1][0], lds[i & 1][1], a_off, b_off, steps, acc);
        }
    };
    if constexpr (B_OC) {
        OcOperand<T, BO, TT> weight;
        weight.init(w, a.N, nullptr, 0, K, K, n0, a.N);
        loop(weight, [&](int k0) { weight.load(k0); });
    } else {
        KcOperand<T, BO, TT> weight;
        weight.init([&](int i) { return w + (int64_t)(n0 + i < a.N ? n0 + i : a.N - 1) * a.K; });
        loop(weight, [&](int k0) { weight.load(k0, K); });
    }

    const int l = threadIdx.x & 63, c = n0 + b_off + TT * (l & 15), left = a.N - c;
    if (left <= 0) return;
    float bias[TT] = {};
    if (a.bias && !none) load_cols<T, TT>(a.bias + (int64_t)s.group * a.N + c, left, bias);
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int32_t r = row_of[a_off + TT * (4 * (l >> 4) + j) + t];
            if (r < 0) continue;
            float v[TT], res[TT] = {};
            if (a.residual_mode) load_cols<T, TT>(a.residual + r * a.residual_stride + c, left, res);
#pragma unroll
            for (int u = 0; u < TT; ++u) v[u] = acc[t][u][j] + bias[u] + (a.residual_mode == BGL_RESIDUAL_BEFORE ? res[u] : 0.0f);
            if (a.saved) store_cols<T, TT>(a.saved + r * a.saved_stride + c, left, v);
#pragma unroll
            for (int u = 0; u < TT; ++u) v[u] = activate<ACT>(v[u]) + (a.residual_mode == BGL_RESIDUAL_AFTER ? res[u] : 0.0f);
            store_cols<T, TT>(a.y + r * a.y_stride + c, left, v);
        }
}

// ----------------------------------------------------------------- dz
template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void k_linear_dz(const typename T::elem *dy, int64_t dy_stride, const typename T::elem *saved,
                                                        int64_t saved_stride, typename T::elem *dz, int64_t dz_stride, int64_t n, int N)
{
    constexpr int V = T::VEC;
    const int per_row = (N + V - 1) / V;
    const int64_t total = n * per_row;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t r = i / per_row;
        const int c = (int)(i % per_row) * V, left = N - c;
        float d[V], z[V];
        load_cols<T, V>(dy + r * dy_stride + c, left, d);
        if constexpr (ACT != BGL_ACT_NONE) {
            load_cols<T, V>(saved + r * saved_stride + c, left, z);
#pragma unroll
            for (int e = 0; e < V; ++e) d[e] *= slope<ACT>(z[e]);
        }
        store_cols<T, V>(dz + r * dz_stride + c, left, d);
    }
}

// ----------------------------------------------------------------- dW, db
// A workgroup takes one tile of dW and one range of a group's rows; partial sums go to `part`, range by range: N * K of dW, N of db.
template <class T>
struct WeightArgs {
    const typename T::elem *dz, *x;
    float *part;
    int64_t n, dz_stride, x_stride, ranges;
    int N, K, range_rows, n_tiles, k_tiles;
    bool with_bias;
    Groups q;
};

template <class T, int TT>
__global__ __launch_bounds__(kThreads, 2) void k_linear_dw(WeightArgs<T> a)
{
    constexpr int BO = 32 * TT;
    __shared__ __attribute__((aligned(16))) uint32_t lds[2][2][BO * kDwords];
    int64_t range;
    int tile;
    if (!tile_of(blockIdx.x, a.ranges, a.n_tiles * a.k_tiles, range, tile)) return;
    const Span s = find_span(a.q, a.n, a.q.groups, a.range_rows, range);
    if (s.group < 0) return;
    const int n0 = tile / a.k_tiles * BO, k0 = tile % a.k_tiles * BO;
    using Op = OcOperand<T, BO, TT>;
    Op up, rows;
    up.init(a.dz, a.dz_stride, a.q.index, s.start, s.count, a.n, n0, a.N);
    rows.init(a.x, a.x_stride, a.q.index, s.start, s.count, a.n, k0, a.K);
    const bool bias = a.with_bias && k0 == 0;
    float sum[T::VEC] = {};
    f32x4 acc[TT][TT] = {};
    const int wave = threadIdx.x / kWave, a_off = (wave >> 1) * 16 * TT, b_off = (wave & 1) * 16 * TT;
    const int tiles = (s.count + Op::BK - 1) / Op::BK;
    up.load(0);
    rows.load(0);
    for (int i = 0; i < tiles; ++i) {
        up.store(lds[i & 1][0]);
        rows.store(lds[i & 1][1]);
        if (bias) {
#pragma unroll
            for (int p = 0; p < Op::PASSES; ++p)
#pragma unroll
                for (int h = 0; h < T::PER; ++h) {
                    struct Pack { typename T::elem e[T::VEC]; };
                    const Pack v = __builtin_bit_cast(Pack, up.reg[p][h]);
#pragma unroll
                    for (int e = 0; e < T::VEC; ++e) sum[e] += T::get(v.e[e]);
                }
        }
        __syncthreads();
        if (i + 1 < tiles) {
            up.load((int64_t)(i + 1) * Op::BK);
            rows.load((int64_t)(i + 1) * Op::BK);
        }
        const int steps = (s.count - i * Op::BK + 16 * T::PER - 1) / (16 * T::PER);
        multiply<T, true, true, BO, TT>(lds[i & 1][0], lds[i & 1][1], a_off, b_off, steps, acc);
    }
    float *part = a.part + range * ((int64_t)a.N * a.K + a.N);
    const int l = threadIdx.x & 63, c = k0 + b_off + TT * (l & 15), left = a.K - c;
    if (left > 0) {
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = n0 + a_off + TT * (4 * (l >> 4) + j) + t;
                if (r >= a.N) continue;
                float v[TT];
#pragma unroll
                for (int u = 0; u < TT; ++u) v[u] = acc[t][u][j];
                store_cols<F32, TT>(part + (int64_t)r * a.K + c, left, v);
            }
    }
    if (bias) {  // the threads of one column chunk, in order
        __syncthreads();
        float *sums = reinterpret_cast<float *>(&lds[0][0][0]);
#pragma unroll
        for (int e = 0; e < T::VEC; ++e) sums[threadIdx.x * T::VEC + e] = sum[e];
        __syncthreads();
        if ((int)threadIdx.x < BO && n0 + (int)threadIdx.x < a.N) {
            float v = 0.0f;
            for (int i = 0; i < Op::ROWS; ++i) v += sums[i * BO + threadIdx.x];
            part[(int64_t)a.N * a.K + n0 + threadIdx.x] = v;
        }
    }
}

// dW and db of group blockIdx.y: the partial sums of its ranges, added in a fixed order.
template <class T>
__global__ __launch_bounds__(kThreads) void k_linear_reduce(const float *part, int64_t n, int range_rows, int64_t NK, int N, Groups q,
                                                            typename T::elem *dw, typename T::elem *db)
{
    __shared__ float4 sums[kThreads];
    const int g = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x / kWave;
    int64_t first;
    int count;
    tiles_before(q, n, range_rows, g, first, count);
    const int64_t len = NK + N, e = ((int64_t)blockIdx.x * 64 + lane) * 4;
    const int left = len - e < 4 ? (int)(len - e) : 4;
    float v[4] = {};
    if (left > 0)
        for (int i = wave; i < count; i += kThreads / kWave) {
            float w[4];
            load_cols<F32, 4>(part + (first + i) * len + e, left, w);
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] += w[u];
        }
    sums[threadIdx.x] = float4{v[0], v[1], v[2], v[3]};
    __syncthreads();
    if (wave || left <= 0) return;
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) {
        const float4 o = sums[w * 64 + lane];
        v[0] += o.x, v[1] += o.y, v[2] += o.z, v[3] += o.w;
    }
    for (int u = 0; u < left; ++u) {
        const int64_t at = e + u;
        if (at < NK) dw[g * NK + at] = T::put(v[u]);
        else if (db) db[(int64_t)g * N + at - NK] = T::put(v[u]);
    }
}

// ----------------------------------------------------------------- grouping
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
    int carry = 0;
    for (int g0 = 0; g0 < classes; g0 += kGroupThreads) {
        const int g = g0 + threadIdx.x;
        int total = 0, below = 0;
        if (g < classes) {
            if (SINGLE) {
                for (int w = 0; w < WAVES; ++w) total += sh[w * classes + g];
            } else {
                for (int t = 0; t < (int)gridDim.x; ++t) {
                    const int c = a.counts[(int64_t)t * classes + g];
                    total += c;
                    if (t < (int)blockIdx.x) below += c;
                }
            }
        }
        int all;
        const int before = block_excl_scan<kGroupThreads>(total, scan, all);
        if (g < classes) {
            base[g] = carry + before + below;
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
struct Shape {
    const bgl_linear_t *l;
    int64_t n;
    int classes;  // groups at least one
};

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

int check_rows(const char *name, const void *p, int64_t stride, int width, int es, bool needed)
{
    if (!p) {
        if (needed) BGL_FAIL(BGL_EINVAL, "%s is null", name);
        return BGL_OK;
    }
    if (!aligned(p, es)) BGL_FAIL(BGL_EINVAL, "%s must be aligned to its elements", name);
    if (stride < width) BGL_FAIL(BGL_EINVAL, "%s: stride %lld is less than the row's %d values", name, (long long)stride, width);
    return BGL_OK;
}

#define BGL_TRY(call)                  \
    do {                               \
        const int rc__ = (call);       \
        if (rc__ != BGL_OK) return rc__; \
    } while (0)

// How the backward pass cuts a layer's rows.  128 x 128 tiles of dW where both sides fill one, else 64 x 64; ranges of rows so that some
// 512 workgroups (two on each CU) have one tile and one range each.
struct WeightPlan {
    int tt, n_tiles, k_tiles, range_rows;
    int64_t ranges;  // upper bound; with groups each may end in a short one
    size_t dz_bytes, dz_stride, part_bytes;
};

WeightPlan plan_weight(const bgl_linear_t *l, int64_t n)
{
    WeightPlan p;
    p.tt = l->in_dim > 64 && l->out_dim > 64 ? 4 : 2;
    const int bo = 32 * p.tt;
    p.n_tiles = (int)ceil_div(l->out_dim, bo);
    p.k_tiles = (int)ceil_div(l->in_dim, bo);
    const int64_t tiles = (int64_t)p.n_tiles * p.k_tiles;
    int64_t rows = ceil_div(n * tiles, 512);
    rows = rows < 256 ? 256 : rows > n ? (n > 0 ? n : 1) : rows;
    p.range_rows = (int)(ceil_div(rows, 64) * 64 > INT32_MAX ? INT32_MAX / 64 * 64 : ceil_div(rows, 64) * 64);
    p.ranges = n / p.range_rows + (l->num_groups > 0 ? (l->num_groups < n ? l->num_groups : n) : 1);
    const int per = 16 / elem_bytes(l);
    p.dz_stride = round_up(l->out_dim, per);
    p.dz_bytes = l->activation == BGL_ACT_NONE ? 0 : round_up((size_t)n * p.dz_stride * elem_bytes(l), 256);
    p.part_bytes = (size_t)p.ranges * ((size_t)l->out_dim * l->in_dim + l->out_dim) * sizeof(float);
    return p;
}

template <class T, bool B_OC, int TT>
void launch_rows_act(const RowsArgs<T> &a, int act, int64_t blocks, hipStream_t st)
{
    if constexpr (B_OC) {
        k_linear_rows<T, B_OC, TT, BGL_ACT_NONE><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a);
    } else {
        if (act == BGL_ACT_RELU) k_linear_rows<T, B_OC, TT, BGL_ACT_RELU><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a);
        else if (act == BGL_ACT_GELU) k_linear_rows<T, B_OC, TT, BGL_ACT_GELU><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a);
        else if (act == BGL_ACT_SILU) k_linear_rows<T, B_OC, TT, BGL_ACT_SILU><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a);
        else k_linear_rows<T, B_OC, TT, BGL_ACT_NONE><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a);
    }
}

// 128 x 128 tiles where they are enough for the 256 CUs and the width fills one, else 64 x 64.
template <class T, bool B_OC>
int launch_rows(RowsArgs<T> &a, int act, hipStream_t st)
{
    const int64_t extra = a.q.groups > 0 ? (a.q.groups + 1 < a.n ? a.q.groups + 1 : a.n) : 1;
    const bool big = a.N > 64 && ceil_div(a.n, 128) * ceil_div(a.N, 128) >= 256;
    const int bo = big ? 128 : 64;
    a.row_tiles = a.n / bo + extra;
    a.col_tiles = (int)ceil_div(a.N, bo);
    const int64_t blocks = tile_count(a.row_tiles, a.col_tiles);
    if (blocks > INT32_MAX) BGL_FAIL(BGL_EUNSUPPORTED, "%lld rows of width %d need too many workgroups", (long long)a.n, a.N);
    if (big) launch_rows_act<T, B_OC, 4>(a, act, blocks, st);
    else launch_rows_act<T, B_OC, 2>(a, act, blocks, st);
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
    a.residual_mode = l->residual;
    a.q = q;
    return launch_rows<T, false>(a, l->activation, st);
}

template <class T>
int launch_dz(int act, const void *dy, int64_t dy_stride, const void *saved, int64_t saved_stride, void *dz, int64_t dz_stride, int64_t n, int N, hipStream_t st)
{
    using E = typename T::elem;
    const int64_t total = n * ceil_div(N, T::VEC), blocks = ceil_div(total, kThreads);
    const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192)), block(kThreads);
#define BGL_DZ(ACT) k_linear_dz<T, ACT><<<grid, block, 0, st>>>((const E *)dy, dy_stride, (const E *)saved, saved_stride, (E *)dz, dz_stride, n, N)
    if (act == BGL_ACT_RELU) BGL_DZ(BGL_ACT_RELU);
    else if (act == BGL_ACT_GELU) BGL_DZ(BGL_ACT_GELU);
    else if (act == BGL_ACT_SILU) BGL_DZ(BGL_ACT_SILU);
    else BGL_DZ(BGL_ACT_NONE);
#undef BGL_DZ
    BGL_HIP(hipGetLastError());
    return BGL_OK;
}

template <class T, int TT>
void launch_dw(const WeightArgs<T> &a, hipStream_t st)
{
    const int64_t blocks = tile_count(a.ranges, a.n_tiles * a.k_tiles);
    k_linear_dw<T, TT><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a);
}

template <class T>
int backward(const bgl_linear_t *l, int64_t n, const Groups &q, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *weight,
             const void *saved, int64_t saved_stride, void *dx, int64_t dx_stride, void *dweight, void *dbias, void *dresidual,
             int64_t dresidual_stride, void *workspace, hipStream_t st)
{
    using E = typename T::elem;
    const WeightPlan p = plan_weight(l, n);
    const int classes = l->num_groups > 0 ? l->num_groups : 1;
    const void *dz = dy;
    int64_t dz_stride = dy_stride;
    if (n > 0 && (dresidual || l->activation != BGL_ACT_NONE)) {
        void *to = dresidual ? dresidual : workspace;
        dz_stride = dresidual ? dresidual_stride : (int64_t)p.dz_stride;
        BGL_TRY(launch_dz<T>(l->activation, dy, dy_stride, saved, saved_stride, to, dz_stride, n, l->out_dim, st));
        dz = to;
    }
    if (dx && n > 0) {
        RowsArgs<T> a{};
        a.x = (const E *)dz, a.w = (const E *)weight, a.y = (E *)dx;
        a.n = n, a.x_stride = dz_stride, a.y_stride = dx_stride;
        a.K = l->out_dim, a.N = l->in_dim;
        a.q = q;
        BGL_TRY((launch_rows<T, true>(a, BGL_ACT_NONE, st)));
    }
    if (dweight || dbias) {
        WeightArgs<T> a{};
        a.dz = (const E *)dz, a.x = (const E *)x, a.part = reinterpret_cast<float *>((char *)workspace + p.dz_bytes);
        a.n = n, a.dz_stride = dz_stride, a.x_stride = x_stride, a.ranges = p.ranges;
        a.N = l->out_dim, a.K = l->in_dim, a.range_rows = p.range_rows, a.n_tiles = p.n_tiles, a.k_tiles = p.k_tiles;
        a.with_bias = dbias != nullptr;
        a.q = q;
        if (n > 0) {
            if (p.tt == 4) launch_dw<T, 4>(a, st);
            else launch_dw<T, 2>(a, st);
            BGL_HIP(hipGetLastError());
        }
        const int64_t NK = (int64_t)l->out_dim * l->in_dim, len = NK + l->out_dim;
        k_linear_reduce<T><<<dim3((unsigned)ceil_div(len, 256), (unsigned)classes), dim3(kThreads), 0, st>>>(a.part, n, p.range_rows, NK, l->out_dim, q,
                                                                                                         (E *)dweight, (E *)dbias);
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

size_t group_bytes(int64_t n, int groups)
{
    int64_t tile_rows;
    const int tiles = group_tiles(n, tile_rows);
    return round_up((size_t)n * sizeof(uint16_t), 256) + (size_t)(tiles > 0 ? tiles : 1) * (groups + 1) * sizeof(int32_t);
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
    *bytes = p.dz_bytes + p.part_bytes;
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
    if (p.dz_bytes + p.part_bytes > 0) {
        if (!workspace || !aligned(workspace, 256)) BGL_FAIL(BGL_EINVAL, "workspace is null or not 256-byte aligned");
        if (workspace_bytes < p.dz_bytes + p.part_bytes)
            BGL_FAIL(BGL_ECAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.dz_bytes + p.part_bytes);
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
    const size_t classes = (size_t)num_groups + 1, place = (kGroupThreads / kWave + 1) * classes * sizeof(int32_t);
    if (tiles <= 1) {
        k_group_place<true><<<dim3(1), dim3(kGroupThreads), place, st>>>(a);
    } else {
        k_group_count<<<dim3((unsigned)tiles), dim3(kGroupThreads), classes * sizeof(int32_t), st>>>(a);
        k_group_place<false><<<dim3((unsigned)tiles), dim3(kGroupThreads), place, st>>>(a);
    }
    BGL_HIP(hipGetLastError());
    return BGL_OK;
} BGL_NOTHROW_END
