// Device templates for tiles of matrix products on the matrix units (gfx950): operands come from global memory through
// registers into LDS and from there as fragments of 16 x 16 MFMA instructions.  Shared by the layers and the orthogonalised updates.
//
// A tile of an operand is BO rows (the index that survives the product) by 32 dwords of the summed index: 32 values of fp32, 64 of
// bf16 (BK).  Operands come in two orders:
//   summed index contiguous (Kc)    LDS [BO][32 dwords] of 16-byte chunks; chunk c of row r lies at c ^ (r & 7), so that the 8 lanes a
//                                   16-byte read serves at a time, each with a row of its own, meet all banks
//   kept index contiguous (Oc)      LDS [BK][BO], blocks of 16 columns moved about within a row so that the rows a read meets lie in
//                                   different banks.  fp32 fragments are read value by value; bf16 fragments, which need neighbouring summed
//                                   indices in a register, by the LDS read that transposes 4 x 16 values among 16 lanes
// Which summed index sits in which lane is free as long as both operands agree: lane group g = lane / 16 has dwords 4g .. 4g+3 of
// each 16 (8 values of bf16, 4 of fp32).  Loads need no alignment beyond the element's (global memory takes unaligned vector accesses).
#pragma once

#include "bgl_internal.h"

namespace bgl {
namespace tile {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kDwords = 32;  // of the summed index per tile

struct F32 {
    typedef float elem;
    typedef uint32_t bits;
    static constexpr int PER = 1, VEC = 4;  // values per dword, per 16 bytes
    static __device__ __forceinline__ float get(elem v) { return v; }
    static __device__ __forceinline__ elem put(float v) { return v; }
    static __device__ __forceinline__ float sum(const uint32_t (&a)[4], float c)
    {
        return c + ((__uint_as_float(a[0]) + __uint_as_float(a[1])) + (__uint_as_float(a[2]) + __uint_as_float(a[3])));
    }
    // 16 dwords of the summed index: four instructions of 4 values
    static __device__ __forceinline__ f32x4 mma(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c)
    {
#pragma unroll
        for (int p = 0; p < 4; ++p) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[p]), __uint_as_float(b[p]), c, 0, 0, 0);
        return c;
    }
};

struct BF16 {
    typedef uint16_t elem;
    typedef uint16_t bits;
    static constexpr int PER = 2, VEC = 8;
    static __device__ __forceinline__ float get(elem v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ elem put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }  // to nearest even
    static __device__ __forceinline__ float sum(const uint32_t (&a)[4], float c)
    {
        const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
        for (int p = 0; p < 4; ++p) c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a[p]), ones, c, false);
        return c;
    }
    static __device__ __forceinline__ f32x4 mma(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

// The thread's number among the 256 that make one product; a workgroup may have several such teams.
__device__ __forceinline__ int team_thread() { return threadIdx.x & (kThreads - 1); }

// A workgroup of WA x WB wavefronts, each with FA x FB fragments.
template <int WA, int WB, int FA_, int FB_>
struct Cut {
    static_assert(WA * WB * kWave == kThreads, "");
    static constexpr int FA = FA_, FB = FB_, BA = 16 * WA * FA, BB = 16 * WB * FB;
    static __device__ __forceinline__ int a_off() { return team_thread() / kWave / WB * 16 * FA; }
    static __device__ __forceinline__ int b_off() { return team_thread() / kWave % WB * 16 * FB; }
};

constexpr int up_to_power(int x)
{
    int p = 16;
    while (p < x) p *= 2;
    return p;
}

template <class V>
__device__ __forceinline__ V load_any(const void *p)
{
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}

// The values of 16 bytes moved `by` places towards the first, zeros behind them; nothing is left of them from VEC places on.
template <class T>
__device__ __forceinline__ uint4 move_down(const uint4 &v, int by)
{
    const int bits = by * (32 / T::PER);
    uint32_t d[5] = {v.x, v.y, v.z, v.w, 0};
    if constexpr (T::PER == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = __builtin_amdgcn_alignbit(d[i + 1], d[i], bits & 31);
    }
    const bool one = bits & 32, two = bits & 64, none = bits >= 128;
    uint32_t e[4] = {one ? d[1] : d[0], one ? d[2] : d[1], one ? d[3] : d[2], one ? 0 : d[3]};
    return uint4{none ? 0 : two ? e[2] : e[0], none ? 0 : two ? e[3] : e[1], none || two ? 0 : e[2], none || two ? 0 : e[3]};
}

// The first `left` values at p (any number: none for left <= 0, at most VEC), zeros behind them, for a row of `width` values whose end is
// p + left: one load that ends where the row does.  Rows shorter than 16 bytes are read value by value.
template <class T>
__device__ __forceinline__ uint4 load_end(const typename T::elem *p, int left, int width)
{
    if (width >= T::VEC) {
        const int back = left >= T::VEC ? 0 : T::VEC - left;
        return move_down<T>(load_any<uint4>(p - back), back);
    }
    uint32_t d[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < T::VEC - 1; ++e) {
        if (e < left) d[e / T::PER] |= (uint32_t)__builtin_bit_cast(typename T::bits, p[e]) << (e % T::PER * 16);
        __builtin_amdgcn_sched_barrier(0);  // (one at a time: this rare case would take 64 registers beside the products')
    }
    return uint4{d[0], d[1], d[2], d[3]};
}

// Both operands keep the next tile on its way in registers while the present one is multiplied out of LDS.  Loads of whole tiles have no
// branch among them: with branches every load waits for those before it.

// A Kc operand: the thread brings chunk (tid & 7) of rows (tid >> 3) + 32 * pass.
template <class T, int BO>
struct KcOperand {
    static constexpr int PASSES = (BO + 31) / 32;
    static constexpr int BK = kDwords * T::PER;
    static constexpr int LDS = PASSES * 32 * kDwords;  // dwords
    const typename T::elem *at[PASSES];
    uint4 reg[PASSES];

    // row(i): the address of tile row i's first value; any readable row for one that has none
    template <class Row>
    __device__ __forceinline__ void init(Row row)
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) at[p] = row((team_thread() >> 3) + 32 * p) + (team_thread() & 7) * T::VEC;
    }
    __device__ __forceinline__ void load_whole(int tile)
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) reg[p] = load_any<uint4>(at[p] + tile * BK);
    }
    __device__ __forceinline__ void load(int tile, int K)
    {
        if ((tile + 1) * BK <= K) return load_whole(tile);
        const int left = K - tile * BK - (int)(team_thread() & 7) * T::VEC;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) reg[p] = load_end<T>(at[p] + tile * BK, left, K);
    }
    __device__ __forceinline__ void store(uint32_t *lds) const
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = (team_thread() >> 3) + 32 * p, c = team_thread() & 7;
            *reinterpret_cast<uint4 *>(lds + r * kDwords + ((c ^ (r & 7)) << 2)) = reg[p];
        }
    }
    // F fragments of rows from `off`, 16 dwords of the summed index from 16 * step
    template <int F>
    static __device__ __forceinline__ void read(const uint32_t *lds, int off, int step, uint32_t (&f)[F][4])
    {
        const int l = threadIdx.x & 63;
        const uint32_t *from = lds + (off + (l & 15)) * kDwords + (((step * 4 + (l >> 4)) ^ (l & 7)) << 2);
#pragma unroll
        for (int t = 0; t < F; ++t) {
            const uint4 v = *reinterpret_cast<const uint4 *>(from + t * 16 * kDwords);
            f[t][0] = v.x, f[t][1] = v.y, f[t][2] = v.z, f[t][3] = v.w;
        }
    }
};

// An Oc operand: values (k, o) at base + row(k) * stride + o, k counted in a range of `count` > 0 summed rows.  LIST: row(k) = rows[k], and
// numbers outside [0, total) have no row; else row(k) = first + k.  Rows outside are read from one that exists and zeroed on the way to
// LDS; columns that do not exist hold anything (they make columns of the result that are not stored).  NARROW:
// rows may be shorter than 16 bytes (a template's affair because that code, never run, still took the others' registers).
template <class T, int BO, bool LIST, bool NARROW>
struct OcOperand {
    static constexpr int BK = kDwords * T::PER;
    static constexpr int W = up_to_power(BO);        // columns of a row in LDS
    static constexpr int LDS = kDwords * W;          // dwords
    static constexpr int PER_ROW = W / T::VEC;       // threads a row takes
    static constexpr int ROWS = kThreads / PER_ROW;  // rows a pass takes
    static constexpr int PASSES = ROWS < BK ? BK / ROWS : 1;
    static constexpr int ALL = (1 << PASSES) - 1;
    const typename T::elem *base;  // of the thread's first value (of its chunk, moved back so that it ends with the row)
    uint32_t stride;
    const int32_t *rows;           // of the range's first row
    int32_t first, total, count;
    int back;                      // how far base was moved; VEC where the thread has no columns
    bool ends;                     // a chunk of the tile is cut by the row's end
    bool narrow;                   // rows shorter than 16 bytes
    int32_t next[LIST ? PASSES : 1];  // row numbers of the tile that is loaded next
    int live;                      // which rows of the tile in reg exist, one bit each
    uint4 reg[PASSES];

    __device__ __forceinline__ int kk(int pass) const { return team_thread() / PER_ROW + ROWS * pass; }
    __device__ __forceinline__ bool idle() const { return ROWS > BK && kk(0) >= BK; }
    __device__ __forceinline__ void init(const typename T::elem *p, int64_t ld, int64_t of, int o0, int O)
    {
        const int o = o0 + team_thread() % PER_ROW * T::VEC, left = O - o;
        narrow = NARROW && O < T::VEC;
        ends = o0 + W > O && O % T::VEC != 0;
        back = left >= T::VEC ? 0 : left > 0 ? T::VEC - left : T::VEC;
        base = p + (narrow ? 0 : left > 0 ? o - back : 0);
        stride = (uint32_t)ld;
        total = (int32_t)of;
    }
    // The range of summed rows: from position `from` of the row order, n of them.
    __device__ __forceinline__ void range(const int32_t *index, int64_t from, int n)
    {
        if constexpr (LIST) rows = index + from;
        first = (int32_t)from;
        count = n;
        seek(0);
    }
    // LIST: asks for the row numbers of a tile
    __device__ __forceinline__ void seek(int tile)
    {
        if constexpr (LIST) {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int k = tile * BK + kk(p);
                next[p] = rows[k < count ? k : count - 1];
            }
        }
    }
    __device__ __forceinline__ void load(int tile)
    {
        uint32_t now[PASSES];
        live = 0;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int k = tile * BK + kk(p);
            const uint32_t r = LIST ? next[LIST ? p : 0] : first + (k < count ? k : count - 1);
            const bool named = !LIST || r < (uint32_t)total;
            now[p] = named ? r : 0;
            live |= (int)(named && k < count) << p;
        }
        seek(tile + 1);  // before the loads: waiting for these numbers then waits for no later load
        if (idle()) return;
        if constexpr (NARROW) {
            if (narrow) {
#pragma unroll
                for (int p = 0; p < PASSES; ++p) reg[p] = load_end<T>(base + (uint64_t)now[p] * stride, T::VEC - back, 0);
                return;
            }
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) reg[p] = load_any<uint4>(base + (uint64_t)now[p] * stride);
    }
    // Zeroes rows that do not exist and puts cut chunks in place; once for each loaded tile, before store().
    __device__ __forceinline__ void settle()
    {
        if (!ends && __all(live == ALL)) return;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) reg[p] = move_down<T>(reg[p], !(live >> p & 1) ? T::VEC : narrow ? 0 : back);
    }
    // where column c of row k lies, in values from the tile's start
    static __device__ __forceinline__ int place(int k, int c)
    {
        constexpr int BLOCKS = W / 16;
        int move;
        if constexpr (T::PER == 1) {
            return k * W + ((c + 16 * (k >> 2)) & (W - 1));
        } else {
            if constexpr (BLOCKS == 8) move = (k & 3) | (k >> 3 & 1) << 2;
            else if constexpr (BLOCKS == 4) move = (k >> 1 & 1) | (k >> 3 & 1) << 1;
            else if constexpr (BLOCKS == 2) move = k >> 3 & 1;
            else move = 0;
            return k * W + (((c >> 4) ^ move) << 4 | (c & 15));
        }
    }
    __device__ __forceinline__ void store(uint32_t *lds) const
    {
        if (idle()) return;
        typename T::elem *to = reinterpret_cast<typename T::elem *>(lds);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) *reinterpret_cast<uint4 *>(to + place(kk(p), team_thread() % PER_ROW * T::VEC)) = reg[p];
    }
    template <int F>
    static __device__ __forceinline__ void read(const uint32_t *lds, int off, int step, uint32_t (&f)[F][4])
    {
        const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
        if constexpr (T::PER == 1) {
#pragma unroll
            for (int t = 0; t < F; ++t)
#pragma unroll
                for (int p = 0; p < 4; ++p) f[t][p] = lds[place(step * 16 + 4 * g, off + 16 * t + i) + p * W];
        } else {
            // lane (i / 4, i % 4) of 16 names columns 4 (i % 4) .. +3 of row i / 4, and gets column i of the four rows
#pragma unroll
            for (int t = 0; t < F; ++t) {
                const uint16_t *from = reinterpret_cast<const uint16_t *>(lds) + place(step * 32 + 8 * g + (i >> 2), off + 16 * t + 4 * (i & 3));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const auto at = (__attribute__((address_space(3))) s16x4 *)(uint16_t *)(from + 4 * h * W);
                    const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at));
                    f[t][2 * h] = v.x, f[t][2 * h + 1] = v.y;
                }
            }
        }
    }
};

// The tiles of one product: load(tile) into registers, store(tile) from there to LDS, compute(tile) out of LDS.  One LDS buffer and two
// barriers a tile: the room a second buffer would take holds another workgroup, which fills the waits of this one.
template <class Load, class Store, class Compute>
__device__ __forceinline__ void pipeline(int tiles, Load load, Store store, Compute compute)
{
    if (tiles <= 0) return;
    load(0);
    for (int i = 0; i < tiles; ++i) {
        store(i);
        __syncthreads();
        if (i + 1 < tiles) load(i + 1);
        compute(i);
        __syncthreads();
    }
}

// One tile of both operands into the accumulators; `steps` of 16 dwords hold values.  also(a, b) sees each step's fragments.
template <class T, class A, class B, class C, class Also>
__device__ __forceinline__ void multiply(const uint32_t *a_lds, const uint32_t *b_lds, int steps, f32x4 (&acc)[C::FA][C::FB], Also also)
{
    const auto products = [&](const uint32_t(&a)[C::FA][4], const uint32_t(&b)[C::FB][4]) {
#pragma unroll
        for (int i = 0; i < C::FA; ++i)
#pragma unroll
            for (int j = 0; j < C::FB; ++j) acc[i][j] = T::mma(a[i], b[j], acc[i][j]);
    };
#pragma unroll
    for (int step = 0; step < 2; ++step) {
        if (step >= steps) break;
        uint32_t a[C::FA][4], b[C::FB][4];
        A::read(a_lds, C::a_off(), step, a);
        B::read(b_lds, C::b_off(), step, b);
        products(a, b);
        also(a, b);
    }
}

// A lane's accumulators: row 4 * (lane / 16) + j of a fragment's 16, column lane % 16.  Through LDS they become rows that threads read
// in pieces of 4 columns or more: fp32, blocks of 16 columns moved on by a block for every 4 rows.  Fragments go there FH of FA at a time
// (WA * 16 * FH rows of the tile): as many as the operands' LDS has room for.
template <int W>
__device__ __forceinline__ int result_place(int r, int c) { return r * W + ((c + 16 * (r >> 2)) & (W - 1)); }

template <class C, int LDS>
struct Result {
    static constexpr int W = up_to_power(C::BB), WA = C::BA / 16 / C::FA;
    static constexpr int fit(int fh) { return fh == 1 || (C::FA % fh == 0 && WA * 16 * fh * W <= LDS) ? fh : fit(fh - 1); }
    static constexpr int FH = fit(C::FA), PARTS = C::FA / FH, ROWS = WA * 16 * FH, SIZE = ROWS * W;
    // the tile's row that row r of a part is
    static __device__ __forceinline__ int row(int part, int r) { return r / (16 * FH) * 16 * C::FA + part * 16 * FH + r % (16 * FH); }
    static __device__ __forceinline__ void put(float *lds, int part, const f32x4 (&acc)[C::FA][C::FB], bool add = false)
    {
        int l = threadIdx.x & 63;
        asm volatile("" : "+v"(l));  // (the addresses are made here: around an outer loop they would be kept in 32 registers)
#pragma unroll
        for (int i = 0; i < C::FA; ++i) {
            if (i / FH != part) continue;
#pragma unroll
            for (int t = 0; t < C::FB; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float *to = lds + result_place<W>(C::a_off() / C::FA * FH + 16 * (i % FH) + 4 * (l >> 4) + j, C::b_off() + 16 * t + (l & 15));
                    *to = add ? *to + acc[i][t][j] : acc[i][t][j];
                }
        }
    }
};

// Work is dealt to workgroups in an order that keeps the tiles of one row block, which read the same rows, on one XCD (workgroup
// numbers go round the eight XCDs).
__device__ __forceinline__ bool tile_of(int64_t id, int64_t row_tiles, int col_tiles, int64_t &row, int &col)
{
    const int64_t j = id >> 3;
    col = (int)(j % col_tiles);
    row = (j / col_tiles) * 8 + (id & 7);
    return row < row_tiles;
}
inline int64_t tile_count(int64_t row_tiles, int col_tiles) { return (row_tiles + 7) / 8 * 8 * col_tiles; }

}  // namespace tile
}  // namespace bgl
