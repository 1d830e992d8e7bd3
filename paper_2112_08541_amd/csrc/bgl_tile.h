// Device templates for tiles of matrix products on the matrix units (gfx950): operands come from global memory through
// registers into LDS and from there as fragments of 16 x 16 MFMA instructions.  Shared by the layers and the orthogonalised updates.
//
// A tile of an operand is BO rows (the index that survives the product) by 32 dwords of the summed index: 32 values of fp32, 64 of
// bf16.  Operands come in two orders:
//   summed index contiguous (Kc)    LDS [BO][32 dwords] of 16-byte chunks; chunk c of row r lies at c ^ ((r / T) & 7), so that the 8
//                                   lanes a 16-byte read serves at a time, whose rows are T apart, meet all banks
//   kept index contiguous (Oc)      LDS [32 dwords][BO]: a dword is one value (fp32), or the values of two neighbouring summed indices
//                                   (bf16), paired in registers on the way from global memory
// A wavefront computes T x T fragments of 16 x 16.  Fragment t holds rows T * i + t (not 16 * t + i): a lane's T fragments then are T
// neighbouring rows, which makes an Oc read one 4T-byte load, and its T accumulators T neighbouring columns of the result.
// Which summed index sits in which lane is free as long as both operands agree: lane group g = lane / 16 has dwords 4g .. 4g+3 of
// each 16.  Loads need no alignment beyond the element's (global memory takes unaligned vector accesses).
#pragma once

#include "bgl_internal.h"

namespace bgl {
namespace tile {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kDwords = 32;  // of the summed index per tile

struct F32 {
    typedef float elem;
    static constexpr int PER = 1, VEC = 4;  // values per dword, per 16 bytes
    static __device__ __forceinline__ float get(elem v) { return v; }
    static __device__ __forceinline__ elem put(float v) { return v; }
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
    static constexpr int PER = 2, VEC = 8;
    static __device__ __forceinline__ float get(elem v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ elem put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }  // to nearest even
    static __device__ __forceinline__ f32x4 mma(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

template <class V>
__device__ __forceinline__ V load_any(const void *p)
{
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}

// Values [0, left) of up to 16 bytes, the others zero.
template <class T>
__device__ __forceinline__ uint4 load_part(const typename T::elem *p, int left)
{
    typename T::elem v[T::VEC];
#pragma unroll
    for (int e = 0; e < T::VEC; ++e) v[e] = e < left ? p[e] : (typename T::elem)0;
    return __builtin_bit_cast(uint4, v);
}

template <class T>
__device__ __forceinline__ uint4 load_upto(const typename T::elem *p, int left)
{
    if (left >= T::VEC) return load_any<uint4>(p);
    return left > 0 ? load_part<T>(p, left) : uint4{0, 0, 0, 0};
}

// A Kc operand: the thread brings chunk (tid & 7) of rows (tid >> 3) + 32 * pass.
template <class T, int BO, int TT>
struct KcOperand {
    static constexpr int PASSES = BO / 32;
    static constexpr int BK = kDwords * T::PER;
    const typename T::elem *at[PASSES];
    uint4 reg[PASSES];

    // row(i): the address of tile row i's first value; any readable row for one that has none
    template <class Row>
    __device__ __forceinline__ void init(Row row)
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) at[p] = row((int)(threadIdx.x >> 3) + 32 * p) + (threadIdx.x & 7) * T::VEC;
    }
    __device__ __forceinline__ void load(int k0, int K)
    {
        if (k0 + BK <= K) {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) reg[p] = load_any<uint4>(at[p] + k0);
        } else {
            const int left = K - k0 - (int)(threadIdx.x & 7) * T::VEC;
#pragma unroll
            for (int p = 0; p < PASSES; ++p) reg[p] = load_upto<T>(at[p] + k0, left);
        }
    }
    __device__ __forceinline__ void store(uint32_t *lds) const
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = (threadIdx.x >> 3) + 32 * p, c = threadIdx.x & 7;
            *reinterpret_cast<uint4 *>(lds + r * kDwords + ((c ^ ((r / TT) & 7)) << 2)) = reg[p];
        }
    }
};

// An Oc operand: values (k, o) at base + row(k) * stride + o, k counted in the tile's range of `count` summed rows.
template <class T, int BO, int TT>
struct OcOperand {
    static constexpr int BK = kDwords * T::PER;
    static constexpr int PER_ROW = BO / T::VEC;              // threads a row takes
    static constexpr int ROWS = kThreads / PER_ROW;          // dword rows a pass takes
    static constexpr int PASSES = kDwords / ROWS;
    const typename T::elem *base;  // of the thread's first value
    int64_t stride;
    const int32_t *rows;           // of the range's first row, or null: rows first, first + 1, ...
    int64_t first, total;
    int64_t count;
    int left;                      // values from the thread's first one to the row's end
    int32_t next[PASSES][T::PER];  // row numbers of the tile that is loaded next, -1 for none
    uint4 reg[PASSES][T::PER];

    __device__ __forceinline__ int kk(int pass) const { return (int)threadIdx.x / PER_ROW + ROWS * pass; }
    __device__ __forceinline__ void init(const typename T::elem *p, int64_t ld, const int32_t *index, int64_t from, int64_t n, int64_t of, int o0, int O)
    {
        const int o = o0 + (int)(threadIdx.x % PER_ROW) * T::VEC;
        left = O - o;
        base = p + (left > 0 ? o : 0);
        stride = ld;
        rows = index ? index + from : nullptr;
        first = from;
        count = n;
        total = of;
        seek(0);
    }
    __device__ __forceinline__ void seek(int64_t k0)
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
            for (int h = 0; h < T::PER; ++h) {
                const int64_t k = k0 + kk(p) * T::PER + h;
                int32_t r = -1;
                if (k < count) {
                    r = rows ? rows[k] : (int32_t)(first + k);
                    if ((uint32_t)r >= (uint64_t)total) r = -1;
                }
                next[p][h] = r;
            }
    }
    __device__ __forceinline__ void load(int64_t k0)
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
            for (int h = 0; h < T::PER; ++h) {
                const int32_t r = next[p][h];
                reg[p][h] = r >= 0 ? load_upto<T>(base + r * stride, left) : uint4{0, 0, 0, 0};
            }
        seek(k0 + BK);
    }
    __device__ __forceinline__ void store(uint32_t *lds) const
    {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            uint32_t *to = lds + kk(p) * BO + (threadIdx.x % PER_ROW) * T::VEC;
            if constexpr (T::PER == 1) {
                *reinterpret_cast<uint4 *>(to) = reg[p][0];
            } else {
                const uint32_t lo[4] = {reg[p][0].x, reg[p][0].y, reg[p][0].z, reg[p][0].w};
                const uint32_t hi[4] = {reg[p][1].x, reg[p][1].y, reg[p][1].z, reg[p][1].w};
                uint32_t out[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    out[2 * i] = __builtin_amdgcn_perm(hi[i], lo[i], 0x05040100);      // low halves of (lo, hi)
                    out[2 * i + 1] = __builtin_amdgcn_perm(hi[i], lo[i], 0x07060302);  // high halves
                }
                *reinterpret_cast<uint4 *>(to) = uint4{out[0], out[1], out[2], out[3]};
                *reinterpret_cast<uint4 *>(to + 4) = uint4{out[4], out[5], out[6], out[7]};
            }
        }
    }
};

// The T fragments of a wavefront whose rows start at `off`, 16 dwords of the summed index from 16 * step.
template <int BO, int TT>
__device__ __forceinline__ void read_kc(const uint32_t *lds, int off, int step, uint32_t (&f)[TT][4])
{
    const int l = threadIdx.x & 63;
    const uint32_t *from = lds + (off + TT * (l & 15)) * kDwords + (((step * 4 + (l >> 4)) ^ (l & 7)) << 2);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const uint4 v = *reinterpret_cast<const uint4 *>(from + t * kDwords);
        f[t][0] = v.x, f[t][1] = v.y, f[t][2] = v.z, f[t][3] = v.w;
    }
}
template <int BO, int TT>
__device__ __forceinline__ void read_oc(const uint32_t *lds, int off, int step, uint32_t (&f)[TT][4])
{
    const int l = threadIdx.x & 63;
    const uint32_t *from = lds + (step * 16 + 4 * (l >> 4)) * BO + off + TT * (l & 15);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if constexpr (TT == 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(from + p * BO);
            f[0][p] = v.x, f[1][p] = v.y, f[2][p] = v.z, f[3][p] = v.w;
        } else {
            static_assert(TT == 2, "");
            const uint2 v = *reinterpret_cast<const uint2 *>(from + p * BO);
            f[0][p] = v.x, f[1][p] = v.y;
        }
    }
}

// One tile of both operands into the accumulators; `steps` of 16 dwords hold values.
template <class T, bool A_OC, bool B_OC, int BO, int TT>
__device__ __forceinline__ void multiply(const uint32_t *a_lds, const uint32_t *b_lds, int a_off, int b_off, int steps, f32x4 (&acc)[TT][TT])
{
#pragma unroll
    for (int s = 0; s < kDwords / 16; ++s) {
        if (s >= steps) break;
        uint32_t a[TT][4], b[TT][4];
        if constexpr (A_OC) read_oc<BO, TT>(a_lds, a_off, s, a); else read_kc<BO, TT>(a_lds, a_off, s, a);
        if constexpr (B_OC) read_oc<BO, TT>(b_lds, b_off, s, b); else read_kc<BO, TT>(b_lds, b_off, s, b);
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int j = 0; j < TT; ++j) acc[i][j] = T::mma(a[i], b[j], acc[i][j]);
    }
}

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
