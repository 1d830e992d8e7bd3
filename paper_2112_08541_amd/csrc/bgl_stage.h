// Device templates for large products of bf16 matrices on the matrix units (gfx950): tiles go from global memory straight into LDS, in stages of 32 or 64
// summed values, and from there as fragments of 16 x 16 x 32 MFMA instructions.
//
// Against the tiles of bgl_tile.h, which pass through registers: the loads take none, so that a wavefront keeps up to 128 x 64 sums (a fragment read from LDS
// meets 8 or 4 others instead of 4) and two workgroups still share a CU, one's epilogue beside the other's products; and a stage waits for loads that were asked
// for a stage or two before, behind one barrier.  In return rows are read in whole 16-byte pieces: they begin on multiples of 16 bytes and are padded with
// zeros to whole stages.
//
// What a load asks the L2 for are lines of 128 bytes: rows read 64 bytes at a time (stages of 32) took twice the requests and a third more time than
// rows read 128 bytes at a time.  So rows that are given are read in stages of 64, and what is written for these products alone lies in blocks of
// 16 rows x 32 values (1,024 bytes that one load of a wavefront takes, whichever index is summed).
//
// A fp32 value is three bf16 (its first 8 bits, the next 8 of what is left, the last): all 24 bits as long as the value is above 2^-110.  A product of two is
// the six products of parts that count, what is left out is below 2^-23 of it.  The parts lie one after the other ("planes"): of a row, or of a block.
//
// A tile of an operand in LDS:
//   Kc        the summed index contiguous: BO rows of 2 STEP bytes, 16-byte piece p of row r at p ^ (r & 7) (64) or p ^ (r / 2 & 3) (32), so that 8 lanes that
//             read 16 bytes each, from rows in a row, meet all banks
//   Oc        the kept index contiguous: 32 rows of BO values, blocks of 16 values moved about within a row (as in bgl_tile.h); fragments by the LDS read
//             that transposes 4 x 16 values among 16 lanes
//   OcBlocks  the same from blocks of 16 x 32: 16-byte piece p of row r at p ^ 2 (r / 2 + r / 8 & 1)
// A load of a wavefront fills 1,024 consecutive bytes of LDS, so it is the addresses it reads from that are exchanged.
#pragma once

#include "bgl_internal.h"
#include "bgl_tile.h"

namespace bgl {
namespace stage {

using tile::bf16x8;
using tile::f32x4;
using tile::s16x4;

constexpr int kThreads = 256, kWaves = kThreads / kWave;

__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
// A buffer of all memory from `base` (the same in every lane) on.
__device__ __forceinline__ i32x4 whole_memory_from(const char *base)
{
    const uint64_t at = (uint64_t)base;
    return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)at), __builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xffff)), -1, 0x00020000};
}
// LOADS times 16 bytes for each lane, from base + off[i] to lds + 1,024 i + 16 lane.  In assembly because the compiler puts a wait for all loads before the next read of LDS
// where it makes these loads itself; multiply() counts them.  (No vector register is written, so none can be lost to a load on its way.)
// Nothing in a block of assembly is known to the compiler as a load, so the block itself has what a load needs: the buffer's words may have been written by the vector
// instruction (a v_readfirstlane) right before the block, 5 wait states before a load may read them, two s_mov and s_nop 2; m0 1 before a load into LDS, s_nop 0.
// The compiler does not take m0 as something a block writes: it is put back.
template <int LOADS>
__device__ __forceinline__ void load_to_lds(i32x4 from, char *lds, const uint32_t (&off)[LOADS])
{
#define BGL_FIRST "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dwordx4 %3, %2, 0 offen lds\n\t"
#define BGL_NEXT(V) "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 " V ", %2, 0 offen lds\n\t"
#define BGL_END "s_mov_b32 m0, %0"
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    uint32_t m0;
    static_assert(LOADS == 2 || LOADS == 4 || LOADS == 6, "");
    if constexpr (LOADS == 2)
        asm volatile(BGL_FIRST BGL_NEXT("%4") BGL_END : "=&s"(m0) : "s"(to), "s"(from), "v"(off[0]), "v"(off[1]) : "memory", "scc");
    else if constexpr (LOADS == 4)
        asm volatile(BGL_FIRST BGL_NEXT("%4") BGL_NEXT("%5") BGL_NEXT("%6") BGL_END
                     : "=&s"(m0)
                     : "s"(to), "s"(from), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3])
                     : "memory", "scc");
    else
        asm volatile(BGL_FIRST BGL_NEXT("%4") BGL_NEXT("%5") BGL_NEXT("%6") BGL_NEXT("%7") BGL_NEXT("%8") BGL_END
                     : "=&s"(m0)
                     : "s"(to), "s"(from), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "v"(off[4]), "v"(off[5])
                     : "memory", "scc");
#undef BGL_FIRST
#undef BGL_NEXT
#undef BGL_END
}

template <int BO, int STEP_>
struct Kc {
    static constexpr int STEP = STEP_, PIECES = STEP / 8, BYTES = BO * STEP * 2, LOADS = BYTES / 1024 / kWaves;
    static_assert(LOADS * kWaves * 1024 == BYTES, "");
    const char *base;
    uint32_t off[LOADS];
    static __device__ __forceinline__ int move(int r) { return STEP == 64 ? r & 7 : r >> 1 & 3; }
    // row(i): the byte offset of the tile's row i from base, less than 2^32; of any readable row for one that does not exist
    template <class Row>
    __device__ __forceinline__ void init(const char *start, Row row)
    {
        base = start;
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = (wave_number() * LOADS + i) * (64 / PIECES) + l / PIECES;
            off[i] = row(r) + (((l % PIECES) ^ move(r)) << 4);
        }
    }
    __device__ __forceinline__ void load(char *lds, uint64_t offset, int) const
    {
        load_to_lds(whole_memory_from(base + offset), lds + wave_number() * LOADS * 1024, off);
    }
    // F fragments of rows from `first` on, the part'th 32 of the stage's summed values
    template <int F>
    static __device__ __forceinline__ void read(const char *lds, int first, int part, bf16x8 (&f)[F])
    {
        const int l = threadIdx.x & 63;
        const char *at = lds + (first + (l & 15)) * STEP * 2 + (((part * 4 + (l >> 4)) ^ move(l & 15)) << 4);
#pragma unroll
        for (int t = 0; t < F; ++t) f[t] = *reinterpret_cast<const bf16x8 *>(at + t * 16 * STEP * 2);
    }
};

// A fragment of 16 kept x 32 summed values where the kept index is contiguous: lane (i / 4, i % 4) of 16 names 4 kept values of summed row i / 4, and 4 rows
// further on, and gets kept value i of all eight.
__device__ __forceinline__ bf16x8 transposed(const char *at, int four_rows)
{
    uint2 h[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
        h[u] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + u * four_rows)));
    const uint4 both{h[0].x, h[0].y, h[1].x, h[1].y};
    return __builtin_bit_cast(bf16x8, both);
}

template <int BO>
struct Oc {
    static constexpr int STEP = 32, BYTES = BO * STEP * 2, LOADS = BYTES / 1024 / kWaves, ROW = BO * 2;
    const char *base;
    uint32_t off[LOADS], stride;
    static __device__ __forceinline__ int move(int k) { return (k & 3) | (k >> 3 & 1) << 2; }
    static __device__ __forceinline__ int place(int k, int c) { return k * ROW + ((((c >> 4) ^ move(k)) << 4 | (c & 15)) << 1); }
    // which of the 32 summed rows the thread's load i is of
    static __device__ __forceinline__ int row_of(int i) { return ((wave_number() * LOADS + i) * 1024 + (int)(threadIdx.x & 63) * 16) / ROW; }
    // base: the first summed row; columns o0 .. o0 + BO - 1 of `width` readable ones (a multiple of 8); what is behind them is anything
    __device__ __forceinline__ void init(const char *start, uint32_t stride_bytes, int o0, int width)
    {
        base = start;
        stride = stride_bytes;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (wave_number() * LOADS + i) * 1024 + (int)(threadIdx.x & 63) * 16, k = at / ROW, p = at % ROW / 16;
            const int column = o0 + (((p >> 1) ^ move(k)) << 4 | (p & 1) << 3);
            off[i] = k * stride + (column < width ? column * 2 : 0);
        }
    }
    // left: summed rows that exist from this step on; the last one stands in for others
    __device__ __forceinline__ void load(char *lds, uint64_t offset, int left) const
    {
        const auto from = whole_memory_from(base + offset);
        char *const to = lds + wave_number() * LOADS * 1024;
        if (left >= STEP) return load_to_lds(from, to, off);
        uint32_t there[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int k = row_of(i), beyond = k >= left ? k - (left - 1) : 0;
            there[i] = off[i] - beyond * stride;
        }
        load_to_lds(from, to, there);
    }
    template <int F>
    static __device__ __forceinline__ void read(const char *lds, int first, int, bf16x8 (&f)[F])
    {
        const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
#pragma unroll
        for (int t = 0; t < F; ++t) f[t] = transposed(lds + place(8 * g + (i >> 2), first + 16 * t + 4 * (i & 3)), 4 * ROW);
    }
};

// Blocks of 16 summed rows x 32 kept values, 1,024 bytes each, those of 16 summed rows one after the other.  The summed rows exist to a multiple of 32.
template <int BO>
struct OcBlocks {
    static constexpr int STEP = 32, ACROSS = BO / 32, BYTES = BO * STEP * 2, LOADS = BYTES / 1024 / kWaves;
    const char *base;
    uint32_t off[LOADS];
    static __device__ __forceinline__ int move(int r) { return ((r >> 1) ^ (r >> 3)) & 1 ? 2 : 0; }
    // down: bytes from 16 summed rows to the next 16, across: from a block to the next; first: of the tile's ACROSS blocks, of `blocks` that exist
    __device__ __forceinline__ void init(const char *start, uint32_t down, uint32_t across, int first, int blocks)
    {
        base = start;
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int q = wave_number() * LOADS + i, b = first + q % ACROSS;
            off[i] = q / ACROSS * down + (b < blocks ? b : blocks - 1) * across + (l >> 2) * 64 + (((l & 3) ^ move(l >> 2)) << 4);
        }
    }
    __device__ __forceinline__ void load(char *lds, uint64_t offset, int) const
    {
        load_to_lds(whole_memory_from(base + offset), lds + wave_number() * LOADS * 1024, off);
    }
    template <int F>
    static __device__ __forceinline__ void read(const char *lds, int first, int, bf16x8 (&f)[F])
    {
        const int l = threadIdx.x & 63, i = l & 15, g = l >> 4, r = 8 * (g & 1) + (i >> 2);
#pragma unroll
        for (int t = 0; t < F; ++t) {
            const int c = first + 16 * t + 4 * (i & 3);
            f[t] = transposed(lds + ((g >> 1) * ACROSS + (c >> 5)) * 1024 + r * 64 + (((c >> 3 & 3) ^ move(r)) << 4) + (c & 4) * 2, 4 * 64);
        }
    }
};

// Tiles in an order for eight XCDs (workgroup numbers go round them): each takes every eighth of the slow tiles, `group` of these at a time, which share its L2
// while the fast ones go by.  With few slow tiles that would leave XCDs with less to do, or with nothing: then all tiles in a row.
constexpr int64_t kDealtFrom = 64;
inline int64_t tile_count(int64_t slow_tiles, int64_t fast_tiles) { return (slow_tiles < kDealtFrom ? slow_tiles : (slow_tiles + 7) / 8 * 8) * fast_tiles; }
__device__ __forceinline__ bool tile_of(uint32_t id, uint32_t slow_tiles, uint32_t fast_tiles, uint32_t group, int64_t &slow, int &fast)
{
    if (slow_tiles < kDealtFrom) {
        slow = __builtin_amdgcn_readfirstlane(id / fast_tiles);
        fast = __builtin_amdgcn_readfirstlane(id % fast_tiles);
        return true;
    }
    const uint32_t j = id >> 3, mine = (slow_tiles + 7) / 8, g = j / (group * fast_tiles) * group, in = j - g * fast_tiles;
    const uint32_t wide = mine - g < group ? mine - g : group;
    fast = __builtin_amdgcn_readfirstlane(in / wide);
    slow = __builtin_amdgcn_readfirstlane((g + in % wide) * 8 + (id & 7));
    return slow < slow_tiles;
}

// How a product goes through its operands: bytes from one stage's summed values to the next, and from one plane to the next.
struct Walk {
    uint32_t a_block, b_block, a_plane, b_plane;
    int count;  // of the summed index, more than 0
    int first;  // stage the product begins with, less than their number; it goes round
};

// A workgroup of 2 x 2 wavefronts, each with FA x FB fragments.
template <int FA_, int FB_>
struct Cut {
    static constexpr int FA = FA_, FB = FB_, BA = 32 * FA, BB = 32 * FB;
    static __device__ __forceinline__ int a_off() { return wave_number() / 2 * 16 * FA; }
    static __device__ __forceinline__ int b_off() { return wave_number() % 2 * 16 * FB; }
};

// Two workgroups a CU: as many stages as 80 KB hold.
template <class A, class B>
constexpr int stages() { return 81920 / (A::BYTES + B::BYTES); }
template <class A, class B>
constexpr int lds_bytes() { return stages<A, B>() * (A::BYTES + B::BYTES); }

// What operands are made of: a bf16; two bf16 of A's values and one of B's; three bf16 of a value; a half.  PLANES: A's.  A, B: the planes of product p, hexadecimal digit p.
enum Kind { ONE_BF16, TWO_BF16, THREE_BF16, ONE_HALF };
template <Kind KIND>
struct Pairs {
    static constexpr int PLANES = KIND == THREE_BF16 ? 3 : KIND == TWO_BF16 ? 2 : 1, COUNT = PLANES == 3 ? 6 : PLANES;
    static constexpr uint32_t A = PLANES == 3 ? 0x010210 : 0x10, B = PLANES == 3 ? 0x211000 : 0;
};
template <Kind KIND>
__device__ __forceinline__ f32x4 mma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c)
{
    if constexpr (KIND == ONE_HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Adds the product to acc: of a fragment pair a lane has rows 4 (lane / 16) .. + 3 of a and row lane % 16 of b, TURNED the other way round.  also(stage, plane of b, a's fragments) sees every 32 summed values.  Ends with all of LDS free.
template <Kind KIND, bool TURNED, class A, class B, class C, class Also>
__device__ __forceinline__ void multiply(char *lds, const A &a, const B &b, const Walk &w, f32x4 (&acc)[C::FA][C::FB], Also also)
{
    static_assert(A::STEP == B::STEP, "");
    constexpr int STEP = A::STEP, STAGES = stages<A, B>(), PLANES = Pairs<KIND>::PLANES, PAIRS = Pairs<KIND>::COUNT, BYTES = A::BYTES + B::BYTES, LOADS = A::LOADS + B::LOADS;
    static_assert(STAGES == 2 || STAGES == 3, "");
    constexpr uint32_t PLANE_A = Pairs<KIND>::A, PLANE_B = Pairs<KIND>::B;
    const int blocks = (w.count + STEP - 1) / STEP, steps = blocks * PAIRS;
    int block = w.first, pair = 0, to = 0;  // of the next stage to load
    const auto load = [&] {
        char *at = lds + to * BYTES;
        const int left = w.count - block * STEP;
        a.load(at, (uint64_t)block * w.a_block + (PLANES > 1 ? (PLANE_A >> 4 * pair & 3) * w.a_plane : 0), left);
        b.load(at + A::BYTES, (uint64_t)block * w.b_block + (PLANES > 1 ? (PLANE_B >> 4 * pair & 3) * w.b_plane : 0), left);
        if (++pair == PAIRS) {
            pair = 0;
            if (++block == blocks) block = 0;
        }
        if (++to == STAGES) to = 0;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if (s < steps) load();
    int at = 0, plane = 0;
    int s = 0;
    do {  // (a loop that may not run at all kept the sums before it beside those after it)
        // this stage's loads have come (all wavefronts': the barrier), and the buffer of the stage before has been read by all
        if (STAGES == 3 && s + 1 < steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + STAGES - 1 < steps) load();
        const char *from = lds + at * BYTES;
#pragma unroll
        for (int part = 0; part < STEP / 32; ++part) {
            bf16x8 fa[C::FA], fb[C::FB];
            B::read(from + A::BYTES, C::b_off(), part, fb);
            A::read(from, C::a_off(), part, fa);
#pragma unroll
            for (int i = 0; i < C::FA; ++i)
#pragma unroll
                for (int j = 0; j < C::FB; ++j)
                    acc[i][j] = TURNED ? mma<KIND>(fb[j], fa[i], acc[i][j]) : mma<KIND>(fa[i], fb[j], acc[i][j]);
            also(s, PLANE_B >> 4 * plane & 3, fa);
        }
        if (++plane == PAIRS) plane = 0;
        if (++at == STAGES) at = 0;
        asm volatile("" ::: "memory");
    } while (++s < steps);
    __syncthreads();
}

}  // namespace stage
}  // namespace bgl
