// Layer norm over each row of a batch, and its gradients.
//
//   m = mean x, v = mean (x - m)^2, r = 1 / sqrt(v + eps), h = (x - m) r, y = h g + b            k_norm_forward
//   d = dy g, dx = r (d - mean d - h mean(d h)), dg = sum over rows of dy h, db = of dy            k_norm_backward, k_norm_reduce
//
// Memory bounds both: a row is read once into the registers of a team of threads, 16 values a thread, and everything else happens there.
#include "bgl_internal.h"
#include "bgl_reduce.h"
#include "bgl_tile.h"

#include <cmath>
#include <type_traits>

namespace bgl {
namespace {

using namespace tile;

constexpr int kValues = 16;          // of a row a thread holds
constexpr int64_t kMostThreads = (int64_t)1 << 31;     // of a launch, which has room for 2^32 - 1
constexpr int kMaxParts = 512;       // workgroups of a backward call that sums weight gradients, so rows of its partial sums
constexpr float kFar = 0x1p-80f;     // scales rows whose squares leave fp32's range
constexpr float kAway = 16.0f;       // deviations from zero that a row's mean has at most to be used as it is kept: h is off by 2^-24 of these

template <class T>
struct NormArgs {
    const typename T::elem *x, *dy, *weight, *bias;
    typename T::elem *out, *dweight, *dbias;  // out: y or dx
    float *saved;        // n x {m, r}
    float *partial;      // parts x {dg, db} x width
    int64_t n, x_stride, dy_stride, out_stride;
    int width, parts;
    float eps;
};

// A team's threads hold chunks t, t + TEAM, t + 2 TEAM, ... of 16 bytes each.  Of the row they may have FULL ones alone, WHOLE ones
// or none, or any part.
enum Fit { ANY, WHOLE, FULL };
template <class T, int TEAM, int VALUES = kValues, Fit FIT = ANY>
struct Piece {
    static constexpr int CHUNKS = VALUES / T::VEC;
    int first;  // the thread's first value
    int width;
    __device__ __forceinline__ Piece(int t, int w) : first(t * T::VEC), width(w) {}
    __device__ __forceinline__ int left(int c) const
    {
        const int values = width - first - c * TEAM * T::VEC;
        return FIT == FULL || (FIT == WHOLE && values > 0) ? T::VEC : values;
    }
    __device__ __forceinline__ void read(const typename T::elem *row, uint4 (&raw)[CHUNKS]) const
    {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            raw[c] = uint4{0, 0, 0, 0};
            const typename T::elem *from = row + first + c * TEAM * T::VEC;
            // (of rows of any width, the pieces that the whole team has: 100,000 x 1,001 f32 backward 289 us without this)
            if (FIT == ANY && (c + 1) * TEAM * T::VEC <= width) raw[c] = load_any<uint4>(from);
            else if (left(c) > 0) raw[c] = FIT != ANY ? load_any<uint4>(from) : load_end<T>(from, left(c), width);
        }
    }
    static __device__ __forceinline__ void values(const uint4 (&raw)[CHUNKS], float (&v)[VALUES])
    {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const uint32_t d[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (T::PER == 1) v[c * 4 + i] = __uint_as_float(d[i]);
                else v[c * 8 + 2 * i] = __uint_as_float(d[i] << 16), v[c * 8 + 2 * i + 1] = __uint_as_float(d[i] & 0xffff0000u);
            }
        }
    }
    __device__ __forceinline__ void load(const typename T::elem *row, float (&v)[VALUES]) const
    {
        uint4 raw[CHUNKS];
        read(row, raw);
        values(raw, v);
    }
    // f(i): does value i exist
    __device__ __forceinline__ bool has(int i) const { return FIT == WHOLE ? left(i / T::VEC) > 0 : i % T::VEC < left(i / T::VEC); }
    __device__ __forceinline__ void store(typename T::elem *row, const float (&v)[VALUES]) const
    {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            typename T::elem e[T::VEC];
#pragma unroll
            for (int i = 0; i < T::VEC; ++i) e[i] = T::put(v[c * T::VEC + i]);
            typename T::elem *to = row + first + c * TEAM * T::VEC;
            if (left(c) >= T::VEC) {
                __builtin_memcpy(to, e, 16);
            } else if (FIT == ANY) {
#pragma unroll
                for (int i = 0; i < T::VEC; ++i)
                    if (i < left(c)) to[i] = e[i];
            }
        }
    }
};

// Two sums over a team.  lds: two floats for each wavefront, and as many again for every other call (a wavefront may be a call ahead).
template <int TEAM>
__device__ __forceinline__ void team_sums(float &a, float &b, float *lds, int &turn)
{
    a = sum_across<(TEAM < 64 ? TEAM : 64)>(a);
    b = sum_across<(TEAM < 64 ? TEAM : 64)>(b);
    if constexpr (TEAM > 64) {
        constexpr int WAVES = TEAM / 64;
        const int t = threadIdx.x % TEAM;
        float *at = lds + (threadIdx.x / TEAM * 2 + turn) * WAVES * 2;
        turn ^= 1;
        if (t % 64 == 0) at[t / 64 * 2] = a, at[t / 64 * 2 + 1] = b;
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) a += at[2 * w], b += at[2 * w + 1];
    }
}

template <int TEAM>
constexpr int norm_threads() { return TEAM < 256 ? 256 : TEAM; }

// The mean, in two parts (m, what fp32 has of the values' mean, and the mean of what is left then, so that rows far from zero keep their spread), and r of the row
// that the team holds.  The sum that m is made of rounds as the values are large: where they differ no more than that (the mean square of x - m is below 2^-28 m^2), or their
// squares leave fp32's range, m is made once more, of the differences from the row's first value, which are exact for values near each other, and 0 for equal ones: rows of
// equal values are normalised to 0 whatever they are.  Beyond the range all of that is of values scaled by a power of two (the same for the whole team).
template <class T, int TEAM, Fit FIT>
__device__ __forceinline__ void moments(const Piece<T, TEAM, kValues, FIT> &p, float (&v)[kValues], float eps, float *lds, int &turn, float &mean, float &rest, float &r)
{
#pragma clang fp contract(off)  // (v - m with the product m unrounded would not fit the m that is kept)
    const float share = 1.0f / (float)p.width;
    float scale = 1.0f;
    float s = 0.0f, unused = 0.0f;
#pragma unroll
    for (int i = 0; i < kValues; ++i) s += v[i];
    team_sums<TEAM>(s, unused, lds, turn);
    float m = s * share, c = 0.0f, q = 0.0f;
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
        const float d = p.has(i) ? v[i] - m : 0.0f;
        c += d;
        q = fmaf(d, d, q);
    }
    team_sums<TEAM>(c, q, lds, turn);
    const bool far = !(q < INFINITY), again = far || q * share <= m * m * 0x1p-28f;
    // (a workgroup's teams of more than a wavefront share barriers: where one goes again all do, and the others leave what they have)
    if (TEAM > 64 ? __syncthreads_or(again) : again) {
        if (far) scale = kFar;
        float one = p.first == 0 ? v[0] * scale : 0.0f, c1 = 0.0f, q1 = 0.0f;
        team_sums<TEAM>(one, unused, lds, turn);
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < kValues; ++i) s += p.has(i) ? v[i] * scale - one : 0.0f;
        team_sums<TEAM>(s, unused, lds, turn);
        const float m1 = one + s * share;
#pragma unroll
        for (int i = 0; i < kValues; ++i) {
            const float d = p.has(i) ? v[i] * scale - m1 : 0.0f;
            c1 += d;
            q1 = fmaf(d, d, q1);
        }
        team_sums<TEAM>(c1, q1, lds, turn);
        if (again) m = m1, c = c1, q = q1;
    }
    c *= share;
    const float var = fmaxf(fmaf(q, share, -c * c), 0.0f) + (q - q);  // (fmaxf would hide a NaN)
    const float most = 1.0f / sqrtf(eps);
    r = scale / sqrtf(var + eps * scale * scale);
    if (r > most) r = most;  // (scaled, eps may be nothing beside the variance, and that nothing too)
    mean = m / scale, rest = c / scale;
}

// A row's threads: 16 values each, a team of 1 to 1,024.  A workgroup has 256 threads or one team.  What fits the team
// better asks less often whether a value is there: 302,709 x 512 bf16 with 29 vector instructions for a value took 40 % longer, bound by these and not by the memory; now
// 101 us (6.1 TB/s), 428,377 x 256 f32 140 (6.3 TB/s).
template <class T, int TEAM, Fit FIT>
__global__ void __launch_bounds__(norm_threads<TEAM>()) k_norm_forward(NormArgs<T> a)
{
    constexpr int TEAMS = norm_threads<TEAM>() / TEAM;
    __shared__ float lds[TEAM > 64 ? norm_threads<TEAM>() / 64 * 4 : 1];
    int turn = 0;
    const Piece<T, TEAM, kValues, FIT> p(threadIdx.x % TEAM, a.width);
    const int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM;
    const bool live = row < a.n;
    if (TEAM <= 64 && !live) return;
    float v[kValues], g[kValues], b[kValues], mean, rest, r;
    p.load(a.x + (live ? row : a.n - 1) * a.x_stride, v);
#pragma unroll
    for (int i = 0; i < kValues; ++i) g[i] = 1.0f, b[i] = 0.0f;
    if (a.weight) p.load(a.weight, g);
    if (a.bias) p.load(a.bias, b);
    moments<T, TEAM, FIT>(p, v, a.eps, lds, turn, mean, rest, r);
    if (!live) return;
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
        const float h = ((v[i] - mean) - rest) * r;
        v[i] = fmaf(h, g[i], b[i]);
    }
    p.store(a.out + row * a.out_stride, v);
    if (a.saved && threadIdx.x % TEAM == 0) a.saved[2 * row] = mean + rest, a.saved[2 * row + 1] = r;
}

// SUMS: the weight's gradients are asked for; a thread then keeps those of its 16 columns over the rows of its team, the workgroup adds up its teams' and
// leaves a row of partial sums.  The widest rows are then 512 threads of 32 values: 1,024 of 16 have 128 registers each, which these sums exceed.
// Behind the forward call of the same rows 428,377 x 256 f32 253 us, 302,709 x 512 bf16 186 (5.2 and 5.0 TB/s); of rows that the caches have in part 158 and 120.
template <class T, int TEAM, bool SUMS, Fit FIT, int VALUES = kValues>
__global__ void __launch_bounds__(norm_threads<TEAM>()) k_norm_backward(NormArgs<T> a)
{
    constexpr int TEAMS = norm_threads<TEAM>() / TEAM;
    __shared__ float lds[TEAM > 64 ? norm_threads<TEAM>() / 64 * 4 : 1];
    __shared__ float sums[SUMS && TEAMS > 1 ? TEAMS * TEAM * VALUES : 1];
    int turn = 0;
    const Piece<T, TEAM, VALUES, FIT> p(threadIdx.x % TEAM, a.width);
    const float share = 1.0f / (float)a.width;
    float g[VALUES], dg[VALUES], db[VALUES];
#pragma unroll
    for (int i = 0; i < VALUES; ++i) g[i] = 1.0f, dg[i] = db[i] = 0.0f;
    if (a.weight) p.load(a.weight, g);
    const int64_t step = (int64_t)gridDim.x * TEAMS;
    // (all teams of a workgroup go round equally often: they share barriers)
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.n; first += step) {
        const int64_t row = first + threadIdx.x / TEAM;
        const bool live = row < a.n;
        float dy[VALUES], h[VALUES];
        float c1 = 0.0f, c2 = 0.0f, mean = 0.0f, r = 0.0f;
        if (live) {
            p.load(a.dy + row * a.dy_stride, dy);
            p.load(a.x + row * a.x_stride, h);
            mean = a.saved[2 * row], r = a.saved[2 * row + 1];
        }
        // what the mean's rounding left, in rows so far from zero that it counts beside their spread; there, places behind the row could be beyond the type, too
        const bool away = !(fabsf(mean) * r <= kAway);
        bool any = away;
        if constexpr (TEAM > 64 && TEAMS > 1)
            for (int64_t other = first; other < first + TEAMS && other < a.n; ++other) any |= !(fabsf(a.saved[2 * other]) * a.saved[2 * other + 1] <= kAway);
        if (any) {
            float rest = 0.0f, unused = 0.0f;
#pragma unroll
            for (int i = 0; i < VALUES; ++i) rest += away && p.has(i) ? h[i] - mean : 0.0f;
            team_sums<TEAM>(rest, unused, lds, turn);
            rest *= share;
            if (away) {
#pragma unroll
                for (int i = 0; i < VALUES; ++i) h[i] = p.has(i) ? (h[i] - mean) - rest : 0.0f;
                mean = 0.0f;
            }
        }
        if (live) {
#pragma unroll
            for (int i = 0; i < VALUES; ++i) {
                h[i] = (h[i] - mean) * r;  // (behind the row a number up to kAway: dy is 0 there)
                if constexpr (SUMS) dg[i] = fmaf(dy[i], h[i], dg[i]), db[i] += dy[i];
                dy[i] *= g[i];
                c1 += dy[i];
                c2 = fmaf(dy[i], h[i], c2);
            }
        }
        if (!a.out) continue;
        team_sums<TEAM>(c1, c2, lds, turn);
        if (live) {
            c1 *= share, c2 *= share;
#pragma unroll
            for (int i = 0; i < VALUES; ++i) dy[i] = r * (dy[i] - fmaf(h[i], c2, c1));
            p.store(a.out + row * a.out_stride, dy);
        }
    }
    if constexpr (SUMS) {
        const int team = threadIdx.x / TEAM;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float *to = a.partial + ((int64_t)blockIdx.x * 2 + which) * a.width;
            if constexpr (TEAMS > 1) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < VALUES; ++i) sums[(team * VALUES + i) * TEAM + threadIdx.x % TEAM] = which ? db[i] : dg[i];
                __syncthreads();
                for (int j = threadIdx.x; j < TEAM * VALUES; j += norm_threads<TEAM>()) {
                    float s = 0.0f;
#pragma unroll
                    for (int t = 0; t < TEAMS; ++t) s += sums[t * VALUES * TEAM + j];
                    const int i = j / TEAM, at = (j % TEAM + i / T::VEC * TEAM) * T::VEC + i % T::VEC;
                    if (at < a.width) to[at] = s;
                }
            } else {
#pragma unroll
                for (int i = 0; i < VALUES; ++i)
                    if (p.has(i)) to[p.first + i / T::VEC * TEAM * T::VEC + i % T::VEC] = which ? db[i] : dg[i];
            }
        }
    }
}

// The partial rows' sums: 32 columns a workgroup, every 32nd row a thread, eight of them on their way at a time.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_reduce(NormArgs<T> a)
{
    constexpr int LANES = 32, AHEAD = 8;
    __shared__ float part[LANES][33];
    const int64_t all = 2 * (int64_t)a.width, at = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
    const int lane = threadIdx.x / 32;
    const float *from = a.partial + (at < all ? at : 0);
    float s = 0.0f;
    for (int p = lane; p < a.parts; p += LANES * AHEAD) {
        float v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = p + u * LANES < a.parts ? from[(p + u * LANES) * all] : 0.0f;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) s += v[u];
    }
    part[lane][threadIdx.x % 32] = s;
    __syncthreads();
    // a column's sums to neighbouring lanes
    s = sum_across<32>(part[threadIdx.x % 32][lane]);
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    if (threadIdx.x % 32 > 0 || c >= all) return;
    typename T::elem *to = c < a.width ? a.dweight : a.dbias;
    if (to) to[c < a.width ? c : c - a.width] = T::put(s);
}

int team_of(int width)
{
    int team = 1;
    while (team * kValues < width) team *= 2;
    return team;
}
int teams_of(int team) { return team < 256 ? 256 / team : 1; }

int parts_of(int width, int64_t n)
{
    // (a row of partial sums is as wide as two of x: with one for each of few wide rows they took longer than these)
    const int teams = teams_of(team_of(width));
    const int64_t groups = teams > 1 ? ceil_div(n, teams) : ceil_div(n, 4), most = teams > 1 ? kMaxParts : kMaxParts / 2;
    return (int)(groups < most ? groups : most);
}

template <class F>
void with_team(int team, F f)
{
    switch (team) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    case 16: return f(std::integral_constant<int, 16>{});
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    case 128: return f(std::integral_constant<int, 128>{});
    case 256: return f(std::integral_constant<int, 256>{});
    case 512: return f(std::integral_constant<int, 512>{});
    default: return f(std::integral_constant<int, 1024>{});
    }
}

template <class T>
int forward(NormArgs<T> a, hipStream_t st)
{
    with_team(team_of(a.width), [&](auto team) {
        constexpr int TEAM = decltype(team)::value;
        const int64_t n = a.n, most = kMostThreads / TEAM;
        for (int64_t row0 = 0; row0 < n; row0 += most) {
            a.n = n - row0 < most ? n - row0 : most;
            const dim3 grid((unsigned)ceil_div(a.n, teams_of(TEAM))), threads(norm_threads<TEAM>());
            if (a.width == TEAM * kValues) k_norm_forward<T, TEAM, FULL><<<grid, threads, 0, st>>>(a);
            else if (a.width % T::VEC == 0) k_norm_forward<T, TEAM, WHOLE><<<grid, threads, 0, st>>>(a);
            else k_norm_forward<T, TEAM, ANY><<<grid, threads, 0, st>>>(a);
            a.x += a.n * a.x_stride, a.out += a.n * a.out_stride, a.saved = a.saved ? a.saved + 2 * a.n : nullptr;
        }
    });
    BGL_HIP(hipGetLastError());
    return BGL_OK;
}

template <class T>
int backward(NormArgs<T> a, hipStream_t st)
{
    const bool sums = a.dweight || a.dbias;
    if (a.n > 0 && (sums || a.out)) {
        with_team(team_of(a.width), [&](auto team) {
            constexpr int TEAM = decltype(team)::value;
            constexpr int LEAST = TEAM < 512 ? TEAM : 512;
            const auto go = [&](auto fit) {
                constexpr Fit FIT = decltype(fit)::value;
                if (sums) k_norm_backward<T, LEAST, true, FIT, kValues * TEAM / LEAST><<<dim3((unsigned)a.parts), dim3(norm_threads<LEAST>()), 0, st>>>(a);
                else k_norm_backward<T, TEAM, false, FIT><<<dim3((unsigned)ceil_div(a.n < kMostThreads / TEAM ? a.n : kMostThreads / TEAM, teams_of(TEAM))), dim3(norm_threads<TEAM>()), 0, st>>>(a);
            };
            if (a.width == TEAM * kValues) go(std::integral_constant<Fit, FULL>{});
            else if (a.width % T::VEC == 0) go(std::integral_constant<Fit, WHOLE>{});
            else go(std::integral_constant<Fit, ANY>{});
        });
        BGL_HIP(hipGetLastError());
    }
    if (sums) {
        k_norm_reduce<T><<<dim3((unsigned)ceil_div(2 * (int64_t)a.width, 32)), dim3(1024), 0, st>>>(a);
        BGL_HIP(hipGetLastError());
    }
    return BGL_OK;
}

int check_norm(const bgl_layer_norm_t *norm, int64_t n)
{
    if (!norm) BGL_FAIL(BGL_EINVAL, "norm is null");
    if (norm->dtype != BGL_F32 && norm->dtype != BGL_BF16) BGL_FAIL(BGL_EINVAL, "unknown dtype %d", norm->dtype);
    if (norm->width < 1) BGL_FAIL(BGL_EINVAL, "width %d", norm->width);
    if (norm->width > BGL_MAX_DIM) BGL_FAIL(BGL_EUNSUPPORTED, "width %d is more than %d", norm->width, BGL_MAX_DIM);
    if (!(norm->eps >= 1e-12f && norm->eps < INFINITY)) BGL_FAIL(BGL_EINVAL, "eps %g is not in [1e-12, inf)", (double)norm->eps);
    if (n < 0 || n >= (int64_t)1 << 31) BGL_FAIL(BGL_EINVAL, "%lld rows", (long long)n);
    return BGL_OK;
}
size_t norm_bytes(const bgl_layer_norm_t *norm, int64_t n) { return (size_t)parts_of(norm->width, n) * 2 * norm->width * sizeof(float); }

}  // namespace
}  // namespace bgl

using namespace bgl;

extern "C" int bgl_layer_norm_workspace_bytes(const bgl_layer_norm_t *norm, int64_t n, size_t *bytes)
try {
    if (!bytes) BGL_FAIL(BGL_EINVAL, "bytes is null");
    BGL_TRY(check_norm(norm, n));
    *bytes = norm_bytes(norm, n);
    return BGL_OK;
} BGL_NOTHROW_END

extern "C" int bgl_layer_norm_forward(const bgl_layer_norm_t *norm, int64_t n, const void *x, int64_t x_stride, const void *weight, const void *bias,
                                      void *y, int64_t y_stride, float *saved, void *stream)
try {
    BGL_TRY(check_norm(norm, n));
    const int es = norm->dtype == BGL_F32 ? 4 : 2;
    BGL_TRY(check_rows("x", x, x_stride, norm->width, es, n > 0));
    BGL_TRY(check_rows("y", y, y_stride, norm->width, es, n > 0));
    if (!aligned(weight, es) || !aligned(bias, es) || !aligned(saved, 4)) BGL_FAIL(BGL_EINVAL, "weight, bias or saved is misaligned");
    if (n == 0) return BGL_OK;
    const auto run = [&](auto type) {
        using T = decltype(type);
        using E = typename T::elem;
        NormArgs<T> a{};
        a.x = (const E *)x, a.weight = (const E *)weight, a.bias = (const E *)bias, a.out = (E *)y, a.saved = saved;
        a.n = n, a.x_stride = x_stride, a.out_stride = y_stride, a.width = norm->width, a.eps = norm->eps;
        return forward<T>(a, (hipStream_t)stream);
    };
    return norm->dtype == BGL_F32 ? run(tile::F32{}) : run(tile::BF16{});
} BGL_NOTHROW_END

extern "C" int bgl_layer_norm_backward(const bgl_layer_norm_t *norm, int64_t n, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                                       const void *weight, const float *saved, void *dx, int64_t dx_stride, void *dweight, void *dbias,
                                       void *workspace, size_t workspace_bytes, void *stream)
try {
    BGL_TRY(check_norm(norm, n));
    const int es = norm->dtype == BGL_F32 ? 4 : 2;
    BGL_TRY(check_rows("dy", dy, dy_stride, norm->width, es, n > 0));
    BGL_TRY(check_rows("x", x, x_stride, norm->width, es, n > 0));
    BGL_TRY(check_rows("dx", dx, dx_stride, norm->width, es, false));
    if (n > 0 && !saved) BGL_FAIL(BGL_EINVAL, "saved is null");
    if (!aligned(weight, es) || !aligned(saved, 4) || !aligned(dweight, es) || !aligned(dbias, es))
        BGL_FAIL(BGL_EINVAL, "weight, saved, dweight or dbias is misaligned");
    const size_t need = dweight || dbias ? norm_bytes(norm, n) : 0;
    if (need > 0) {
        if (!workspace || !aligned(workspace, 256)) BGL_FAIL(BGL_EINVAL, "workspace is null or not 256-byte aligned");
        if (workspace_bytes < need) BGL_FAIL(BGL_ECAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    }
    const auto run = [&](auto type) {
        using T = decltype(type);
        using E = typename T::elem;
        NormArgs<T> a{};
        a.x = (const E *)x, a.dy = (const E *)dy, a.weight = (const E *)weight, a.out = (E *)dx, a.dweight = (E *)dweight, a.dbias = (E *)dbias;
        a.saved = const_cast<float *>(saved), a.partial = (float *)workspace;
        a.n = n, a.x_stride = x_stride, a.dy_stride = dy_stride, a.out_stride = dx_stride;
        a.width = norm->width, a.parts = parts_of(norm->width, n), a.eps = norm->eps;
        return backward<T>(a, (hipStream_t)stream);
    };
    return norm->dtype == BGL_F32 ? run(tile::F32{}) : run(tile::BF16{});
} BGL_NOTHROW_END
