// Norms of queries and keys for each head, and their rotation by position, in one pass (gfx950).
//
//   y = x / sqrt(mean x^2 + eps) w over the d elements of a head,   (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin) for its pairs
//
// with the angle position base^(-2 p / rot) for pair p.  Memory bound: every element is read once and written once.  A lane holds a unit of
// sixteen elements of a head, both of each of its eight pairs, so that the rotation needs no other lane and the norm a sum over the few lanes of a head.
// Angles are formed in 64 bits as parts of a turn (a position of 100000 has lost 0.004 rad in 32), once for a row and a pair, by one thread
// of the workgroup; all heads of the row take cosine and sine from LDS.
// Backward: with dy the gradient turned back, x^ = x / sqrt(...): dw = sum dy x^ over rows and heads, dx = r (dy w - x^ mean(dy w x^)).  A workgroup keeps
// its sums for the weights in registers over all of its rows; a second launch adds up the workgroups'.
// 8192 rows of 32 + 8 heads of 128 in bf16: 35 us, 4.7 TB/s (kernel 29).  Backward, 64 x 197 rows of 2 x 12 heads of 64: 35 us (3.3 TB/s; wavefronts wait for two thirds of
// it, one turn of rows a workgroup whose angles come before its first load) and 5.  fp32, 8192 rows of 32 + 8 heads of 128: 70 us (4.8 TB/s), backward 115 (4.4).
// Where 16 divides d and rot a unit is two chunks of 8; elsewhere each element is loaded and stored by itself: 8192 rows of 32 + 8 heads in bf16, d 80 and rot 20: 120 us (0.9 TB/s),
// backward 163; d 96 and rot 24: 135 and 175.
#include "seq_kernels.h"
#include "../csrc/lm/lm_device.h"

namespace stl {
namespace seq {

using lm::Chunk;

// Pairs 0 .. rot / 2 - 1 are turned; those behind them are the other elements two by two (the second of the last one may not exist), left as they are.
struct Pair {
    int a, b;
};
template <bool ADJ>
__device__ __forceinline__ Pair pair_of(int p, int rot)
{
    const int half = rot / 2;
    if (p >= half || ADJ) return Pair{2 * p, 2 * p + 1};
    return Pair{p, p + half};
}

// The sixteen elements of a unit (pairs 8 u .. 8 u + 7) in registers.  VEC: as two chunks of 8, where 16 divides d and rot.
// ADJ: pair k is (x[2 k], x[2 k + 1]), otherwise (x[k], x[8 + k]).
template <typename T, bool ADJ, bool VEC>
struct Unit {
    static __device__ __forceinline__ int second_chunk(int u, int rot)
    {
        return ADJ || 16 * u >= rot ? 16 * u + 8 : rot / 2 + 8 * u;
    }
    static __device__ __forceinline__ int first_chunk(int u, int rot) { return ADJ || 16 * u >= rot ? 16 * u : 8 * u; }
    // as loaded, and as numbers
    struct Raw {
        Chunk<T> c[VEC ? 2 : 1];
        float f[VEC ? 1 : 16];
    };
    static __device__ __forceinline__ void load(const T *p, int u, int d, int rot, Raw &r)
    {
        if constexpr (VEC) {
            r.c[0].load(p + first_chunk(u, rot), 8);
            r.c[1].load(p + second_chunk(u, rot), 8);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Pair at = pair_of<ADJ>(8 * u + k, rot);
                r.f[ADJ ? 2 * k : k] = at.a < d ? Elem<T>::ld(p + at.a) : 0.f;
                r.f[ADJ ? 2 * k + 1 : 8 + k] = at.b < d ? Elem<T>::ld(p + at.b) : 0.f;
            }
        }
    }
    static __device__ __forceinline__ void clear(Raw &r)
    {
        r.c[0].fill(0.f);
        if constexpr (VEC) r.c[1].fill(0.f);
#pragma unroll
        for (int e = 0; e < (VEC ? 1 : 16); ++e) r.f[e] = 0.f;
    }
    static __device__ __forceinline__ void numbers(const Raw &r, float *x)
    {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = VEC ? r.c[e >> 3 & (VEC ? 1 : 0)].get(e & 7) : r.f[VEC ? 0 : e];
    }
    static __device__ __forceinline__ void load(const T *p, int u, int d, int rot, float *x)
    {
        Raw r;
        load(p, u, d, rot, r);
        numbers(r, x);
    }
    static __device__ __forceinline__ void store(T *p, int u, int d, int rot, const float *x)
    {
        if constexpr (VEC) {
            Chunk<T>::store(p + first_chunk(u, rot), 8, x);
            Chunk<T>::store(p + second_chunk(u, rot), 8, x + 8);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Pair at = pair_of<ADJ>(8 * u + k, rot);
                if (at.a < d) Elem<T>::st(p + at.a, x[ADJ ? 2 * k : k]);
                if (at.b < d) Elem<T>::st(p + at.b, x[ADJ ? 2 * k + 1 : 8 + k]);
            }
        }
    }
    // the first n pairs turned by the angles whose cosines and sines lie at `cs`, or back
    static __device__ __forceinline__ void turn(const f32x2_t *cs, int n, float *x, float back)
    {
        if (VEC && n <= 0) return;                               // (whole units are turned, or none of it)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (!VEC && k >= n) break;
            float &a = x[ADJ ? 2 * k : k], &b = x[ADJ ? 2 * k + 1 : 8 + k];
            const f32x2_t t = cs[k];
            const float s = back * t[1], was = a;
            a = fmaf(was, t[0], -(b * s));
            b = fmaf(was, s, b * t[0]);
        }
    }
};

// sum over groups of `lanes` lanes next to each other (a power of two), in every one of them
__device__ __forceinline__ float group_sum(float v, int lanes)
{
    if (lanes > 1) v += lm::dpp<0xb1, 0xf>(v, 0.f);
    if (lanes > 2) v += lm::dpp<0x4e, 0xf>(v, 0.f);
    if (lanes > 4) v += lm::dpp<0x141, 0xf>(v, 0.f);
    if (lanes > 8) v += lm::dpp<0x140, 0xf>(v, 0.f);
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
    return v;
}

struct HeadPlan {
    int units, lanes, together;              // of a head; rows whose angles are formed together
    int grid;
    bool vec;
};
HeadPlan head_plan(const HeadArgs &a, bool back)
{
    HeadPlan p;
    p.units = ((a.d + 1) / 2 + 7) / 8;
    p.lanes = 1;
    while (p.lanes < p.units) p.lanes *= 2;
    p.together = a.rows >= 8192 ? 8 : a.rows >= 4096 ? 4 : a.rows >= 2048 ? 2 : 1;
    // (backward, few heads: twice as many where the heads of these rows leave workgroups with idle lanes and there are 512 of them all the same: 12 heads of 64 in
    // eight rows are 96 of 128 places)
    if (back && p.together * a.heads[0] % (256 / p.lanes) && a.rows / (2 * p.together) >= 512) p.together *= 2;
    const int turns = (a.rows + p.together - 1) / p.together, each = (turns + 1023) / 1024;
    p.grid = (turns + each - 1) / each;                          // every workgroup as many turns, but for the last
    p.vec = a.d % 16 == 0 && a.rot % 16 == 0;
    return p;
}

// cosines and sines of the pairs of `rows` rows from `row` on, 8 units pairs a row (those that are not turned: 1 and 0)
__device__ __forceinline__ void angles(const HeadArgs &a, int pairs, int row, int rows, f32x2_t *table)
{
    const int half = a.rot / 2;
    for (int i = (int)threadIdx.x; i < rows * pairs; i += 256) {
        const int r = i / pairs, p = i % pairs;
        f32x2_t cs = {1.f, 0.f};
        if (p < half) {
            // quarters of a turn, position base^(-2 p / rot) 2 / pi: whole ones in 64 bits, so that what is left is small and the smaller of cosine and sine as
            // exact, relative to itself, as the larger
            const double quarters = (double)a.position[row + r] * (exp2(-a.log2_base * (2.0 * p / a.rot)) * 0.63661977236758134308), n = rint(quarters);
            float s, c;
            sincospif(0.5f * (float)(quarters - n), &s, &c);
            const int q = (int)(n - 4.0 * floor(0.25 * n));
            if (q & 1) {
                const float was = c;
                c = -s, s = was;
            }
            if (q & 2) c = -c, s = -s;
            cs = f32x2_t{c, s};
        }
        table[i] = cs;
    }
}

template <typename T, bool ADJ, bool VEC>
__global__ __launch_bounds__(256) void head_kernel(const HeadArgs a, const HeadPlan plan, T *out_q, T *out_k)
{
    extern __shared__ __align__(16) char smem[];
    f32x2_t *table = reinterpret_cast<f32x2_t *>(smem);
    using U = Unit<T, ADJ, VEC>;
    const int lanes = plan.lanes, pairs = 8 * plan.units;
    const int u = (int)threadIdx.x % lanes, group = (int)threadIdx.x / lanes, groups = 256 / lanes;
    const bool mine = u < plan.units;
    float w[2][16];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
#pragma unroll
        for (int e = 0; e < 16; ++e) w[side][e] = 1.f;
        if (a.w[side] && mine) U::load((const T *)a.w[side], u, a.d, a.rot, w[side]);
    }
    const float inv = 1.f / (float)a.d;
    for (int64_t row = (int64_t)blockIdx.x * plan.together; row < a.rows; row += (int64_t)gridDim.x * plan.together) {
        const int rows = a.rows - row < plan.together ? (int)(a.rows - row) : plan.together;
        __syncthreads();
        angles(a, pairs, (int)row, rows, table);
        __syncthreads();
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const int heads = a.heads[side];
            T *out = side ? out_k : out_q;
            // (every lane takes part in the sums)
            for (int from = 0; from < rows * heads; from += groups) {
                const int i = from + group, r = i / heads, h = i - r * heads;
                const bool live = mine && i < rows * heads;
                float x[16] = {};
                if (live) U::load((const T *)a.in[side] + (row + r) * a.ld_in[side] + (size_t)h * a.d, u, a.d, a.rot, x);
                if (a.norm) {
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum = fmaf(x[e], x[e], sum);
                    const float by = rsqrtf(fmaf(group_sum(sum, lanes), inv, a.eps));
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] *= by * w[side][e];
                }
                if (live) {
                    U::turn(table + r * pairs + 8 * u, a.rot / 2 - 8 * u, x, 1.f);
                    U::store(out + (row + r) * a.ld_out[side] + (size_t)h * a.d, u, a.d, a.rot, x);
                }
            }
        }
    }
}

// parts: for each workgroup the sums for the two weights, d each.  Queries first, then keys: with one side's weights and sums at a time four workgroups share a CU
template <typename T, bool ADJ, bool VEC>
__global__ __launch_bounds__(256, VEC && sizeof(T) == 2 ? 4 : 2) void head_back_kernel(const HeadArgs a, const HeadGrads g, const HeadPlan plan, float *parts)
{
    extern __shared__ __align__(16) char smem[];
    f32x2_t *table = reinterpret_cast<f32x2_t *>(smem);
    using U = Unit<T, ADJ, VEC>;
    const int lanes = plan.lanes, pairs = 8 * plan.units;
    const int u = (int)threadIdx.x % lanes, group = (int)threadIdx.x / lanes, groups = 256 / lanes;
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const bool mine = u < plan.units;
    const float inv = 1.f / (float)a.d;
    float *red = reinterpret_cast<float *>(smem + plan.together * 64 * plan.units);          // [wavefront][unit][16]
    float *weights = red + 4 * 16 * plan.units;                  // [unit][16]: in registers they would cost a workgroup of four on a CU
    bool formed = false;                                         // whether the angles of all of this workgroup's rows are in LDS
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const int heads = a.heads[side];
        const T *in = (const T *)a.in[side], *up = (const T *)g.up[side];
        T *out = (T *)g.d_in[side];
        if (heads == 0 || (!out && !g.dw[side])) continue;
        const size_t ld_in = a.ld_in[side], ld_up = a.ld_out[side];
        float dw[16] = {};
        if (side > 0) __syncthreads();                           // everybody is done with the queries' weights and sums
        if ((int)threadIdx.x < plan.units) {
            float w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = 1.f;
            if (a.w[side]) U::load((const T *)a.w[side], (int)threadIdx.x, a.d, a.rot, w);
#pragma unroll
            for (int e = 0; e < 16; ++e) weights[16 * threadIdx.x + e] = w[e];
        }
        __syncthreads();
        for (int64_t row = (int64_t)blockIdx.x * plan.together; row < a.rows; row += (int64_t)gridDim.x * plan.together) {
            const int rows = a.rows - row < plan.together ? (int)(a.rows - row) : plan.together;
            // a group of lanes has one head at a time
            typename U::Raw x_raw, t_raw;
            auto fetch = [&](int from) __attribute__((always_inline)) {
                const int i = from + group, r = i / heads, h = i - r * heads;
                U::clear(x_raw), U::clear(t_raw);
                if (!mine || i >= rows * heads) return;
                if (a.norm) U::load(in + (row + r) * ld_in + (size_t)h * a.d, u, a.d, a.rot, x_raw);
                if (up) U::load(up + (row + r) * ld_up + (size_t)h * a.d, u, a.d, a.rot, t_raw);
            };
            if (!formed) {
                __syncthreads();
                angles(a, pairs, (int)row, rows, table);
                __syncthreads();
                formed = (int)gridDim.x * plan.together >= a.rows;
            }
            fetch(0);
            for (int from = 0; from < rows * heads; from += groups) {
                const int i = from + group, r = i / heads, h = i - r * heads;
                const bool live = mine && i < rows * heads;
                float x[16], t[16];
                U::numbers(x_raw, x);
                U::numbers(t_raw, t);
                if (live) U::turn(table + r * pairs + 8 * u, a.rot / 2 - 8 * u, t, -1.f);
                if (a.norm) {
                    float squares = 0.f, dot = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) squares = fmaf(x[e], x[e], squares);
                    const float by = rsqrtf(fmaf(group_sum(squares, lanes), inv, a.eps));
                    const float *w = weights + 16 * (mine ? u : 0);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        x[e] *= by;
                        dw[e] = fmaf(t[e], x[e], dw[e]);
                        t[e] *= w[e];
                        dot = fmaf(t[e], x[e], dot);
                    }
                    dot = group_sum(dot, lanes) * inv;
#pragma unroll
                    for (int e = 0; e < 16; ++e) t[e] = by * fmaf(-x[e], dot, t[e]);
                }
                if (live && out) U::store(out + (row + r) * ld_in + (size_t)h * a.d, u, a.d, a.rot, t);
                if (from + groups < rows * heads) fetch(from + groups);
            }
        }
        if (!g.dw[side]) continue;
        // over the groups of a wavefront, then over the wavefronts, in an order of their own each
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float v = dw[e];
            for (int n = lanes; n < 64; n *= 2) v += __shfl_xor(v, n);
            if (lane < lanes && mine) red[(wave * plan.units + u) * 16 + e] = v;
        }
        __syncthreads();
        for (int i = (int)threadIdx.x; i < 16 * plan.units; i += 256) {
            float v = 0.f;
            for (int k = 0; k < 4; ++k) v += red[k * plan.units * 16 + i];
            const int unit = i / 16, e = i % 16;
            int at;
            if (VEC) at = (e < 8 ? U::first_chunk(unit, a.rot) : U::second_chunk(unit, a.rot)) + e % 8;
            else {
                const Pair p = pair_of<ADJ>(8 * unit + (ADJ ? e / 2 : e % 8), a.rot);
                at = (ADJ ? e % 2 : e / 8) ? p.b : p.a;
            }
            if (at < a.d) parts[((size_t)blockIdx.x * 2 + side) * a.d + at] = v;
        }
    }
}

// dw (+)= sum over `n` workgroups' parts; four columns, 64 threads a column that take every 64th part
__global__ __launch_bounds__(256) void head_sum_kernel(const float *parts, int n, int d, float *dw_q, float *dw_k, int accumulate)
{
    __shared__ float red[4][4];
    const int x = (int)threadIdx.x & 3, y = (int)threadIdx.x >> 2, c = (int)blockIdx.x * 4 + x, side = (int)blockIdx.y;
    float *dw = side ? dw_k : dw_q;
    if (!dw) return;
    float v = 0.f;
    if (c < d) {
#pragma unroll 4
        for (int b = y; b < n; b += 64) v += parts[((size_t)b * 2 + side) * d + c];
    }
    for (int m = 4; m < 64; m *= 2) v += __shfl_xor(v, m);
    if ((y & 15) == 0) red[y >> 4][x] = v;
    __syncthreads();
    if (y == 0 && c < d) {
        v = (red[0][x] + red[1][x]) + (red[2][x] + red[3][x]);
        dw[c] = accumulate ? dw[c] + v : v;
    }
}

size_t head_workspace_bytes(const HeadArgs &a)
{
    return ((size_t)head_plan(a, true).grid * 2 * a.d * 4 + 255) / 256 * 256;
}

template <typename T, bool ADJ, bool VEC>
hipError_t forward(const HeadArgs &a, const HeadPlan &p, void *const out[2], hipStream_t s)
{
    hipLaunchKernelGGL((head_kernel<T, ADJ, VEC>), dim3(p.grid), dim3(256), p.together * 64 * p.units, s, a, p, (T *)out[0], (T *)out[1]);
    return hipGetLastError();
}
template <typename T, bool ADJ, bool VEC>
hipError_t backward(const HeadArgs &a, const HeadGrads &g, const HeadPlan &p, float *parts, hipStream_t s)
{
    hipLaunchKernelGGL((head_back_kernel<T, ADJ, VEC>), dim3(p.grid), dim3(256), (p.together + 5) * 64 * p.units, s, a, g, p, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!g.dw[0] && !g.dw[1])) return e;
    hipLaunchKernelGGL(head_sum_kernel, dim3((a.d + 3) / 4, 2), dim3(256), 0, s, parts, p.grid, a.d, g.dw[0], g.dw[1], g.accumulate);
    return hipGetLastError();
}

// f(a value of the storage type, whether pairs are adjacent, whether heads are whole chunks)
template <typename F>
hipError_t by_kind(int dtype, bool adjacent, bool vec, F f)
{
    auto rest = [&](auto t) {
        if (adjacent) return vec ? f(t, std::true_type(), std::true_type()) : f(t, std::true_type(), std::false_type());
        return vec ? f(t, std::false_type(), std::true_type()) : f(t, std::false_type(), std::false_type());
    };
    return dtype ? rest(bf16_t()) : rest(float());
}

hipError_t launch_head_forward(int dtype, const HeadArgs &a, void *const out[2], hipStream_t s)
{
    const HeadPlan p = head_plan(a, false);
    return by_kind(dtype, a.adjacent, p.vec, [&](auto t, auto adj, auto vec) { return forward<decltype(t), adj.value, vec.value>(a, p, out, s); });
}

hipError_t launch_head_backward(int dtype, const HeadArgs &a, const HeadGrads &g, void *ws, hipStream_t s)
{
    const HeadPlan p = head_plan(a, true);
    return by_kind(dtype, a.adjacent, p.vec, [&](auto t, auto adj, auto vec) { return backward<decltype(t), adj.value, vec.value>(a, g, p, (float *)ws, s); });
}

}  // namespace seq
}  // namespace stl
