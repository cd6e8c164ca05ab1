// The step between two blocks of a residual network, in one pass over the rows:
//     u = POST ? norm(H) w_post + b_post : H,    Xout = skip X + scale g (.) u,    Z = PRE ? norm(Xout) w_pre + b_pre : -,
// norm(v) = (v - mean v) / sqrt(mean (v - mean v)^2 + eps), without the means unless CENTER, and its gradients.
//
// What bounds it: memory.  The forward pass reads X and H and writes Xout and Z, the backward pass reads Xout, H, dXout and dZ and writes dX
// and dH; a row is loaded once, stays in registers as fp32 (8 NV elements a thread) through all its statistics, and every output is rounded
// once.  The statistics of the saved rows are formed again in the backward pass (they cost sums, not bytes), so nothing is saved for it.
// A row has TPR threads (a wavefront up to 512 elements, 512 threads up to 4096); a workgroup walks over rows and has the next ones' loads in
// flight while it sums.  Vectors over the columns (weights, offsets, a gate that all rows share) stay in registers over the walk.
#pragma once
#include "lm_kernels.h"
#include "lm_device.h"

#include <type_traits>

namespace stl {
namespace lm {

// K sums (at most kSums) over the TPR threads of a row, in every thread of the row.  red: 2 x (workgroup's wavefronts) x kSums floats, used in turn,
// so that one barrier a call is enough: who writes a half again has passed the barrier behind which all have read it.
constexpr int kSums = 5;
template <int TPR, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float *red, int &half, int waves)
{
    if constexpr (TPR == 64) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
    } else {
        constexpr int WPR = TPR / 64;
        const int wave = (int)threadIdx.x >> 6;
        float *mine = red + half * waves * kSums;
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = wave_sum_last(v[k]);
        if ((threadIdx.x & 63) == 63) {
#pragma unroll
            for (int k = 0; k < K; ++k) mine[wave * kSums + k] = v[k];
        }
        __syncthreads();
        const float *row = mine + wave / WPR * WPR * kSums;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float t = row[k];
#pragma unroll
            for (int w = 1; w < WPR; ++w) t += row[w * kSums + k];
            v[k] = t;
        }
        half ^= 1;
    }
}

// fp32 storage takes a mean twice, the second time of the centred row (its sum comes with the squares'): the rounding of the first would otherwise be
// the whole of an element that is close to the mean.
template <typename T, int TPR, int NV, bool CENTER>
__global__ __launch_bounds__(TPR < 512 ? 512 : TPR) void residual_forward_kernel(const ResidualArgs a, void *Xout_, void *Z_)
{
    constexpr int THREADS = TPR < 512 ? 512 : TPR, RL = THREADS / TPR, WAVES = THREADS / 64;
    constexpr bool TWICE = CENTER && sizeof(T) == 4;
    __shared__ float red[2 * WAVES * kSums];
    int half = 0;
    const int t = (int)threadIdx.x % TPR, n = a.n;
    const float inv_n = 1.f / (float)n;
    const T *X = (const T *)a.X, *H = (const T *)a.H, *gate = (const T *)a.gate;
    T *Xout = (T *)Xout_, *Z = (T *)Z_;
    int col[NV], left[NV];
    Chunk<T> wo[NV], bo[NV], wp[NV], bp[NV], g[NV];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        col[c] = (c * TPR + t) * 8;
        left[c] = n - col[c];
        wo[c].fill(1.f), bo[c].fill(0.f), wp[c].fill(1.f), bp[c].fill(0.f), g[c].fill(1.f);
        if (left[c] > 0) {
            if (a.w_post) wo[c].load((const T *)a.w_post + col[c], left[c]);
            if (a.b_post) bo[c].load((const T *)a.b_post + col[c], left[c]);
            if (a.w_pre) wp[c].load((const T *)a.w_pre + col[c], left[c]);
            if (a.b_pre) bp[c].load((const T *)a.b_pre + col[c], left[c]);
        }
    }
    const int step = (int)gridDim.x * RL;
    int row = (int)blockIdx.x * RL + (int)threadIdx.x / TPR, grow = -1;
    Chunk<T> xr[NV], hr[NV];
    auto fetch = [&](int r) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            xr[c].fill(0.f), hr[c].fill(0.f);
            if (r < a.rows && left[c] > 0) {
                xr[c].load(X + (size_t)r * n + col[c], left[c]);
                hr[c].load(H + (size_t)r * n + col[c], left[c]);
            }
        }
    };
    fetch(row);
    // all rows of a workgroup take the same number of turns: they share its barriers
    for (int first = (int)blockIdx.x * RL; first < a.rows; first += step, row += step) {
        if (gate && row < a.rows && row / a.per_gate != grow) {
            grow = row / a.per_gate;
#pragma unroll
            for (int c = 0; c < NV; ++c)
                if (left[c] > 0) g[c].load(gate + (size_t)grow * n + col[c], left[c]);
        }
        float x[NV][8], h[NV][8];
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] = xr[c].get(e), h[c][e] = hr[c].get(e);
        fetch(row + step);
        // 1 / deviation of the row in v, which is centred in place
        auto normalise = [&](float (&v)[NV][8]) {
            if constexpr (CENTER) {
                float s[1] = {0.f};
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[0] += v[c][e];
                row_sums<TPR>(s, red, half, WAVES);
                const float mean = s[0] * inv_n;
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[c][e] = e < left[c] ? v[c][e] - mean : 0.f;
            }
            float s[TWICE ? 2 : 1] = {};
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[0] = fmaf(v[c][e], v[c][e], s[0]);
                    if constexpr (TWICE) s[1] += v[c][e];
                }
            row_sums<TPR>(s, red, half, WAVES);
            if constexpr (TWICE) {
                const float rest = s[1] * inv_n;
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[c][e] = e < left[c] ? v[c][e] - rest : 0.f;
                s[0] = fmaf(-rest, s[1], s[0]);
            }
            return rsqrtf(s[0] * inv_n + a.eps);
        };
        const float rh = a.post ? normalise(h) : 1.f;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = fmaf(h[c][e] * rh, wo[c].get(e), bo[c].get(e));
                x[c][e] = e < left[c] ? fmaf(a.scale * g[c].get(e), u, a.skip * x[c][e]) : 0.f;
            }
#pragma unroll
        for (int c = 0; c < NV; ++c)
            if (row < a.rows && left[c] > 0) Chunk<T>::store(Xout + (size_t)row * n + col[c], left[c], x[c]);
        if (a.pre) {
            const float rx = normalise(x);
#pragma unroll
            for (int c = 0; c < NV; ++c) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c][e] = fmaf(x[c][e] * rx, wp[c].get(e), bp[c].get(e));
                if (row < a.rows && left[c] > 0) Chunk<T>::store(Z + (size_t)row * n + col[c], left[c], x[c]);
            }
        }
    }
}

// Gradients.  The rows are dealt in items: item i holds `chunk` rows (or what is left) of group i / pieces, all of which share a row of the gate;
// the weights' and offsets' sums run over all items of a workgroup.  Partials are added in a fixed order by residual_sums_kernel: results are the same
// from run to run.
//   d = dXout + r (t - [mean t] - x^ mean(t x^)),  t = dZ w_pre,  x^ = norm(Xout);   du = scale g d;   dH likewise from th = du w_post.
// What bounds it beside memory is the vector unit (some 30 operations an element and row on two wavefronts a SIMD), so what a column's gate and
// weights multiply is multiplied once an item: with A = sum h^ d and B = sum d over an item's rows,
//   dgate = scale (w_post A + b_post B),   dw_post = scale sum over items g A,   db_post = scale sum over items g B.
// Where every row has its own gate (gate_rows), A and B are summed with it and the row's gate gradient is written as it is found.
struct ResidualItems {
    int groups, pieces, chunk, per;          // per: rows of a group
    bool gate_rows;
    float *gate_part, *vec_part;             // groups x pieces x n;  workgroups x 4 x n (dw_pre, db_pre, dw_post, db_post)
};
// (workgroups of 256 threads, two a CU: 94 us for 8192 x 4096 bf16 instead of 88)
constexpr int kBackThreads = 512;

template <typename T, int TPR, int NV, bool CENTER, bool OFFSETS>
__global__ __launch_bounds__(TPR < kBackThreads ? kBackThreads : TPR) void residual_backward_kernel(const ResidualArgs a, const ResidualGrads o, const ResidualItems it)
{
    constexpr int THREADS = TPR < kBackThreads ? kBackThreads : TPR, RL = THREADS / TPR, WAVES = THREADS / 64;
    constexpr bool TWICE = CENTER && sizeof(T) == 4;
    __shared__ float red[2 * WAVES * kSums];
    __shared__ f32x4_t fold[RL > 1 ? THREADS * 2 : 1];
    int half = 0;
    const int t = (int)threadIdx.x % TPR, lane_row = (int)threadIdx.x / TPR, n = a.n;
    const float inv_n = 1.f / (float)n;
    const T *X = (const T *)a.X, *H = (const T *)a.H, *gate = (const T *)a.gate, *dXout = (const T *)o.dXout, *dZ = (const T *)o.dZ;
    T *dX = (T *)o.dX, *dH = (T *)o.dH;
    const bool need_h = a.post || o.dgate;
    int col[NV], left[NV];
    Chunk<T> wo[NV], wp[NV], g[NV];
    float s_wp[NV][8], s_wo[NV][8], s_a[NV][8];              // sums over rows: dZ x^, g A over items, A
    float s_bp[OFFSETS ? NV : 1][8], s_bo[OFFSETS ? NV : 1][8], s_b[OFFSETS ? NV : 1][8];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        col[c] = (c * TPR + t) * 8;
        left[c] = n - col[c];
        wo[c].fill(1.f), wp[c].fill(1.f), g[c].fill(1.f);
        if (left[c] > 0) {
            if (a.w_post) wo[c].load((const T *)a.w_post + col[c], left[c]);
            if (a.w_pre) wp[c].load((const T *)a.w_pre + col[c], left[c]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s_wp[c][e] = s_wo[c][e] = s_a[c][e] = 0.f;
            if constexpr (OFFSETS) s_bp[c][e] = s_bo[c][e] = s_b[c][e] = 0.f;
        }
    }
    // a sum over the rows of the workgroup's row lanes, written as the row `dst` of a partial
    auto flush = [&](float (&s)[NV][8], float *dst) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            if constexpr (RL > 1) {
                __syncthreads();
                fold[threadIdx.x * 2] = f32x4_t{s[c][0], s[c][1], s[c][2], s[c][3]};
                fold[threadIdx.x * 2 + 1] = f32x4_t{s[c][4], s[c][5], s[c][6], s[c][7]};
                __syncthreads();
                const float *f = reinterpret_cast<const float *>(fold);
                for (int i = (int)threadIdx.x; i < TPR * 8; i += THREADS) {
                    float v = f[i];
#pragma unroll
                    for (int l = 1; l < RL; ++l) v += f[l * TPR * 8 + i];
                    if (c * TPR * 8 + i < n) dst[c * TPR * 8 + i] = v;
                }
            } else if (left[c] > 0) {
                Chunk<float>::store(dst + col[c], left[c], s[c]);
            }
        }
    };
    // the rows r0 + lane_row, + RL, ... below r1; GATES: each with its own row of the gate
    auto rows = [&](const int r0, const int r1, auto gates_c) {
        constexpr bool GATES = decltype(gates_c)::value;
        Chunk<T> xr[NV], hr[NV], dr[NV], zr[NV];
        auto fetch = [&](int r) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                xr[c].fill(0.f), hr[c].fill(0.f), dr[c].fill(0.f), zr[c].fill(0.f);
                if (r < r1 && left[c] > 0) {
                    const size_t at = (size_t)r * n + col[c];
                    if (a.pre) {
                        xr[c].load(X + at, left[c]);
                        if (dZ) zr[c].load(dZ + at, left[c]);
                    }
                    if (need_h) hr[c].load(H + at, left[c]);
                    if (dXout) dr[c].load(dXout + at, left[c]);
                }
            }
        };
        int row = r0 + lane_row;
        fetch(row);
        for (int first = r0; first < r1; first += RL, row += RL) {
            float x[NV][8], h[NV][8], tz[NV][8];
            Chunk<T> d_now[NV], z_now[NV];
            if (GATES && row < r1) {
#pragma unroll
                for (int c = 0; c < NV; ++c)
                    if (left[c] > 0) g[c].load(gate + (size_t)row * n + col[c], left[c]);
            }
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                d_now[c] = dr[c], z_now[c] = zr[c];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[c][e] = xr[c].get(e), h[c][e] = hr[c].get(e);
                    tz[c][e] = zr[c].get(e) * wp[c].get(e);
                }
            }
            fetch(row + RL);
            float mean_t = 0.f;
            if constexpr (CENTER) {
                float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[0] += x[c][e], s[1] += h[c][e], s[2] += tz[c][e];
                row_sums<TPR>(s, red, half, WAVES);
                const float mx = s[0] * inv_n, mh = a.post ? s[1] * inv_n : 0.f;
                mean_t = s[2] * inv_n;
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[c][e] = e < left[c] ? x[c][e] - mx : 0.f;
                        h[c][e] = e < left[c] ? h[c][e] - mh : 0.f;
                    }
            }
            float s[TWICE ? 5 : 3] = {};
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[0] = fmaf(x[c][e], x[c][e], s[0]);
                    s[1] = fmaf(h[c][e], h[c][e], s[1]);
                    s[2] = fmaf(tz[c][e], x[c][e], s[2]);
                    if constexpr (TWICE) s[3] += x[c][e], s[4] += h[c][e];
                }
            row_sums<TPR>(s, red, half, WAVES);
            if constexpr (TWICE) {
                const float rest_x = s[3] * inv_n, rest_h = a.post ? s[4] * inv_n : 0.f;
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[c][e] = e < left[c] ? x[c][e] - rest_x : 0.f;
                        h[c][e] = e < left[c] ? h[c][e] - rest_h : 0.f;
                    }
                s[0] = fmaf(-rest_x, s[3], s[0]);
                s[1] = fmaf(-rest_h, s[4], s[1]);
                s[2] = fmaf(-rest_x * (float)n, mean_t, s[2]);
            }
            const float rx = a.pre ? rsqrtf(s[0] * inv_n + a.eps) : 0.f, rh = a.post ? rsqrtf(s[1] * inv_n + a.eps) : 1.f, cx = -rx * rx * s[2] * inv_n;
            float q[2] = {0.f, 0.f}, d[NV][8];
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                z_now[c].opaque();
                d_now[c].opaque();
                float gate_grad[GATES ? 8 : 1];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = z_now[c].get(e), xh = x[c][e] * rx, hh = h[c][e] * rh, ge = g[c].get(e);
                    d[c][e] = fmaf(rx, CENTER ? tz[c][e] - mean_t : tz[c][e], fmaf(xh, cx, d_now[c].get(e)));
                    if (CENTER && e >= left[c]) d[c][e] = 0.f;
                    s_wp[c][e] = fmaf(z, xh, s_wp[c][e]);
                    const float du = ge * d[c][e];
                    s_a[c][e] = fmaf(hh, GATES ? du : d[c][e], s_a[c][e]);
                    if constexpr (OFFSETS) s_bp[c][e] += z, s_b[c][e] += GATES ? du : d[c][e];
                    if constexpr (GATES) gate_grad[e] = hh * wo[c].get(e) * d[c][e];
                    tz[c][e] = du * wo[c].get(e);
                    if constexpr (CENTER) q[0] += tz[c][e];
                    q[1] = fmaf(tz[c][e], h[c][e], q[1]);
                }
                if constexpr (GATES) {
                    if (o.dgate && row < r1 && left[c] > 0) {
                        const size_t at = (size_t)row * n + col[c];
                        Chunk<T> bo;
                        Chunk<float> old;
                        bo.fill(0.f), old.fill(0.f);
                        if (a.b_post) bo.load((const T *)a.b_post + col[c], left[c]);
                        if (o.accumulate) old.load(o.dgate + at, left[c]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) gate_grad[e] = fmaf(a.scale, fmaf(bo.get(e), d[c][e], gate_grad[e]), old.get(e));
                        Chunk<float>::store(o.dgate + at, left[c], gate_grad);
                    }
                }
            }
            float out = a.scale, mean_th = 0.f, ch = 0.f;
            if (a.post) {
                row_sums<TPR>(q, red, half, WAVES);
                mean_th = CENTER ? q[0] * inv_n : 0.f, ch = -rh * rh * q[1] * inv_n;
                out *= rh;
            }
            if (row < r1) {
#pragma unroll
                for (int c = 0; c < NV; ++c) {
                    if (left[c] <= 0) continue;
                    const size_t at = (size_t)row * n + col[c];
                    if (dH) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) tz[c][e] = out * fmaf(h[c][e], ch, CENTER ? tz[c][e] - mean_th : tz[c][e]);
                        Chunk<T>::store(dH + at, left[c], tz[c]);
                    }
                    if (dX) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) d[c][e] *= a.skip;
                        Chunk<T>::store(dX + at, left[c], d[c]);
                    }
                }
            }
        }
    };
    const int items = it.groups * it.pieces;
    for (int i = (int)blockIdx.x; i < items; i += (int)gridDim.x) {
        const int group = i / it.pieces, r0 = group * it.per + (i - group * it.pieces) * it.chunk;
        int r1 = r0 + it.chunk;
        if (r1 > (group + 1) * it.per) r1 = (group + 1) * it.per;
        if (r1 > a.rows) r1 = a.rows;
        if (it.gate_rows) {
            rows(r0, r1, std::true_type{});
        } else {
            if (gate) {
#pragma unroll
                for (int c = 0; c < NV; ++c)
                    if (left[c] > 0) g[c].load(gate + (size_t)group * n + col[c], left[c]);
            }
            rows(r0, r1, std::false_type{});
        }
        // the item's sums: into the workgroup's, and the gate's partial
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            Chunk<T> bo;
            bo.fill(0.f);
            if (OFFSETS && a.b_post && left[c] > 0) bo.load((const T *)a.b_post + col[c], left[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float mul = it.gate_rows ? 1.f : g[c].get(e);
                s_wo[c][e] = fmaf(mul, s_a[c][e], s_wo[c][e]);
                s_a[c][e] = a.scale * s_a[c][e] * wo[c].get(e);
                if constexpr (OFFSETS) {
                    s_bo[c][e] = fmaf(mul, s_b[c][e], s_bo[c][e]);
                    s_a[c][e] = fmaf(a.scale * s_b[c][e], bo.get(e), s_a[c][e]);
                    s_b[c][e] = 0.f;
                }
            }
        }
        if (o.dgate && !it.gate_rows) flush(s_a, it.gate_part + (size_t)i * n);
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) s_a[c][e] = 0.f;
    }
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s_wo[c][e] *= a.scale;
            if constexpr (OFFSETS) s_bo[c][e] *= a.scale;
        }
    float *mine = it.vec_part + (size_t)blockIdx.x * 4 * n;
    if (o.dw_pre) flush(s_wp, mine);
    if (o.dw_post) flush(s_wo, mine + 2 * (size_t)n);
    if constexpr (OFFSETS) {
        if (o.db_pre) flush(s_bp, mine + (size_t)n);
        if (o.db_post) flush(s_bo, mine + 3 * (size_t)n);
    }
}

// threads of a row and chunks of eight elements a thread: a wavefront for up to 512 elements, then as many threads as there are chunks
template <class F>
hipError_t residual_shape(int n, F &&f)
{
    if (n <= 512) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (n <= 1024) return f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
    if (n <= 2048) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (n <= 4096) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
    if (n <= 8192) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
    if (n <= 16384) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
}

template <typename T>
hipError_t residual_forward(const ResidualArgs &a, void *Xout, void *Z, hipStream_t s)
{
    return residual_shape(a.n, [&](auto tpr_c, auto nv_c) {
        constexpr int TPR = decltype(tpr_c)::value, NV = decltype(nv_c)::value, THREADS = TPR < 512 ? 512 : TPR, RL = THREADS / TPR;
        const int wanted = (a.rows + RL - 1) / RL, grid = wanted < 1024 ? wanted : 1024;
        if (a.center) {
            auto kern = residual_forward_kernel<T, TPR, NV, true>;
            hipLaunchKernelGGL(kern, dim3(grid), dim3(THREADS), 0, s, a, Xout, Z);
        } else {
            auto kern = residual_forward_kernel<T, TPR, NV, false>;
            hipLaunchKernelGGL(kern, dim3(grid), dim3(THREADS), 0, s, a, Xout, Z);
        }
        return hipGetLastError();
    });
}

template <typename T>
hipError_t residual_backward(const ResidualArgs &a, const ResidualGrads &g, const ResidualItems &it, int grid, hipStream_t s)
{
    return residual_shape(a.n, [&](auto tpr_c, auto nv_c) {
        constexpr int TPR = decltype(tpr_c)::value, NV = decltype(nv_c)::value, THREADS = TPR < kBackThreads ? kBackThreads : TPR;
        auto run = [&](auto kern) {
            hipLaunchKernelGGL(kern, dim3(grid), dim3(THREADS), 0, s, a, g, it);
            return hipGetLastError();
        };
        const bool offsets = g.db_pre || g.db_post || a.b_post;
        if (a.center) return offsets ? run(residual_backward_kernel<T, TPR, NV, true, true>) : run(residual_backward_kernel<T, TPR, NV, true, false>);
        return offsets ? run(residual_backward_kernel<T, TPR, NV, false, true>) : run(residual_backward_kernel<T, TPR, NV, false, false>);
    });
}

hipError_t residual_forward_f32(const ResidualArgs &a, void *Xout, void *Z, hipStream_t s);
hipError_t residual_backward_f32(const ResidualArgs &a, const ResidualGrads &g, const ResidualItems &it, int grid, hipStream_t s);

}  // namespace lm
}  // namespace stl
