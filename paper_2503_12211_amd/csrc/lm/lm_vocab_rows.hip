// Vocabulary loss, everything but the matrix products: the list of rows that have a term, their rows of X side by side, the losses and the
// gradient in the logits row by row, and the last stage of the gradients' sums.
#include "lm_kernels.h"
#include "lm_device.h"

namespace stl {
namespace lm {

// ---- which rows have a term --------------------------------------------------------------------------------------------------------
struct Terms {
    const int64_t *label, *top_id;
    const float *top_logit;
    int vocab, ntop;
    __device__ __forceinline__ bool labelled(int row) const { return label && (uint64_t)label[row] < (uint64_t)vocab; }
    // entry j of the row's teacher counts: its id is in the vocabulary and its logit above minus infinity (not a number counts: it shows)
    __device__ __forceinline__ bool entry(int row, int j) const
    {
        const size_t at = (size_t)row * ntop + j;
        return (uint64_t)top_id[at] < (uint64_t)vocab && !(top_logit[at] == -INFINITY);
    }
    __device__ __forceinline__ bool taught(int row) const
    {
        if (!top_id) return false;
        for (int j = 0; j < ntop; ++j)
            if (entry(row, j)) return true;
        return false;
    }
    __device__ __forceinline__ bool any(int row) const { return labelled(row) || taught(row); }
};
static Terms terms_of(const VocabArgs &a) { return Terms{a.label, a.top_id, a.top_logit, a.vocab, a.ntop}; }

// dz_scale.  The gradient in the logits is rounded to bf16 on its way into the products.  What it is made of is at most the row's weight, w = |dlabel| +
// |dtop| / tau, and its largest entries (a label's, -(1 - p) dlabel) are close below; so all rows are multiplied by the factor that takes the
// largest w to 1.97 times a power of two, where bf16's steps are finest relative to what they hold, and the products' sums by its reciprocal: the
// rounding of a label's entry falls from up to 2.3e-3 (root mean square, just above a power of two) to 1.15e-3.  A power of two of no
// matter: the factor lies in (0.98, 1.97].
__device__ __forceinline__ float dz_scale(float w)
{
    const uint32_t bits = __float_as_uint(w);
    const uint32_t e = bits >> 23;
    if (e == 0 || e >= 254) return 1.f;                      // zero, smaller than is normal, or not finite
    return 1.96875f / __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
}

struct Weights {
    const float *dlabel, *dtop;
    float inv_tau;
    __device__ __forceinline__ float of(int r, bool labelled, bool taught) const
    {
        return (labelled && dlabel ? fabsf(dlabel[r]) : 0.f) + (taught && dtop ? fabsf(dtop[r]) * inv_tau : 0.f);
    }
};
static Weights weights_of(const VocabArgs &a, const VocabGrads *g) { return Weights{g ? g->dlabel : nullptr, g ? g->dtop : nullptr, 1.f / a.tau}; }

// Over the THREADS of a workgroup: `n` of this one and the threads before it, and of all; the largest `top`.
template <int THREADS>
__device__ __forceinline__ int scan_rows(int n, int &all, float &top)
{
    __shared__ int sums[THREADS / 64];
    __shared__ float tops[THREADS / 64];
    const int lane = (int)threadIdx.x & 63;
    int upto = n;
    for (int step = 1; step < 64; step *= 2) {
        const int v = __shfl_up(upto, step);
        if (lane >= step) upto += v;
    }
    top = wave_max(top);
    if (lane == 63) {
        sums[threadIdx.x >> 6] = upto;
        tops[threadIdx.x >> 6] = top;
    }
    __syncthreads();
    all = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < (int)threadIdx.x >> 6) upto += sums[w];
        all += sums[w];
        top = fmaxf(top, tops[w]);
    }
    return upto;
}

// One workgroup: every thread counts a run of neighbouring rows, the counts are added up over the workgroup, and every thread lists its rows.
__global__ __launch_bounds__(1024) void select_rows_kernel(Terms t, int rows, Weights w, int *list, int *count, float *scale)
{
    const int per = (rows + 1023) / 1024, r0 = (int)threadIdx.x * per, r1 = r0 + per < rows ? r0 + per : rows;
    int n = 0, all;
    float top = 0.f;
    uint32_t has = 0;                                        // of the first 32 rows
    for (int r = r0; r < r1; ++r) {
        const bool l = t.labelled(r), q = t.taught(r);
        n += l || q;
        if (r - r0 < 32) has |= (uint32_t)(l || q) << (r - r0);
        top = fmaxf(top, w.of(r, l, q));
    }
    int at = scan_rows<1024>(n, all, top) - n;
    for (int r = r0; r < r1; ++r)
        if (r - r0 < 32 ? has >> (r - r0) & 1 : t.any(r)) list[at++] = r;
    if (threadIdx.x == 0) {
        *count = all;
        scale[0] = dz_scale(top);
        scale[1] = 1.f / scale[0];
    }
}

hipError_t launch_select_rows(const VocabArgs &a, const VocabGrads *g, RowList rl, hipStream_t s)
{
    hipLaunchKernelGGL(select_rows_kernel, dim3(1), dim3(1024), 0, s, terms_of(a), a.rows, weights_of(a, g), rl.list, rl.count, rl.scale);
    return hipGetLastError();
}

// ---- rows side by side ---------------------------------------------------------------------------------------------------------------
// threads of a workgroup of 256 that share a row of d elements, eight each at a time
__host__ __device__ inline int threads_of(int d)
{
    int n = 8;
    while (n < 256 && n * 8 < d) n *= 2;
    return n;
}

// row `from` of `in` (none: zeros) to row `to` of `out`, zeros behind its end, by thread t of n
template <typename T>
__device__ __forceinline__ void copy_row(const T *in, long from, int d, T *out, size_t to, int ld, int t, int n)
{
    for (int c = t * 8; c < ld; c += n * 8) {
        Chunk<T> v;
        v.fill(0.f);
        if (from >= 0 && c < d) v.load(in + (size_t)from * d + c, d - c);
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v.get(e);
        Chunk<T>::store(out + to * ld + c, ld - c, f);
    }
}

// a workgroup a row: the listed row first + b to row b of `out` (b < cap) and to its second row's place (held: second_row), and zeros where row b (b <
// zeros) is not listed.  FEW: there is no list yet, and first is 0; every workgroup goes over all rows.
template <typename T, bool FEW>
__global__ __launch_bounds__(256) void arrange_rows_kernel(Terms t, int rows, Weights w, const T *X, int *list, int *count, float *scale, int first, int cap, int d,
                                                           int ld, T *out, int held, int zeros, T *dX, float *label_loss, float *top_loss)
{
    const int b = (int)blockIdx.x;
    long from = -1;
    if constexpr (FEW) {
        __shared__ int mine;
        const int per = (rows + 255) / 256, r0 = (int)threadIdx.x * per;     // at most four rows a thread
        int n = 0, all;
        float top = 0.f;
        uint32_t has = 0;
        for (int r = r0; r < r0 + per && r < rows; ++r) {
            const bool l = t.labelled(r), q = t.taught(r);
            n += l || q;
            has |= (uint32_t)(l || q) << (r - r0);
            top = fmaxf(top, w.of(r, l, q));
        }
        int at = scan_rows<256>(n, all, top) - n;
        const int second = second_row(all, held), want = second && b >= second ? b - second : b;
        if (threadIdx.x == 0) mine = -1;
        __syncthreads();
        for (; has; has &= has - 1, ++at) {
            const int r = r0 + __builtin_ctz(has);
            if (at == want) mine = r;
            if (b == 0) list[at] = r;
        }
        if (b == 0 && threadIdx.x == 0) {
            *count = all;
            scale[0] = dz_scale(top);
            scale[1] = 1.f / scale[0];
        }
        __syncthreads();
        from = mine;
    } else {
        const int second = second_row(*count, held), want = second && b >= second ? b - second : b;
        if (b < cap && first + want < *count) from = list[first + want];
    }
    if (b < cap) copy_row(X, from, d, out, b, ld, (int)threadIdx.x, 256);
    if (b < zeros && !t.any(b)) {
        if (threadIdx.x == 0) {
            if (label_loss) label_loss[b] = 0.f;
            if (top_loss) top_loss[b] = 0.f;
        }
        if (dX) copy_row(X, -1L, d, dX, b, d, (int)threadIdx.x, 256);
    }
}

hipError_t launch_arrange_rows(const VocabArgs &a, const VocabGrads *g, RowList rl, int first, int cap, int ld, void *out, int held, void *dX, float *label_loss, float *top_loss,
                               hipStream_t s)
{
    const int zeros = first == 0 ? a.rows : 0;
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        hipLaunchKernelGGL(kern, dim3(cap > zeros ? cap : zeros), dim3(256), 0, s, terms_of(a), a.rows, weights_of(a, g), (const T *)a.X, rl.list, rl.count, rl.scale,
                           first, cap, a.d, ld, (T *)out, held, zeros, (T *)dX, label_loss, top_loss);
        return hipGetLastError();
    };
    const bool few = few_rows(a) && first == 0;              // later chunks have the list
    if (a.bf16) return few ? run(arrange_rows_kernel<bf16_t, true>, (bf16_t *)nullptr) : run(arrange_rows_kernel<bf16_t, false>, (bf16_t *)nullptr);
    return few ? run(arrange_rows_kernel<float, true>, (float *)nullptr) : run(arrange_rows_kernel<float, false>, (float *)nullptr);
}

// (a workgroup a row: 71 us for 97624 x 205, several: 34)
__global__ __launch_bounds__(256) void pad_rows_kernel(const bf16_t *in, int rows, int d, bf16_t *out, int ld)
{
    const int n = threads_of(ld), r = (int)blockIdx.x * (256 / n) + (int)threadIdx.x / n;
    if (r < rows) copy_row(in, r, d, out, r, ld, (int)threadIdx.x % n, n);
}

hipError_t launch_pad_rows(const void *in, int rows, int d, int ld, void *out, hipStream_t s)
{
    const int per = 256 / threads_of(ld);
    hipLaunchKernelGGL(pad_rows_kernel, dim3((rows + per - 1) / per), dim3(256), 0, s, (const bf16_t *)in, rows, d, (bf16_t *)out, ld);
    return hipGetLastError();
}

// ---- losses and the gradient in the logits -----------------------------------------------------------------------------------------
constexpr int kRowThreads = 512, kRowWaves = kRowThreads / 64;

__device__ __forceinline__ float block_max(float v, float *red)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < kRowWaves; ++w) v = fmaxf(v, red[w]);
    return v;
}
__device__ __forceinline__ float block_sum(float v, float *red)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < kRowWaves; ++w) v += red[w];
    return v;
}

// f of every logit of a row of fp32 storage (STORE: which takes its place), by a workgroup: eight a thread at a time where each thread has some (40 rows of
// 53504, three sweeps: 43 us, 86 by ones), one where there are fewer (2048 rows of 1000: 16.0 us, 19 by eights)
template <bool STORE, class F>
__device__ __forceinline__ void each_logit(float *Z, int vocab, F &&f)
{
    const int tid = (int)threadIdx.x;
    if (vocab < kRowThreads * 8) {
        for (int v = tid; v < vocab; v += kRowThreads) {
            const float z = f(Z[v]);
            if (STORE) Z[v] = z;
        }
        return;
    }
    for (int v = tid * 8; v < vocab; v += kRowThreads * 8) {
        Chunk<float> in;
        in.load(Z + v, vocab - v);
        float out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < vocab - v) out[e] = f(in.get(e));
        if (STORE) Chunk<float>::store(Z + v, vocab - v, out);
    }
}

// what rounding x to y left (none where y is no number)
__device__ __forceinline__ float rest_of(float x, float y) { return fabsf(y) < INFINITY ? x - y : 0.f; }

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// One listed row a workgroup.  With p = softmax(z), p_tau = softmax(z / tau), q the teacher's shares and their entries id_j:
//     label_loss = lse - z_label,   top_loss = sum_j q_j (log q_j - z_id_j / tau + lse_tau),
//     dz_v = dlabel (p_v - [v = label]) + dtop / tau (p_tau,v - sum_{j: id_j = v} q_j).
// The row is written in one sweep without the label's and the entries' own terms, which then overwrite their places: their logits are taken in
// fp32 (p - 1 of a label that is nearly certain loses everything in 16 bits).  bf16 storage: the sweep reads a logit as 16-bit steps below its group's
// maximum (kSteps) and writes the bf16 gradient over it; the row's dot products with the label's and the entries' rows of W give their logits.
// Few rows (second_row) have few entries that count, whose roundings do not average out: what rounding leaves is a second row of the products
// (the gradients' errors of 3 rows of 1216, vocabulary 103168: 2.6e-3 -> 1.7e-3, their own rounding; 16 x 4096, 65536: 362 -> 392 us).
// What bounds it: reading and writing the row, 4 bytes a logit (bf16) or 8.
template <typename T, bool GRADS>
__global__ __launch_bounds__(kRowThreads) void vocab_rows_kernel(Terms t, const VocabGrads g, const T *W, int d, float tau, const int *list, const int *count,
                                                                 const float *scale, VocabChunk c, float *label_loss, float *top_loss)
{
    // (no contraction: the losses have the same bits with and without gradients)
#pragma clang fp contract(off)
    constexpr bool BF16 = sizeof(T) == 2;
    __shared__ float red[kRowWaves];
    __shared__ int ids[kMostTop + 1];        // the entries', and behind them the label's
    __shared__ float y[kMostTop], q[kMostTop], all[kMostTop + 1], z[kMostTop + 1];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, r = (int)blockIdx.x, vocab = t.vocab;
    T *codes = (T *)c.codes + (size_t)r * c.ld;
    const int listed = *count - c.first;
    const size_t second = BF16 ? (size_t)second_row(*count, c.held) * c.ld : 0;           // from a row's place to its second one's
    if (r >= listed) {
        // behind the list: the products read whole stages of 32 rows (fp32 storage: all rows of the chunk)
        const int read = BF16 ? whole_stages(listed) : c.cap;
        if (GRADS && r < read)
            for (size_t v = tid; v < c.ld; v += kRowThreads) {
                codes[v] = 0;
                if (second) codes[v + second] = 0;
            }
        return;
    }
    const int row = list[c.first + r];
    const bool labelled = t.labelled(row);
    const int ntop = t.top_id ? t.ntop : 0;
    const float inv_tau = 1.f / tau;

    // the teacher's shares
    float top = -INFINITY;
    bool any = false;
    for (int j = tid; j < ntop; j += kRowThreads) {
        const bool ok = t.entry(row, j);
        y[j] = ok ? t.top_logit[(size_t)row * ntop + j] : -INFINITY;
        ids[j] = ok ? (int)t.top_id[(size_t)row * ntop + j] : -1;
        top = fmaxf(top, y[j]);
        any |= ok;
    }
    if (tid == 0) ids[ntop] = labelled ? (int)t.label[row] : -1;
    const bool taught = ntop > 0 && block_max(any ? 1.f : 0.f, red) > 0.f;
    float y_sum = 0.f, log_y_sum = 0.f, y_top = 0.f;
    if (taught) {
        y_top = block_max(top, red);
        for (int j = tid; j < ntop; j += kRowThreads)
            if (ids[j] >= 0) y_sum += expf((y[j] - y_top) * inv_tau);
        y_sum = block_sum(y_sum, red);
        log_y_sum = logf(y_sum);
    }
    __syncthreads();

    // log of the sums over the vocabulary; bf16 storage, in powers of two: y of VocabChunk, whose first sum is of the labels' temperature, 1, or, without
    // labels, of the teacher's; the second is there where both are and differ
    float m = -INFINITY, sum = 0.f, sum_tau = 0.f, lse, lse_tau;
    float lse2 = 0.f, lse2_tau = 0.f, ratio = 1.f;
    const GroupSums *groups = nullptr;
    if constexpr (BF16) {
        groups = c.sums + (size_t)r * c.groups;
        ratio = c.two ? inv_tau : 1.f;
        for (int i = tid; i < c.groups; i += kRowThreads) m = fmaxf(m, groups[i].m);
        m = block_max(m, red);
        for (int i = tid; i < c.groups; i += kRowThreads) {
            const GroupSums g = groups[i];
            const float below = g.m - m;
            sum += g.sum * __builtin_amdgcn_exp2f(below);
            if (c.two) sum_tau += g.sum_tau * __builtin_amdgcn_exp2f(below * ratio);
        }
        sum = block_sum(sum, red);
        sum_tau = c.two ? block_sum(sum_tau, red) : sum;
        lse2 = m + log2f(sum), lse2_tau = m * ratio + log2f(sum_tau);
        lse = lse2 * kLn2, lse_tau = lse2_tau * kLn2;
    } else {
        float *Z = (float *)codes;
        each_logit<false>(Z, vocab, [&](float z) { return m = fmaxf(m, z); });
        m = block_max(m, red);
        each_logit<false>(Z, vocab, [&](float z) {
            sum += expf(z - m);
            if (ntop) sum_tau += expf((z - m) * inv_tau);
            return z;
        });
        sum = block_sum(sum, red);
        sum_tau = block_sum(sum_tau, red);
        lse = m + logf(sum), lse_tau = m * inv_tau + logf(sum_tau);
    }

    // the logits of the label and the teacher's entries
    if constexpr (BF16) {
        const bf16_t *x = (const bf16_t *)c.Xc + (size_t)r * c.ldx;
        if (!t.top_id) {
            // a label alone: its product is shared by the workgroup
            float dot = 0.f;
            if (labelled) {
                const bf16_t *w = (const bf16_t *)W + (size_t)ids[0] * d;
                for (int e0 = tid * 8; e0 < d; e0 += kRowThreads * 8) {
                    Chunk<bf16_t> a, b;
                    a.load(x + e0, d - e0);
                    b.load(w + e0, d - e0);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot = fmaf(a.get(e), b.get(e), dot);
                }
            }
            dot = block_sum(dot, red);
            if (tid == 0) z[0] = dot;
        }
        // four entries of a wavefront at a time: the loads of four rows of W in flight (an entry that is none reads the first row)
        constexpr int AT_ONCE = 4;
        for (int j0 = t.top_id ? wave * AT_ONCE : 1; j0 <= ntop; j0 += kRowWaves * AT_ONCE) {
            const bf16_t *w[AT_ONCE];
            float dot[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int id = j0 + k <= ntop ? ids[j0 + k] : -1;
                w[k] = (const bf16_t *)W + (size_t)(id < 0 ? 0 : id) * d;
                dot[k] = 0.f;
            }
            for (int e0 = lane * 8; e0 < d; e0 += 512) {
                Chunk<bf16_t> a, b[AT_ONCE];
                a.load(x + e0, d - e0);
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) b[k].load(w[k] + e0, d - e0);
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot[k] = fmaf(a.get(e), b[k].get(e), dot[k]);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const float sum = wave_sum(dot[k]);
                if (lane == 0 && j0 + k <= ntop) z[j0 + k] = sum;
            }
        }
    } else {
        for (int j = tid; j <= ntop; j += kRowThreads)
            if (ids[j] >= 0) z[j] = ((const float *)codes)[ids[j]];
    }
    __syncthreads();
    if (label_loss && tid == 0) label_loss[row] = labelled ? lse - z[ntop] : 0.f;
    if (taught) {
        for (int j = tid; j < ntop; j += kRowThreads) {
            y[j] = (y[j] - y_top) * inv_tau - log_y_sum;     // log q_j
            q[j] = ids[j] >= 0 ? expf(y[j]) : 0.f;
        }
        __syncthreads();
        // the same entry may be there more than once: `all` is its share, of which q_j is a part
        float part = 0.f;
        for (int j = tid; j <= ntop; j += kRowThreads) {
            float share = 0.f;
            for (int i = 0; i < ntop; ++i) share += ids[i] == ids[j] ? q[i] : 0.f;
            all[j] = share;
            // an entry so far below the first that its share is zero adds nothing
            if (j < ntop && ids[j] >= 0 && share != 0.f) part += q[j] * ((share == q[j] ? y[j] : logf(share)) - (z[j] * inv_tau - lse_tau));
        }
        part = block_sum(part, red);
        if (top_loss && tid == 0) top_loss[row] = part;
    } else if (top_loss && tid == 0) {
        top_loss[row] = 0.f;
    }
    if constexpr (GRADS) {
        const float factor = BF16 ? *scale : 1.f;
        const float cl = labelled && g.dlabel ? g.dlabel[row] * factor : 0.f, ct = taught && g.dtop ? g.dtop[row] * inv_tau * factor : 0.f;
        if constexpr (BF16) {
            auto sweep = [&](auto two_c) {
                constexpr bool TWO = decltype(two_c)::value;
                // chunks of eight logits lie in one group of 64
                for (size_t v = (size_t)tid * 8; v < c.ld; v += kRowThreads * 8) {
                    const u32x4_t in = *reinterpret_cast<const u32x4_t *>(codes + v);
                    const float mg = groups[v / 64].m, step = groups[v / 64].step;
                    const float at = mg - lse2, at_tau = mg * ratio - lse2_tau;
                    // two temperatures: below the maximum by the higher one of two lines (Steps)
                    const float step1 = step > 0.f ? step : c.bend * (1.f / kBendSteps), step2 = fabsf(step), off2 = step > 0.f ? 0.f : fmaf(-kBendSteps, step2, c.bend);
                    float out[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t code = (in[e >> 1] >> (16 * (e & 1))) & 0xffffu;
                        float dz = 0.f;
                        if constexpr (TWO) {
                            const float below = fmaxf((float)code * step1, fmaf((float)code, step2, off2));
                            if (labelled) dz = cl * __builtin_amdgcn_exp2f(at - below);
                            if (taught) dz = fmaf(ct, __builtin_amdgcn_exp2f(fmaf(-below, ratio, at_tau)), dz);
                        } else {
                            if (labelled) dz = cl * __builtin_amdgcn_exp2f(fmaf(-(float)code, step, at));
                            if (taught) dz = fmaf(ct, __builtin_amdgcn_exp2f(fmaf(-(float)code, step, at_tau)), dz);
                        }
                        // a row whose sums are not a number stays one throughout
                        out[e] = code == 65535u && m + sum == m + sum ? 0.f : dz;
                    }
                    const u32x4_t packed = {pack_bf16x2(out[0], out[1]), pack_bf16x2(out[2], out[3]), pack_bf16x2(out[4], out[5]), pack_bf16x2(out[6], out[7])};
                    *reinterpret_cast<u32x4_t *>(codes + v) = packed;
                    if (second) {
                        u32x4_t rest;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            rest[k] = pack_bf16x2(rest_of(out[2 * k], __uint_as_float(packed[k] << 16)), rest_of(out[2 * k + 1], __uint_as_float(packed[k] & 0xffff0000u)));
                        *reinterpret_cast<u32x4_t *>(codes + v + second) = rest;
                    }
                }
            };
            if (c.two) sweep(std::true_type{});
            else sweep(std::false_type{});
        } else {
            each_logit<true>((float *)codes, vocab, [&](float z) {
                float dz = 0.f;
                if (labelled) dz = cl * expf(z - lse);
                if (taught) dz = fmaf(ct, expf(fmaf(z, inv_tau, -lse_tau)), dz);
                return dz;
            });
        }
        __syncthreads();                     // the sweep's stores are done before the entries' places are written again
        for (int j = tid; j <= ntop; j += kRowThreads) {
            const int v = ids[j];
            if (v < 0) continue;
            float dz = 0.f;
            if (labelled) dz = cl * (expf(z[j] - lse) - (ids[ntop] == v ? 1.f : 0.f));
            if (taught) dz = fmaf(ct, expf(fmaf(z[j], inv_tau, -lse_tau)) - all[j], dz);
            Elem<T>::st(codes + v, dz);
            if (second) {
                const float held = __uint_as_float(pack_bf16x2(dz, 0.f) << 16);
                Elem<T>::st(codes + v + second, rest_of(dz, held));
            }
        }
    }
}

hipError_t launch_vocab_rows(const VocabArgs &a, const VocabGrads *g, RowList rl, const VocabChunk &c, float *label_loss, float *top_loss, hipStream_t s)
{
    const VocabGrads none{};
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        // with gradients of bf16 storage also the rows up to a whole stage of the products' contraction
        const int rows = a.bf16 && g ? whole_stages(c.cap) : c.cap;
        hipLaunchKernelGGL(kern, dim3(rows), dim3(kRowThreads), 0, s, terms_of(a), g ? *g : none, (const T *)a.W, a.d, a.tau, (const int *)rl.list,
                           (const int *)rl.count, (const float *)rl.scale, c, label_loss, top_loss);
        return hipGetLastError();
    };
    if (a.bf16) return g ? run(vocab_rows_kernel<bf16_t, true>, (bf16_t *)nullptr) : run(vocab_rows_kernel<bf16_t, false>, (bf16_t *)nullptr);
    return g ? run(vocab_rows_kernel<float, true>, (float *)nullptr) : run(vocab_rows_kernel<float, false>, (float *)nullptr);
}

// ---- the gradients' last stage ---------------------------------------------------------------------------------------------------------
// eight elements of a row's parts p0, p0 + step, ...: their sum
__device__ __forceinline__ void sum_parts(const float *part, int p0, int parts, int step, size_t stride, int left, float (&f)[8])
{
    constexpr int AT_ONCE = 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 0.f;
    int p = p0;
    for (; p + (AT_ONCE - 1) * step < parts; p += AT_ONCE * step) {
        Chunk<float> v[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) v[k].load(part + (size_t)(p + k * step) * stride, left);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += v[k].get(e);
    }
    for (; p < parts; p += step) {
        Chunk<float> v;
        v.load(part + (size_t)p * stride, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] += v.get(e);
    }
}

template <typename T>
__device__ __forceinline__ void store_scaled(T *out, int left, float (&f)[8], float factor)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= factor;
    Chunk<T>::store(out, left, f);
}

// a workgroup a row of the chunk, to where the row came from
template <typename T>
__global__ __launch_bounds__(256) void finish_dx_kernel(const float *part, int known, int ld, const int *list, const int *count, const float *scale, int first,
                                                        int cap, int d, int held, T *dX)
{
    int rows = *count - first;
    if (rows > cap) rows = cap;
    const int r = (int)blockIdx.x;
    if (r >= rows) return;
    const bool bf16 = sizeof(T) == 2;
    const int parts = bf16 ? count[1] : known, n = threads_of(d), groups = 256 / n, group = (int)threadIdx.x / n, t = (int)threadIdx.x % n;
    const int second = bf16 ? second_row(*count, held) : 0;
    const size_t stride = (size_t)(second ? 2 * second : bf16 ? rows : cap) * ld;
    const float *from = part + (size_t)r * ld, factor = bf16 ? scale[1] : 1.f;
    T *to = dX + (size_t)list[first + r] * d;
    // short rows: several groups of threads share the parts, and the first adds them up in order
    __shared__ f32x4_t red[512];
    for (int c0 = 0; c0 < d; c0 += n * 8) {
        const int c = c0 + t * 8;
        float f[8] = {};
        if (c < d) {
            sum_parts(from + c, group, parts, groups, stride, d - c, f);
            if (second) {
                float rest[8];
                sum_parts(from + (size_t)second * ld + c, group, parts, groups, stride, d - c, rest);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] += rest[e];
            }
        }
        if (groups > 1) {                                    // (then c0 takes one turn)
            red[threadIdx.x * 2] = f32x4_t{f[0], f[1], f[2], f[3]};
            red[threadIdx.x * 2 + 1] = f32x4_t{f[4], f[5], f[6], f[7]};
            __syncthreads();
            if (group == 0)
                for (int k = 1; k < groups; ++k) {
                    const f32x4_t a = red[(k * n + t) * 2], b = red[(k * n + t) * 2 + 1];
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] += a[e], f[e + 4] += b[e];
                }
        }
        if (group == 0 && c < d) store_scaled(to + c, d - c, f, factor);
    }
}

hipError_t launch_finish_dx(bool bf16, const float *part, int parts, int ld, RowList rl, int first, int cap, int d, int held, void *dX, hipStream_t s)
{
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        hipLaunchKernelGGL(kern, dim3(cap), dim3(256), 0, s, part, parts, ld, (const int *)rl.list, (const int *)rl.count, (const float *)rl.scale, first, cap, d, held, (T *)dX);
        return hipGetLastError();
    };
    return bf16 ? run(finish_dx_kernel<bf16_t>, (bf16_t *)nullptr) : run(finish_dx_kernel<float>, (float *)nullptr);
}

// as many rows a workgroup as it has threads for (97624 x 205, a workgroup a row: 49 us, several: 24)
template <typename T>
__global__ __launch_bounds__(256) void finish_dw_kernel(const float *part, int parts, size_t stride, int ld, size_t rows, int d, const float *scale, T *dW)
{
    const int n = threads_of(d);
    const size_t r = (size_t)blockIdx.x * (256 / n) + threadIdx.x / n;
    if (r >= rows) return;
    const float factor = scale[1];
    for (int c = (int)threadIdx.x % n * 8; c < d; c += n * 8) {
        float f[8];
        sum_parts(part + r * ld + c, 0, parts, 1, stride, d - c, f);
        store_scaled(dW + r * d + c, d - c, f, factor);
    }
}

hipError_t launch_finish_dw(bool bf16, RowList rl, const float *part, int parts, size_t stride, int ld, size_t rows, int d, void *dW, hipStream_t s)
{
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        const size_t per = 256 / threads_of(d);
        hipLaunchKernelGGL(kern, dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, s, part, parts, stride, ld, rows, d, (const float *)rl.scale, (T *)dW);
        return hipGetLastError();
    };
    return bf16 ? run(finish_dw_kernel<bf16_t>, (bf16_t *)nullptr) : run(finish_dw_kernel<float>, (float *)nullptr);
}

}  // namespace lm
}  // namespace stl
