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

// One workgroup: every thread counts a run of neighbouring rows, the counts are added up over the workgroup, and every thread lists its rows.
__global__ __launch_bounds__(1024) void select_rows_kernel(Terms t, int rows, int *list, int *count)
{
    __shared__ int sums[1024];
    const int per = (rows + 1023) / 1024, r0 = (int)threadIdx.x * per, r1 = r0 + per < rows ? r0 + per : rows;
    int n = 0;
    for (int r = r0; r < r1; ++r) n += t.any(r);
    sums[threadIdx.x] = n;
    __syncthreads();
    for (int step = 1; step < 1024; step *= 2) {
        const int v = (int)threadIdx.x >= step ? sums[threadIdx.x - step] : 0;
        __syncthreads();
        sums[threadIdx.x] += v;
        __syncthreads();
    }
    int at = sums[threadIdx.x] - n;
    for (int r = r0; r < r1; ++r)
        if (t.any(r)) list[at++] = r;
    if (threadIdx.x == 1023) *count = sums[1023];
}

hipError_t launch_select_rows(const VocabArgs &a, RowList rl, hipStream_t s)
{
    hipLaunchKernelGGL(select_rows_kernel, dim3(1), dim3(1024), 0, s, terms_of(a), a.rows, rl.list, rl.count);
    return hipGetLastError();
}

// ---- rows side by side ---------------------------------------------------------------------------------------------------------------
// a workgroup a row: the row list[first + b] (or, without a list, first + b) of `in`, zeros where there is none and behind its end
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(const T *in, const int *list, const int *count, int first, int d, int ld, T *out)
{
    const int r = first + (int)blockIdx.x;
    const int row = !list ? r : r < *count ? list[r] : -1;
    T *o = out + (size_t)blockIdx.x * ld;
    for (int c = (int)threadIdx.x * 8; c < ld; c += 2048) {
        Chunk<T> v;
        v.fill(0.f);
        if (row >= 0 && c < d) v.load(in + (size_t)row * d + c, d - c);
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v.get(e);
        Chunk<T>::store(o + c, ld - c, f);
    }
}

hipError_t launch_gather_rows(bool bf16, const void *X, RowList rl, int first, int cap, int d, int ld, void *out, hipStream_t s)
{
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        hipLaunchKernelGGL(kern, dim3(cap), dim3(256), 0, s, (const T *)X, (const int *)rl.list, (const int *)rl.count, first, d, ld, (T *)out);
        return hipGetLastError();
    };
    return bf16 ? run(copy_rows_kernel<bf16_t>, (bf16_t *)nullptr) : run(copy_rows_kernel<float>, (float *)nullptr);
}

hipError_t launch_pad_rows(const void *in, int rows, int d, int ld, void *out, hipStream_t s)
{
    hipLaunchKernelGGL(copy_rows_kernel<bf16_t>, dim3(rows), dim3(256), 0, s, (const bf16_t *)in, (const int *)nullptr, (const int *)nullptr, 0, d, ld,
                       (bf16_t *)out);
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

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// One listed row a workgroup.  With p = softmax(z), p_tau = softmax(z / tau), q the teacher's shares and their entries id_j:
//     label_loss = lse - z_label,   top_loss = sum_j q_j (log q_j - z_id_j / tau + lse_tau),
//     dz_v = dlabel (p_v - [v = label]) + dtop / tau (p_tau,v - sum_{j: id_j = v} q_j).
// The row is written in one sweep without the label's and the entries' own terms, which then overwrite their places: their logits are taken in
// fp32 (p - 1 of a label that is nearly certain loses everything in 16 bits).  bf16 storage: the sweep reads a logit as 16-bit steps below its group's
// maximum (kSteps) and writes the bf16 gradient over it; the row's dot products with the label's and the entries' rows of W give their logits.
// What bounds it: reading and writing the row, 4 bytes a logit (bf16) or 8.
template <typename T, bool GRADS>
__global__ __launch_bounds__(kRowThreads) void vocab_rows_kernel(Terms t, const VocabGrads g, const T *W, int d, float tau, const int *list, const int *count,
                                                                 VocabChunk c, float *label_loss, float *top_loss)
{
    constexpr bool BF16 = sizeof(T) == 2;
    __shared__ float red[kRowWaves];
    __shared__ int ids[kMostTop + 1];        // the entries', and behind them the label's
    __shared__ float y[kMostTop], q[kMostTop], all[kMostTop + 1], z[kMostTop + 1];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, r = (int)blockIdx.x, vocab = t.vocab;
    T *codes = (T *)c.codes + (size_t)r * c.ld;
    if (c.first + r >= *count) {
        // behind the list: the products read whole stages of 32 rows (fp32 storage: all rows of the chunk)
        const int listed = *count - c.first, read = BF16 ? (listed + 31) / 32 * 32 : c.cap;
        if (GRADS && r < read)
            for (size_t v = tid; v < c.ld; v += kRowThreads) codes[v] = 0;
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

    // log of the sums over the vocabulary; with one term the product keeps one sum, of that term's temperature
    float m = -INFINITY, sum = 0.f, sum_tau = 0.f;
    const float *gm = nullptr;
    if constexpr (BF16) {
        gm = c.group_max + (size_t)r * c.groups;
        const float *gs = c.group_sum + (size_t)r * c.groups, *gt = c.group_sum_tau ? c.group_sum_tau + (size_t)r * c.groups : nullptr;
        for (int i = tid; i < c.groups; i += kRowThreads) m = fmaxf(m, gm[i]);
        m = block_max(m, red);
        for (int i = tid; i < c.groups; i += kRowThreads) {
            const float below = gm[i] - m;
            sum += gs[i] * exp_fast(t.label ? below : below * inv_tau);
            if (gt) sum_tau += gt[i] * exp_fast(below * inv_tau);
        }
    } else {
        const float *Z = (const float *)codes;
        for (int v = tid; v < vocab; v += kRowThreads) m = fmaxf(m, Z[v]);
        m = block_max(m, red);
        for (int v = tid; v < vocab; v += kRowThreads) {
            sum += expf(Z[v] - m);
            if (ntop) sum_tau += expf((Z[v] - m) * inv_tau);
        }
    }
    sum = block_sum(sum, red);
    sum_tau = block_sum(sum_tau, red);
    if constexpr (BF16)
        if (!c.group_sum_tau) sum_tau = sum;
    const float lse = m + logf(sum), lse_tau = m * inv_tau + logf(sum_tau);

    // the logits of the label and the teacher's entries
    if constexpr (BF16) {
        const bf16_t *x = (const bf16_t *)c.Xc + (size_t)r * c.ldx;
        for (int j = wave; j <= ntop; j += kRowWaves) {
            if (ids[j] < 0) continue;
            const bf16_t *w = (const bf16_t *)W + (size_t)ids[j] * d;
            float dot = 0.f;
            for (int e0 = lane * 8; e0 < d; e0 += 512) {
                Chunk<bf16_t> a, b;
                a.load(x + e0, d - e0);
                b.load(w + e0, d - e0);
#pragma unroll
                for (int e = 0; e < 8; ++e) dot = fmaf(a.get(e), b.get(e), dot);
            }
            dot = wave_sum(dot);
            if (lane == 0) z[j] = dot;
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
        const float cl = labelled && g.dlabel ? g.dlabel[row] : 0.f, ct = taught && g.dtop ? g.dtop[row] * inv_tau : 0.f;
        if constexpr (BF16) {
            // chunks of eight logits lie in one group of 64
            const float *gstep = c.group_step + (size_t)r * c.groups;
            for (size_t v = (size_t)tid * 8; v < c.ld; v += kRowThreads * 8) {
                const u32x4_t in = *reinterpret_cast<const u32x4_t *>(codes + v);
                const float mg = gm[v / 64], step = gstep[v / 64];
                const float at = mg - lse, at_tau = mg * inv_tau - lse_tau;
                float out[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t code = (in[e >> 1] >> (16 * (e & 1))) & 0xffffu;
                    const float below = -(float)code * step;
                    float dz = 0.f;
                    if (labelled) dz = cl * exp_fast(at + below);
                    if (taught) dz = fmaf(ct, exp_fast(fmaf(below, inv_tau, at_tau)), dz);
                    // a row whose sums are not a number stays one throughout
                    out[e] = code == 65535u && lse == lse ? 0.f : dz;
                }
                *reinterpret_cast<u32x4_t *>(codes + v) =
                    u32x4_t{pack_bf16x2(out[0], out[1]), pack_bf16x2(out[2], out[3]), pack_bf16x2(out[4], out[5]), pack_bf16x2(out[6], out[7])};
            }
        } else {
            float *Z = (float *)codes;
            for (int v = tid; v < vocab; v += kRowThreads) {
                float dz = 0.f;
                if (labelled) dz = cl * expf(Z[v] - lse);
                if (taught) dz = fmaf(ct, expf(fmaf(Z[v], inv_tau, -lse_tau)), dz);
                Z[v] = dz;
            }
        }
        __syncthreads();                     // the sweep's stores are done before the entries' places are written again
        for (int j = tid; j <= ntop; j += kRowThreads) {
            const int v = ids[j];
            if (v < 0) continue;
            float dz = 0.f;
            if (labelled) dz = cl * (expf(z[j] - lse) - (ids[ntop] == v ? 1.f : 0.f));
            if (taught) dz = fmaf(ct, expf(fmaf(z[j], inv_tau, -lse_tau)) - all[j], dz);
            Elem<T>::st(codes + v, dz);
        }
    }
}

hipError_t launch_vocab_rows(const VocabArgs &a, const VocabGrads *g, RowList rl, const VocabChunk &c, float *label_loss, float *top_loss, hipStream_t s)
{
    const VocabGrads none{};
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        // with gradients of bf16 storage also the rows up to a whole stage of the products' contraction
        const int rows = a.bf16 && g ? (c.cap + 31) / 32 * 32 : c.cap;
        hipLaunchKernelGGL(kern, dim3(rows), dim3(kRowThreads), 0, s, terms_of(a), g ? *g : none, (const T *)a.W, a.d, a.tau, (const int *)rl.list,
                           (const int *)rl.count, c, label_loss, top_loss);
        return hipGetLastError();
    };
    if (a.bf16) return g ? run(vocab_rows_kernel<bf16_t, true>, (bf16_t *)nullptr) : run(vocab_rows_kernel<bf16_t, false>, (bf16_t *)nullptr);
    return g ? run(vocab_rows_kernel<float, true>, (float *)nullptr) : run(vocab_rows_kernel<float, false>, (float *)nullptr);
}

// ---- the gradients' last stage ---------------------------------------------------------------------------------------------------------
// a workgroup a row of the chunk: the sum of its parts, rounded once, to where the row came from
template <typename T>
__global__ __launch_bounds__(256) void finish_rows_kernel(const float *part, int parts, size_t stride, int ld, const int *list, const int *count, int first,
                                                          int d, T *out)
{
    const size_t r = blockIdx.x + (size_t)blockIdx.y * 32768;
    if (list && first + (int)r >= *count) return;
    const size_t row = list ? (size_t)list[first + r] : r;
    for (int c = (int)threadIdx.x * 8; c < d; c += 2048) {
        float f[8] = {};
        for (int p = 0; p < parts; ++p) {
            Chunk<float> v;
            v.load(part + p * stride + r * ld + c, d - c);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += v.get(e);
        }
        Chunk<T>::store(out + row * d + c, d - c, f);
    }
}

hipError_t launch_finish_dx(bool bf16, const float *part, int parts, size_t stride, int ld, RowList rl, int first, int cap, int d, void *dX, hipStream_t s)
{
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        hipLaunchKernelGGL(kern, dim3(cap), dim3(256), 0, s, part, parts, stride, ld, (const int *)rl.list, (const int *)rl.count, first, d, (T *)dX);
        return hipGetLastError();
    };
    return bf16 ? run(finish_rows_kernel<bf16_t>, (bf16_t *)nullptr) : run(finish_rows_kernel<float>, (float *)nullptr);
}

hipError_t launch_finish_dw(bool bf16, const float *part, int parts, size_t stride, int ld, size_t rows, int d, void *dW, hipStream_t s)
{
    auto run = [&](auto kern, auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        // 32768 rows of workgroups at a time
        for (size_t at = 0; at < rows; at += 32768) {
            const size_t now = rows - at < 32768 ? rows - at : 32768;
            hipLaunchKernelGGL(kern, dim3((unsigned)now), dim3(256), 0, s, part + at * ld, parts, stride, ld, (const int *)nullptr, (const int *)nullptr, 0, d,
                               (T *)dW + at * d);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    return bf16 ? run(finish_rows_kernel<bf16_t>, (bf16_t *)nullptr) : run(finish_rows_kernel<float>, (float *)nullptr);
}

// zeros in dX's rows without a term, and in their losses' places
template <typename T>
__global__ __launch_bounds__(256) void zero_others_kernel(Terms t, int d, T *out, float *label_loss, float *top_loss)
{
    const int row = (int)blockIdx.x;
    if (t.any(row)) return;
    if (threadIdx.x == 0) {
        if (label_loss) label_loss[row] = 0.f;
        if (top_loss) top_loss[row] = 0.f;
    }
    if (out) {
        const float f[8] = {};
        for (int c = (int)threadIdx.x * 8; c < d; c += 2048) Chunk<T>::store(out + (size_t)row * d + c, d - c, f);
    }
}

hipError_t launch_zero_others(const VocabArgs &a, void *dX, float *label_loss, float *top_loss, hipStream_t s)
{
    if (a.bf16) hipLaunchKernelGGL(zero_others_kernel<bf16_t>, dim3(a.rows), dim3(256), 0, s, terms_of(a), a.d, (bf16_t *)dX, label_loss, top_loss);
    else hipLaunchKernelGGL(zero_others_kernel<float>, dim3(a.rows), dim3(256), 0, s, terms_of(a), a.d, (float *)dX, label_loss, top_loss);
    return hipGetLastError();
}

}  // namespace lm
}  // namespace stl
