// Embedding: rows of a vocabulary by token, and their gradient by sorted tokens (gfx950).
//
//   X[i] = scale W[token i]                      memory: rows of W read where they lie, X written once
//   dW[v] (+)= scale sum_{i: token i = v} dX[i]
//
// The gradient is formed without floating-point atomics, so that its bits do not depend on the order in which workgroups run.  Three launches:
//  1. the rows sorted by id.  The vocabulary is cut into ranges, a workgroup each.  It reads all tokens twice: once to count its ids (and, for the place at
//     which its rows begin, the tokens of lower ids), once to write its rows down, in order.  A wavefront walks over consecutive tokens and has counts of
//     its own, so the order of rows with one id is that of the batch.  Ids that do not occur are noted as bits.
//  2. sums over the sorted rows, cut into segments of equal length whatever the ids: a common token's many rows are shared by many workgroups.
//     A run of one id that lies in one segment is finished there; parts of others go to the workspace in fp32.  Zeros for absent ids beside them.
//  3. parts of a run that several segments share are added up in order.
#include "seq_kernels.h"
#include "../lm/lm_device.h"

namespace stl {
namespace seq {

using lm::Chunk;

// rows of `per` threads with a chunk of 8 elements each, 256 / per rows a workgroup; wider rows take several in blockIdx.y
template <typename T>
__global__ __launch_bounds__(256) void embed_kernel(const EmbedArgs a, int per, const int64_t *token, const T *W, T *X)
{
    const int sub = (int)threadIdx.x / per, at = 8 * ((int)blockIdx.y * per + (int)threadIdx.x % per);
    const size_t row = (size_t)blockIdx.x * (256 / per) + sub;
    const int left = a.d - at;
    if (row >= (size_t)a.rows || left <= 0) return;
    const int64_t id = token[row];
    Chunk<T> c;
    c.fill(0.f);
    if (id >= 0 && id < a.vocab) c.load(W + (size_t)id * a.d + at, left);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = a.scale * c.get(e);
    Chunk<T>::store(X + row * a.d + at, left, v);
}

constexpr int kWaves = 16, kMostWidth = 960;                   // 60 KB of counts

// The lanes' ids that lie in [first, first + width), one after the other: lanes of the same id go together.  f(id - first, their mask)
template <typename F>
__device__ __forceinline__ void each_id(int rel, int width, F f)
{
    uint64_t todo = __ballot((unsigned)rel < (unsigned)width);
    while (todo) {
        const int one = __builtin_amdgcn_readlane(rel, __builtin_ctzll(todo));
        const uint64_t same = __ballot(rel == one) & todo;
        f(one, same);
        todo &= ~same;
    }
}

__global__ __launch_bounds__(64 * kWaves) void embed_sort_kernel(const EmbedArgs a, const EmbedPlan plan, const int64_t *token, int *order, int *ids, int *total,
                                                                 uint64_t *absent)
{
    __shared__ int count[kWaves][kMostWidth];
    __shared__ int below[kWaves];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int first = (int)blockIdx.x * plan.width, width = a.vocab - first < plan.width ? a.vocab - first : plan.width;
    for (int w = 0; w < kWaves; ++w)
        if ((int)threadIdx.x < width) count[w][threadIdx.x] = 0;
    __syncthreads();
    // tokens of this wavefront: whole steps of 64
    const int steps = (a.rows + 63) / 64, per = (steps + kWaves - 1) / kWaves;
    const int begin = wave * per, end = begin + per < steps ? begin + per : steps;
    auto id_of = [&](int step) {
        const int row = 64 * step + lane;
        const int64_t id = row < a.rows ? token[row] : -1;
        return id >= 0 && id < a.vocab ? (int)id : -1;
    };
    int lower = 0;
    for (int step = begin; step < end; step += 8) {
        int id[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) id[u] = step + u < end ? id_of(step + u) : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            lower += (int)__popcll(__ballot((unsigned)id[u] < (unsigned)first));
            const int rel = id[u] < 0 ? -1 : id[u] - first;
            if ((unsigned)rel < (unsigned)width) atomicAdd(&count[wave][rel], 1);
        }
    }
    if (lane == 0) below[wave] = lower;
    __syncthreads();
    // where each id's rows of each wavefront begin: ids in order, then wavefronts; thread i sums id i, then a scan over ids
    const int id = (int)threadIdx.x;
    int mine = 0;
    if (id < width)
        for (int w = 0; w < kWaves; ++w) mine += count[w][id];
    __shared__ int wave_sum[kWaves];
    int upto = mine;                                             // inclusive, over the wavefront
    for (int n = 1; n < 64; n *= 2) {
        const int other = __shfl_up(upto, n);
        if (lane >= n) upto += other;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < kWaves; ++w) base += below[w] + (w < wave ? wave_sum[w] : 0);
    if (id < width) {
        int at = base + upto - mine;
        for (int w = 0; w < kWaves; ++w) {
            const int n = count[w][id];
            count[w][id] = at;
            at += n;
        }
    }
    if ((int)blockIdx.x == plan.ranges - 1 && threadIdx.x == 64 * kWaves - 1) *total = base + upto;
    // ids that do not occur, a bit each, for the zeros that the sums' launch writes
    const uint64_t gone = __ballot(id < width && mine == 0);
    if (lane == 0) absent[(size_t)blockIdx.x * kWaves + wave] = gone;
    __syncthreads();
    for (int step = begin; step < end; step += 8) {
        int got[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) got[u] = step + u < end ? id_of(step + u) : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int rel = got[u] < 0 ? -1 : got[u] - first;
            const int row = 64 * (step + u) + lane;
            each_id(rel, width, [&](int one, uint64_t same) {
                const int at = count[wave][one];                  // all lanes read it before one of them moves it on
                asm volatile("" ::: "memory");
                if (same >> lane & 1) {
                    const int rank = (int)__popcll(same & ((1ull << lane) - 1));
                    order[at + rank] = row;
                    ids[at + rank] = first + one;
                    if (rank == 0) count[wave][one] = at + (int)__popcll(same);
                }
                asm volatile("" ::: "memory");
            });
        }
    }
}

// zeros for the absent ones of 64 ids
template <typename T>
__device__ __forceinline__ void write_zeros(const EmbedArgs &a, const EmbedPlan &plan, int some, const uint64_t *absent, T *dW)
{
    const int each = (plan.width + 63) / 64, range = some / each, word = some % each, lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const uint64_t bits = absent[(size_t)range * kWaves + word];
    constexpr int per16 = 16 / (int)sizeof(T);
    for (int i = wave; i < 64; i += 4) {
        if (!(bits >> i & 1)) continue;
        T *out = dW + ((size_t)range * plan.width + 64 * word + i) * a.d;
        // whole 16-byte pieces at such addresses, lane by lane, and single elements in front of them and behind
        int head = (int)(-(uintptr_t)out % 16 / sizeof(T));
        head = head < a.d ? head : a.d;
        const int pieces = (a.d - head) / per16, rest = a.d - head - pieces * per16;
        for (int c = lane; c < pieces; c += 64) *reinterpret_cast<u32x4_t *>(out + head + c * per16) = u32x4_t{0u, 0u, 0u, 0u};
        if (lane < head) Elem<T>::st(out + lane, 0.f);
        if (lane < rest) Elem<T>::st(out + a.d - 1 - lane, 0.f);
    }
}

// A chunk of 8 columns a thread.  parts[2 s]: the sum of segment s's rows that go on from segment s - 1; parts[2 s + 1]: of those that go on behind it.
// Workgroups behind the segments': zeros for up to 64 ids that do not occur, most of dW, while the sums wait for their rows.
template <typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(const EmbedArgs a, const EmbedPlan plan, const int *order, const int *ids, const int *total,
                                                        const uint64_t *absent, const T *dX, T *dW, float *parts, int accumulate)
{
    if ((int)blockIdx.x >= plan.segments) {
        if (blockIdx.y == 0) write_zeros(a, plan, (int)blockIdx.x - plan.segments, absent, dW);
        return;
    }
    const int seg = (int)blockIdx.x, col = 8 * ((int)blockIdx.y * 256 + (int)threadIdx.x), left = a.d - col;
    const int count = *total;
    const int64_t first = (int64_t)seg * plan.length;
    if (first >= count || left <= 0) return;
    const int begin = (int)first, end = begin + plan.length < count ? begin + plan.length : count;
    float sum[8] = {};
    bool whole = begin == 0 || ids[begin - 1] != ids[begin];      // the present run begins in this segment
    for (int at = begin; at < end; at += 8) {
        Chunk<T> c[8];
        int id[9];
#pragma unroll
        for (int u = 0; u < 9; ++u) id[u] = at + u < count ? ids[at + u] : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (at + u < end) c[u].load(dX + (size_t)order[at + u] * a.d + col, left);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (at + u >= end) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += c[u].get(e);
            const bool last = at + u == end - 1, over = id[u + 1] != id[u];
            if (!last && !over) continue;
            if (whole && over) {
                T *out = dW + (size_t)id[u] * a.d + col;
                Chunk<T> old;
                old.fill(0.f);
                if (accumulate) old.load(out, left);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = a.scale * sum[e] + old.get(e);
                Chunk<T>::store(out, left, sum);
            } else {
                Chunk<float>::store(parts + (2 * (size_t)seg + (whole ? 1 : 0)) * a.d + col, left, sum);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            whole = true;
        }
    }
}

// The run that begins in this segment and goes on behind it, if there is one: a wavefront has 512 columns, the four of a workgroup take the run's segments eight at a
// time in turn, and their sums are added in order.
template <typename T>
__global__ __launch_bounds__(256) void embed_join_kernel(const EmbedArgs a, const EmbedPlan plan, const int *ids, const int *total, const float *parts, T *dW,
                                                         int accumulate)
{
    constexpr int kStep = 8;
    __shared__ __align__(16) float sums[3][512];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int seg = (int)blockIdx.x, col = 512 * (int)blockIdx.y + 8 * lane, left = a.d - col;
    // (all at once: what lies behind the last sorted row is no id, and not used)
    const int64_t begin = (int64_t)seg * plan.length, next = begin + plan.length, mine = next + (int64_t)plan.length * lane;
    const int count = *total, id = ids[next], before = ids[next - 1], first = ids[begin], earlier = begin > 0 ? ids[begin - 1] : -1;
    int there = ids[mine < a.rows ? mine : begin];
    if (next >= count || before != id) return;
    // (a run that covers all of this segment and begins before it is another segment's)
    if (first == id && earlier == id) return;
    // segments whose first row is the run's, 64 at a time
    int more = 0;
    for (;;) {
        const int64_t row = next + (int64_t)plan.length * (more + lane);
        const uint64_t other = ~__ballot(row < count && there == id);
        more += other ? (int)__builtin_ctzll(other) : 64;
        if (other) break;
        const int64_t ahead = next + (int64_t)plan.length * (more + lane);
        there = ids[ahead < a.rows ? ahead : begin];
    }
    float sum[8] = {};
    if (wave == 0) {
        Chunk<float> c;
        c.load(parts + (2 * (size_t)seg + 1) * a.d + col, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = c.get(e);
    }
    for (int at = kStep * wave; at < more; at += 4 * kStep) {
        Chunk<float> c[kStep];
#pragma unroll
        for (int u = 0; u < kStep; ++u) c[u].load(parts + 2 * (size_t)(seg + 1 + (at + u < more ? at + u : at)) * a.d + col, left);
#pragma unroll
        for (int u = 0; u < kStep; ++u)
            if (at + u < more)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += c[u].get(e);
    }
    if (wave > 0) Chunk<float>::store(&sums[wave - 1][8 * lane], 8, sum);
    __syncthreads();
    if (wave > 0 || left <= 0) return;
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += sums[w][8 * lane + e];
    T *out = dW + (size_t)id * a.d + col;
    Chunk<T> old;
    old.fill(0.f);
    if (accumulate) old.load(out, left);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = a.scale * sum[e] + old.get(e);
    Chunk<T>::store(out, left, sum);
}

EmbedPlan embed_plan(const EmbedArgs &a)
{
    EmbedPlan p{};
    p.ranges = a.vocab < 256 ? a.vocab : 256;
    if ((a.vocab + p.ranges - 1) / p.ranges > kMostWidth) p.ranges = (a.vocab + kMostWidth - 1) / kMostWidth;
    p.width = (a.vocab + p.ranges - 1) / p.ranges;
    p.ranges = (a.vocab + p.width - 1) / p.width;
    p.length = (a.rows + 2047) / 2048;
    if (p.length < 16) p.length = 16;
    p.segments = (a.rows + p.length - 1) / p.length;
    auto whole = [](size_t n) { return (n + 255) / 256 * 256; };
    p.ids_at = 256 + whole((size_t)a.rows * 4);
    p.absent_at = p.ids_at + whole((size_t)a.rows * 4);
    p.parts_at = p.absent_at + whole((size_t)p.ranges * kWaves * 8);
    p.bytes = p.parts_at + whole((size_t)p.segments * 2 * a.d * 4);
    return p;
}

template <typename T>
hipError_t forward(const EmbedArgs &a, const int64_t *token, const void *W, void *X, hipStream_t s)
{
    const int chunks = (a.d + 7) / 8;
    int per = 1;
    while (per < chunks && per < 256) per *= 2;
    const int rows = 256 / per;
    hipLaunchKernelGGL(embed_kernel<T>, dim3((a.rows + rows - 1) / rows, (chunks + per - 1) / per), dim3(256), 0, s, a, per, token, (const T *)W, (T *)X);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const EmbedArgs &a, const int64_t *token, const void *dX, void *dW, int accumulate, void *ws, hipStream_t s)
{
    const EmbedPlan p = embed_plan(a);
    int *total = (int *)ws, *order = (int *)((char *)ws + 256), *ids = (int *)((char *)ws + p.ids_at);
    uint64_t *absent = (uint64_t *)((char *)ws + p.absent_at);
    float *parts = (float *)((char *)ws + p.parts_at);
    hipLaunchKernelGGL(embed_sort_kernel, dim3(p.ranges), dim3(64 * kWaves), 0, s, a, p, token, order, ids, total, absent);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int zeros = accumulate ? 0 : p.ranges * ((p.width + 63) / 64);
    hipLaunchKernelGGL(embed_sum_kernel<T>, dim3(p.segments + zeros, (a.d + 2047) / 2048), dim3(256), 0, s, a, p, order, ids, total, absent, (const T *)dX, (T *)dW, parts,
                       accumulate);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.segments == 1) return hipSuccess;
    hipLaunchKernelGGL(embed_join_kernel<T>, dim3(p.segments - 1, (a.d + 511) / 512), dim3(256), 0, s, a, p, ids, total, parts, (T *)dW, accumulate);
    return hipGetLastError();
}

hipError_t launch_embed_forward(int dtype, const EmbedArgs &a, const int64_t *token, const void *W, void *X, hipStream_t s)
{
    return dtype ? forward<bf16_t>(a, token, W, X, s) : forward<float>(a, token, W, X, s);
}

hipError_t launch_embed_backward(int dtype, const EmbedArgs &a, const int64_t *token, const void *dX, void *dW, int accumulate, void *ws, hipStream_t s)
{
    return dtype ? backward<bf16_t>(a, token, dX, dW, accumulate, ws, s) : backward<float>(a, token, dX, dW, accumulate, ws, s);
}

}  // namespace seq
}  // namespace stl
