// Embedding: rows of a vocabulary by token, and their gradient by sorted tokens (gfx950).
//
//   X[i] = scale W[token i]                      memory: rows of W read where they lie, X written once
//   dW[v] (+)= scale sum_{i: token i = v} dX[i]
//
// The gradient is formed without floating-point atomics, so that its bits do not depend on the order in which workgroups run.  Three launches:
//  1. the rows sorted by id.  The vocabulary is cut into ranges, a workgroup each.  It reads all tokens twice: once to count its ids (and, for the place at
//     which its rows begin, the tokens of lower ids), once to write its rows down, in order.  A wavefront walks over consecutive tokens and has counts of
//     its own, so the order of rows with one id is that of the batch.  Other workgroups write zeros to all of dW meanwhile: few of its rows are any token's.
//  2. sums over the sorted rows, cut into segments of equal length whatever the ids: a common token's many rows are shared by many workgroups.
//     A run of one id that lies in one segment is finished there; parts of others go to the workspace in fp32.
//  3. parts of a run that several segments share are added up, in four sums that take eight of them in turn.
// 16384 rows of 2048 in bf16, 32000 ids: 33 us (131 MB of zeros; the sort alone takes 17), 20 (96 MB, 4.7 TB/s) and 7 (a chain of loads: the commonest id has 102
// segments); a forward call of 8192 rows of 4096: 21 us, 5.4 TB/s.  The sort reads all tokens in every range, which takes over for many rows: 131072 rows of 1024: 119 us, 76 and 11.
#include "seq_kernels.h"
#include "../csrc/lm/lm_device.h"

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
    const bool there = id >= 0 && id < a.vocab;
    if (there) c.load(W + (size_t)id * a.d + at, left);
    const float scale = there ? a.scale : 0.f;                   // (zeros also where the scale is no finite number)
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = scale * c.get(e);
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

// `bytes` zeros from an address of 16 bytes on, by `of` workgroups
constexpr int kZeros = 4;                    // pieces of a thread and turn
__device__ __forceinline__ void write_zeros(char *to, size_t bytes, int block, int of)
{
    const size_t pieces = bytes / 16, step = (size_t)64 * kWaves;
    for (size_t at = (size_t)block * kZeros * step + threadIdx.x; at < pieces; at += (size_t)of * kZeros * step)
#pragma unroll
        for (int u = 0; u < kZeros; ++u)
            if (at + u * step < pieces) reinterpret_cast<u32x4_t *>(to)[at + u * step] = u32x4_t{0u, 0u, 0u, 0u};
    if (block == 0 && threadIdx.x < bytes % 16 / 2) reinterpret_cast<uint16_t *>(to + 16 * pieces)[threadIdx.x] = 0;
}

// Workgroups behind the ranges': zeros for dW, of which most rows are not any token's, while the others sort.
__global__ __launch_bounds__(64 * kWaves) void embed_sort_kernel(const EmbedArgs a, const EmbedPlan plan, const int64_t *token, int *order, int *ids, int *total,
                                                                 char *zeros, size_t bytes)
{
    if ((int)blockIdx.x >= plan.ranges) {
        write_zeros(zeros, bytes, (int)blockIdx.x - plan.ranges, (int)gridDim.x - plan.ranges);
        return;
    }
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

// A chunk of 8 columns a thread.  parts[2 s]: the sum of segment s's rows that go on from segment s - 1; parts[2 s + 1]: of those that go on behind it.
template <typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(const EmbedArgs a, const EmbedPlan plan, const int *order, const int *ids, const int *total,
                                                        const T *dX, T *dW, float *parts, int accumulate)
{
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
        // (rows behind the segment's are its last one; one branch for all of them, so that their loads are in flight together)
        const T *from[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) from[u] = dX + (size_t)order[at + u < end ? at + u : end - 1] * a.d + col;
        if (left >= 8) {
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u].load(from[u], 8);
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u].load(from[u], left);
        }
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
// time in turn (0 to 7, 32 to 39, ... the first), and the four sums are added up: an order that the tokens alone decide, but not that of the rows.
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
    // 16 rows a segment, or more where that makes 2048 of them; 8 where they are few and a workgroup's chain of loads is what takes the time (3001 rows of 1021 in
    // fp32: 17 -> 11 us for the sums; 16384 rows of 2048 in bf16 in eights: 20 -> 21, and joining them 7 -> 12)
    const bool few = a.rows <= 8192;
    p.length = few ? 8 : (a.rows + 2047) / 2048 > 16 ? (a.rows + 2047) / 2048 : 16;
    p.segments = (a.rows + p.length - 1) / p.length;
    const int sixteens = (a.rows + 15) / 16, room = few ? p.segments : sixteens < 1024 ? 1024 : sixteens < 2048 ? sixteens : 2048;   // (never less for more rows)
    auto whole = [](size_t n) { return (n + 255) / 256 * 256; };
    p.ids_at = 256 + whole((size_t)a.rows * 4);
    p.parts_at = p.ids_at + whole((size_t)a.rows * 4);
    p.bytes = p.parts_at + whole((size_t)room * 2 * a.d * 4);
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
    float *parts = (float *)((char *)ws + p.parts_at);
    // zeros: 256 KB a workgroup, at most two for each CU
    const size_t bytes = accumulate ? 0 : (size_t)a.vocab * a.d * sizeof(T), blocks = (bytes + 262143) / 262144;
    hipLaunchKernelGGL(embed_sort_kernel, dim3(p.ranges + (unsigned)(blocks < 512 ? blocks : 512)), dim3(64 * kWaves), 0, s, a, p, token, order, ids, total, (char *)dW, bytes);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(embed_sum_kernel<T>, dim3(p.segments, (a.d + 2047) / 2048), dim3(256), 0, s, a, p, order, ids, total, (const T *)dX, (T *)dW, parts, accumulate);
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
