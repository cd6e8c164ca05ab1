// The residual step: bf16 storage, the dealing of rows, and the last stage of the sums over rows.
#include "lm_residual.h"

namespace stl {
namespace lm {

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T *p, size_t n)
{
    for (size_t i = blockIdx.x * (size_t)256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

hipError_t launch_zero_elements(bool bf16, void *p, size_t n, hipStream_t s)
{
    const size_t blocks = (n + 255) / 256;
    const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048));
    if (n == 0) return hipSuccess;
    if (bf16) hipLaunchKernelGGL(zero_kernel<bf16_t>, grid, dim3(256), 0, s, (bf16_t *)p, n);
    else hipLaunchKernelGGL(zero_kernel<float>, grid, dim3(256), 0, s, (float *)p, n);
    return hipGetLastError();
}

// out[c] (+)= sum of nb partials part[b * stride + c], c < n, in an order that depends on nb alone: 16 threads a column take every 16th each
// and are added up in turn.
struct SumJob {
    const float *part;
    float *out;
    int nb;
    size_t stride;
};
struct SumJobs {
    SumJob job[4];
    // then one for every group of rows that share a gate row: its partials lie one after the other
    const float *gate_part;
    float *dgate;
    int vectors, pieces;
};
__global__ __launch_bounds__(1024) void residual_sums_kernel(const SumJobs jobs, int n, int accumulate)
{
    __shared__ float red[1024];
    const int x = (int)threadIdx.x & 63, y = (int)threadIdx.x >> 6, c = (int)blockIdx.x * 64 + x;
    SumJob j;
    if ((int)blockIdx.y < jobs.vectors) {
        j = jobs.job[blockIdx.y];
    } else {
        const size_t group = blockIdx.y - jobs.vectors;
        j = SumJob{jobs.gate_part + group * jobs.pieces * n, jobs.dgate + group * n, jobs.pieces, (size_t)n};
    }
    float v = 0.f;
    if (c < n)
        for (int b = y; b < j.nb; b += 64) {
            float u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = b + 16 * k < j.nb ? j.part[(size_t)(b + 16 * k) * j.stride + c] : 0.f;
            v += (u[0] + u[1]) + (u[2] + u[3]);
        }
    red[threadIdx.x] = v;
    __syncthreads();
    if (y == 0 && c < n) {
        for (int k = 1; k < 16; ++k) v += red[k * 64 + x];
        j.out[c] = accumulate ? j.out[c] + v : v;
    }
}

// One workgroup a CU (two take 97 us instead of 92 for 8192 x 4096 bf16: twice the partials, and no more wavefronts are resident): the rows of a
// group are dealt in as many pieces as give each of them one, but no fewer rows a piece than a workgroup takes at a time.
static ResidualItems residual_items(int rows, int n, int per_gate, bool gate, int *grid)
{
    ResidualItems it{};
    it.gate_rows = gate && per_gate == 1;
    it.per = !gate || it.gate_rows || per_gate > rows ? rows : per_gate;
    it.groups = (rows + it.per - 1) / it.per;
    const int tpr = n <= 512 ? 64 : n <= 1024 ? 128 : n <= 2048 ? 256 : 512, lanes = tpr < kBackThreads ? kBackThreads / tpr : 1, target = 256;
    int pieces = (target + it.groups - 1) / it.groups;
    const int most = (it.per + lanes - 1) / lanes;
    if (pieces > most) pieces = most;
    it.chunk = (it.per + pieces - 1) / pieces;
    it.pieces = (it.per + it.chunk - 1) / it.chunk;
    const long items = (long)it.groups * it.pieces;
    *grid = (int)(items < target ? items : target);
    return it;
}

static inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t residual_workspace_bytes(int rows, int n, int per_gate)
{
    if (rows == 0) return 0;
    // with a gate or without one: the vectors' partials of at most 256 workgroups and the gate's, one an item
    int grid = 0, gateless = 0;
    const ResidualItems it = residual_items(rows, n, per_gate, true, &grid);
    residual_items(rows, n, per_gate, false, &gateless);
    const size_t vec = round256((size_t)(grid > gateless ? grid : gateless) * 4 * n * sizeof(float));
    return vec + (it.gate_rows ? 0 : round256((size_t)it.groups * it.pieces * n * sizeof(float)));
}

hipError_t launch_residual_forward(int dtype, const ResidualArgs &a, void *Xout, void *Z, hipStream_t s)
{
    return dtype == 0 ? residual_forward_f32(a, Xout, Z, s) : residual_forward<bf16_t>(a, Xout, Z, s);
}

hipError_t launch_residual_backward(int dtype, const ResidualArgs &a, const ResidualGrads &g, void *ws, hipStream_t s)
{
    int grid = 0;
    ResidualItems it = residual_items(a.rows, a.n, a.per_gate, a.gate != nullptr, &grid);
    it.vec_part = (float *)ws;
    it.gate_part = (float *)((char *)ws + round256((size_t)grid * 4 * a.n * sizeof(float)));
    const hipError_t e = dtype == 0 ? residual_backward_f32(a, g, it, grid, s) : residual_backward<bf16_t>(a, g, it, grid, s);
    if (e != hipSuccess) return e;
    SumJobs jobs{};
    float *outs[4] = {g.dw_pre, g.db_pre, g.dw_post, g.db_post};
    for (int i = 0; i < 4; ++i)
        if (outs[i]) jobs.job[jobs.vectors++] = SumJob{it.vec_part + (size_t)i * a.n, outs[i], grid, (size_t)4 * a.n};
    const int cols = (a.n + 63) / 64;
    int gates = 0;
    if (g.dgate && !it.gate_rows) jobs.gate_part = it.gate_part, jobs.dgate = g.dgate, jobs.pieces = it.pieces, gates = it.groups;
    // a launch has at most 32768 rows of workgroups
    for (int at = 0; jobs.vectors + gates > 0; at += 32768) {
        const int now = gates < 32768 ? gates : 32768;
        hipLaunchKernelGGL(residual_sums_kernel, dim3(cols, jobs.vectors + now), dim3(1024), 0, s, jobs, a.n, g.accumulate);
        const hipError_t e2 = hipGetLastError();
        if (e2 != hipSuccess) return e2;
        gates -= now;
        jobs.vectors = 0;
        jobs.gate_part += (size_t)now * jobs.pieces * a.n;
        if (jobs.dgate) jobs.dgate += (size_t)now * a.n;
    }
    return hipSuccess;
}

}  // namespace lm
}  // namespace stl
