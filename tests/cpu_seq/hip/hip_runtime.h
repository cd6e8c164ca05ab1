// The stand-in for the HIP runtime that runs kernels as they are meant to run (tests/cpu_emu/), with what the kernels of csrc_seq use beside.
#pragma once
#include "../../cpu_emu/hip/hip_runtime.h"
inline unsigned long long __ballot(int v)
{
    int *s = emu::Exchange<int>::all(v != 0);
    unsigned long long r = 0;
    for (int l = 0; l < 64; ++l) r |= (unsigned long long)(s[l] != 0) << l;
    emu::Exchange<int>::release();
    return r;
}
inline int __shfl(int v, int from) { return emu::from_lane(v, [&](int) { return from; }); }
inline int __popcll(unsigned long long v) { return __builtin_popcountll(v); }
inline int atomicAdd(int *p, int v) { const int old = *p; *p += v; return old; }
inline void sincospif(float x, float *s, float *c) { *s = (float)sin(M_PI * (double)x), *c = (float)cos(M_PI * (double)x); }
inline float fmul_legacy(float a, float b) { return a == 0.0f || b == 0.0f ? 0.0f : a * b; }
// D[i][j] += sum_k A[i][k] B[k][j] of 16 x 16 by 4 contractions: a lane holds row (column) lane % 16, k = lane / 16, and of D column lane % 16, rows 4 (lane / 16) + e
inline emu_f32x4 emu_mfma16f(float a, float b, emu_f32x4 c)
{
    struct Two { float a, b; };
    Two *s = emu::Exchange<Two>::all(Two{a, b});
    const int l = emu::lane();
    for (int e = 0; e < 4; ++e)
        for (int k = 0; k < 4; ++k) c[e] += s[4 * (l / 16) + e + 16 * k].a * s[l % 16 + 16 * k].b;
    emu::Exchange<Two>::release();
    return c;
}
#undef __builtin_amdgcn_mfma_f32_16x16x4f32
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) emu_mfma16f(a, b, c)
// STL_LAUNCHES: a file that takes the sizes of launches, whose kernels do not run
template <class F>
inline void seq_launch(const char *name, const void *kern, dim3 grid, dim3 block, size_t smem, F f)
{
    const char *to = getenv("STL_LAUNCHES");
    if (!to) return emu::launch(name, kern, grid, block, smem, f);
    FILE *out = fopen(to, "a");
    fprintf(out, "%u %u %u %u %s\n", grid.x, grid.y, grid.z, block.x, name);
    fclose(out);
}
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kern, grid, block, smem, stream, ...) seq_launch(#kern, (const void *)(kern), grid, block, (size_t)(smem), [&]() { kern(__VA_ARGS__); })
