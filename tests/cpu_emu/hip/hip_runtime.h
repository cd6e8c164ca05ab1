// Host stand-in for <hip/hip_runtime.h> that runs kernels as they are meant to run, test infrastructure only (tests/test_cpu_lm.py): the threads of
// a workgroup are fibers that meet at barriers, the lanes of a wavefront meet at cross-lane operations, and matrix-core products, transposing LDS
// reads and LDS-DMA loads do what the instructions do.  So results can be compared with the oracle, and AddressSanitizer sees every access of
// the real index arithmetic, also where addresses depend on data.  Workgroups run one after the other.
#pragma once
#include <sys/mman.h>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <map>
#include <utility>
#include <vector>
#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __shared__ static
#define __launch_bounds__(...)
#define __align__(n) __attribute__((aligned(n)))
struct dim3 { unsigned x, y, z; dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {} };
inline dim3 threadIdx, blockIdx, blockDim, gridDim;
typedef int hipError_t;
typedef void *hipStream_t;
constexpr hipError_t hipSuccess = 0, hipErrorInvalidValue = 1;
enum { hipFuncAttributeMaxDynamicSharedMemorySize = 0, hipDeviceAttributeMultiprocessorCount = 1 };
inline hipError_t hipGetLastError() { return 0; }
inline const char *hipGetErrorString(hipError_t) { return "cpu"; }
inline std::map<const void *, int> g_lds_granted;
inline hipError_t hipFuncSetAttribute(const void *f, int, int bytes) { g_lds_granted[f] = bytes; return 0; }
inline hipError_t hipGetDevice(int *d) { *d = 0; return 0; }
inline hipError_t hipDeviceGetAttribute(int *v, int, int) { *v = 24; return 0; }      // few CUs: persistent kernels walk over several blocks each
#define HIP_SYMBOL(x) (&(x))
inline hipError_t hipGetSymbolAddress(void **p, const void *sym) { *p = const_cast<void *>(sym); return 0; }

// ---- fibers --------------------------------------------------------------------------------------------------------------------
extern "C" void emu_switch(void **from, void *to);
namespace emu {
enum State { ready, at_wave, at_barrier, done };
struct Fiber { void *sp; char *stack; State state; dim3 tid; };
inline std::vector<Fiber> fibers;
inline void *main_sp;
inline int current = -1, live_threads = 0;
inline std::function<void()> body;
inline size_t dyn_lds = 0;
inline char *dyn_lds_ptr = nullptr;
inline const char *kernel = "";
constexpr size_t kStack = 128 * 1024;
[[noreturn]] inline void die(const char *why)
{
    fprintf(stderr, "runtime error: %s in %s, block (%u,%u), thread %u\n", why, kernel, blockIdx.x, blockIdx.y, threadIdx.x);
    abort();
}
inline void yield(State s)
{
    Fiber &f = fibers[current];
    f.state = s;
    emu_switch(&f.sp, main_sp);
    threadIdx = fibers[current].tid;
}
inline void entry()
{
    threadIdx = fibers[current].tid;
    body();
    Fiber &f = fibers[current];
    f.state = done;
    emu_switch(&f.sp, main_sp);
    die("a finished thread was resumed");
}
inline void prepare(Fiber &f)
{
    if (!f.stack) f.stack = (char *)mmap(nullptr, kStack, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
    void **sp = (void **)(f.stack + kStack - 64);
    *--sp = nullptr;                       // return address of entry: never used
    *--sp = (void *)&entry;
    for (int i = 0; i < 6; ++i) *--sp = nullptr;
    f.sp = sp;
    f.state = ready;
}
inline void run_block(dim3 block)
{
    const int n = (int)(block.x * block.y * block.z), waves = (n + 63) / 64;
    if ((int)fibers.size() < n) fibers.resize(n, Fiber{nullptr, nullptr, done, dim3()});
    for (int i = 0; i < n; ++i) {
        prepare(fibers[i]);
        fibers[i].tid = dim3(i % block.x, i / block.x % block.y, i / (block.x * block.y));
    }
    for (;;) {
        int finished = 0, waiting = 0;
        for (int w = 0; w < waves; ++w) {
            const int lo = w * 64, hi = lo + 64 < n ? lo + 64 : n;
            for (;;) {
                for (int i = lo; i < hi; ++i)
                    if (fibers[i].state == ready) {
                        current = i;
                        emu_switch(&main_sp, fibers[i].sp);
                    }
                int meet = 0, rest = 0;
                for (int i = lo; i < hi; ++i) {
                    meet += fibers[i].state == at_wave;
                    rest += fibers[i].state != at_wave;
                }
                if (!meet) break;
                if (rest) die("a cross-lane operation that not all lanes reach");
                for (int i = lo; i < hi; ++i) fibers[i].state = ready;
            }
            for (int i = lo; i < hi; ++i) {
                finished += fibers[i].state == done;
                waiting += fibers[i].state == at_barrier;
            }
        }
        if (finished == n) return;
        if (waiting != n) die("a barrier that not all threads reach");
        for (int i = 0; i < n; ++i) fibers[i].state = ready;
    }
}
// values of the 64 lanes of the calling wavefront
template <class T>
struct Exchange {
    static inline T slot[1024];
    static T *all(const T &mine)
    {
        slot[current] = mine;
        yield(at_wave);
        return slot + current / 64 * 64;
    }
    static void release() { yield(at_wave); }
};
inline int lane() { return current & 63; }
template <class T, class F>
T from_lane(T v, F &&which)
{
    T *s = Exchange<T>::all(v);
    const T got = s[which(lane())];
    Exchange<T>::release();
    return got;
}
template <class F>
inline void launch(const char *name, const void *kern, dim3 grid, dim3 block, size_t smem, F f)
{
    kernel = name;
    const unsigned long threads = (unsigned long)block.x * block.y * block.z;
    if (smem > 160 * 1024 || threads > 1024 || threads == 0 || grid.x > 0x7fffffffu || grid.y > 65535u || grid.z > 65535u || !grid.x || !grid.y || !grid.z)
        die("launch outside device limits");
    if (smem > 64 * 1024 && g_lds_granted[kern] < (int)smem) die("dynamic LDS not granted");
    // LDS in the low 4 GB (its addresses are 32-bit in the kernels), 64 KB aligned, ending where a page without access begins
    static char *arena = nullptr;
    if (!arena) {
        char *p = (char *)mmap(nullptr, 1 << 20, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_32BIT, -1, 0);
        if (p == MAP_FAILED) die("no memory below 4 GB");
        arena = (char *)(((uintptr_t)p + 65535) & ~(uintptr_t)65535);
    }
    mprotect(arena, 512 * 1024, PROT_NONE);
    const size_t pages = (smem + 4095) / 4096 * 4096;
    if (pages) mprotect(arena, pages, PROT_READ | PROT_WRITE);
    memset(arena, 0x7f, pages);
    dyn_lds = smem;
    dyn_lds_ptr = arena;
    gridDim = grid;
    blockDim = block;
    body = f;
    for (unsigned z = 0; z < grid.z; ++z)
        for (unsigned y = 0; y < grid.y; ++y)
            for (unsigned x = 0; x < grid.x; ++x) {
                blockIdx = dim3(x, y, z);
                run_block(block);
            }
}
}  // namespace emu
#define hipLaunchKernelGGL(kern, grid, block, smem, stream, ...) emu::launch(#kern, (const void *)(kern), grid, block, (size_t)(smem), [&]() { kern(__VA_ARGS__); })
inline void __syncthreads() { emu::yield(emu::at_barrier); }
inline void emu_barrier() { emu::yield(emu::at_barrier); }
inline void emu_wave() { emu::yield(emu::at_wave); }
inline char *cpu_dyn_lds_ptr() { return emu::dyn_lds_ptr; }
inline float __uint_as_float(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
inline uint32_t __float_as_uint(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
inline float rsqrtf(float x) { return 1.0f / sqrtf(x); }
typedef unsigned short emu_u16x2 __attribute__((ext_vector_type(2)));
inline emu_u16x2 emu_pknorm(float a, float b)
{
    auto one = [](float x) { return (unsigned short)(x >= 1.0f ? 65535 : x > 0.0f ? (int)nearbyintf(x * 65535.0f) : 0); };
    return emu_u16x2{one(a), one(b)};
}
#define __builtin_amdgcn_cvt_pknorm_u16(a, b) emu_pknorm(a, b)
// uniform by construction where the kernels use it
#define __builtin_amdgcn_readfirstlane(x) (x)
#define __builtin_amdgcn_sched_barrier(x) ((void)0)
#define __builtin_amdgcn_sched_group_barrier(a, b, c) ((void)0)
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
inline float __shfl_xor(float v, int m) { return emu::from_lane(v, [&](int l) { return l ^ m; }); }
inline int __shfl_up(int v, int n) { return emu::from_lane(v, [&](int l) { return l < n ? l : l - n; }); }
inline int __builtin_amdgcn_readlane_emu(int v, int from) { return emu::from_lane(v, [&](int) { return from; }); }
#define __builtin_amdgcn_readlane(v, l) __builtin_amdgcn_readlane_emu(v, l)
inline int emu_dpp(int old, int v, int ctrl, int rows)
{
    const int got = emu::from_lane(v, [&](int l) {
        if (ctrl < 0x100) return (l & ~3) | (ctrl >> (2 * (l & 3)) & 3);      // quad_perm
        if (ctrl == 0x141) return (l & ~7) | (7 - (l & 7));                   // row_half_mirror
        if (ctrl == 0x140) return (l & ~15) | (15 - (l & 15));                // row_mirror
        if (ctrl == 0x142) return l < 16 ? l : (l & ~15) - 1;                 // row_bcast 15
        if (ctrl == 0x143) return l < 32 ? l : 31;                            // row_bcast 31
        emu::die("a DPP control that is not known here");
    });
    return rows >> (emu::lane() / 16) & 1 ? got : old;
}
#define __builtin_amdgcn_update_dpp(old, v, ctrl, rows, banks, bound) emu_dpp(old, v, ctrl, rows)
typedef __bf16 emu_bf16x8 __attribute__((ext_vector_type(8)));
typedef float emu_f32x4 __attribute__((ext_vector_type(4)));
typedef float emu_f32x16 __attribute__((ext_vector_type(16)));
struct EmuBits8 { uint16_t v[8]; };
inline float emu_bf16(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
// D[i][j] += sum_k A[i][k] B[k][j]: a lane holds row (column) lane % 16, k = 8 (lane / 16) ..., and of D column lane % 16, rows 4 (lane / 16) ...
inline emu_f32x4 emu_mfma16(emu_bf16x8 a, emu_bf16x8 b, emu_f32x4 c)
{
    struct Two { EmuBits8 a, b; } mine;
    memcpy(&mine.a, &a, 16);
    memcpy(&mine.b, &b, 16);
    Two *s = emu::Exchange<Two>::all(mine);
    const int l = emu::lane();
    for (int e = 0; e < 4; ++e) {
        const int i = 4 * (l / 16) + e, j = l % 16;
        float t = c[e];
        for (int k = 0; k < 32; ++k) t += emu_bf16(s[i + 16 * (k / 8)].a.v[k % 8]) * emu_bf16(s[j + 16 * (k / 8)].b.v[k % 8]);
        c[e] = t;
    }
    emu::Exchange<Two>::release();
    return c;
}
inline emu_f32x16 emu_mfma32f(float a, float b, emu_f32x16 c)
{
    struct Two { float a, b; };
    Two *s = emu::Exchange<Two>::all(Two{a, b});
    const int l = emu::lane();
    for (int e = 0; e < 16; ++e) {
        const int i = 8 * (e >> 2) + 4 * (l / 32) + (e & 3), j = l % 32;
        for (int k = 0; k < 2; ++k) c[e] += s[i + 32 * k].a * s[j + 32 * k].b;
    }
    emu::Exchange<Two>::release();
    return c;
}
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) emu_mfma16(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, x, y, z) emu_mfma32f(a, b, c)
// not in the kernels that are run here
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) (c)
typedef short emu_v4i16 __attribute__((ext_vector_type(4)));
// sixteen lanes give the addresses of four rows of 16 elements, four lanes a row; lane i gets element i of the four rows
template <class P>
inline emu_v4i16 emu_read_tr(P p)
{
    struct Four { uint16_t v[4]; } mine;
    const char *at = (const char *)(uintptr_t)(uint32_t)(uintptr_t)p;
    if (at < emu::dyn_lds_ptr || at + 8 > emu::dyn_lds_ptr + emu::dyn_lds) emu::die("a transposing read outside LDS");
    memcpy(&mine, at, 8);
    Four *s = emu::Exchange<Four>::all(mine);
    const int l = emu::lane(), g = l & ~15, i = l & 15;
    emu_v4i16 r;
    for (int j = 0; j < 4; ++j) r[j] = (short)s[g + 4 * j + (i >> 2)].v[i & 3];
    emu::Exchange<Four>::release();
    return r;
}
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) emu_read_tr(p)
// LDS-DMA load: lane L's 16 bytes land at byte lds + 16 L of the dynamic LDS
inline void cpu_touch16(const void *g, uint32_t lds)
{
    const size_t to = lds + 16 * (size_t)emu::lane();
    if ((uintptr_t)g & 15) emu::die("an LDS-DMA source that is not 16-byte aligned");
    if ((lds & 15) || to + 16 > emu::dyn_lds) emu::die("an LDS-DMA destination outside LDS");
    uint64_t v[2] = {((const uint64_t *)g)[0], ((const uint64_t *)g)[1]};
    memcpy(emu::dyn_lds_ptr + to, v, 16);
}
#define __HIP_MEMORY_SCOPE_AGENT 0
#define __hip_atomic_load(p, order, scope) (0xffffffffu)
#define __hip_atomic_fetch_add(p, v, order, scope) (*(p) += (v), *(p) - (v))
#define __hip_atomic_fetch_or(p, v, order, scope) (*(p) |= (v))
#define __builtin_amdgcn_fence(order, scope) ((void)0)
#define __builtin_amdgcn_s_sleep(n) ((void)0)
