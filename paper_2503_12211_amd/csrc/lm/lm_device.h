// Device helpers of the residual step and the vocabulary loss (gfx950 only).
#pragma once
#include "../stl_device.h"

namespace stl {
namespace lm {

// Sum (maximum) over the 64 lanes of a wavefront: four DPP steps leave each row of 16 lanes with its own in every lane, two more take rows 0 and 2, then
// row 1, into the rows above; the last lane has it all.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float v, float old)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(old), (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63)); }
__device__ __forceinline__ float wave_sum_last(float v)          // in lane 63
{
    v += dpp<0xb1, 0xf>(v, 0.f);       // quad_perm 1 0 3 2
    v += dpp<0x4e, 0xf>(v, 0.f);       // quad_perm 2 3 0 1
    v += dpp<0x141, 0xf>(v, 0.f);      // row_half_mirror
    v += dpp<0x140, 0xf>(v, 0.f);      // row_mirror
    v += dpp<0x142, 0xa>(v, 0.f);      // row_bcast 15
    v += dpp<0x143, 0xc>(v, 0.f);      // row_bcast 31
    return v;
}
__device__ __forceinline__ float wave_sum(float v) { return last_lane(wave_sum_last(v)); }
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, dpp<0xb1, 0xf>(v, v));
    v = fmaxf(v, dpp<0x4e, 0xf>(v, v));
    v = fmaxf(v, dpp<0x141, 0xf>(v, v));
    v = fmaxf(v, dpp<0x140, 0xf>(v, v));
    v = fmaxf(v, dpp<0x142, 0xa>(v, v));
    v = fmaxf(v, dpp<0x143, 0xc>(v, v));
    return last_lane(v);
}

// Eight consecutive elements of a row, held as loaded; `left` of them (or fewer) are in the row, the others are zeros.  Rows start at
// any element: gfx950 loads and stores 16 bytes at any address, and the last, incomplete chunk of a row goes element by element.
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
    u32x4_t v;
    __device__ __forceinline__ void fill(float f)
    {
        const uint32_t w = pack_bf16x2(f, f);
        v = u32x4_t{w, w, w, w};
    }
    __device__ __forceinline__ void load(const bf16_t *p, int left)
    {
        if (left >= 8) {
            v = *reinterpret_cast<const u32x4_any_t *>(p);
        } else {
            v = u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) v[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
        }
    }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
    // an opaque value from here on: what is computed from it is not kept over the turns of a loop
    __device__ __forceinline__ void opaque() { asm volatile("" : "+v"(v)); }
    static __device__ __forceinline__ void store(bf16_t *p, int left, const float *f)
    {
        const u32x4_t w = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
        if (left >= 8) {
            *reinterpret_cast<u32x4_any_t *>(p) = w;
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) p[e] = (bf16_t)(w[e >> 1] >> (16 * (e & 1)));
        }
    }
};
template <> struct Chunk<float> {
    f32x4_t a, b;
    __device__ __forceinline__ void fill(float f) { a = b = f32x4_t{f, f, f, f}; }
    __device__ __forceinline__ void load(const float *p, int left)
    {
        if (left >= 8) {
            a = *reinterpret_cast<const f32x4_any_t *>(p);
            b = *reinterpret_cast<const f32x4_any_t *>(p + 4);
        } else {
            a = b = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) (e < 4 ? a : b)[e & 3] = p[e];
        }
    }
    __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
    __device__ __forceinline__ void opaque() {}
    static __device__ __forceinline__ void store(float *p, int left, const float *f)
    {
        if (left >= 8) {
            *reinterpret_cast<f32x4_any_t *>(p) = f32x4_t{f[0], f[1], f[2], f[3]};
            *reinterpret_cast<f32x4_any_t *>(p + 4) = f32x4_t{f[4], f[5], f[6], f[7]};
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) p[e] = f[e];
        }
    }
};

}  // namespace lm
}  // namespace stl
