// Matrix products of the vocabulary loss in fp32 storage, on the fp32 matrix cores (v_mfma_f32_32x32x2_f32):
//     Out[i][j] (+)= sum_l A(i, l) B(l, j),   A stored [i][l] or [l][i], B stored [j][l] or [l][j], any sizes.
//
// What bounds it: the matrix cores, 64 cycles a product of 32 x 32 x 2 (157 TFLOP/s at 2.4 GHz).  A workgroup has a block of 64 x 64 outputs, a quarter
// for each of four wavefronts; where there are fewer than two blocks a CU, two or four groups of four wavefronts share a block's contraction,
// each with every second or fourth stage, and add their sums up in LDS.  (Blocks of 32 x 32 as in ../stl_gemm_generic.hip move twice the
// bytes through LDS; 2048 rows of 768, 1000 classes, us of the three products under the profiler: 80, 64 and 62 there, 52, 64 and 68 here, the
// whole call 192 and 153.  The matrix cores are busy for 60, 61 and 59 % of the time that CUs have wavefronts, and for 45, 39 and 37 % of the three launches:
// 512, 384 and 192 equal blocks on 256 CUs.)  A stage holds 32 elements
// of the contraction; the next two's are on their way through registers while it is multiplied, into the other half of LDS.  Operands keep their orientation in LDS,
// with rows padded so that a fragment's lanes fall on all banks: [row][l] 36 floats (a lane reads four l at once, one for each of four
// products), [l][row] 72.
#include "lm_kernels.h"
#include "lm_device.h"

namespace stl {
namespace lm {
namespace f32 {

constexpr int BT = 64, BK = 32, LD_ROW = BK + 4, LD_L = BT + 8, TILE = BT * LD_ROW;        // floats; BK * LD_L is as many
static_assert(BK * LD_L == TILE, "one size of LDS tile");

struct Operand {
    const float *p;
    long ld;
    int rows;                // i or j
    bool along;              // rows of l
};

// a stage of one operand on its way through registers: 64 x 32 floats, two pieces of four for each of 256 threads
struct Staged {
    f32x4_t v[2];
    __device__ __forceinline__ void load(const Operand &o, int r0, int l0, int L, int t)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int q = t + 256 * k;
            if (o.along) {
                const int row = r0 + (q >> 3), l = l0 + 4 * (q & 7);
                v[k] = row < o.rows && l < L ? load4<float>(o.p + row * o.ld + l, L - l) : f32x4_t{0.f, 0.f, 0.f, 0.f};
            } else {
                const int l = l0 + (q >> 4), row = r0 + 4 * (q & 15);
                v[k] = l < L && row < o.rows ? load4<float>(o.p + l * o.ld + row, o.rows - row) : f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
        }
    }
    __device__ __forceinline__ void put(float *tile, bool along, int t) const
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int q = t + 256 * k;
            *reinterpret_cast<f32x4_t *>(tile + (along ? (q >> 3) * LD_ROW + 4 * (q & 7) : (q >> 4) * LD_L + 4 * (q & 15))) = v[k];
        }
    }
};

// four products' values of a lane: row `row` of the tile, l = l0 .. l0 + 3
template <bool ALONG>
__device__ __forceinline__ f32x4_t fragment(const float *tile, int row, int l0)
{
    if constexpr (ALONG) {
        return *reinterpret_cast<const f32x4_t *>(tile + row * LD_ROW + l0);
    } else {
        f32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = tile[(l0 + e) * LD_L + row];
        return v;
    }
}

template <int GROUPS, bool A_ALONG, bool B_ALONG, bool ACC>
__global__ __launch_bounds__(256 * GROUPS) void gemm_f32_kernel(Operand a, Operand b, int L, float *out, int tiles_m, int tiles_n, int tiles)
{
    extern __shared__ __align__(16) char smem[];
    const int t = (int)threadIdx.x & 255, group = (int)threadIdx.x >> 8, lane = t & 63, wave = t >> 6;
    // each XCD takes a contiguous eighth of the blocks
    const int v = (int)((long)(blockIdx.x & 7) * tiles / 8) + (int)(blockIdx.x >> 3);
    if (v >= (int)((long)((blockIdx.x & 7) + 1) * tiles / 8)) return;
    // down the columns of eight block rows first: the 128 blocks that an XCD has at a time share 8 rows of one operand and 16 columns of the other
    const int per = 8 * tiles_n, q = v / per, rem = v - q * per, in_group = tiles_m - 8 * q < 8 ? tiles_m - 8 * q : 8;
    const int i0 = (8 * q + rem % in_group) * BT, j0 = rem / in_group * BT, wi = wave >> 1 << 5, wj = (wave & 1) << 5;
    a.along = A_ALONG, b.along = B_ALONG;
    float *mine = reinterpret_cast<float *>(smem) + group * 4 * TILE;
    f32x16_t acc = {};
    const int all = (L + BK - 1) / BK, s0 = (int)((long)all * blockIdx.y / gridDim.y), stages = (int)((long)all * (blockIdx.y + 1) / gridDim.y) - s0;
    const int turns = (stages + GROUPS - 1) / GROUPS;
    if (s0 + stages < all) L = (s0 + stages) * BK;
    out += (size_t)blockIdx.y * a.rows * b.rows;
    Staged sa[2], sb[2];
    auto load = [&](int s, int k) {
        if (s < turns) {
            sa[k].load(a, i0, (s0 + s * GROUPS + group) * BK, L, t);
            sb[k].load(b, j0, (s0 + s * GROUPS + group) * BK, L, t);
        }
    };
    auto turn = [&](int s, auto k_c) {
        constexpr int k = decltype(k_c)::value;
        float *ta = mine + k * 2 * TILE, *tb = ta + TILE;
        sa[k].put(ta, A_ALONG, t);
        sb[k].put(tb, B_ALONG, t);
        // (a half is written again two turns later, behind the next turn's barrier, which all reach after they have read it)
        __syncthreads();
        load(s + 2, k);
#pragma unroll
        for (int l = 0; l < BK; l += 8) {
            const f32x4_t fa = fragment<A_ALONG>(ta, wi + (lane & 31), l + 4 * (lane >> 5)), fb = fragment<B_ALONG>(tb, wj + (lane & 31), l + 4 * (lane >> 5));
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[e], fb[e], acc, 0, 0, 0);
        }
    };
    load(0, 0);
    load(1, 1);
    for (int s = 0; s < turns; s += 2) {
        turn(s, std::integral_constant<int, 0>{});
        if (s + 1 < turns) turn(s + 1, std::integral_constant<int, 1>{});
    }
    if constexpr (GROUPS > 1) {
        __syncthreads();
        float *sums = reinterpret_cast<float *>(smem);       // [group - 1][wave][16][64]
        if (group > 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[(((group - 1) * 4 + wave) * 16 + e) * 64 + lane] = acc[e];
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] += sums[((g * 4 + wave) * 16 + e) * 64 + lane];
    }
    const int j = j0 + wj + (lane & 31);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int i = i0 + wi + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
        if (i < a.rows && j < b.rows) {
            float *o = out + (size_t)i * b.rows + j;
            *o = ACC ? *o + acc[e] : acc[e];
        }
    }
}

template <int GROUPS, bool A_ALONG, bool B_ALONG, bool ACC>
hipError_t launch_as(const Operand &a, const Operand &b, int L, float *out, int tiles_m, int tiles_n, int tiles, int splits, hipStream_t s)
{
    auto kern = gemm_f32_kernel<GROUPS, A_ALONG, B_ALONG, ACC>;
    constexpr int lds = GROUPS * 4 * TILE * (int)sizeof(float);
    static std::atomic<uint64_t> granted{0};                 // of this instantiation
    if (const hipError_t e = allow_lds(reinterpret_cast<const void *>(kern), lds, lds, granted); e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((tiles + 7) / 8 * 8, splits), dim3(256 * GROUPS), lds, s, a, b, L, out, tiles_m, tiles_n, tiles);
    return hipGetLastError();
}

}  // namespace f32

int gemm_f32_splits(int I, int J, int L)
{
    using namespace f32;
    const long tiles = (long)((I + BT - 1) / BT) * ((J + BT - 1) / BT);
    const int stages = (L + BK - 1) / BK;
    long n = tiles >= 512 ? 1 : 512 / tiles;
    if (n > stages / 32) n = stages / 32;
    return n > 16 ? 16 : n < 1 ? 1 : (int)n;
}

hipError_t launch_gemm_f32(const GemmF32 &g, hipStream_t s)
{
    using namespace f32;
    const Operand a{g.A, g.a_along ? g.L : g.I, g.I, g.a_along}, b{g.B, g.b_along ? g.L : g.J, g.J, g.b_along};
    const long tiles_m = (g.I + BT - 1) / BT, tiles_n = (g.J + BT - 1) / BT, tiles = tiles_m * tiles_n;
    if (tiles > (1L << 30)) return hipErrorInvalidValue;
    const int stages = (g.L + BK - 1) / BK / g.splits;
    auto run = [&](auto groups_c) {
        constexpr int G = decltype(groups_c)::value;
        if (g.a_along && !g.b_along) return launch_as<G, true, false, false>(a, b, g.L, g.Out, (int)tiles_m, (int)tiles_n, (int)tiles, g.splits, s);
        if (g.a_along) return launch_as<G, true, true, false>(a, b, g.L, g.Out, (int)tiles_m, (int)tiles_n, (int)tiles, g.splits, s);
        return g.accumulate ? launch_as<G, false, false, true>(a, b, g.L, g.Out, (int)tiles_m, (int)tiles_n, (int)tiles, g.splits, s)
                            : launch_as<G, false, false, false>(a, b, g.L, g.Out, (int)tiles_m, (int)tiles_n, (int)tiles, g.splits, s);
    };
    if ((!g.a_along && g.b_along) || (g.accumulate && g.a_along)) return hipErrorInvalidValue;         // forms that no product here has
    // as many groups as make two blocks' worth of wavefronts a CU, where each has two stages at least
    if (tiles * g.splits < 256 && stages >= 8) return run(std::integral_constant<int, 4>{});
    if (tiles * g.splits < 512 && stages >= 4) return run(std::integral_constant<int, 2>{});
    return run(std::integral_constant<int, 1>{});
}

}  // namespace lm
}  // namespace stl
