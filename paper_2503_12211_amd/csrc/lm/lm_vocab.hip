// Vocabulary loss: the matrix products of bf16 storage on the matrix cores, and the order of launches for both storage types.
//
// Rows with a term are listed on the device and taken in chunks; the logits of a chunk are never in memory as such.  bf16 storage:
//   1. logits product  X W^T: every wavefront turns its 64 columns of a row into their maximum and the sum of their exponentials, and (for
//      gradients) writes the logits as 16-bit steps below that maximum;
//   2. a pass over the rows gives the losses and writes the bf16 gradient dz over the steps (lm_vocab_rows.hip);
//   3. dX = dz W, contraction over the vocabulary, split where there are few blocks;  4. dW = dz^T X, contraction over the rows.
// Three products of 2 T V d operations, where forming the logits twice would take four; what bounds them is the matrix cores (lm_gemm.h).
// fp32 storage: the same steps on the fp32 products of lm_f32.hip, the chunk's logits in fp32.
#include "lm_gemm.h"
#include "lm_kernels.h"
#include "lm_device.h"

namespace stl {
namespace lm {

// ---- logits ------------------------------------------------------------------------------------------------------------------------
struct LogitsOut {
    GroupSums *sums;
    int groups;
    uint16_t *codes;
    long ld;
    float scale;         // log2(e) over the temperature of the first sum: y = scale z
    float ratio;         // the first temperature over the second
    float deepest;       // below a group's maximum by this much in y, no share is left in fp32
    float bend;          // as much for the lower of two temperatures (kSteps)
};

// From a group's largest y and its spread to its smallest: what a step is, and what takes y to [0, 1] for the conversion to 16 bits, in which 1
// is 65535.  The smallest y comes to lie on 65534.  (The order of the bounds makes any spread that is not a number a finite one.)
// TWO: of two lines the lower one is taken, the second of which has the steps below the bend; without a bend they are the same.
template <bool TWO>
struct Steps {
    float size, mul, add, mul2, add2;
    __device__ __forceinline__ Steps(float ref, float spread, const LogitsOut &out)
    {
        const float deep = fminf(fmaxf(spread, 1e-3f), out.deepest);
        const bool bent = TWO && deep > 2.f * out.bend;
        const float whole = bent ? out.bend * (kSteps / kBendSteps) : deep * (kSteps / (kSteps - 1.f));
        size = whole * (1.f / kSteps);
        mul = -__builtin_amdgcn_rcpf(whole);                 // (an error of 1e-7 of it is 0.007 steps at the far end)
        add = -ref * mul;
        if constexpr (TWO) {
            const float below = (deep - out.bend) * (kSteps / kBendSteps);
            mul2 = bent ? -__builtin_amdgcn_rcpf(below) : mul;
            add2 = bent ? fmaf(out.bend - ref, mul2, kBendSteps / kSteps) : add;
            if (bent) size = -below * (1.f / kSteps);
        }
    }
    __device__ __forceinline__ float at(float y) const
    {
        const float t = fmaf(y, mul, add);
        if constexpr (TWO) return fminf(t, fmaf(y, mul2, add2));
        return t;
    }
    __device__ __forceinline__ uint32_t codes(float y0, float y1) const { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pknorm_u16(at(y0), at(y1))); }
};

typedef Ring<256, 256, 2, 4, 4, false, false, false> LogitsFull;
typedef Ring<128, 256, 2, 4, 5, false, false, false> LogitsHalf;
static_assert(LogitsFull::WN == 64 && LogitsHalf::WN == 64, "a wavefront's columns are one group");
static_assert(LogitsHalf::SLABS_AT <= LogitsFull::SLABS_AT && LogitsHalf::LDS_BYTES <= LogitsFull::LDS_BYTES, "LDS of walk_list");

// What a wavefront makes of its 16 FM x 64 products: the group's sums for every row, and the codes.  WHOLE: all columns are in the vocabulary.
// A lane has the columns col0 + 16 b + 4 (lane / 16) + e of the rows row0 + 16 a + lane % 16.
template <int FM, bool CODES, bool TWO, bool WHOLE>
__device__ __forceinline__ void logits_out(pipe::acc4_t (&acc)[FM][4], int row0, int col0, int rows, int vocab, char *slab, int lane, const LogitsOut &out)
{
    // no contraction of y's product with what follows it: the losses have the same bits with and without gradients
#pragma clang fp contract(off)
    using pipe::static_for;
    constexpr int PA = 2;                                    // fragment rows that the slab holds: 16 rows of 128 bytes each
    int el = lane;                                           // opaque: what follows from it is not kept over the products
    asm volatile("" : "+v"(el));
    const int quad = el >> 4, rl = el & 15, col = col0 + 4 * quad, group = col0 / 64;
    static_for<0, FM / PA>([&](auto pass_c) {
        constexpr int a0 = decltype(pass_c)::value * PA;
        static_for<0, PA>([&](auto a_c) {
            constexpr int a = a0 + decltype(a_c)::value;
            // (scaled first: of products the compiler knows that they are in canonical form, into which it has to bring every operand of a maximum
            // that may not be)
            float y[16], m = -INFINITY, least = INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                y[i] = acc[a][i / 4][i % 4] * out.scale;
                if constexpr (!WHOLE) {
                    const bool in = col + 16 * (i / 4) + i % 4 < vocab;
                    if constexpr (CODES) least = fminf(least, in ? y[i] : INFINITY);
                    y[i] = in ? y[i] : -INFINITY;
                } else if constexpr (CODES) {
                    least = fminf(least, y[i]);
                }
                m = fmaxf(m, y[i]);
            }
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            if constexpr (CODES) {
                least = fminf(least, __shfl_xor(least, 16));
                least = fminf(least, __shfl_xor(least, 32));
            }
            // a group of nothing but minus infinities: 2^(-inf - 0), not 2^(-inf + inf)
            const float ref = m == -INFINITY ? 0.f : m;
            float s = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float below = y[i] - ref;
                s += __builtin_amdgcn_exp2f(below);
                if constexpr (TWO) s2 += __builtin_amdgcn_exp2f(below * out.ratio);
            }
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if constexpr (TWO) {
                s2 += __shfl_xor(s2, 16);
                s2 += __shfl_xor(s2, 32);
            }
            const Steps<TWO> st(ref, ref - least, out);
            const int row = row0 + 16 * a + rl;
            if (quad == 0 && row < rows) out.sums[(size_t)row * out.groups + group] = GroupSums{m, s, s2, st.size};
            if constexpr (CODES) {
                char *rowp = slab + (16 * (a - a0) + rl) * 128;
                const int swz = (rl >> 1) & 7;
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<u32x2_t *>(rowp + (((2 * b + (quad >> 1)) ^ swz) << 4) + (quad & 1) * 8) =
                        u32x2_t{st.codes(y[4 * b], y[4 * b + 1]), st.codes(y[4 * b + 2], y[4 * b + 3])};
            }
        });
        if constexpr (CODES) {
            // rows leave as whole 128-byte lines; a wavefront's LDS operations execute in order
            asm volatile("" ::: "memory");
            const int rr = el >> 3, rc = el & 7;
#pragma unroll
            for (int i = 0; i < PA * 2; ++i) {
                const int row = i * 8 + rr, gi = row0 + a0 * 16 + row;
                const u32x4_t piece = *reinterpret_cast<const u32x4_t *>(slab + row * 128 + ((rc ^ ((row >> 1) & 7)) << 4));
                if (gi < rows) *reinterpret_cast<u32x4_t *>(out.codes + (size_t)gi * out.ld + col0 + rc * 8) = piece;
            }
            asm volatile("" ::: "memory");
        }
    });
}

// listed rows of the chunk: count - first, a device value, at most cap
template <bool CODES, bool TWO>
__global__ __launch_bounds__(512) void vocab_logits_kernel(const Operands o, const int *count, int first, int cap, int vocab, const LogitsOut out)
{
    using namespace pipe;
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t smem_lds = (uint32_t)(uintptr_t)STL_LDS(smem);
    int rows = *count - first;
    if (rows > cap) rows = cap;
    if (rows <= 0) return;
    const int tiles_m = (rows + 255) / 256, tiles_n = (vocab + 255) / 256, size = group_rows(tiles_m), nks = o.Kl / BKS;
    walk_list<LogitsFull, LogitsHalf>(
        tiles_m * tiles_n, rows, o, smem, smem_lds, wave, lane,
        [&](int v, Operands &, int &stages, int &i0, int &j0) {
            int bi, bj;
            block_at(v, tiles_m, tiles_n, size, bi, bj);
            stages = nks;
            i0 = bi * 256;
            j0 = bj * 256;
        },
        [&](auto &w, int, int i0, int j0) {
            constexpr int FM = sizeof(w.acc) / sizeof(w.acc[0]);
            char *slab = smem + (FM == LogitsFull::FM ? LogitsFull::SLABS_AT : LogitsHalf::SLABS_AT) + wave * LogitsFull::SLAB;
            const int row0 = i0 + wave / 4 * 16 * FM, col0 = j0 + wave % 4 * 64;
            if (col0 + 64 <= vocab) logits_out<FM, CODES, TWO, true>(w.acc, row0, col0, rows, vocab, slab, lane, out);
            else if (col0 < vocab) logits_out<FM, CODES, TWO, false>(w.acc, row0, col0, rows, vocab, slab, lane, out);
        });
}

// Few rows (at most 16 FM listed ones of the chunk): reading W once is the work, and how it is read decides.  Memory gives 512 MB in rows of 8 KB, of which
// a visit takes 64 (128, 256, 512, 1024) bytes side by side, at 4.1 (4.3, 4.7, 5.3, 6.0) TB/s, a plain loop 6.2; the LDS-DMA rings ask for 64 or 128.  So
// a workgroup has one group of 64 columns, that is 64 rows of W, and takes 1 KB (512 elements of the contraction) of each at a time, a wavefront's
// instruction a row: through registers, on the way while the stage before is multiplied, into LDS (two workgroups a CU: one multiplies while the
// other waits).  Each of the four wavefronts multiplies a quarter of a stage, X coming straight from L2 into fragments, and their sums meet in LDS,
// where a lane then has a column.  16 rows x 4096, vocabulary 65536 (537 MB): 97 us (5.5 TB/s), 128 in blocks of the LDS-DMA ring.
// LDS: row stride 1 KB, 16-byte chunk c of row r at c ^ (r & 15): the 16 rows of a fragment fall on all banks.
template <int FM, bool CODES, bool TWO>
__global__ __launch_bounds__(256, 2) void vocab_logits_few_kernel(const Operands o, const int *count, int first, int cap, int vocab, const LogitsOut out)
{
    constexpr int NW = 4, ROWS = 16 * FM, STAGE = 512, STEPS = STAGE / 32 / NW;      // a wavefront's steps of 32 elements in a stage
    __shared__ __align__(16) char tile[64 * 1024];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, kq = lane >> 4, col0 = (int)blockIdx.x * 64;
    int rows = *count - first;
    if (rows > cap) rows = cap;
    if (rows <= 0) return;
    const int stages = (o.Kl + STAGE - 1) / STAGE;
    u32x4_t rb[16], ra[STEPS][FM];
    f32x4_t acc[FM][4];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[f][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto fetch = [&](int s) {
        const int l0 = s * STAGE;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = col0 + 4 * i + wave, l = l0 + 8 * lane;          // rows behind the last feed columns that are masked below
            rb[i] = l < o.Kl ? *reinterpret_cast<const u32x4_t *>(o.B + (long)(row < vocab ? row : vocab - 1) * o.ldb + l) : u32x4_t{0u, 0u, 0u, 0u};
        }
    };
    fetch(0);
    for (int s = 0; s < stages; ++s) {
        // (X's fragments come from L2 while W's rows go into LDS)
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                const int l = s * STAGE + (STEPS * wave + k) * 32 + 8 * kq;
                ra[k][f] = l < o.Kl ? *reinterpret_cast<const u32x4_t *>(o.A + (long)(16 * f + n16) * o.lda + l) : u32x4_t{0u, 0u, 0u, 0u};
            }
        if (s > 0) __syncthreads();                          // all have read the stage before
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = 4 * i + wave;
            *reinterpret_cast<u32x4_t *>(tile + row * 1024 + ((lane ^ (row & 15)) << 4)) = rb[i];
        }
        __syncthreads();
        if (s + 1 < stages) fetch(s + 1);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int chunk = 4 * (STEPS * wave + k) + kq;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const bf16x8_t b = *reinterpret_cast<const bf16x8_t *>(tile + (16 * c + n16) * 1024 + ((chunk ^ n16) << 4));
#pragma unroll
                for (int f = 0; f < FM; ++f) acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ra[k][f]), b, acc[f][c], 0, 0, 0);
            }
        }
    }
    // accumulator e of fragment (f, c): row 16 f + 4 kq + e, column 16 c + n16
    __syncthreads();
    float *sums = reinterpret_cast<float *>(tile);           // [wavefront][row][64]
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(wave * ROWS + 16 * f + 4 * kq + e) * 64 + 16 * c + n16] = acc[f][c][e];
    __syncthreads();
    const bool in = col0 + lane < vocab;
    for (int r = wave; r < ROWS && r < rows; r += NW) {
#pragma clang fp contract(off)
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) y += sums[(w * ROWS + r) * 64 + lane];
        y = in ? y * out.scale : -INFINITY;
        const float m = wave_max(y), ref = m == -INFINITY ? 0.f : m, below = y - ref;
        const float s = wave_sum(__builtin_amdgcn_exp2f(below));
        float s2 = 0.f, spread = 0.f;
        if constexpr (TWO) s2 = wave_sum(__builtin_amdgcn_exp2f(below * out.ratio));
        if constexpr (CODES) spread = wave_max(in ? -below : 0.f);
        const Steps<TWO> st(ref, spread, out);
        if (lane == 0) {
            const size_t at = (size_t)r * out.groups + blockIdx.x;
            out.sums[at] = GroupSums{m, s, s2, st.size};
        }
        if constexpr (CODES) out.codes[(size_t)r * out.ld + col0 + lane] = (uint16_t)(st.codes(y, y) & 0xffffu);
    }
}

// ---- dX and dW -----------------------------------------------------------------------------------------------------------------------
// dX parts: part s, rows x ldx = dz (columns of split s) W.  The number of parts is left behind the count.
template <int BM, int WAVES_M, int WAVES_N, int NS>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64) void vocab_dx_kernel(const Operands o, int *count, int first, int cap, int d, int held, Splits sps, float *part, int ldx)
{
    using namespace pipe;
    typedef Ring<BM, 256, WAVES_M, WAVES_N, NS, false, true, true> R;
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char *slab = smem + NS * R::STAGE_BYTES + wave * R::SLAB;
    const uint32_t smem_lds = (uint32_t)(uintptr_t)STL_LDS(smem);
    int rows = *count - first;
    if (rows > cap) rows = cap;
    if (rows <= 0) return;
    if (const int second = second_row(*count, held)) rows = 2 * second;
    const int tiles_m = (rows + BM - 1) / BM, tiles_n = sps.tiles_n, size = group_rows(tiles_m), per = tiles_m * tiles_n, splits = sps.of(rows), total = per * splits, stages = sps.stages;
    const size_t stride = (size_t)rows * ldx;
    if (blockIdx.x == 0 && tid == 0) count[1] = splits;
    auto begin_of = [&](int sp) { return (int)((long)stages * sp / splits); };
    walk(R{}, first_block(total), end_block(total), block_step(), o, smem, smem_lds, wave, lane,
         [&](int v, Operands &mine, int &n, int &i0, int &j0) {
             const int sp = v / per, s0 = begin_of(sp), s1 = begin_of(sp + 1);
             int bi, bj;
             block_at(v - sp * per, tiles_m, tiles_n, size, bi, bj);
             mine.A += (long)s0 * BKS;
             mine.B += (long)s0 * BKS * o.ldb;
             mine.Kl = (o.Kl < s1 * BKS ? o.Kl : s1 * BKS) - s0 * BKS;
             n = s1 - s0;
             i0 = bi * BM;
             j0 = bj * 256;
         },
         [&](typename R::Tile &w, int v, int i0, int j0) {
             int el = lane;
             asm volatile("" : "+v"(el));
             w.template store<float, false, false>(slab, part + v / per * stride, i0 + wave / R::WAVES_N * R::WM, j0 + wave % R::WAVES_N * R::WN, rows, ldx, 0, 1 << 30, 1,
                                                   el);
         });
}

// dW = dz^T X over the listed rows of a chunk: straight to dW (bf16), or to parts in fp32, added to what is there behind the first chunk.
typedef Ring<256, 256, 2, 4, 4, true, true, false> DwFull;
typedef Ring<128, 256, 2, 4, 5, true, true, false> DwHalf;
static_assert(DwHalf::SLABS_AT <= DwFull::SLABS_AT && DwHalf::LDS_BYTES <= DwFull::LDS_BYTES, "LDS of walk_list");

template <typename TO, bool ACC>
__global__ __launch_bounds__(512) void vocab_dw_kernel(const Operands o, const int *count, const float *scale, int first, int cap, int held, int vocab, int splits, TO *out,
                                                       size_t stride, int ldo)
{
    using namespace pipe;
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t smem_lds = (uint32_t)(uintptr_t)STL_LDS(smem);
    int rows = *count - first;
    if (rows > cap) rows = cap;
    if (rows <= 0) {
        if (ACC) return;                                     // nothing to add
        rows = 0;
    } else if (const int second = second_row(*count, held)) {
        rows = 2 * second;
    }
    const int tiles_m = (vocab + 255) / 256, tiles_n = (ldo + 255) / 256, size = group_rows(tiles_m), per = tiles_m * tiles_n, stages = (rows + BKS - 1) / BKS;
    auto begin_of = [&](int sp) { return (int)((long)stages * sp / splits); };
    walk_list<DwFull, DwHalf>(
        per * splits, vocab, o, smem, smem_lds, wave, lane,
        [&](int v, Operands &mine, int &n, int &i0, int &j0) {
            const int sp = v / per, s0 = begin_of(sp);
            int bi, bj;
            block_at(v - sp * per, tiles_m, tiles_n, size, bi, bj);
            mine.A += (long)s0 * BKS * o.lda;
            mine.B += (long)s0 * BKS * o.ldb;
            n = begin_of(sp + 1) - s0;
            i0 = bi * 256;
            j0 = bj * 256;
        },
        [&](auto &w, int v, int i0, int j0) {
            constexpr int FM = sizeof(w.acc) / sizeof(w.acc[0]);
            char *slab = smem + (FM == DwFull::FM ? DwFull::SLABS_AT : DwHalf::SLABS_AT) + wave * DwFull::SLAB;
            int el = lane;
            asm volatile("" : "+v"(el));
            if constexpr (sizeof(TO) == 2) {
                const float factor = scale[1];
                static_for<0, FM>([&](auto a_c) {
                    static_for<0, 4>([&](auto b_c) { w.acc[decltype(a_c)::value][decltype(b_c)::value] *= factor; });
                });
            }
            w.template store<TO, ACC, false>(slab, out + v / per * stride, i0 + wave / 4 * 16 * FM, j0 + wave % 4 * 64, vocab, ldo, 0, 1 << 30, 1, el);
        });
}

// ---- launches ------------------------------------------------------------------------------------------------------------------------
template <class K, class... Args>
static hipError_t launch_ring(K kern, std::atomic<uint64_t> &granted, int lds, int threads, long blocks, hipStream_t s, Args... args)
{
    if (const hipError_t e = allow_lds(reinterpret_cast<const void *>(kern), lds, lds, granted); e != hipSuccess) return e;
    if (blocks > 0x7fffffffL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, dim3(pipe::list_grid(blocks, pipe::cu_count())), dim3(threads), lds, s, args...);
    return hipGetLastError();
}

template <bool CODES, bool TWO>
static hipError_t launch_logits_as(const Operands &o, const int *count, int first, int cap, int vocab, const LogitsOut &out, hipStream_t s)
{
    // Up to 32 rows are few: whole calls at 4096 x 65536, us, there / in blocks of 256 rows: 16 rows 109 / 149, 32 rows 116 / 149; 64 rows 166 / 149, for
    // whose fragments and sums there are not enough registers.
    auto few = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(out.groups), dim3(256), 0, s, o, count, first, cap, vocab, out);
        return hipGetLastError();
    };
    if (cap <= 16) return few(vocab_logits_few_kernel<1, CODES, TWO>);
    if (cap <= 32) return few(vocab_logits_few_kernel<2, CODES, TWO>);
    typedef LogitsFull R;
    static std::atomic<uint64_t> granted{0};                 // of this instantiation
    return launch_ring(vocab_logits_kernel<CODES, TWO>, granted, R::LDS_BYTES, R::THREADS, 2L * ((cap + 255) / 256) * ((vocab + 255) / 256), s, o, count, first, cap,
                       vocab, out);
}
static hipError_t launch_logits(const Operands &o, const int *count, int first, int cap, int vocab, const LogitsOut &out, bool two, hipStream_t s)
{
    if (out.codes) return two ? launch_logits_as<true, true>(o, count, first, cap, vocab, out, s) : launch_logits_as<true, false>(o, count, first, cap, vocab, out, s);
    return two ? launch_logits_as<false, true>(o, count, first, cap, vocab, out, s) : launch_logits_as<false, false>(o, count, first, cap, vocab, out, s);
}

template <int BM, int WAVES_M, int WAVES_N, int NS>
static hipError_t launch_dx(const Operands &o, int *count, int first, int cap, int d, int held, const Splits &sp, float *part, int ldx, hipStream_t s)
{
    typedef Ring<BM, 256, WAVES_M, WAVES_N, NS, false, true, true> R;
    static std::atomic<uint64_t> granted{0};
    return launch_ring(vocab_dx_kernel<BM, WAVES_M, WAVES_N, NS>, granted, R::LDS_BYTES, R::THREADS, pipe::cu_count(), s, o, count, first, cap, d, held, sp, part, ldx);
}

template <typename TO, bool ACC>
static hipError_t launch_dw(const Operands &o, const RowList &rl, int first, int cap, int held, int vocab, int splits, TO *out, size_t stride, int ldo, hipStream_t s)
{
    typedef DwFull R;
    static std::atomic<uint64_t> granted{0};
    return launch_ring(vocab_dw_kernel<TO, ACC>, granted, R::LDS_BYTES, R::THREADS, 2L * ((vocab + 255) / 256) * ((ldo + 255) / 256) * splits, s, o,
                       (const int *)rl.count, (const float *)rl.scale, first, cap, held, vocab, splits, out, stride, ldo);
}

// ---- the whole of a call -----------------------------------------------------------------------------------------------------------------
namespace {

inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
inline long round_up(long x, long to) { return (x + to - 1) / to * to; }

// How a call is cut, and where things lie in the workspace.
struct Plan {
    int cap;                 // listed rows of a chunk
    int chunks;
    int rows_held;           // rows that Xc has
    int ldx;                 // elements of a row of Xc (and of a packed W)
    bool pack_w;             // W's rows are copied to ldx elements each
    size_t ldz;              // elements of a row of the logits' codes / of the gradient in the logits
    int groups;
    bool small;              // blocks of 64 rows
    int held;                // rows that the chunk's buffers have for two numbers a row (second_row)
    Splits dx;
    int dw_splits;
    bool dw_parts;           // dW through fp32 parts
    size_t list, count, scale, xc, wp, sums, codes, dx_part, dw_part, dw_stride, total;
};

Plan plan_of(const VocabArgs &a, bool grads)
{
    Plan p{};
    const int cus = 256;     // of an MI355X; the workspace has to be the same on a machine without one
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round256(bytes);
        return here;
    };
    p.list = take((size_t)a.rows * sizeof(int));
    p.count = take(2 * sizeof(int));
    p.scale = take(2 * sizeof(float));
    if (a.bf16) {
        long cap = kChunkCodes / a.vocab / 256 * 256;
        cap = cap > kChunkMost ? kChunkMost : cap < kChunkLeast ? kChunkLeast : cap;
        p.cap = (int)(a.rows < cap ? a.rows : cap);
        p.chunks = (a.rows + p.cap - 1) / p.cap;
        // up to 64 rows, twice: blocks of 64 (64 x 64, vocabulary 109807: 97 us, 108 in blocks of 256; 64 x 4096, 65536: 505 and 508)
        p.small = p.cap <= 64;
        const int twice = grads ? 2 * whole_stages(p.cap < kPairRows ? p.cap : kPairRows) : 0, product_rows = p.cap > twice ? p.cap : twice;
        p.rows_held = (int)round_up(product_rows, p.small ? 64 : 256);
        p.held = grads ? p.rows_held : 0;
        p.ldx = (int)round_up(a.d, pipe::BKS);                 // whole stages of the products
        p.pack_w = p.ldx != a.d;
        p.groups = (a.vocab + 63) / 64;
        p.ldz = (size_t)p.groups * 64;
        p.xc = take((size_t)p.rows_held * p.ldx * 2);
        if (p.pack_w) p.wp = take((size_t)a.vocab * p.ldx * 2);
        p.sums = take((size_t)p.cap * p.groups * sizeof(GroupSums));
        if (grads) {
            p.codes = take((size_t)p.rows_held * p.ldz * 2);
            p.dx = Splits{p.small ? 64 : 256, (a.d + 255) / 256, (a.vocab + pipe::BKS - 1) / pipe::BKS};
            p.dx_part = take((size_t)p.dx.rows(product_rows) * p.ldx * sizeof(float));
            const long dw_blocks = (long)((a.vocab + 255) / 256) * ((a.d + 255) / 256);
            const int row_stages = (product_rows + pipe::BKS - 1) / pipe::BKS;
            p.dw_splits = (int)(dw_blocks >= cus ? 1 : cus / dw_blocks);
            if (p.dw_splits > row_stages / 8) p.dw_splits = row_stages / 8 > 0 ? row_stages / 8 : 1;
            p.dw_parts = p.chunks > 1 || p.dw_splits > 1 || a.d % 8 != 0;
            p.dw_stride = (size_t)a.vocab * p.ldx;
            if (p.dw_parts) p.dw_part = take(p.dw_stride * p.dw_splits * sizeof(float));
        }
    } else {
        long cap = kChunkLogits / a.vocab;
        cap = cap < kChunkLeastF32 ? kChunkLeastF32 : cap > kChunkMostF32 ? kChunkMostF32 : cap;
        p.cap = (int)(a.rows < cap ? a.rows : cap);
        p.chunks = (a.rows + p.cap - 1) / p.cap;
        p.ldx = a.d;
        p.ldz = a.vocab;
        p.xc = take((size_t)p.cap * a.d * 4);
        p.codes = take((size_t)p.cap * p.ldz * 4);
        if (grads) {
            // the last chunk has fewer rows, and may have more parts
            const int last = a.rows - (p.chunks - 1) * p.cap;
            const size_t some = (size_t)p.cap * gemm_f32_splits(p.cap, a.d, a.vocab), end = (size_t)last * gemm_f32_splits(last, a.d, a.vocab);
            p.dx_part = take((some > end ? some : end) * a.d * 4);
        }
    }
    p.total = at;
    return p;
}

#define LM_TRY(call)                                   \
    do {                                               \
        const hipError_t e_ = (call);                  \
        if (e_ != hipSuccess) return e_;               \
    } while (0)

hipError_t loss_bf16(const VocabArgs &a, const VocabGrads *g, float *label_loss, float *top_loss, const Plan &p, char *base, const RowList &rl, hipStream_t s)
{
    bf16_t *xc = (bf16_t *)(base + p.xc), *codes = g ? (bf16_t *)(base + p.codes) : nullptr;
    const bf16_t *W = (const bf16_t *)a.W;
    if (p.pack_w) {
        LM_TRY(launch_pad_rows(a.W, a.vocab, a.d, p.ldx, base + p.wp, s));
        W = (const bf16_t *)(base + p.wp);
    }
    const bool two = a.label && a.ntop && a.tau != 1.f;
    const float inv_tau = 1.f / a.tau, scale = 1.44269504088896340736f * (a.label ? 1.f : inv_tau);
    const float deepest = kNoShare * (two ? fmaxf(1.f, a.tau) : 1.f), bend = kNoShare * (two ? fminf(1.f, a.tau) : 1.f);
    for (int ch = 0; ch < p.chunks; ++ch) {
        const int first = ch * p.cap;
        LM_TRY(launch_arrange_rows(a, g, rl, first, p.rows_held, p.ldx, xc, p.held, g ? g->dX : nullptr, label_loss, top_loss, s));
        const Operands logits{xc, W, p.ldx, p.ldx, p.rows_held, a.vocab, p.ldx};
        const LogitsOut lo{(GroupSums *)(base + p.sums), p.groups, codes, (long)p.ldz, scale, inv_tau, deepest, bend};
        LM_TRY(launch_logits(logits, rl.count, first, p.cap, a.vocab, lo, two, s));
        const VocabChunk c{first, p.cap, codes, p.ldz, lo.sums, two, bend, p.groups, xc, p.ldx, p.held};
        LM_TRY(launch_vocab_rows(a, g, rl, c, label_loss, top_loss, s));
        if (g && g->dX) {
            const Operands o{codes, W, (long)p.ldz, p.ldx, p.rows_held, p.ldx, a.vocab};
            float *part = (float *)(base + p.dx_part);
            LM_TRY((p.small ? launch_dx<64, 1, 4, 7>(o, rl.count, first, p.cap, a.d, p.held, p.dx, part, p.ldx, s)
                            : launch_dx<256, 2, 4, 4>(o, rl.count, first, p.cap, a.d, p.held, p.dx, part, p.ldx, s)));
            LM_TRY(launch_finish_dx(true, part, 0, p.ldx, rl, first, p.cap, a.d, p.held, g->dX, s));
        }
        if (g && g->dW) {
            const Operands o{codes, xc, (long)p.ldz, p.ldx, (int)p.ldz, p.ldx, 0};
            float *part = (float *)(base + p.dw_part);
            if (!p.dw_parts) LM_TRY((launch_dw<bf16_t, false>(o, rl, first, p.cap, p.held, a.vocab, 1, (bf16_t *)g->dW, 0, a.d, s)));
            else if (ch == 0) LM_TRY((launch_dw<float, false>(o, rl, first, p.cap, p.held, a.vocab, p.dw_splits, part, p.dw_stride, p.ldx, s)));
            else LM_TRY((launch_dw<float, true>(o, rl, first, p.cap, p.held, a.vocab, p.dw_splits, part, p.dw_stride, p.ldx, s)));
        }
    }
    if (g && g->dW && p.dw_parts)
        LM_TRY(launch_finish_dw(true, rl, (const float *)(base + p.dw_part), p.dw_splits, p.dw_stride, p.ldx, a.vocab, a.d, g->dW, s));
    return hipSuccess;
}

hipError_t loss_f32(const VocabArgs &a, const VocabGrads *g, float *label_loss, float *top_loss, const Plan &p, char *base, const RowList &rl, hipStream_t s)
{
    float *xc = (float *)(base + p.xc), *z = (float *)(base + p.codes), *dx = (float *)(base + p.dx_part);
    const float *W = (const float *)a.W;
    for (int ch = 0; ch < p.chunks; ++ch) {
        const int first = ch * p.cap, cap = a.rows - first < p.cap ? a.rows - first : p.cap;
        LM_TRY(launch_arrange_rows(a, g, rl, first, cap, a.d, xc, 0, g ? g->dX : nullptr, label_loss, top_loss, s));
        LM_TRY(launch_gemm_f32({cap, a.vocab, a.d, xc, true, W, true, z, false, 1}, s));
        const VocabChunk c{first, cap, z, p.ldz, nullptr, false, 0.f, 0, xc, a.d, 0};
        LM_TRY(launch_vocab_rows(a, g, rl, c, label_loss, top_loss, s));
        if (g && g->dX) {
            const int parts = gemm_f32_splits(cap, a.d, a.vocab);
            LM_TRY(launch_gemm_f32({cap, a.d, a.vocab, z, true, W, false, dx, false, parts}, s));
            LM_TRY(launch_finish_dx(false, dx, parts, a.d, rl, first, cap, a.d, 0, g->dX, s));
        }
        if (g && g->dW) LM_TRY(launch_gemm_f32({a.vocab, a.d, cap, z, false, xc, false, (float *)g->dW, ch > 0, 1}, s));
    }
    return hipSuccess;
}

}  // namespace

size_t vocab_workspace_bytes(const VocabArgs &a, bool grads) { return a.rows == 0 ? 0 : plan_of(a, grads).total; }

hipError_t launch_vocab_loss(const VocabArgs &a, const VocabGrads *g, float *label_loss, float *top_loss, void *ws, hipStream_t s)
{
    const Plan p = plan_of(a, g != nullptr);
    char *base = (char *)ws;
    const RowList rl{(int *)(base + p.list), (int *)(base + p.count), (float *)(base + p.scale)};
    if (!few_rows(a)) LM_TRY(launch_select_rows(a, g, rl, s));
    return a.bf16 ? loss_bf16(a, g, label_loss, top_loss, p, base, rl, s) : loss_f32(a, g, label_loss, top_loss, p, base, rl, s);
}

}  // namespace lm
}  // namespace stl
