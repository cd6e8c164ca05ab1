// Matrix products of the vocabulary loss: a block of BM x BN outputs on a ring of LDS stages, with an epilogue of the caller's.
//
// The stages themselves -- LDS-DMA sources, swizzles, fragments, the order of reads, loads and products within a stage -- are those of the plane
// products (../stl_gemm_pipe.h).  What differs is around them: one plane with a leading dimension of its own for each operand, a contraction
// that may end inside a stage (KTAIL: the second operand's missing rows are read as its last one, the first operand holds zeros there), an
// epilogue that gets the accumulators, and a block order in groups of rows.
#pragma once
#include "../stl_gemm_pipe.h"

namespace stl {
namespace lm {

struct Operands {
    const bf16_t *A, *B;
    long lda, ldb;
    int a_rows, b_rows;      // rows behind which nothing is read ([l][row] form: columns, a multiple of 8)
    int Kl;
};

// Blocks in groups of about four block rows, down the columns of a group first: the 32 workgroups of an XCD, side by side in the list, then share 4 rows
// of the first operand and 8 columns of the second in their L2 instead of 1 and 32 (4096 x 65536 x 4096: 1735 us, 2090 row by row, 1846 in groups of
// 16).  Groups are of even size: of five rows one group of five, not of four and one (1280 x 50176 x 1024: 124 us and 135).
__device__ __forceinline__ int group_rows(int tiles_m)
{
    const int groups = tiles_m < 7 ? 1 : (tiles_m + 1) / 4;
    return (tiles_m + groups - 1) / groups;
}
__device__ __forceinline__ void block_at(int v, int tiles_m, int tiles_n, int size, int &bi, int &bj)
{
    const int per = size * tiles_n, q = v / per, rem = v - q * per;
    const int rows = tiles_m - q * size < size ? tiles_m - q * size : size;
    bj = rem / rows;
    bi = q * size + rem - bj * rows;
}

template <int BM_, int BN_, int WAVES_M, int WAVES_N_, int NS, bool A_T, bool B_T, bool KTAIL>
struct Ring {
    static constexpr int BM = BM_, BN = BN_, WAVES_N = WAVES_N_, NW = WAVES_M * WAVES_N, THREADS = NW * 64;
    static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, FM = WM / 16, FN = WN / 16;
    static constexpr int OPER_BYTES = BM * pipe::BKS * 2, STAGE_BYTES = (BM + BN) * pipe::BKS * 2;
    static constexpr int D = (BM + BN) / 16 / NW;          // DMA instructions per wavefront and stage
    static constexpr int SLAB = 4096, SLABS_AT = NS * STAGE_BYTES, LDS_BYTES = SLABS_AT + NW * SLAB;
    static_assert(LDS_BYTES <= 160 * 1024 && NS >= 3, "LDS");
    typedef pipe::WaveTile<FM, FN> Tile;
    pipe::Frag<A_T, BM> fa;
    pipe::Frag<B_T, BN> fb;
    pipe::Src<A_T, BM, NW, false> sa;
    pipe::Src<B_T, BN, NW, KTAIL> sb;
    __device__ __forceinline__ void init(int wave, int lane)
    {
        fa.init(wave / WAVES_N * WM, lane);
        fb.init(wave % WAVES_N * WN, lane);
    }
    // point the DMA sources at the block whose first row and column are i0, j0 and put its first NS - 1 stages in flight
    __device__ __forceinline__ void start(const Operands &o, int nks, int i0, int j0, uint32_t smem_lds, int wave, int lane)
    {
        // the lane id as an opaque value: what the sources derive from it is computed per block and occupies no registers meanwhile
        int sl = lane;
        asm volatile("" : "+v"(sl));
        sa.init(o.A, o.lda, i0, o.a_rows, wave, sl, 0, 1, 1 << 30, 0, o.Kl);
        sb.init(o.B, o.ldb, j0, o.b_rows, wave, sl, 0, 1, 1 << 30, 0, o.Kl);
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) {
            if (s < nks) {
                sa.issue(smem_lds + s * STAGE_BYTES, wave, sl);
                sb.issue(smem_lds + s * STAGE_BYTES + OPER_BYTES, wave, sl);
            }
        }
    }
    // The block whose first loads are in flight: its nks stages, next() (the loads of what follows) and epilogue(accumulators).
    template <class N, class E>
    __device__ __forceinline__ void block(int nks, const char *smem, uint32_t smem_lds, int wave, int lane, N &&next, E &&epilogue)
    {
        using namespace pipe;
        Tile w;
        w.clear();
        // Stage s+NS-1 is issued in iteration s; stage s+1 must have landed at the top of iteration s (its fragments are
        // fetched during stage s).  Stores of the previous epilogue may still be in flight: "at most N operations
        // outstanding" then over-waits but never under-waits.
        wait_stages<D, NS - 2>(nks - 1);
        block_barrier();
#pragma unroll
        for (int a = 0; a < FM; ++a) w.va[a] = fa.read(smem, a);
#pragma unroll
        for (int b = 0; b < FN; ++b) w.vb[0][b] = fb.read(smem + OPER_BYTES, b);
        auto stage = [&](int s, auto par_c, auto steady_c) {
            constexpr int PAR = decltype(par_c)::value;
            constexpr bool STEADY = decltype(steady_c)::value;
            const bool refill = STEADY || s + NS - 1 < nks;
            if (STEADY) wait_vmcnt<D * (NS - 3)>();
            else wait_stages<D, NS - 3>(nks - 2 - s < 0 ? 0 : nks - 2 - s);
            block_barrier();   // stage s+1 visible to all; nobody reads stage s-1 any more
            const uint32_t dst = smem_lds + ((s + NS - 1) % NS) * STAGE_BYTES;
            const char *nxt = smem + ((s + 1) % NS) * STAGE_BYTES;
            w.template stage<PAR>([&](int f) { return fa.read(nxt, f); }, [&](int f) { return fb.read(nxt + OPER_BYTES, f); },
                                  [&](auto a_c) {
                                      constexpr int a = decltype(a_c)::value, NA = decltype(sa)::NI, NB = decltype(sb)::NI;
                                      static_for<0, NA + NB>([&](auto j_c) {
                                          constexpr int j = decltype(j_c)::value;
                                          if constexpr (j * FM / (NA + NB) == a) {
                                              if (refill) {
                                                  if constexpr (j < NA) sa.issue_one(dst, wave, j);
                                                  else sb.issue_one(dst + OPER_BYTES, wave, j - NA);
                                              }
                                          }
                                      });
                                  });
            if (refill) {
                sa.next_stage(wave, lane);
                sb.next_stage(wave, lane);
            }
        };
        using I0 = std::integral_constant<int, 0>;
        using I1 = std::integral_constant<int, 1>;
        const int n_refill = nks > NS - 1 ? nks - (NS - 1) : 0;
        int s = 0;
        for (; s + 1 < n_refill; s += 2) {
            stage(s, I0{}, std::true_type{});
            stage(s + 1, I1{}, std::true_type{});
        }
        for (; s < nks; s += 2) {
            stage(s, I0{}, std::false_type{});
            if (s + 1 < nks) stage(s + 1, I1{}, std::false_type{});
        }
        // every wavefront is done with the ring: refill it for the next block before this one's epilogue
        block_barrier();
        next();
        epilogue(w);
    }
};

// A workgroup's way through its share of a list of blocks: every step-th from v on, below end.  place(v, o, stages, i0, j0) says what block v is;
// epilogue(accumulators, v, i0, j0).
template <class R, class P, class E>
__device__ __forceinline__ void walk(R, int v, int end, int step, const Operands &o, const char *smem, uint32_t smem_lds, int wave, int lane, P &&place, E &&epilogue)
{
    R ring;
    ring.init(wave, lane);
    auto start = [&](int u) {
        Operands mine = o;
        int stages, i0, j0;
        place(u, mine, stages, i0, j0);
        ring.start(mine, stages, i0, j0, smem_lds, wave, lane);
    };
    if (v < end) start(v);
    for (; v < end; v += step) {
        Operands mine = o;
        int stages, i0, j0;
        place(v, mine, stages, i0, j0);
        ring.block(
            stages, smem, smem_lds, wave, lane,
            [&]() {
                if (v + step < end) start(v + step);
            },
            [&](typename R::Tile &w) { epilogue(w, v, i0, j0); });
    }
}

// The same over the blocks of 256 x 256 of a whole list, in which those of a last round that would leave half of the workgroups idle are cut into two halves
// of 128 rows, one for each of twice as many workgroups (Half); a half that begins behind the last of the output's `rows` rows is none.  777 rows,
// 1024, vocabulary 50001, 784 blocks on 256 CUs: the whole call 122 -> 115 us.
template <class Full, class Half, class P, class E>
__device__ __forceinline__ void walk_list(int total, int rows, const Operands &o, const char *smem, uint32_t smem_lds, int wave, int lane, P &&place, E &&epilogue)
{
    const int first = pipe::first_block(total), end = pipe::end_block(total), step = pipe::block_step(), whole = pipe::whole_end(total), rest = end - whole;
    if (rows <= 128) {                                       // the upper halves are all there is
        walk(Half{}, first, end, step, o, smem, smem_lds, wave, lane, place, epilogue);
        return;
    }
    if (2 * rest > step) {
        walk(Full{}, first, end, step, o, smem, smem_lds, wave, lane, place, epilogue);
        return;
    }
    walk(Full{}, first, whole, step, o, smem, smem_lds, wave, lane, place, epilogue);
    // (its ring lies in that of the whole blocks, which all wavefronts have left, and ends below their slabs)
    const int u = (int)(blockIdx.x >> 3);
    if (u >= 2 * rest) return;
    auto half = [&](int h, Operands &mine, int &stages, int &i0, int &j0) {
        place(whole + h / 2, mine, stages, i0, j0);
        i0 += (h & 1) * 128;
    };
    Operands mine = o;
    int stages, i0, j0;
    half(u, mine, stages, i0, j0);
    if (i0 < rows) walk(Half{}, u, u + 1, 1, o, smem, smem_lds, wave, lane, half, [&](typename Half::Tile &w, int h, int r, int c) { epilogue(w, whole + h / 2, r, c); });
}

}  // namespace lm
}  // namespace stl
