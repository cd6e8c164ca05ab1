// Internal launcher interface between the C ABI (lm_api.hip) and the kernels of the residual step and the vocabulary loss.
#pragma once
#include "../stl_kernels.h"

#include <type_traits>

namespace stl {
namespace lm {

// n zeros (a kernel: memset nodes in a captured graph are avoided)
hipError_t launch_zero_elements(bool bf16, void *p, size_t n, hipStream_t s);

// ---- residual step (lm_residual.h) -------------------------------------------------------------------------------------------
struct ResidualArgs {
    int rows, n;
    int per_gate;                            // rows that share a row of the gate
    float skip, scale, eps;
    bool post, pre, center;
    const void *X, *H, *gate, *w_post, *b_post, *w_pre, *b_pre;      // storage type; gate, weights and offsets may be NULL
};
struct ResidualGrads {                       // what the backward pass reads besides (X is the stream behind the sum) and writes; any may be NULL
    const void *dXout, *dZ;
    void *dX, *dH;
    float *dgate, *dw_post, *db_post, *dw_pre, *db_pre;
    int accumulate;
};
constexpr int kResidualWidest = 32768;       // a row is held in the registers of one workgroup
size_t residual_workspace_bytes(int rows, int n, int per_gate);
hipError_t launch_residual_forward(int dtype, const ResidualArgs &a, void *Xout, void *Z, hipStream_t s);
hipError_t launch_residual_backward(int dtype, const ResidualArgs &a, const ResidualGrads &g, void *ws, hipStream_t s);

// ---- fp32 products (lm_f32.hip) ------------------------------------------------------------------------------------------------
// Out (I x J) (+)= A B over L, dense rows: A stored [i][l] (a_along) or [l][i], B stored [j][l] (b_along) or [l][j]
struct GemmF32 {
    int I, J, L;
    const float *A;
    bool a_along;
    const float *B;
    bool b_along;
    float *Out;
    bool accumulate;         // of [l][i] and [l][j] only
    int splits;              // of the contraction over workgroups: part s of the output lies s * I * J floats on
};
// as many as make two blocks a CU where there are fewer, of 32 stages at least
int gemm_f32_splits(int I, int J, int L);
hipError_t launch_gemm_f32(const GemmF32 &g, hipStream_t s);

// ---- vocabulary loss (lm_vocab.hip, lm_vocab_rows.hip) -----------------------------------------------------------------------
struct VocabArgs {
    int rows, d, vocab, ntop;
    float tau;
    bool bf16;
    const void *X, *W;
    const int64_t *label, *top_id;           // NULL: no such term
    const float *top_logit;
};
struct VocabGrads {
    const float *dlabel, *dtop;              // rows; upstream gradients of the two losses
    void *dX, *dW;                           // storage type, either may be NULL
};
constexpr int kMostTop = 1024;
// Rows of a chunk.  bf16: as many as have kChunkCodes logits (4.3 GB of codes), kChunkLeast to kChunkMost of them, which fill the chip several times
// over; fp32: as many as have kChunkLogits (1 GiB), kChunkLeastF32 at least, and no more than kChunkMostF32: a launch of a workgroup of 512 a row has fewer
// than 2^32 threads.
constexpr long kChunkCodes = 1L << 31, kChunkLogits = 1L << 28;
constexpr int kChunkLeast = 256, kChunkMost = 8192, kChunkLeastF32 = 64, kChunkMostF32 = 1 << 22;
// A logit between its product and its gradient is held (bf16 storage) in 16 bits: y = z log2(e) / t, t = 1 where there are labels and tau otherwise, in steps
// from its group's maximum down to its minimum, 65534; 65535 is what is below every share that fp32 can hold (minus infinity among it): 2^-kNoShare.
// One temperature: even steps over at most kNoShare; half a step is at most 1.1e-3, that is 8e-4 of a share.  A group of 64 normal logits spreads over
// five deviations: at a deviation of 2 a step is 2.2e-4, an error of 4e-5 (root mean square), a fortieth of the rounding of the gradient to
// bf16 that follows (as bf16 exponentials they would add that rounding once more).
// Two temperatures that differ (their ratio is up to 16): the lower one's shares end at kNoShare min(1, tau) below the maximum, but the other's go on to
// kNoShare max(1, tau).  A group that spreads over more than twice the first, `bend`, has half of its steps above the bend and half below, so that
// a share of either is off by 1.6e-3 at most (even steps, tau = 16: 1.3e-2).
constexpr float kSteps = 65535.f, kLowestTau = 0.25f, kHighestTau = 16.f, kNoShare = 150.041f;
constexpr float kBendSteps = 32767.f;
size_t vocab_workspace_bytes(const VocabArgs &a, bool grads);
// label_loss, top_loss: rows fp32 or NULL; g NULL: losses alone
hipError_t launch_vocab_loss(const VocabArgs &a, const VocabGrads *g, float *label_loss, float *top_loss, void *ws, hipStream_t s);

// The rows that have a label or a teacher, in order: list[0 .. count), and count itself, on the device; list has room for `rows`,
// count for a second number.
// scale: a factor for the gradient in the logits of bf16 storage, and its reciprocal (dz_scale in lm_vocab_rows.hip).
struct RowList {
    int *list, *count;
    float *scale;
};
hipError_t launch_select_rows(const VocabArgs &a, const VocabGrads *g, RowList rl, hipStream_t s);
// rows first .. first + cap of the list of X, side by side with ld elements each (zeros behind a row's end and behind the list's).  With the
// first chunk also: zeros for the rows that are not listed, in dX and the losses (each may be NULL).
// Few rows are listed by every workgroup of the first chunk's launch for itself, and by the first of them for the launches that follow, later chunks' among
// them: 1024 labels are 8 KB for each, lists of a teacher lie far apart.  In the place of a launch that lists them (us): labels, 1024 x 64, vocabulary 1000: 16.0 ->
// 14.7, 1500 rows 18.0 -> 17.8, 2048 19.4 -> 21.7, 4096 26 -> 54; a teacher's 16 entries, 256 x 256, 8000: 20.2 -> 18.8, 400 rows 21.7 -> 20.5, 700 23.6 ->
// 23.7, 1024 25.7 -> 27.4.
inline bool few_rows(const VocabArgs &a) { return a.rows <= (a.top_id ? 256 : 1024); }
hipError_t launch_arrange_rows(const VocabArgs &a, const VocabGrads *g, RowList rl, int first, int cap, int ld, void *out, int held, void *dX, float *label_loss, float *top_loss,
                               hipStream_t s);
// rows of an array, ld elements each in `out`, zeros behind a row's end (bf16)
hipError_t launch_pad_rows(const void *in, int rows, int d, int ld, void *out, hipStream_t s);

// Logits of one chunk of listed rows on their way to the gradient (storage fp32: the logits themselves).  bf16: what the product leaves for
// every listed row and group of 64 columns, with y as for kSteps: the largest y, m, the sums of
// 2^(y - m) and of 2^((y - m) / tau), and with gradients y as 16-bit steps below m and the size of a step; minus the size of those below the bend
// where there is one.
struct alignas(16) GroupSums {
    float m, sum, sum_tau, step;
};
// Up to so many listed rows the gradient in the logits of bf16 storage is held as two numbers (vocab_rows_kernel): what rounding that of row r leaves goes
// to row r + second_row, itself rounded.  The errors of dX and dW over those of one rounding of each, the largest of 420 outputs of small calls (most of them
// of 64 to 128 columns, labels, a teacher's 5 to 100 entries or both): with one number 1.60, 1.74, 1.65, 1.49, 1.50, 1.56, 1.47, 1.52 and 1.46 at 33, 48, 64, 96,
// 128, 140, 192, 256 and 400 rows (the median is 1.33 throughout; two equal roundings give 1.41), with two 1.00.  They double the rows of dX's and dW's
// products: 64 x 4096, vocabulary 65536: 430 -> 502 us, 100 x 4096: 479 -> 535, 64 x 64, 109807: 90 -> 97.
constexpr int kPairRows = 128;
__host__ __device__ inline int whole_stages(int rows) { return (rows + 31) / 32 * 32; }
// 0: one number a row.  listed: of all chunks; held: rows of the chunk's buffers (0: no gradients), which have room for both
__host__ __device__ inline int second_row(int listed, int held) { return listed <= kPairRows && 2 * whole_stages(listed) <= held ? whole_stages(listed) : 0; }
struct VocabChunk {
    int first, cap;                          // listed rows first .. first + cap (those that exist)
    void *codes;                             // cap x ld: 16 bits (bf16 storage) or fp32 logits; the gradient is written in their place
    size_t ld;
    const GroupSums *sums;                   // cap x groups (bf16 storage)
    bool two;                                // they have the second sum: both terms are there and tau is not 1
    float bend;
    int groups;
    const void *Xc;                          // the listed rows, ldx elements each
    int ldx;
    int held;                                // second_row
};
hipError_t launch_vocab_rows(const VocabArgs &a, const VocabGrads *g, RowList rl, const VocabChunk &c, float *label_loss, float *top_loss, hipStream_t s);
// How the contraction of dX over the vocabulary is cut, on the device, where the rows of the chunk are known: in as many runs of whole stages (16 at
// least) as take the least time, in 10 ns: rounds of blocks over the CUs of an MI355X, of 53 a stage and 500 beside, and 12 a block and run for writing
// its fp32 part and adding it up (34 rows of 64, vocabulary 109807: 117 us in 16 runs, 36 in up to 64).
// Whole calls with 1, 2, 4, 8, 12, 16, 24, 32, 48 and 64 runs, ten shapes from 3 x 512, vocabulary 60000, to 1500 x 512, 16000: the choice is within 1 % of the
// best of them at each (300 x 1024, 50001: 202 us, 238 in 12 runs, 219 in 64; 1201 x 1024: 431, 495 in 16).  Part s of `rows` rows lies s * rows * ld
// floats on; the product leaves the number of runs at count[1] for the kernel that adds them up.
struct Splits {
    int block_rows, tiles_n, stages;
    static constexpr int kMost = 64, kBlocks = 1024;         // runs, and blocks of all runs where there is more than one
    __host__ __device__ int of(int rows) const
    {
        const int tiles = (rows + block_rows - 1) / block_rows * tiles_n;      // at most 32 * 4096
        int best = 1;
        int64_t least = 0;
        for (int s = 1; s == 1 || (s <= kMost && s * tiles <= kBlocks && 16 * s <= stages); s += s < 16 ? 1 : 8) {
            const int64_t time = (int64_t)((s * tiles + 255) / 256) * (53 * stages / s + 500) + 12 * s * tiles;
            if (s == 1 || time < least) least = time, best = s;
        }
        return best;
    }
    // rows of all parts together, at most, for up to `cap` rows
    __host__ long rows(int cap) const
    {
        const long full = (long)kBlocks / tiles_n * block_rows, all = (long)cap * kMost, some = full < all ? full : all;
        return some > cap ? some : cap;
    }
};
// dX rows of the list from the parts (bf16 storage: as many as the product left behind the count), a row and its second one (held: second_row) together
hipError_t launch_finish_dx(bool bf16, const float *part, int parts, int ld, RowList rl, int first, int cap, int d, int held, void *dX, hipStream_t s);
// out[i][j] = sum over parts of part[p][i][j], rows of ld in the parts and of d in `out`, and 1 / scale
hipError_t launch_finish_dw(bool bf16, RowList rl, const float *part, int parts, size_t stride, int ld, size_t rows, int d, void *dW, hipStream_t s);

}  // namespace lm
}  // namespace stl
