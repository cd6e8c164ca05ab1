// Attention whose past decays, chunk by chunk (gfx950).
//
//   S_t = lambda S_{t-1} + k_t v_t^T,   o_t = c q_t S_t,   lambda = exp(a) of the head
//
// Written out for a chunk of C tokens behind a state S, i and j counting from the chunk's first token:
//   o_i = c ( lambda^(i+1) q_i S + sum_{j <= i} lambda^(i-j) (q_i . k_j) v_j ),     S <- lambda^C S + sum_j lambda^(C-1-j) k_j v_j^T
// so that all but the masking is matrix products.  The gradients are the same thing with other operands: dQ is this attention of (dO, V, K), and, with
// time reversed, dV that of (K, Q, dO) and dK that of (V, dO, Q) (DecayPass).
//
// A workgroup takes a segment of a sequence, a head and 128 columns of v at most, chunk after chunk.  Where there are too few heads to fill the chip, a sequence has
// several segments: a sweep without outputs first forms what each adds to the state, a small kernel joins these in order to the state in front of each
// segment (decay_join_kernel), and all segments run at once.  That reads K and V twice (largely from the last-level cache: 108 of 201 MB come from memory the second
// time in the sizes below).
// A wavefront owns 16 columns of v: its part of S stays in accumulators (dk x 16, fp32) all along, in 128 registers with all else (4 to 8 of a thread's in scratch memory
// for rows of 97 to 128 in bf16), so that two workgroups share a CU.  Products are formed so that accumulators are the next product's operand as they lie:
//   P^T = K Q^T (tokens j x i)   ->   O^T += V^T P^T,      S (dk x columns) as S^T in   O^T = S^T Q^T
// An accumulator's lane holds rows 4 g + e of its column (g = lane / 16), an operand's lane eight elements of the contraction, whose order is free as long as
// both operands have it: along the rows it is the order that two tiles of accumulators have (state_row), over tokens 8 g + e.  P is the same for all columns:
// the wavefronts form a quarter of its tile each and share them through LDS, which is one more barrier a chunk and saves each wavefront three quarters of it.
//
// Chunks of 32 tokens come through a ring of LDS stages, loaded without a register between (rows of whole 16-byte pieces at such addresses; others go through
// registers and one stage).
//
// A value of V that is no finite number must not reach earlier tokens, as it would with a zero of the masked P: it is multiplied as a zero, and its column
// of the outputs from its token on, and of the state, becomes NaN.
//
// bf16 storage: operands that come from fp32 (P, S, V scaled by the decay up to the chunk's end) are given to the matrix cores as sums of bf16 numbers, two of
// them (a relative error of 2^-16) for what goes into outputs that are rounded to bf16, three (2^-24) for what goes into the fp32 state.  With one, P's
// and S's roundings would each be as large as the output's own.  fp32 storage: fp32 matrix instructions.
//
// What bounds it, 8192 tokens x 32 heads of 128 in bf16, 8 segments: states 43 us, join 8, outputs 82 (matrix cores busy for 30 % of it, vector unit, which splits S, V and P,
// for half, wavefronts waiting for 40 %).  With the loads and stores alone the last takes 61, with the products alone 67: both at once are near what there is.
// Tried without gain: matrix and vector instructions in turn by scheduling groups (equal), the products of P behind the state's update (3 % slower), the remainders of
// a split by two-element dot products in the place of shifts and subtractions (6 % slower), 32 columns a wavefront and two of them on a SIMD (5 to 7 % slower but for
// gradients of bf16, 3 % faster; fp32 a fifth slower).
#pragma once
#include "seq_kernels.h"
#include "../csrc/lm/lm_device.h"
#include "../csrc/stl_gemm_pipe.h"

#include <atomic>

namespace stl {
namespace seq {

using lm::Chunk;
using pipe::v4i16_t;

// One sweep: "queries" A, "keys" B (width da), "values" V (width dv); forward in time, or backward.  Heads of A, B and V that several heads
// share: head h takes h / share.
struct DecayPass {
    int rows, sequences, length, heads, seq_step, token_step;
    int da, dv;
    const void *A, *B, *V;
    size_t lda, ldb, ldv, ldo;
    int share_a, share_b, share_v;
    void *O;                                 // storage type, or fp32 (out32); NULL: the state alone
    bool out32, reverse;
    // factors of probabilities, of what outputs take from the state, and of what goes into it: c, c and 1 forward in time; backward, where the state is the gradient as the
    // formula has it (what is handed in belongs to it as it is), c, 1 and c
    float out_scale, state_scale, value_scale;
    const float *log_decay;
    const int64_t *offset;
    // states lie [sequence][head][da][dv], or [dv][da] (turned).  The first is multiplied, for the first token, by lambda^init_power (1 forward in time, 0 backward,
    // where what is given belongs to the last token itself); the last by lambda^last_power.
    const float *init;
    float *last;
    bool turned;
    int init_power, last_power;
    // segments of seg_tokens (a multiple of 32).  starts [sequence][head][segments][da dv]: number s holds what segment s adds to the state, and behind decay_join_kernel
    // the state in front of segment s + 1; the last one `init` as it was, where the last state may be written over it.
    int segments, seg_tokens;
    float *starts;
    bool ring;                               // rows are whole 16-byte pieces at such addresses
};

// tokens of sequence b: the row of the first, and how many (never outside the rows there are, whatever the offsets are)
struct Tokens {
    int64_t first;
    int count;
};
__device__ __forceinline__ Tokens tokens_of(const DecayPass &p, int b)
{
    if (!p.offset) return Tokens{(int64_t)b * p.seq_step, p.length};
    int64_t lo = p.offset[b], hi = p.offset[b + 1];
    lo = lo < 0 ? 0 : lo > p.rows ? p.rows : lo;
    hi = hi < lo ? lo : hi > p.rows ? p.rows : hi;
    return Tokens{lo, hi - lo < p.length ? (int)(hi - lo) : p.length};
}

// a b, and zero where either is zero, whatever the other is (v_mul_legacy_f32, which has no builtin)
__device__ float fmul_legacy(float a, float b) __asm("llvm.amdgcn.fmul.legacy");

// lambda^n, a not below -100000 (where it is 0 for every n > 0)
__device__ __forceinline__ double power(double a, int n) { return n == 0 ? 1.0 : exp(a * n); }


constexpr int kChunk = 32;                   // tokens

// 32 rows of an operand in LDS, in groups of four 16-byte pieces of every row (64 bytes a row, 2 KB a group).  Piece c of row r lies in its row's place
// c % 4 ^ r / 4 % 4: a read of one piece of 32 rows, or of four pieces of four rows, meets every bank alike, and group and operand are constants of an address.
constexpr int kGroupBytes = 64 * kChunk;
__device__ __forceinline__ int piece_at(int r, int c) { return kGroupBytes * (c >> 2) + 64 * r + 16 * ((c ^ r >> 2) & 3); }

// The state's row, within 32, of element e of a lane's accumulators of tile t (g = lane / 16), and so the order of a contraction along the rows.
__device__ __forceinline__ int state_row(int g, int t, int e) { return 16 * t + 4 * g + e; }

// The tile of probabilities (tokens i of the queries by tokens j of the keys) is formed by a workgroup's wavefronts in quarters of 16 by 16: 0, 1 and 2 are (i, j) from
// (0, 0), (16, 0) and (16, 16) on, and the fourth is all masked.  A lane has one i and four j from `j` on.
struct Quarter {
    int i, j;
    __device__ __forceinline__ Quarter(int which, int lane) : i((which > 0 ? 16 : 0) + (lane & 15)), j((which > 1 ? 16 : 0) + 4 * (lane >> 4)) {}
};

template <typename T> struct Ops;

template <> struct Ops<bf16_t> {
    static constexpr int kOutParts = 2, kStateParts = 3;
    typedef bf16x8_t Frag;                   // operand: row or column lane % 16, eight elements of a contraction of 32
    static __device__ __forceinline__ f32x4_t mma(const Frag &a, const Frag &b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    // a lane's places: of its two times four elements of row lane % 16; of its piece of that row; and of what it gives to the transposing reads of a matrix'
    // first 16 columns, for rows 8 g .. and 8 g + 4 ..
    struct Places {
        int row[2], piece, across[2];
    };
    static __device__ __forceinline__ Places places(int lane)
    {
        const int n = lane & 15, g = lane >> 4, r = 8 * g + (n >> 2), c = n >> 1 & 1;
        return Places{{piece_at(n, g >> 1) + 8 * (g & 1), piece_at(n, 2 + (g >> 1)) + 8 * (g & 1)}, piece_at(n, -g & 3), {piece_at(r, c) + 8 * (n & 1), piece_at(r + 4, c) + 8 * (n & 1)}};
    }
    // contraction along the rows, columns 32 k + state_row(g, t, e); row lane % 16 + 16 half
    static __device__ __forceinline__ Frag along(const char *rows, const Places &at, int k, int half)
    {
        const char *from = rows + kGroupBytes * k + kGroupBytes / 2 * half;
        const u32x2_t lo = *reinterpret_cast<const u32x2_t *>(from + at.row[0]), hi = *reinterpret_cast<const u32x2_t *>(from + at.row[1]);
        return __builtin_bit_cast(Frag, u32x4_t{lo[0], lo[1], hi[0], hi[1]});
    }
    static __device__ __forceinline__ Frag transposed(const char *lo, const char *hi)
    {
        struct { v4i16_t lo, hi; } two;
        two.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t *)STL_LDS(lo));
        two.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t *)STL_LDS(hi));
        return __builtin_bit_cast(Frag, two);
    }
    // contraction over the rows, column 16 c + lane % 16  (the other half of a row's 64 bytes: its places with bit 5 the other way round)
    static __device__ __forceinline__ Frag across(const char *rows, const Places &at, int c)
    {
        const int other = 32 * (c & 1);
        rows += kGroupBytes * (c >> 1);
        return transposed(rows + (at.across[0] ^ other), rows + (at.across[1] ^ other));
    }
    // x rounded, and x less by that
    static __device__ __forceinline__ Frag part(float *x)
    {
        u32x4_t w;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
            x[2 * k] -= __uint_as_float(w[k] << 16);
            x[2 * k + 1] -= __uint_as_float(w[k] & 0xffff0000u);
        }
        return __builtin_bit_cast(Frag, w);
    }
    // Probabilities, q_i . k_j times `near`: two parts of four bf16 numbers a lane to where probabilities() finds them.
    template <int KT>
    static __device__ __forceinline__ void quarter(const char *queries, const char *keys, int which, int lane, const float *near, char *probs)
    {
        const Quarter at(which, lane);
        const int c = -(lane >> 4) & 3;
        const char *q = queries + piece_at(at.i, c), *k = keys + piece_at((which > 1 ? 16 : 0) + (lane & 15), c);
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KT; ++i) sum = mma(*reinterpret_cast<const Frag *>(k + kGroupBytes * i), *reinterpret_cast<const Frag *>(q + kGroupBytes * i), sum);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fmul_legacy(near[e], sum[e]);                     // (zero times anything is zero: the masked ones)
        char *to = probs + piece_at(at.i, -(at.j >> 3) & 3) + 8 * (at.j >> 2 & 1);
#pragma unroll
        for (int m = 0; m < kOutParts; ++m) {
            const u32x2_t w = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
            *reinterpret_cast<u32x2_t *>(to + kGroupBytes * m) = w;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] -= __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        }
    }
    // part m of them, contraction over j, column i = lane % 16 + 16 half
    static __device__ __forceinline__ Frag probabilities(const char *probs, const Places &at, int m, int half)
    {
        return *reinterpret_cast<const Frag *>(probs + at.piece + kGroupBytes * m + kGroupBytes / 2 * half);
    }
    static __device__ __forceinline__ float get(const Frag &a, int e)
    {
        const u32x4_t w = __builtin_bit_cast(u32x4_t, a);
        return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
    // zero times them by the matrix cores: one instruction in the place of a dozen
    static __device__ __forceinline__ bool finite(const Frag &a)
    {
        return mma(__builtin_bit_cast(Frag, u32x4_t{0u, 0u, 0u, 0u}), a, f32x4_t{0.f, 0.f, 0.f, 0.f})[0] == 0.f;
    }
    // zeros in the place of what is no finite number; the first row of such an element, 32 if there is none
    static __device__ __forceinline__ int clean(Frag &a, int g)
    {
        int first = kChunk;
        u32x4_t w = __builtin_bit_cast(u32x4_t, a);
#pragma unroll
        for (int e = 7; e >= 0; --e) {
            const uint32_t half = e & 1 ? 0xffff0000u : 0xffffu, ones = half & 0x7f807f80u;
            if ((w[e >> 1] & ones) != ones) continue;
            w[e >> 1] &= ~half;
            first = 8 * g + e;
        }
        a = __builtin_bit_cast(Frag, w);
        return first;
    }
};

template <> struct Ops<float> {
    static constexpr int kOutParts = 1, kStateParts = 1;
    struct Frag {
        float f[8];
    };
    // (four contractions at a time: number 8 (lane / 16) + e of 32 with the e-th instruction)
    static __device__ __forceinline__ f32x4_t mma(const Frag &a, const Frag &b, f32x4_t c)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[e], b.f[e], c, 0, 0, 0);
        return c;
    }
    // where piece c of the probabilities lies: four lanes' pieces 2 (lane / 16) of sixteen rows in places that meet every bank alike
    static __device__ __forceinline__ int gray(int c) { return c ^ (c >> 1 & 1); }
    struct Places {
        int row[2], piece[2], across[2];
    };
    static __device__ __forceinline__ Places places(int lane)
    {
        const int n = lane & 15, g = lane >> 4, r = 8 * g, c = n >> 2, x = 4 * (n & 3);
        return Places{{piece_at(n, g), piece_at(n, 4 + g)}, {piece_at(n, gray(2 * g)), piece_at(n, gray(2 * g + 1))}, {piece_at(r, c) + x, piece_at(r + 4, c) + x}};
    }
    static __device__ __forceinline__ Frag two(const char *first, const char *second)
    {
        const f32x4_t u = *reinterpret_cast<const f32x4_t *>(first), v = *reinterpret_cast<const f32x4_t *>(second);
        return Frag{{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]}};
    }
    static __device__ __forceinline__ Frag along(const char *rows, const Places &at, int k, int half)
    {
        rows += 2 * kGroupBytes * k + kGroupBytes / 2 * half;
        return two(rows + at.row[0], rows + at.row[1]);
    }
    static __device__ __forceinline__ Frag across(const char *rows, const Places &at, int c)
    {
        Frag r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r.f[e] = *reinterpret_cast<const float *>(rows + at.across[e >> 2] + kGroupBytes * c + 64 * (e & 3));
        return r;
    }
    static __device__ __forceinline__ Frag part(const float *x)
    {
        Frag r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r.f[e] = x[e];
        return r;
    }
    template <int KT>
    static __device__ __forceinline__ void quarter(const char *queries, const char *keys, int which, int lane, const float *near, char *probs)
    {
        const Quarter at(which, lane);
        const int c = -(lane >> 4) & 3;
        const char *q = queries + piece_at(at.i, c), *k = keys + piece_at((which > 1 ? 16 : 0) + (lane & 15), c);
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2 * KT; ++i) {
            const f32x4_t u = *reinterpret_cast<const f32x4_t *>(k + kGroupBytes * i), v = *reinterpret_cast<const f32x4_t *>(q + kGroupBytes * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(u[e], v[e], sum, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmul_legacy(near[e], sum[e]);
        *reinterpret_cast<f32x4_t *>(probs + piece_at(at.i, gray(at.j >> 2))) = sum;
    }
    static __device__ __forceinline__ Frag probabilities(const char *probs, const Places &at, int, int half)
    {
        return two(probs + at.piece[0] + kGroupBytes / 2 * half, probs + at.piece[1] + kGroupBytes / 2 * half);
    }
    static __device__ __forceinline__ float get(const Frag &a, int e) { return a.f[e]; }
    // (an exponent of ones carries into its sign bit)
    static __device__ __forceinline__ bool finite(const Frag &a)
    {
        uint32_t carry = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) carry |= (__float_as_uint(a.f[e]) & 0x7f800000u) + 0x00800000u;
        return !(carry & 0x80000000u);
    }
    static __device__ __forceinline__ int clean(Frag &a, int g)
    {
        int first = kChunk;
#pragma unroll
        for (int e = 7; e >= 0; --e) {
            if ((__float_as_uint(a.f[e]) & 0x7f800000u) != 0x7f800000u) continue;
            a.f[e] = 0.f;
            first = 8 * g + e;
        }
        return first;
    }
};

constexpr int kDecayColumns = 128;           // of v, of a workgroup, 16 a wavefront
// 32 KT: width of queries and keys in LDS; NW wavefronts; OUT: with outputs; RING: loaded by LDS-DMA
template <typename T, int KT, int NW, bool OUT, bool RING>
struct DecayShape {
    static constexpr int columns = 16 * NW, threads = 64 * NW, in_group = 64 / (int)sizeof(T);
    static constexpr int groups = 32 * KT / in_group, groups_v = columns / in_group;
    static constexpr int bytes = kGroupBytes * groups, bytes_v = kGroupBytes * groups_v, stage = (OUT ? 2 : 1) * bytes + bytes_v;
    // half of the LDS, so that two workgroups share a CU, where two stages fit into it
    static constexpr int tables = 512, tile = OUT ? 2 * kGroupBytes : 0;
    static constexpr int sharing = 2 * stage + tables + tile <= 80 * 1024 ? 2 : 1;
    static constexpr int room = 160 * 1024 / sharing - tables - tile, fit = room / stage;
    static constexpr int stages = RING ? fit < 4 ? fit : 4 : 1;
    static constexpr int lds = stages * stage + tables + tile;
    static_assert(stages >= (RING ? 2 : 1), "a ring has two stages at least");
};
// wavefronts of a SIMD, whose registers they share: two workgroups'
constexpr int decay_waves(size_t element, int KT) { return KT <= (element == 2 ? 4 : 3) ? 4 : 2; }

// up to four elements of a row of outputs
template <typename T>
__device__ __forceinline__ void put4(T *to, int left, f32x4_t v)
{
    if (left >= 4) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_any_t *>(to) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else *reinterpret_cast<f32x4_any_t *>(to) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) Elem<T>::st(to + e, v[e]);
    }
}

// all but the N youngest loads and stores are done, and all LDS reads
template <int N>
__device__ __forceinline__ void wait_all_but()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// all LDS reads and writes are done
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// eight elements of row r, from element 8 u on, to where they lie in LDS
__device__ __forceinline__ void put8(char *rows, int r, int u, const Chunk<bf16_t> &c) { *reinterpret_cast<u32x4_t *>(rows + piece_at(r, u)) = c.v; }
__device__ __forceinline__ void put8(char *rows, int r, int u, const Chunk<float> &c)
{
    *reinterpret_cast<f32x4_t *>(rows + piece_at(r, 2 * u)) = c.a;
    *reinterpret_cast<f32x4_t *>(rows + piece_at(r, 2 * u + 1)) = c.b;
}

// 16 bytes a lane, from `base` + `off`, to LDS: lane l's to lds_wave_base + 16 l.
__device__ __forceinline__ void dma16_at(const char *base, uint32_t off, uint32_t lds_wave_base)
{
    const uint32_t l = __builtin_amdgcn_readfirstlane(lds_wave_base);
    // M0 has to be written one wait state ahead of the load, a scalar register that a vector instruction writes (the base, where the compiler brings it from
    // one) five; the compiler, which sees to that elsewhere, does not look into the statement
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(l) : "memory", "m0");
}

// One operand's share of a stage that a wavefront loads by LDS-DMA.  Instruction i brings 64 pieces, one a lane: four of each of 16 rows.  Where the row
// ends before the groups do, or instructions are no multiple of the wavefronts, some of them bring the same again: all wavefronts issue as many.
template <typename T, int GROUPS, int NW>
struct RingSource {
    static constexpr int kAll = 2 * GROUPS, kPer = (kAll + NW - 1) / NW, kInGroup = 64 / (int)sizeof(T);
    const char *next;                        // where the next chunk's lowest row is, if it is whole
    int64_t advance;                         // bytes from there to the one behind it
    uint32_t off[kPer];                      // of a lane's pieces, from the chunk's lowest row on
    uint32_t which, step;                    // a bit for each instruction: whether this lane's piece lies within the row; bytes from token to token
    int there, whole;                        // instructions that bring something; whether rows end where a group does
    __device__ __forceinline__ int instruction(int j, int wave) const
    {
        const int i = j * NW + wave;
        return i < there ? i : there - 1;
    }
    static __device__ __forceinline__ int row(int i, int lane) { return 16 * (i & 1) + (lane >> 2); }
    static __device__ __forceinline__ int piece(int i, int lane) { return 4 * (i >> 1) + ((lane ^ row(i, lane) >> 2) & 3); }
    __device__ __forceinline__ void init(const T *base, size_t ld, const Tokens &tokens, int token_step, int from, int wave, int lane, int wide, bool reverse)
    {
        there = 2 * ((wide + kInGroup - 1) / kInGroup), whole = wide % kInGroup == 0;
        const int64_t bytes = (int64_t)token_step * (int64_t)(ld * sizeof(T));
        step = (uint32_t)bytes;
        next = reinterpret_cast<const char *>(base + (size_t)tokens.first * ld) + bytes * (reverse ? tokens.count - from - kChunk : from);
        advance = (reverse ? -kChunk : kChunk) * bytes;
        which = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int i = instruction(j, wave), r = row(i, lane), c = piece(i, lane);
            if (c * (16 / (int)sizeof(T)) < wide) which |= 1u << j;
            off[j] = (uint32_t)(reverse ? kChunk - 1 - r : r) * step + 16 * c;
        }
    }
    // the next `count` tokens.  Rows past them take the last one's values, which are finite where those are
    __device__ __forceinline__ void load(int count, bool reverse, uint32_t lds, int wave, int lane)
    {
        if (there == kAll && count == kChunk && whole) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) dma16_at(next, off[j], lds + 1024 * instruction(j, wave));
        } else {
            const char *base = next + (reverse ? (int64_t)(kChunk - count) * step : 0);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int i = instruction(j, wave);
                uint32_t at = off[j];
                if (count < kChunk) {
                    int r = row(i, lane);
                    r = r < count ? r : count - 1;
                    at = (uint32_t)(reverse ? count - 1 - r : r) * step + 16 * piece(i, lane);
                }
                if (which >> j & 1) dma16_at(base, at, lds + 1024 * i);
            }
        }
        next += advance;
    }
};

struct Two {
    float high, low;
};
// the same in all lanes: to a scalar register
__device__ __forceinline__ float uniform(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v))); }

template <typename T, int KT, int NW, bool OUT, bool RING>
__device__ __forceinline__ void decay_body(const DecayPass &p, int first)
{
    extern __shared__ __align__(16) char smem[];
    using S = DecayShape<T, KT, NW, OUT, RING>;
    using O = Ops<T>;
    using Frag = typename O::Frag;
    constexpr int threads = S::threads;
    // lambda^n, n = 0 .. 32; value_scale lambda^(31 - n), n = 0 .. 31; the same for the last chunk's tokens, and zeros behind them
    float *fade = reinterpret_cast<float *>(smem + S::stages * S::stage), *rising = fade + kChunk + 4, *ending = rising + kChunk;
    char *probs = smem + S::stages * S::stage + S::tables;       // the tile of probabilities of a chunk

    const int blocks = (p.dv + kDecayColumns - 1) / kDecayColumns;
    int at = first + (int)blockIdx.x;
    const int z = at % blocks;
    at /= blocks;
    const int seg = at % p.segments;
    at /= p.segments;
    const int b = at / p.heads, head = at % p.heads;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
    const Tokens tokens = tokens_of(p, b);
    const int begin = seg * p.seg_tokens;
    // the segment that has the last token (the first one where there is none)
    const bool final = OUT && (seg == 0 || begin < tokens.count) && tokens.count <= begin + p.seg_tokens;
    const int end = tokens.count < begin + p.seg_tokens ? tokens.count : begin + p.seg_tokens;
    if (OUT ? begin >= tokens.count && !final : begin + p.seg_tokens >= tokens.count) return;

    const T *gA = (const T *)p.A + (size_t)(head / p.share_a) * p.da, *gB = (const T *)p.B + (size_t)(head / p.share_b) * p.da;
    const T *gV = (const T *)p.V + (size_t)(head / p.share_v) * p.dv + z * kDecayColumns;
    const int vleft = p.dv - z * kDecayColumns;                  // columns of v from this workgroup's first on
    const int col = 16 * wave;                                   // this wavefront's first among them
    const int token_step = p.offset ? 1 : p.token_step;
    const bool reverse = p.reverse;
    auto row_of = [&](int t) { return (size_t)(tokens.first + (int64_t)(reverse ? tokens.count - 1 - t : t) * token_step); };

    // the quarter of the tile whose tokens j are behind all of its i
    if (OUT)
        for (int i = (int)threadIdx.x; i < S::tile / 16; i += threads) *reinterpret_cast<u32x4_t *>(probs + 16 * i) = u32x4_t{0u, 0u, 0u, 0u};
    // pieces behind a row's end are never loaded
    if (RING && (p.da % S::in_group || p.da < 32 * KT || vleft < S::columns)) {
        for (int i = (int)threadIdx.x; i < S::stages * S::stage / 16; i += threads) *reinterpret_cast<u32x4_t *>(smem + 16 * i) = u32x4_t{0u, 0u, 0u, 0u};
        __syncthreads();
    }
    RingSource<T, S::groups, NW> ring_a, ring_b;
    RingSource<T, S::groups_v, NW> ring_v;
    constexpr int kLoads = (OUT ? 2 : 1) * RingSource<T, S::groups, NW>::kPer + RingSource<T, S::groups_v, NW>::kPer;       // a stage, of a wavefront
    if (RING) {
        if (OUT) ring_a.init(gA, p.lda, tokens, token_step, begin, wave, lane, p.da, reverse);
        ring_b.init(gB, p.ldb, tokens, token_step, begin, wave, lane, p.da, reverse);
        ring_v.init(gV, p.ldv, tokens, token_step, begin, wave, lane, vleft < S::columns ? vleft : S::columns, reverse);
    }
    // or the next chunk on its way through registers: 8 elements of a row at a time
    constexpr int kPieces8 = 4 * KT, kPer = (kPieces8 * kChunk + threads - 1) / threads, kPerV = (kChunk * S::columns / 8 + threads - 1) / threads;
    Chunk<T> na[OUT && !RING ? kPer : 1], nb[RING ? 1 : kPer], nv[RING ? 1 : kPerV];
    auto lds_of = [&](int stage) { return (uint32_t)(uintptr_t)STL_LDS(smem) + stage * S::stage; };
    auto fetch = [&](int from, int stage) {
        const int count = end - from < kChunk ? end - from : kChunk;
        if constexpr (RING) {
            const uint32_t to = lds_of(stage);
            ring_b.load(count, reverse, to, wave, lane);
            ring_v.load(count, reverse, to + S::bytes, wave, lane);
            if (OUT) ring_a.load(count, reverse, to + S::bytes + S::bytes_v, wave, lane);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int unit = i * threads + (int)threadIdx.x, r = unit / kPieces8, u = unit % kPieces8, left = r < count ? p.da - 8 * u : 0;
                const size_t row = left > 0 ? row_of(from + r) : 0;
                if (OUT) na[i].load(gA + row * p.lda + 8 * u, left);
                nb[i].load(gB + row * p.ldb + 8 * u, left);
            }
#pragma unroll
            for (int i = 0; i < kPerV; ++i) {
                const int unit = i * threads + (int)threadIdx.x, r = unit / (S::columns / 8), u = unit % (S::columns / 8), left = r < count ? vleft - 8 * u : 0;
                nv[i].load(gV + (left > 0 ? row_of(from + r) : 0) * p.ldv + 8 * u, left);
            }
        }
    };
    const int chunks = end > begin ? (end - begin + kChunk - 1) / kChunk : 0;
#pragma unroll
    for (int c = 0; c < (RING ? S::stages - 1 : 1); ++c)
        if (c < chunks) fetch(begin + c * kChunk, c);

    double a = p.log_decay ? (double)p.log_decay[head] : 0.0;
    a = a < -1e5 ? -1e5 : a;
    for (int i = (int)threadIdx.x; i <= kChunk; i += threads) {
        const double exact = power(a, i);
        fade[i] = (float)exact;
        if (i < kChunk) {
            const float f = (float)(p.value_scale * exact);
            const int last = (end - begin - 1) % kChunk - i;      // (no chunk: nobody reads it)
            rising[kChunk - 1 - i] = f;
            if (last >= 0) ending[last] = f;
            else ending[kChunk + last] = 0.f;
        }
    }

    // the state, element e of tile t of 32 rows k: row 32 k + state_row(g, t, e), column n
    f32x4_t state[KT][2];
    const size_t each = (size_t)p.da * p.dv, state_at = ((size_t)b * p.heads + head) * each;
    const float *init = OUT ? p.init : nullptr;
    size_t init_at = state_at;
    int power_of_first = p.init_power;                           // of lambda, from the state to the next token
    if (OUT && p.segments > 1 && (seg > 0 || (init && p.last))) {
        init = p.starts;
        init_at = (((size_t)b * p.heads + head) * p.segments + (seg > 0 ? seg - 1 : p.segments - 1)) * each;
        if (seg > 0) power_of_first = 1;
    }
    // (loads of elements that there are not go to the last ones and are dropped: without a branch all of them are in flight at once)
    const int j = z * kDecayColumns + col + n, j_in = j < p.dv ? j : p.dv - 1;
    if (init) {
        const float *column = init + init_at + (size_t)j_in * (p.turned ? p.da : 1);
        const size_t step_i = p.turned ? 1 : p.dv;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int i = 32 * k + state_row(g, t, 0);
                if (p.turned && i + 4 <= p.da) {
                    state[k][t] = *reinterpret_cast<const f32x4_any_t *>(column + i);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) state[k][t][e] = column[(i + e < p.da ? i + e : p.da - 1) * step_i];
                }
            }
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) state[k][t][e] = 32 * k + state_row(g, t, e) < p.da && j < p.dv ? state[k][t][e] : 0.f;
    } else {
#pragma unroll
        for (int k = 0; k < KT; ++k) state[k][0] = state[k][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();

    // lambda to a chunk's tokens, in two numbers: of the first one (from the state on), of whole ones, and of the last one
    auto two = [&](int steps) {
        const double exact = power(a, steps);
        const float high = (float)exact;
        return Two{uniform(high), uniform((float)(exact - (double)high))};
    };
    const int last_count = chunks > 0 ? end - begin - (chunks - 1) * kChunk : 0;
    const Two through_first = two((chunks > 1 ? kChunk : last_count) - 1 + power_of_first), through = two(kChunk), through_last = two(last_count);
    // what does not change from chunk to chunk
    const typename O::Places places = O::places(lane);
    float near[4] = {};                                          // c lambda^(i - j) for this lane's i and j, 0 for j > i
    if (OUT && wave < 3) {
        const Quarter at(wave, lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int ago = at.i - at.j - e;
            near[e] = ago >= 0 ? p.out_scale * fade[ago >= 0 ? ago : 0] : 0.f;
        }
    }
    float since[2] = {};                                         // state_scale lambda^(tokens from the state to n and n + 16)
    if (OUT) since[0] = p.state_scale * fade[n + power_of_first], since[1] = p.state_scale * fade[n + 16 + power_of_first];
    // where this lane's outputs of the next chunk go (and those of 16 tokens on), and how many of its columns there are (none: no outputs); bit 0: in fp32,
    // bit 1: not all columns of the wavefront
    char *out_at = nullptr;
    int64_t out_advance = 0, out_half = 0;
    const int out_left = OUT && p.O ? vleft - col - 4 * g : 0;
    int out_kind = (p.out32 ? 1 : 0) | (p.O && vleft - col >= 16 ? 0 : 2);
    asm volatile("" : "+s"(out_kind));                           // (kept, and not read from the arguments again in each chunk)
    if (OUT && p.O) {
        const int64_t size = p.out32 ? 4 : (int64_t)sizeof(T), row = tokens.first + (int64_t)(reverse ? tokens.count - 1 - begin - n : begin + n) * token_step;
        out_at = (char *)p.O + (row * (int64_t)p.ldo + (int64_t)head * p.dv + z * kDecayColumns + col + 4 * g) * size;
        out_advance = (reverse ? -kChunk : kChunk) * token_step * (int64_t)p.ldo * size, out_half = out_advance / 2;
    }
    // What the roundings of a chunk's lambda to fp32 have left out: made good by the next ones.  What the last one leaves out would have the same sign in call after call of
    // few tokens (8 a call, 20000 of them: a state off by 3e-5), so it begins anywhere within half a step of the first product, by the state's own bits, and is nothing in
    // the mean.  (Formed with two numbers, in the last chunk or where the state comes in, the product costs 1 to 8 % of a sweep or 4 to 12 registers that are not there.)
    uint32_t mixed = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) mixed ^= __float_as_uint(state[0][e >> 2][e & 3]);
    float owed = OUT ? (float)(int32_t)(mixed * 0x9e3779b1u) * 0x1p-56f * through_first.high : 0.f;

    int stage = 0;
    for (int c = 0; c < chunks; ++c) {
        const int from = begin + c * kChunk, count = end - from < kChunk ? end - from : kChunk;
        if constexpr (RING) {
            // this chunk's loads are done (younger ones: those of the stages - 2 chunks behind it, and outputs), everybody's after the barrier, where everybody is
            // also done with the chunk before, whose stage takes the next loads
            if (c + S::stages - 1 <= chunks) wait_all_but<kLoads *(S::stages - 2)>();
            else wait_all_but<0>();
            pipe::block_barrier();
            if (c + S::stages - 1 < chunks) fetch(from + (S::stages - 1) * kChunk, stage > 0 ? stage - 1 : S::stages - 1);
        } else {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int unit = i * threads + (int)threadIdx.x, r = unit / kPieces8, u = unit % kPieces8;
                if (kPieces8 * kChunk % threads && unit >= kPieces8 * kChunk) break;
                put8(smem, r, u, nb[i]);
                if (OUT) put8(smem + S::bytes + S::bytes_v, r, u, na[i]);
            }
#pragma unroll
            for (int i = 0; i < kPerV; ++i) {
                const int unit = i * threads + (int)threadIdx.x;
                put8(smem + S::bytes, unit / (S::columns / 8), unit % (S::columns / 8), nv[i]);
            }
            __syncthreads();
            if (c + 1 < chunks) fetch(from + kChunk, 0);
        }
        const char *lB = smem + stage * S::stage, *lV = lB + S::bytes, *lA = lV + S::bytes_v;

        Frag values = O::across(lV, places, wave);
        const bool unclean = __ballot(!O::finite(values)) != 0;
        int bad = kChunk;                                        // the first token whose value in this lane's column is no finite number
        if (unclean) {
            bad = O::clean(values, g);
            for (int m = 16; m < 64; m *= 2) {
                const int other = __shfl_xor(bad, m);
                bad = other < bad ? other : bad;
            }
        }
        const Two by = c == 0 ? through_first : c + 1 == chunks ? through_last : through;
        const float low = by.low + owed, fall = by.high + low;
        owed = low - (fall - by.high);
        const float *weight = count < kChunk ? ending : rising;
        // all products of a chunk in one piece of straight code, so that vector and matrix instructions overlap (the state behind the last token too, which
        // is not always needed)
        f32x4_t out[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};                       // of tokens n and n + 16
        if (OUT) {
            if (wave < 3) O::template quarter<KT>(lA, lB, wave, lane, near, probs);
            Frag q[2][2] = {{O::along(lA, places, 0, 0), O::along(lA, places, 0, 1)}};       // (operands are read a step ahead)
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                if (k + 1 < KT) q[k + 1 & 1][0] = O::along(lA, places, k + 1, 0), q[k + 1 & 1][1] = O::along(lA, places, k + 1, 1);
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = state[k][e >> 2][e & 3];
#pragma unroll
                for (int m = 0; m < O::kOutParts; ++m) {
                    const Frag part = O::part(x);
                    out[0] = O::mma(part, q[k & 1][0], out[0]);
                    out[1] = O::mma(part, q[k & 1][1], out[1]);
                }
            }
            out[0] *= since[0], out[1] *= since[1];
            wait_lds();
            pipe::block_barrier();
#pragma unroll
            for (int m = 0; m < O::kOutParts; ++m)
#pragma unroll
                for (int half = 0; half < 2; ++half) out[half] = O::mma(values, O::probabilities(probs, places, m, half), out[half]);
        }
        float x[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4_t left = *reinterpret_cast<const f32x4_t *>(weight + 8 * g + 4 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = O::get(values, 4 * i + e) * left[e];
        }
        Frag parts[O::kStateParts];
#pragma unroll
        for (int m = 0; m < O::kStateParts; ++m) parts[m] = O::part(x);
        Frag key[2] = {O::across(lB, places, 0)};
#pragma unroll
        for (int c = 0; c < 2 * KT; ++c) {
            if (c + 1 < 2 * KT) key[c + 1 & 1] = O::across(lB, places, c + 1);
            f32x4_t &tile = state[c >> 1][c & 1];
            tile *= fall;
#pragma unroll
            for (int m = 0; m < O::kStateParts; ++m) tile = O::mma(key[c & 1], parts[m], tile);
        }
        if (unclean) {
            const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int first = __shfl(bad, 4 * g + e);
                if (n >= first) out[0][e] = nan;
                if (n + 16 >= first) out[1][e] = nan;
            }
            if (bad < kChunk)
#pragma unroll
                for (int k = 0; k < KT; ++k) state[k][0] = state[k][1] = f32x4_t{nan, nan, nan, nan};
        }
        if (OUT)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (n + 16 * half >= count) continue;
                char *to = out_at + (half ? out_half : 0);
                if (out_kind == 0) put4((T *)to, 4, out[half]);
                else if (out_kind == 1) put4((float *)to, 4, out[half]);
                else if (out_kind == 2) put4((T *)to, out_left, out[half]);
                else put4((float *)to, out_left, out[half]);
            }
        if (OUT) out_at += out_advance;
        if (OUT && !power_of_first) since[0] = p.state_scale * fade[n + 1], since[1] = p.state_scale * fade[n + 17];
        power_of_first = 1;
        if (RING) stage = stage + 1 < S::stages ? stage + 1 : 0;
    }
    if (OUT ? final && p.last : true) {
        float *to = OUT ? p.last + state_at : p.starts + (((size_t)b * p.heads + head) * p.segments + seg) * each;
        const float by = OUT ? (float)(tokens.count > 0 ? power(a, p.last_power) : 1.0) : 1.f;
        float *column = to + j * (p.turned ? p.da : 1);
        const size_t step_i = p.turned ? 1 : p.dv;
        if (j < p.dv)
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = 32 * k + state_row(g, e >> 2, e & 3);
                    if (i < p.da) column[i * step_i] = by * state[k][e >> 2][e & 3];
                }
    }
}

// sweeps of the same widths, one beside the other (blockIdx.y)
constexpr int kMostSweeps = 3;
struct DecaySweeps {
    DecayPass pass[kMostSweeps];
    int count, first;                        // (first: the number of a launch's first workgroup)
};
template <typename T, int KT, int NW, bool OUT, bool RING>
__global__ __launch_bounds__(64 * NW, decay_waves(sizeof(T), KT)) void decay_kernel(const DecaySweeps s)
{
    decay_body<T, KT, NW, OUT, RING>(s.pass[blockIdx.y], s.first);
}

template <typename T, int KT, int NW, bool OUT, bool RING>
hipError_t launch_shape(const DecaySweeps &sw, hipStream_t s)
{
    using S = DecayShape<T, KT, NW, OUT, RING>;
    static std::atomic<uint64_t> granted{0};
    const DecayPass &p = sw.pass[0];
    const int blocks = (p.dv + kDecayColumns - 1) / kDecayColumns;
    const hipError_t e = allow_lds((const void *)decay_kernel<T, KT, NW, OUT, RING>, S::lds, S::lds, granted);
    if (e != hipSuccess) return e;
    // (a dimension's threads have to fit into 32 bits: at most half as many a launch)
    constexpr int kMost = (int)((1u << 31) / S::threads);
    DecaySweeps part = sw;
    for (int all = p.sequences * p.heads * p.segments * blocks, at = 0; at < all; at += kMost) {
        part.first = at;
        hipLaunchKernelGGL((decay_kernel<T, KT, NW, OUT, RING>), dim3(all - at < kMost ? all - at : kMost, sw.count), dim3(S::threads), S::lds, s, part);
        const hipError_t launched = hipGetLastError();
        if (launched != hipSuccess) return launched;
    }
    return hipSuccess;
}

inline int key_tiles(int da) { return da <= 128 ? (da + 31) / 32 : 8; }
inline int value_waves(int dv) { return dv <= 64 ? 4 : 8; }

// sweeps with the same key_tiles, value_waves, blocks of columns, segments and kind of rows
template <typename T, bool OUT>
hipError_t decay_sweeps(const DecaySweeps &sw, hipStream_t s)
{
    const int tiles = key_tiles(sw.pass[0].da), waves = value_waves(sw.pass[0].dv);
    constexpr bool wide = sizeof(T) == 2;                        // fp32: a ring of rows of 256 does not fit
    if (!sw.pass[0].ring || (!wide && tiles == 8)) {
        if (tiles == 8) return launch_shape<T, 8, 8, OUT, false>(sw, s);
        return tiles > 2 ? launch_shape<T, 4, 8, OUT, false>(sw, s) : launch_shape<T, 2, 8, OUT, false>(sw, s);
    }
    auto ring = [&](auto nw) {
        constexpr int NW = decltype(nw)::value;
        if constexpr (wide)
            if (tiles == 8) return launch_shape<T, 8, NW, OUT, true>(sw, s);
        if (tiles == 4) return launch_shape<T, 4, NW, OUT, true>(sw, s);
        if (tiles == 3) return launch_shape<T, 3, NW, OUT, true>(sw, s);
        return tiles == 2 ? launch_shape<T, 2, NW, OUT, true>(sw, s) : launch_shape<T, 1, NW, OUT, true>(sw, s);
    };
    return waves == 4 ? ring(std::integral_constant<int, 4>()) : ring(std::integral_constant<int, 8>());
}
// seq_decay_bf16.hip, seq_decay_f32.hip; seq_decay_states_*.hip: what segments add to the state
hipError_t decay_sweeps_bf16(const DecaySweeps &sw, hipStream_t s);
hipError_t decay_sweeps_f32(const DecaySweeps &sw, hipStream_t s);
hipError_t decay_states_bf16(const DecaySweeps &sw, hipStream_t s);
hipError_t decay_states_f32(const DecaySweeps &sw, hipStream_t s);

}  // namespace seq
}  // namespace stl
