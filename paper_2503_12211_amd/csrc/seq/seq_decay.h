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
// segment (decay_join_kernel), and all segments run at once.  That reads K and V twice (from the last-level cache, if they fit there).  A wavefront owns 32 columns of v: its part of S
// stays in accumulators (dk x 32, fp32) all along.  Products are formed so that accumulators are the next product's operand as they lie:
//   P^T = K Q^T (tokens j x i)   ->   O^T += V^T P^T,      S (dk x columns) as S^T in   O^T = S^T Q^T
// An accumulator's lane holds rows 8 (e / 4) + 4 h + e % 4 of its column (h = lane / 32), an operand's lane eight elements of the contraction, whose
// order is free as long as both operands have it: the contraction goes in the accumulators' order, and Q and K lie in LDS with the middle two of every
// four groups of four elements exchanged, so that a lane still reads 16 bytes at once.
//
// bf16 storage: operands that come from fp32 (P, S, V scaled by the decay up to the chunk's end) are given to the matrix cores as sums of bf16 numbers, two of
// them (a relative error of 2^-16) for what goes into outputs that are rounded to bf16, three (2^-24) for what goes into the fp32 state.  With one, P's
// and S's roundings would each be as large as the output's own.  fp32 storage: fp32 matrix instructions.
#pragma once
#include "seq_kernels.h"
#include "../lm/lm_device.h"

#include <atomic>

namespace stl {
namespace seq {

using lm::Chunk;
typedef short v4i16_t __attribute__((ext_vector_type(4)));
#define SEQ_LDS(p) ((__attribute__((address_space(3))) char *)(p))

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
    float out_scale;
    const float *log_decay;
    const int64_t *offset;
    // states lie [sequence][head][da][dv], or [dv][da] (turned).  The first is multiplied by init_scale and, for the first token, lambda^init_power (1 forward in
    // time, 0 backward, where what is given belongs to the last token itself); the last by last_scale lambda^last_power.
    const float *init;
    float *last;
    bool turned;
    float init_scale, last_scale;
    int init_power, last_power;
    // segments of seg_tokens (a multiple of 32).  starts [sequence][head][segments][da dv]: number s holds what segment s adds to the state, and behind decay_join_kernel
    // the state in front of segment s + 1; the last one `init` as it was, where the last state may be written over it.
    int segments, seg_tokens;
    float *starts;
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

// lambda^n, a not below -100000 (where it is 0 for every n > 0)
__device__ __forceinline__ double power(double a, int n) { return n == 0 ? 1.0 : exp(a * n); }

template <typename T> struct Ops;

template <> struct Ops<bf16_t> {
    static constexpr int kPad = 8, kOutParts = 2, kStateParts = 3;
    // operand for a contraction of 32 in the accumulators' order
    struct Frag {
        bf16x8_t f[2];
    };
    static __device__ __forceinline__ f32x16_t mma(const Frag &a, const Frag &b, f32x16_t c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.f[0], b.f[0], c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.f[1], b.f[1], c, 0, 0, 0);
    }
    // contraction along a row of LDS (rows as put() leaves them), p at the row's 32 elements
    static __device__ __forceinline__ Frag along(const bf16_t *p, int h)
    {
        Frag r;
        r.f[0] = *reinterpret_cast<const bf16x8_t *>(p + 8 * h);
        r.f[1] = *reinterpret_cast<const bf16x8_t *>(p + 16 + 8 * h);
        return r;
    }
    // contraction over 32 rows of LDS, the lane's column of the 32 from p on; PUT: rows as put() leaves them
    template <bool PUT>
    static __device__ __forceinline__ Frag across(const bf16_t *p, int stride, int lane)
    {
        const int h = lane >> 5, q = lane & 15, piece = PUT ? (q & 3) == 1 ? 2 : (q & 3) == 2 ? 1 : q & 3 : q & 3;
        const bf16_t *at = p + (4 * h + (q >> 2)) * stride + 16 * (lane >> 4 & 1) + 4 * piece;
        struct { v4i16_t lo, hi; } two[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            two[b].lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t *)SEQ_LDS((char *)(at + 16 * b * stride)));
            two[b].hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t *)SEQ_LDS((char *)(at + (16 * b + 8) * stride)));
        }
        return Frag{{__builtin_bit_cast(bf16x8_t, two[0]), __builtin_bit_cast(bf16x8_t, two[1])}};
    }
    // sixteen elements of a row on their way to LDS: groups of four in the order 0 2 1 3
    static __device__ __forceinline__ void put(bf16_t *p, const Chunk<bf16_t> &a, const Chunk<bf16_t> &b)
    {
        *reinterpret_cast<u32x4_t *>(p) = u32x4_t{a.v[0], a.v[1], b.v[0], b.v[1]};
        *reinterpret_cast<u32x4_t *>(p + 8) = u32x4_t{a.v[2], a.v[3], b.v[2], b.v[3]};
    }
    static __device__ __forceinline__ void put_plain(bf16_t *p, const Chunk<bf16_t> &a) { *reinterpret_cast<u32x4_t *>(p) = a.v; }
    static __device__ __forceinline__ bool finite(const Chunk<bf16_t> &a)
    {
        bool ok = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) ok &= (a.v[i] & 0x7f80u) != 0x7f80u && (a.v[i] & 0x7f800000u) != 0x7f800000u;
        return ok;
    }
    // the sum of N operands, the last of them rounded
    template <int N>
    static __device__ __forceinline__ void split(const float *x, Frag *out)
    {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t w[N][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float u = x[8 * b + 2 * k], v = x[8 * b + 2 * k + 1];
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    w[n][k] = pack_bf16x2(u, v);
                    u -= __uint_as_float(w[n][k] << 16);
                    v -= __uint_as_float(w[n][k] & 0xffff0000u);
                }
            }
#pragma unroll
            for (int n = 0; n < N; ++n) out[n].f[b] = __builtin_bit_cast(bf16x8_t, u32x4_t{w[n][0], w[n][1], w[n][2], w[n][3]});
        }
    }
    static __device__ __forceinline__ float get(const Frag &a, int e)
    {
        const u32x4_t w = __builtin_bit_cast(u32x4_t, a.f[e >> 3]);
        return __uint_as_float(e & 1 ? w[e >> 1 & 3] & 0xffff0000u : w[e >> 1 & 3] << 16);
    }
};

template <> struct Ops<float> {
    static constexpr int kPad = 4, kOutParts = 1, kStateParts = 1;
    struct Frag {
        float f[16];
    };
    static __device__ __forceinline__ f32x16_t mma(const Frag &a, const Frag &b, f32x16_t c)
    {
#pragma unroll
        for (int e = 0; e < 16; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.f[e], b.f[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ Frag along(const float *p, int h)
    {
        Frag r;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t *>(p + 8 * g + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) r.f[4 * g + e] = v[e];
        }
        return r;
    }
    template <bool PUT>
    static __device__ __forceinline__ Frag across(const float *p, int stride, int lane)
    {
        Frag r;
#pragma unroll
        for (int e = 0; e < 16; ++e) r.f[e] = p[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * stride + (lane & 31)];
        return r;
    }
    static __device__ __forceinline__ void put(float *p, const Chunk<float> &a, const Chunk<float> &b)
    {
        put_plain(p, a);
        put_plain(p + 8, b);
    }
    static __device__ __forceinline__ void put_plain(float *p, const Chunk<float> &a)
    {
        *reinterpret_cast<f32x4_t *>(p) = a.a;
        *reinterpret_cast<f32x4_t *>(p + 4) = a.b;
    }
    static __device__ __forceinline__ bool finite(const Chunk<float> &a)
    {
        bool ok = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) ok &= (__float_as_uint(a.get(e)) & 0x7f800000u) != 0x7f800000u;
        return ok;
    }
    template <int N>
    static __device__ __forceinline__ void split(const float *x, Frag *out)
    {
#pragma unroll
        for (int e = 0; e < 16; ++e) out[0].f[e] = x[e];
    }
    static __device__ __forceinline__ float get(const Frag &a, int e) { return a.f[e]; }
};

// a lane's row within 32 of accumulator element e
__device__ __forceinline__ int acc_row(int e, int h) { return 8 * (e >> 2) + 4 * h + (e & 3); }

constexpr int kDecayColumns = 128;           // of v, of a workgroup, 32 a wavefront
constexpr int kChunk = 32;
template <typename T, int KT, int NW>        // 32 KT: width of queries and keys in LDS; NW wavefronts
struct DecayShape {
    static constexpr int columns = 32 * NW, ld = 32 * KT + Ops<T>::kPad, ldv = columns + Ops<T>::kPad;
    static constexpr int lds(bool outputs) { return (((outputs ? 2 : 1) * ld + ldv) * kChunk * (int)sizeof(T) + 15) / 16 * 16 + (kChunk + 1) * 4 + 8; }
};
// 256 registers, two workgroups a CU, where a wavefront's state and the next chunk fit
constexpr int decay_waves(size_t element, int KT) { return element == 2 && KT <= 4 ? 2 : 1; }

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

// OUT: with outputs; without, what a segment adds to the state
template <typename T, int KT, int NW, bool OUT>
__device__ __forceinline__ void decay_body(const DecayPass &p)
{
    extern __shared__ __align__(16) char smem[];
    using S = DecayShape<T, KT, NW>;
    using O = Ops<T>;
    using Frag = typename O::Frag;
    constexpr int ld = S::ld, ldv = S::ldv, threads = 64 * NW;
    T *lB = reinterpret_cast<T *>(smem), *lV = lB + kChunk * ld, *lA = lV + kChunk * ldv;
    float *fade = reinterpret_cast<float *>(smem + S::lds(OUT) - (kChunk + 1) * 4 - 8);      // lambda^n, n = 0 .. 32
    int *bad = reinterpret_cast<int *>(fade + kChunk + 1);

    const int blocks = (p.dv + kDecayColumns - 1) / kDecayColumns;
    int at = (int)blockIdx.x;
    const int z = at % blocks;
    at /= blocks;
    const int seg = at % p.segments;
    at /= p.segments;
    const int b = at / p.heads, head = at % p.heads;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
    const Tokens tokens = tokens_of(p, b);
    const int begin = seg * p.seg_tokens;
    // the segment that has the last token (the first one where there is none)
    const bool final = OUT && (seg == 0 || begin < tokens.count) && tokens.count <= begin + p.seg_tokens;
    const int end = tokens.count < begin + p.seg_tokens ? tokens.count : begin + p.seg_tokens;
    if (OUT ? begin >= tokens.count && !final : begin + p.seg_tokens >= tokens.count) return;

    const T *gA = (const T *)p.A + (size_t)(head / p.share_a) * p.da, *gB = (const T *)p.B + (size_t)(head / p.share_b) * p.da;
    const T *gV = (const T *)p.V + (size_t)(head / p.share_v) * p.dv + z * kDecayColumns;
    const int vleft = p.dv - z * kDecayColumns;                  // columns of v from this workgroup's first on
    const int col = 32 * wave;                                   // this wavefront's first among them
    auto row_of = [&](int t) { return (size_t)(tokens.first + (int64_t)(p.reverse ? tokens.count - 1 - t : t) * (p.offset ? 1 : p.token_step)); };

    double a = p.log_decay ? (double)p.log_decay[head] : 0.0;
    a = a < -1e5 ? -1e5 : a;
    if (threadIdx.x <= kChunk) fade[threadIdx.x] = (float)power(a, (int)threadIdx.x);
    if (threadIdx.x == 0) bad[0] = bad[1] = 0;
    const double whole = power(a, kChunk);

    // the state, element e of tile k: row 32 k + acc_row(e), column n
    f32x16_t state[KT];
    const size_t each = (size_t)p.da * p.dv, state_at = ((size_t)b * p.heads + head) * each;
    const float *init = p.init;
    float init_scale = p.init_scale;
    size_t init_at = state_at;
    int power_of_first = p.init_power;                           // of lambda, from the state to the next token
    if (!OUT) init = nullptr;
    if (OUT && p.segments > 1 && (seg > 0 || (init && p.last))) {
        init = p.starts;
        init_at = (((size_t)b * p.heads + head) * p.segments + (seg > 0 ? seg - 1 : p.segments - 1)) * each;
        if (seg > 0) init_scale = 1.f, power_of_first = 1;
    }
    auto at_state = [&](int k, int e) {
        const int i = 32 * k + acc_row(e, h), j = z * kDecayColumns + col + n;
        return i < p.da && j < p.dv ? (p.turned ? j * p.da + i : i * p.dv + j) : -1;
    };
#pragma unroll
    for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = init ? at_state(k, e) : -1;
            state[k][e] = i >= 0 ? init_scale * init[init_at + i] : 0.f;
        }
    bool any = init != nullptr;                                  // whether the state may differ from zero

    // the next chunk on its way: 16 elements of a row of A and of B, 8 of V at a time
    constexpr int kUnits = 2 * KT * kChunk, kPer = (kUnits + threads - 1) / threads, kPerV = kChunk * S::columns / 8 / threads;
    Chunk<T> na[OUT ? kPer : 1][2], nb[kPer][2], nv[kPerV];
    auto fetch = [&](int from, int count) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int unit = i * threads + (int)threadIdx.x, r = unit / (2 * KT), u = unit % (2 * KT), left = r < count ? p.da - 16 * u : 0;
            const size_t row = left > 0 ? row_of(from + r) : 0;
            if (OUT) {
                na[i][0].load(gA + row * p.lda + 16 * u, left);
                na[i][1].load(gA + row * p.lda + 16 * u + 8, left - 8);
            }
            nb[i][0].load(gB + row * p.ldb + 16 * u, left);
            nb[i][1].load(gB + row * p.ldb + 16 * u + 8, left - 8);
        }
#pragma unroll
        for (int i = 0; i < kPerV; ++i) {
            const int unit = i * threads + (int)threadIdx.x, r = unit / (S::columns / 8), u = unit % (S::columns / 8), left = r < count ? vleft - 8 * u : 0;
            nv[i].load(gV + (left > 0 ? row_of(from + r) : 0) * p.ldv + 8 * u, left);
        }
    };

    int from = begin, count = end - from < kChunk ? end - from : kChunk, turn = 0, singles = 0;
    if (count > 0) fetch(from, count);
    while (count > 0) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int unit = i * threads + (int)threadIdx.x, r = unit / (2 * KT), u = unit % (2 * KT);
            if (kUnits % threads && unit >= kUnits) break;
            if (OUT) O::put(lA + r * ld + 16 * u, na[i][0], na[i][1]);
            O::put(lB + r * ld + 16 * u, nb[i][0], nb[i][1]);
        }
        bool ok = true;
#pragma unroll
        for (int i = 0; i < kPerV; ++i) {
            const int unit = i * threads + (int)threadIdx.x, r = unit / (S::columns / 8), u = unit % (S::columns / 8);
            ok &= O::finite(nv[i]);
            O::put_plain(lV + r * ldv + 8 * u, nv[i]);
        }
        if (!ok) bad[turn] = 1;
        __syncthreads();
        // A value that is no finite number must not reach earlier tokens, as it would with a zero of the masked P: a chunk with one goes token by token.
        const bool again = bad[turn] && count > 1;
        if (threadIdx.x == 0) bad[turn ^ 1] = 0;
        turn ^= 1;
        if (again) singles = from + count;
        const int next = again ? from : from + count;
        int next_count = end - next < kChunk ? end - next : kChunk;
        if (next < singles) next_count = 1;
        if (next_count > 0) fetch(next, next_count);
        if (!again) {
            if (OUT && p.O) {
                Frag q[KT];
#pragma unroll
                for (int k = 0; k < KT; ++k) q[k] = O::along(lA + n * ld + 32 * k, h);
                f32x16_t out = {};
                if (any) {
#pragma unroll
                    for (int k = 0; k < KT; ++k) {
                        float x[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = state[k][e];
                        Frag parts[O::kOutParts];
                        O::template split<O::kOutParts>(x, parts);
#pragma unroll
                        for (int m = 0; m < O::kOutParts; ++m) out = O::mma(parts[m], q[k], out);
                    }
                    out *= fade[n + (power_of_first ? 1 : 0)];
                }
                f32x16_t prob = {};
#pragma unroll
                for (int k = 0; k < KT; ++k) prob = O::mma(O::along(lB + n * ld + 32 * k, h), q[k], prob);
                float x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int ago = n - acc_row(e, h);
                    x[e] = ago >= 0 ? prob[e] * fade[ago >= 0 ? ago : 0] : 0.f;
                }
                Frag parts[O::kOutParts];
                O::template split<O::kOutParts>(x, parts);
                const Frag v = O::template across<false>(lV + col, ldv, lane);
#pragma unroll
                for (int m = 0; m < O::kOutParts; ++m) out = O::mma(v, parts[m], out);
                if (n < count) {
                    const size_t row = row_of(from + n);
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int c = col + 8 * g + 4 * h, left = vleft - c;
                        f32x4_t w = {out[4 * g], out[4 * g + 1], out[4 * g + 2], out[4 * g + 3]};
                        w *= p.out_scale;
                        const size_t to = row * p.ldo + (size_t)head * p.dv + z * kDecayColumns + c;
                        if (p.out32) put4((float *)p.O + to, left, w);
                        else put4((T *)p.O + to, left, w);
                    }
                }
            }
            // the state behind the chunk's last token (not needed behind the sequence's last one if nobody asks for it)
            if (!OUT || next < end || (final && p.last)) {
                const int steps = count - 1 + power_of_first;
                const double fall = steps == kChunk ? whole : power(a, steps);
                const float fall_hi = (float)fall, fall_lo = (float)(fall - (double)fall_hi);
                if (any)
#pragma unroll
                    for (int k = 0; k < KT; ++k)
#pragma unroll
                        for (int e = 0; e < 16; ++e) state[k][e] = fmaf(state[k][e], fall_hi, state[k][e] * fall_lo);
                const Frag v = O::template across<false>(lV + col, ldv, lane);
                float x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int left = count - 1 - acc_row(e, h);
                    x[e] = left >= 0 ? O::get(v, e) * fade[left >= 0 ? left : 0] : 0.f;
                }
                Frag parts[O::kStateParts];
                O::template split<O::kStateParts>(x, parts);
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    const Frag key = O::template across<true>(lB + 32 * k, ld, lane);
#pragma unroll
                    for (int m = 0; m < O::kStateParts; ++m) state[k] = O::mma(key, parts[m], state[k]);
                }
                any = true;
            }
            power_of_first = 1;
        }
        from = next;
        count = next_count;
    }
    if (OUT ? final && p.last : true) {
        float *to = OUT ? p.last + state_at : p.starts + (((size_t)b * p.heads + head) * p.segments + seg) * each;
        const float by = OUT ? (float)(p.last_scale * (tokens.count > 0 ? power(a, p.last_power) : 1.0)) : 1.f;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = at_state(k, e);
                if (i >= 0) to[i] = by * state[k][e];
            }
    }
}

// sweeps of the same widths, one beside the other (blockIdx.y)
constexpr int kMostSweeps = 3;
struct DecaySweeps {
    DecayPass pass[kMostSweeps];
    int count;
};
template <typename T, int KT, int NW, bool OUT>
__global__ __launch_bounds__(64 * NW, decay_waves(sizeof(T), KT)) void decay_kernel(const DecaySweeps s)
{
    decay_body<T, KT, NW, OUT>(s.pass[blockIdx.y]);
}

template <typename T, int KT, int NW>
hipError_t launch_shape(const DecaySweeps &sw, bool outputs, hipStream_t s)
{
    using S = DecayShape<T, KT, NW>;
    static std::atomic<uint64_t> granted[2];
    const DecayPass &p = sw.pass[0];
    const int blocks = (p.dv + kDecayColumns - 1) / kDecayColumns, bytes = S::lds(outputs);
    const hipError_t e = allow_lds(outputs ? (const void *)decay_kernel<T, KT, NW, true> : (const void *)decay_kernel<T, KT, NW, false>, bytes, bytes, granted[outputs]);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((size_t)p.sequences * p.heads * p.segments * blocks), sw.count);
    if (outputs) hipLaunchKernelGGL((decay_kernel<T, KT, NW, true>), grid, dim3(64 * NW), bytes, s, sw);
    else hipLaunchKernelGGL((decay_kernel<T, KT, NW, false>), grid, dim3(64 * NW), bytes, s, sw);
    return hipGetLastError();
}

inline int key_tiles(int da) { return da <= 32 ? 1 : da <= 64 ? 2 : da <= 128 ? 4 : 8; }
inline int value_waves(int dv) { return dv <= 64 ? 2 : 4; }

// sweeps with the same key_tiles, value_waves, blocks of columns and segments
template <typename T>
hipError_t decay_sweeps(const DecaySweeps &sw, bool outputs, hipStream_t s)
{
    auto wide = [&](auto nw) {
        switch (key_tiles(sw.pass[0].da)) {
        case 1: return launch_shape<T, 1, decltype(nw)::value>(sw, outputs, s);
        case 2: return launch_shape<T, 2, decltype(nw)::value>(sw, outputs, s);
        case 4: return launch_shape<T, 4, decltype(nw)::value>(sw, outputs, s);
        }
        return launch_shape<T, 8, decltype(nw)::value>(sw, outputs, s);
    };
    return value_waves(sw.pass[0].dv) == 2 ? wide(std::integral_constant<int, 2>()) : wide(std::integral_constant<int, 4>());
}
hipError_t decay_sweeps_bf16(const DecaySweeps &sw, bool outputs, hipStream_t s);   // seq_decay_bf16.hip
hipError_t decay_sweeps_f32(const DecaySweeps &sw, bool outputs, hipStream_t s);    // seq_decay_f32.hip

}  // namespace seq
}  // namespace stl
