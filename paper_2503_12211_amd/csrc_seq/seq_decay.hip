// Attention with decay: what the forward and the backward call make of the sweeps, single tokens, and the small kernels around.
#include "seq_decay.h"

namespace stl {
namespace seq {

// Up to so many tokens a sequence go one by one, with the state in registers (decay_few_kernel): a sweep's chunk is 32 tokens whatever it holds.  6 tokens, in
// brackets as a sweep, us of a call among others: 64 sequences x 32 heads of 128: 76 (75); 8 x 32 of 128: 14 (12.5); 1 x 32 of 128: 8 (10); 8 tokens: 86 (75.5), 17 (12.5),
// 9 (10); 4 tokens one by one: 67, 11.6, 8.
constexpr int kFewTokens = 6;

// A few tokens: memory bound by the state, which is read once and written once (64 tokens x 32 heads of 128: 268 MB in 53 us, 5.1 TB/s, the rate of a copy; one token of
// 8 heads of 64: 4 us, a launch).  A thread has four columns of every RG-th row (RG: groups of COLS / 4 threads), RPT
// rows; for each token q and k go through LDS, o is the sum over the rows: lanes, then wavefronts.
template <typename T, int COLS, int RPT>
__global__ __launch_bounds__(256) void decay_few_kernel(const DecayArgs a, T *O, float *state_out)
{
    constexpr int LC = COLS / 4, RG = 256 / LC;
    __shared__ float lq[kDecayWidest], lk[kDecayWidest];
    __shared__ __align__(16) float sums[4][COLS];
    const int blocks = (a.dv + COLS - 1) / COLS, z = (int)blockIdx.x % blocks, bh = (int)blockIdx.x / blocks, b = bh / a.heads, head = bh % a.heads;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, col = z * COLS + 4 * (tid % LC), group = tid / LC, left = a.dv - col;
    DecayPass p{};
    p.rows = a.rows, p.length = a.length, p.seq_step = a.seq_step, p.offset = a.offset;
    const Tokens tokens = tokens_of(p, b);
    const size_t at = (size_t)bh * a.dk * a.dv;
    f32x4_t state[RPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
        const int i = r * RG + group;
        state[r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (a.state && i < a.dk) state[r] = load4(a.state + at + (size_t)i * a.dv + col, left);
    }
    double fall = a.log_decay ? (double)a.log_decay[head] : 0.0;
    fall = power(fall < -1e5 ? -1e5 : fall, 1);
    // lambda in two numbers: its rounding to fp32 has the same sign at every token, and thousands of calls would add it up (3000 tokens: a state off by 7e-5)
    const float by = (float)fall, rest = (float)(fall - (double)by);
    const int share = a.heads / a.kv_heads;
    for (int t = 0; t < tokens.count; ++t) {
        const size_t row = (size_t)(tokens.first + (int64_t)t * (a.offset ? 1 : a.token_step));
        if (tid < a.dk) {
            lq[tid] = a.scale * Elem<T>::ld((const T *)a.Q + row * a.ld_q + (size_t)head * a.dk + tid);
            lk[tid] = Elem<T>::ld((const T *)a.K + row * a.ld_k + (size_t)(head / share) * a.dk + tid);
        }
        const f32x4_t v = load4((const T *)a.V + row * a.ld_v + (size_t)(head / share) * a.dv + col, left);
        __syncthreads();
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            const int i = r * RG + group;
            const float k = lk[i], q = lq[i];                    // (there is LDS behind the last row too, and any value does)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                state[r][e] = fmaf(state[r][e], by, fmaf(state[r][e], rest, k * v[e]));
                sum[e] = i < a.dk ? fmaf(q, state[r][e], sum[e]) : sum[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            for (int n = LC; n < 64; n *= 2) sum[e] += __shfl_xor(sum[e], n);
        if (lane < LC) *reinterpret_cast<f32x4_t *>(&sums[wave][4 * lane]) = sum;
        __syncthreads();
        if (tid < COLS && z * COLS + tid < a.dv)
            Elem<T>::st(O + row * a.ld_o + (size_t)head * a.dv + z * COLS + tid, (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]));
    }
    if (!state_out || (tokens.count == 0 && state_out == a.state)) return;
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
        const int i = r * RG + group;
        if (i < a.dk) put4(state_out + at + (size_t)i * a.dv + col, left, state[r]);
    }
}

template <typename T, int COLS>
hipError_t few_tokens(const DecayArgs &a, void *O, float *state_out, hipStream_t s)
{
    constexpr int RG = 256 / (COLS / 4);
    const dim3 grid((unsigned)((size_t)a.sequences * a.heads * ((a.dv + COLS - 1) / COLS)));
    const int each = (a.dk + RG - 1) / RG;
    if (each <= 64 / RG) hipLaunchKernelGGL((decay_few_kernel<T, COLS, 64 / RG>), grid, dim3(256), 0, s, a, (T *)O, state_out);
    else if (each <= 128 / RG) hipLaunchKernelGGL((decay_few_kernel<T, COLS, 128 / RG>), grid, dim3(256), 0, s, a, (T *)O, state_out);
    else hipLaunchKernelGGL((decay_few_kernel<T, COLS, 256 / RG>), grid, dim3(256), 0, s, a, (T *)O, state_out);
    return hipGetLastError();
}

// What segments add to the state -> the state in front of each.  Four elements a thread; the elements of a state in whichever order they lie.
__global__ __launch_bounds__(256) void decay_join_kernel(const DecaySweeps s)
{
    const DecayPass &p = s.pass[blockIdx.z];
    const int each = p.da * p.dv, bh = (int)blockIdx.x, at = 4 * ((int)blockIdx.y * 256 + (int)threadIdx.x), left = each - at;
    if (left <= 0) return;
    const Tokens tokens = tokens_of(p, bh / p.heads);
    double a = p.log_decay ? (double)p.log_decay[bh % p.heads] : 0.0;
    a = a < -1e5 ? -1e5 : a;
    float *starts = p.starts + (size_t)bh * p.segments * each + at;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    if (p.init) {
        v = load4(p.init + (size_t)bh * each + at, left);
        put4(starts + (size_t)(p.segments - 1) * each, left, v);
    }
    int steps = p.seg_tokens - 1 + p.init_power;
    const int full = (tokens.count - 1) / p.seg_tokens;          // segments with another behind them
    f32x4_t next = full > 0 ? load4(starts, left) : v;
    for (int k = 0; k < full; ++k) {
        const f32x4_t add = next;
        if (k + 1 < full) next = load4(starts + (size_t)(k + 1) * each, left);
        const double exact = power(a, steps);
        const float fall = (float)exact, rest = (float)(exact - (double)fall);       // (as for single tokens: the rounding is in every call's)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(v[e], fall, fmaf(v[e], rest, add[e]));
        put4(starts + (size_t)k * each, left, v);
        steps = p.seg_tokens;
    }
}

// Gradients of key heads that several heads share: out[row][g] = sum over the heads of group g of part[row][head], rows of the sequences alone, of keys and of
// values (blockIdx.z).  A workgroup takes whole rows.
struct Shared {
    const float *part[2];
    void *out[2];
    size_t ld[2];
    int width[2];
};
template <typename T>
__global__ __launch_bounds__(256) void decay_share_kernel(const DecayPass p, const Shared what, int share)
{
    const Tokens tokens = tokens_of(p, (int)blockIdx.y);
    const int z = (int)blockIdx.z, width = what.width[z], wide = p.heads / share * width;
    const float *part = what.part[z];
    T *out = (T *)what.out[z];
    if (!out) return;
    for (int t = (int)blockIdx.x; t < tokens.count; t += (int)gridDim.x) {
        const size_t row = (size_t)(tokens.first + (int64_t)t * (p.offset ? 1 : p.token_step));
        for (int c = (int)threadIdx.x; c < wide; c += 256) {
            const int g = c / width, e = c - g * width;
            const float *from = part + (row * p.heads + (size_t)g * share) * width + e;
            float v = 0.f;
            for (int k = 0; k < share; ++k) v += from[(size_t)k * width];
            Elem<T>::st(out + row * what.ld[z] + c, v);
        }
    }
}

namespace {

size_t whole(size_t n) { return (n + 255) / 256 * 256; }

// Segments of a sequence.  They cost a sweep more, so only where a head has four of them at least for a workgroup a CU (and sweep), and of 128 tokens (fp32, whose
// products take three times as long: 64).  us of a call: 8192 tokens x 32 heads of 128 in bf16: 493 in one piece, 376 in 2, 200 in 4, 120 in 8, 135 in 12, 131 in 16; 13 sequences of
// up to 777 tokens x 16 heads: 52 in one piece, 70 in 2, 82 in 4; fp32, 4096 tokens x 16 heads: 724 in one piece, 152 in 8, 95 in 16; gradients in fp32, 8 x 333 tokens x 4 heads: 99
// in one piece, 81 in 2, 56 in 4 and 8.  In gradients the three sweeps of a launch are not counted: 4 x 2048 tokens x 16 heads of 128 in bf16 take 147 in 4, 154 in 2, 172 in 8, but
// 130 in one piece (192 workgroups).
int most_segments(int dtype, const DecayArgs &a)
{
    const int64_t groups = (int64_t)a.sequences * a.heads * ((a.dv + kDecayColumns - 1) / kDecayColumns), most = 256 / groups, fit = a.length / (dtype ? 128 : 64);
    return most < 4 || fit < 4 ? 1 : (int)(most < fit ? most : fit);
}
void cut(const DecayArgs &a, int64_t n, int *segments, int *tokens)
{
    *tokens = n > 1 ? (int)((a.length + n * kChunk - 1) / (n * kChunk)) * kChunk : a.length > 0 ? a.length : 1;
    *segments = a.length > 0 ? (a.length + *tokens - 1) / *tokens : 1;
}

DecayPass common(int dtype, const DecayArgs &a)
{
    DecayPass p{};
    p.rows = a.rows, p.sequences = a.sequences, p.length = a.length, p.heads = a.heads, p.seq_step = a.seq_step, p.token_step = a.token_step;
    p.log_decay = a.log_decay, p.offset = a.offset;
    p.share_a = p.share_b = p.share_v = 1;
    p.out_scale = p.state_scale = a.scale, p.value_scale = 1.f;
    cut(a, most_segments(dtype, a), &p.segments, &p.seg_tokens);
    return p;
}

size_t starts_bytes(int dtype, const DecayArgs &a)
{
    // (never less for a longer sequence)
    const int segments = most_segments(dtype, a);
    return segments > 1 ? whole((size_t)a.sequences * a.heads * segments * a.dk * a.dv * 4) : 0;
}
size_t parts_bytes(const DecayArgs &a, int width) { return a.heads != a.kv_heads ? whole((size_t)a.rows * a.heads * width * 4) : 0; }

// rows are whole 16-byte pieces at such addresses, and a chunk's bytes are counted by 31 bits
bool whole_rows(int dtype, const DecayPass &p)
{
    const size_t each = dtype ? 8 : 4, step = p.offset || p.token_step < 1 ? 1 : p.token_step, most = ((size_t)1 << 31) / (16 / each) / kChunk / step;
    auto ok = [&](const void *at, size_t ld) { return !at || ((uintptr_t)at % 16 == 0 && ld % each == 0 && ld < most); };
    return ok(p.A, p.lda) && ok(p.B, p.ldb) && ok(p.V, p.ldv) && p.da % each == 0 && p.dv % each == 0;
}
hipError_t sweep(int dtype, DecaySweeps &sw, bool outputs, hipStream_t s)
{
    bool ring = true;
    for (int i = 0; i < sw.count; ++i) ring = ring && whole_rows(dtype, sw.pass[i]);
    for (int i = 0; i < sw.count; ++i) sw.pass[i].ring = ring;
    if (outputs) return dtype ? decay_sweeps_bf16(sw, s) : decay_sweeps_f32(sw, s);
    return dtype ? decay_states_bf16(sw, s) : decay_states_f32(sw, s);
}
hipError_t join(const DecaySweeps &sw, hipStream_t s)
{
    const DecayPass &p = sw.pass[0];
    hipLaunchKernelGGL(decay_join_kernel, dim3(p.sequences * p.heads, (p.da * p.dv + 1023) / 1024, sw.count), dim3(256), 0, s, sw);
    return hipGetLastError();
}

hipError_t share_out(int dtype, const DecayArgs &a, const DecayPass &p, const Shared &all, hipStream_t s)
{
    const size_t size = dtype ? 2 : 4;
    const int blocks = a.length < 4096 ? a.length : 4096;
    for (int b = 0; b < a.sequences; b += 65535) {
        DecayPass q = p;
        Shared what = all;
        const dim3 grid((unsigned)blocks, a.sequences - b < 65535 ? a.sequences - b : 65535, 2);
        if (q.offset) q.offset += b;
        const size_t skip = q.offset ? 0 : (size_t)b * a.seq_step;
        for (int i = 0; i < 2; ++i)
            if (what.out[i]) what.part[i] += skip * a.heads * what.width[i], what.out[i] = (char *)what.out[i] + skip * what.ld[i] * size;
        if (dtype) hipLaunchKernelGGL(decay_share_kernel<bf16_t>, grid, dim3(256), 0, s, q, what, a.heads / a.kv_heads);
        else hipLaunchKernelGGL(decay_share_kernel<float>, grid, dim3(256), 0, s, q, what, a.heads / a.kv_heads);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t decay_workspace_bytes(int dtype, const DecayArgs &a, bool grads)
{
    if (!grads) return a.length > kFewTokens ? starts_bytes(dtype, a) : 0;
    return 2 * starts_bytes(dtype, a) + parts_bytes(a, a.dk) + parts_bytes(a, a.dv);
}

hipError_t launch_decay_forward(int dtype, const DecayArgs &a, void *O, float *state_out, void *ws, hipStream_t s)
{
    if (a.length <= kFewTokens) {
        // 32 columns a workgroup where 128 would leave lanes idle (256 x 8 heads of 64: 15 us for 28) or CUs without one; rows of 512 bytes elsewhere (64 tokens x 32 heads
        // of 128: 54 us for 57)
        const bool narrow = a.dv <= 96 || (int64_t)a.sequences * a.heads < 1024;
        if (dtype) return narrow ? few_tokens<bf16_t, 32>(a, O, state_out, s) : few_tokens<bf16_t, 128>(a, O, state_out, s);
        return narrow ? few_tokens<float, 32>(a, O, state_out, s) : few_tokens<float, 128>(a, O, state_out, s);
    }
    DecaySweeps sw{};
    DecayPass &p = sw.pass[0];
    sw.count = 1;
    p = common(dtype, a);
    p.da = a.dk, p.dv = a.dv;
    p.A = a.Q, p.lda = a.ld_q;
    p.B = a.K, p.ldb = a.ld_k, p.V = a.V, p.ldv = a.ld_v;
    p.share_b = p.share_v = a.heads / a.kv_heads;
    p.O = O, p.ldo = a.ld_o;
    p.init = a.state, p.last = state_out;
    p.init_power = 1;
    p.starts = (float *)ws;
    if (p.segments > 1) {
        hipError_t e = sweep(dtype, sw, false, s);
        if (e == hipSuccess) e = join(sw, s);
        if (e != hipSuccess) return e;
    }
    return sweep(dtype, sw, true, s);
}

hipError_t launch_decay_backward(int dtype, const DecayArgs &a, const DecayGrads &g, void *ws, hipStream_t s)
{
    const int share = a.heads / a.kv_heads;
    char *at = (char *)ws;
    auto take = [&](size_t n) {
        char *was = at;
        at += n;
        return (float *)was;
    };
    float *starts[2] = {take(starts_bytes(dtype, a)), take(starts_bytes(dtype, a))}, *part_k = take(parts_bytes(a, a.dk)), *part_v = take(parts_bytes(a, a.dv));
    // the state forward in time, from K and V
    DecayPass f = common(dtype, a);
    f.da = a.dk, f.dv = a.dv;
    f.B = a.K, f.ldb = a.ld_k, f.V = a.V, f.ldv = a.ld_v;
    f.share_b = f.share_v = share;
    f.init = a.state, f.init_power = 1;
    f.starts = starts[0];
    // its gradient backward in time, from Q and dO
    DecayPass r = common(dtype, a);
    r.reverse = true;
    r.da = a.dk, r.dv = a.dv;
    r.B = a.Q, r.ldb = a.ld_q, r.V = g.dO, r.ldv = a.ld_o;
    r.init = g.dstate_out, r.state_scale = 1.f, r.value_scale = a.scale;
    r.last_power = 1;
    r.starts = starts[1];
    const bool back = g.dK || g.dV || g.dstate_in;
    hipError_t e = hipSuccess;
    if (f.segments > 1) {
        // (the last state is written over none of them: `init` need not be kept, but for dstate_in, which is the last state of the sweep for dV)
        DecaySweeps sw{};
        if (g.dQ) sw.pass[sw.count++] = f;
        if (back) sw.pass[sw.count++] = r;
        e = sweep(dtype, sw, false, s);
        if (e == hipSuccess) e = join(sw, s);
        if (e != hipSuccess) return e;
    }
    DecaySweeps sw{};
    if (g.dQ) {
        DecayPass p = f;
        p.da = a.dv, p.dv = a.dk, p.turned = true;
        p.A = g.dO, p.lda = a.ld_o;
        p.B = a.V, p.ldb = a.ld_v, p.V = a.K, p.ldv = a.ld_k;
        p.O = g.dQ, p.ldo = a.ld_q;
        sw.pass[sw.count++] = p;
    }
    if (g.dK) {
        DecayPass p = r;
        p.da = a.dv, p.dv = a.dk, p.turned = true;
        p.A = a.V, p.lda = a.ld_v, p.share_a = share;
        p.B = g.dO, p.ldb = a.ld_o, p.V = a.Q, p.ldv = a.ld_q;
        p.O = share > 1 ? (void *)part_k : g.dK, p.ldo = share > 1 ? (size_t)a.heads * a.dk : a.ld_k, p.out32 = share > 1;
        sw.pass[sw.count++] = p;
    }
    if (g.dV || g.dstate_in) {
        DecayPass p = r;
        p.A = a.K, p.lda = a.ld_k, p.share_a = share;
        p.O = share > 1 && g.dV ? (void *)part_v : g.dV, p.ldo = share > 1 ? (size_t)a.heads * a.dv : a.ld_v, p.out32 = share > 1;
        p.last = g.dstate_in;
        sw.pass[sw.count++] = p;
    }
    // one launch for sweeps of the same tiles
    for (int i = 0; i < sw.count;) {
        DecaySweeps some{};
        do some.pass[some.count++] = sw.pass[i++];
        while (i < sw.count && key_tiles(sw.pass[i].da) == key_tiles(some.pass[0].da) && value_waves(sw.pass[i].dv) == value_waves(some.pass[0].dv) &&
               (sw.pass[i].dv + kDecayColumns - 1) / kDecayColumns == (some.pass[0].dv + kDecayColumns - 1) / kDecayColumns);
        e = sweep(dtype, some, true, s);
        if (e != hipSuccess) return e;
    }
    if (share == 1 || a.length == 0 || (!g.dK && !g.dV)) return e;
    return share_out(dtype, a, r, Shared{{part_k, part_v}, {g.dK, g.dV}, {a.ld_k, a.ld_v}, {a.dk, a.dv}}, s);
}

}  // namespace seq
}  // namespace stl
