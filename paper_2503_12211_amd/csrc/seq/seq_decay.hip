// Attention with decay: bf16 storage, and what the forward and the backward call make of the sweeps.
#include "seq_decay.h"

namespace stl {
namespace seq {

hipError_t decay_pass_bf16(const DecayPass &p, hipStream_t s) { return decay_pass<bf16_t>(p, s); }

namespace {

DecayPass common(const DecayArgs &a)
{
    DecayPass p{};
    p.rows = a.rows, p.sequences = a.sequences, p.length = a.length, p.heads = a.heads, p.seq_step = a.seq_step, p.token_step = a.token_step;
    p.log_decay = a.log_decay, p.offset = a.offset;
    p.share_a = p.share_b = p.share_v = 1;
    p.out_scale = a.scale, p.init_scale = p.last_scale = 1.f;
    return p;
}

size_t whole(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// Gradients of key heads that several heads share: out[row][g] = sum over the heads of group g of part[row][head], rows of the sequences alone.
template <typename T>
__global__ __launch_bounds__(256) void decay_share_kernel(const DecayPass p, const float *part, T *out, size_t ld, int width, int share)
{
    const int b = (int)blockIdx.y;
    const Tokens tokens = tokens_of(p, b);
    const int groups = p.heads / share, wide = groups * width;
    const int64_t all = (int64_t)tokens.count * wide;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int t = (int)(i / wide), c = (int)(i % wide), g = c / width, e = c % width;
        const size_t row = (size_t)(tokens.first + (int64_t)t * (p.offset ? 1 : p.token_step));
        const float *from = part + (row * p.heads + (size_t)g * share) * width + e;
        float v = 0.f;
        for (int k = 0; k < share; ++k) v += from[(size_t)k * width];
        Elem<T>::st(out + row * ld + c, v);
    }
}

size_t decay_workspace_bytes(int dtype, const DecayArgs &a, bool grads)
{
    size_t n = 0;
    if (grads && a.heads != a.kv_heads) n += whole((size_t)a.rows * a.heads * (a.dk > a.dv ? a.dk : a.dv) * 4);
    return n;
}

hipError_t launch_decay_forward(int dtype, const DecayArgs &a, void *O, float *state_out, void *ws, hipStream_t s)
{
    DecayPass p = common(a);
    p.da = a.dk, p.dv = a.dv;
    p.A = a.Q, p.lda = a.ld_q;
    p.B = a.K, p.ldb = a.ld_k, p.V = a.V, p.ldv = a.ld_v;
    p.share_b = p.share_v = a.heads / a.kv_heads;
    p.O = O, p.ldo = a.ld_o;
    p.init = a.state, p.last = state_out;
    p.init_power = 1;
    return dtype ? decay_pass_bf16(p, s) : decay_pass_f32(p, s);
}

hipError_t launch_decay_backward(int dtype, const DecayArgs &a, const DecayGrads &g, void *ws, hipStream_t s)
{
    const int share = a.heads / a.kv_heads;
    auto sweep = [&](const DecayPass &p) { return dtype ? decay_pass_bf16(p, s) : decay_pass_f32(p, s); };
    // what belongs to a key head: by head in fp32 first where heads share it
    auto shared = [&](DecayPass p, void *out, size_t ld, int width) {
        if (share == 1 || !out) {
            p.O = out, p.ldo = ld;
            return sweep(p);
        }
        p.O = ws, p.ldo = (size_t)a.heads * width, p.out32 = true;
        hipError_t e = sweep(p);
        if (e != hipSuccess) return e;
        const int64_t elements = (int64_t)a.length * a.kv_heads * width;
        int64_t blocks = (elements + 2047) / 2048;
        if (blocks > 4096) blocks = 4096;
        for (int b = 0; b < a.sequences; b += 65535) {
            DecayPass q = p;
            const int some = a.sequences - b < 65535 ? a.sequences - b : 65535;
            const dim3 grid((unsigned)blocks, some);
            float *part = (float *)ws;
            if (q.offset) q.offset += b;
            const size_t skip = q.offset ? 0 : (size_t)b * a.seq_step;
            part += skip * a.heads * width;
            if (dtype) hipLaunchKernelGGL(decay_share_kernel<bf16_t>, grid, dim3(256), 0, s, q, (const float *)part, (bf16_t *)out + skip * ld, ld, width, share);
            else hipLaunchKernelGGL(decay_share_kernel<float>, grid, dim3(256), 0, s, q, (const float *)part, (float *)out + skip * ld, ld, width, share);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    hipError_t e = hipSuccess;
    if (g.dQ) {
        DecayPass p = common(a);
        p.da = a.dv, p.dv = a.dk;
        p.A = g.dO, p.lda = a.ld_o;
        p.B = a.V, p.ldb = a.ld_v, p.V = a.K, p.ldv = a.ld_k;
        p.share_b = p.share_v = share;
        p.O = g.dQ, p.ldo = a.ld_q;
        p.init = a.state, p.turned = true;
        p.init_power = 1;
        e = sweep(p);
        if (e != hipSuccess) return e;
    }
    // the state's gradient is held without the factor c, which its outputs have
    DecayPass p = common(a);
    p.reverse = true;
    p.init = g.dstate_out, p.init_scale = 1.f / a.scale;
    p.last_scale = a.scale, p.last_power = 1;
    if (g.dV || g.dstate_in) {
        DecayPass v = p;
        v.da = a.dk, v.dv = a.dv;
        v.A = a.K, v.lda = a.ld_k, v.share_a = share;
        v.B = a.Q, v.ldb = a.ld_q, v.V = g.dO, v.ldv = a.ld_o;
        v.last = g.dstate_in;
        e = shared(v, g.dV, a.ld_v, a.dv);
        if (e != hipSuccess) return e;
    }
    if (g.dK) {
        DecayPass k = p;
        k.da = a.dv, k.dv = a.dk;
        k.A = a.V, k.lda = a.ld_v, k.share_a = share;
        k.B = g.dO, k.ldb = a.ld_o, k.V = a.Q, k.ldv = a.ld_q;
        k.turned = true;
        e = shared(k, g.dK, a.ld_k, a.dk);
    }
    return e;
}

}  // namespace seq
}  // namespace stl
