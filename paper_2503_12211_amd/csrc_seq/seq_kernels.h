// Internal launcher interface between the C ABI (seq_api.hip) and the kernels of the embedding, the norms and rotation of queries and keys, and
// attention with decay.
#pragma once
#include "../csrc/stl_kernels.h"

#include <stddef.h>
#include <type_traits>

namespace stl {
namespace seq {

// ---- embedding (seq_embed.hip) -------------------------------------------------------------------------------------------------
struct EmbedArgs {
    int rows, d, vocab;
    float scale;
};
// How the backward pass cuts its work: ranges of `width` ids, each sorted by one workgroup, and `segments` of `length` sorted rows.
struct EmbedPlan {
    int ranges, width, length, segments;
    size_t ids_at, parts_at, bytes;          // of the workspace: rows sorted by id, ids in that order, sums of cut runs; all of it
};
EmbedPlan embed_plan(const EmbedArgs &a);
hipError_t launch_embed_forward(int dtype, const EmbedArgs &a, const int64_t *token, const void *W, void *X, hipStream_t s);
hipError_t launch_embed_backward(int dtype, const EmbedArgs &a, const int64_t *token, const void *dX, void *dW, int accumulate, void *ws, hipStream_t s);

// ---- norms and rotation of queries and keys (seq_head.hip) -----------------------------------------------------------------------
constexpr int kHeadWidest = 1024;            // a head's elements are held by the lanes of a wavefront, sixteen each
struct HeadArgs {
    int rows, heads[2], d, rot;              // of queries, of keys
    size_t ld_in[2], ld_out[2];              // elements from row to row
    float eps;
    double log2_base;
    bool norm, adjacent;
    const void *in[2], *w[2];                // storage type; w may be NULL
    const int64_t *position;                 // NULL: no rotation
};
struct HeadGrads {
    const void *up[2];                       // NULL: zeros
    void *d_in[2];
    float *dw[2];
    int accumulate;
};
size_t head_workspace_bytes(const HeadArgs &a);
hipError_t launch_head_forward(int dtype, const HeadArgs &a, void *const out[2], hipStream_t s);
hipError_t launch_head_backward(int dtype, const HeadArgs &a, const HeadGrads &g, void *ws, hipStream_t s);

// ---- attention with decay (seq_decay*.hip) ---------------------------------------------------------------------------------------
constexpr int kDecayWidest = 256;            // a head's state is held by the wavefronts of a workgroup
struct DecayArgs {
    int rows, sequences, length, heads, kv_heads, dk, dv;
    int seq_step, token_step;
    size_t ld_q, ld_k, ld_v, ld_o;
    float scale;
    const void *Q, *K, *V;
    const float *log_decay;                  // NULL: zeros
    const int64_t *offset;                   // NULL: sequences of `length` tokens
    const float *state;                      // NULL: zeros
};
struct DecayGrads {
    const void *dO;
    const float *dstate_out;                 // NULL: zeros
    void *dQ, *dK, *dV;                      // any may be NULL
    float *dstate_in;
};
size_t decay_workspace_bytes(int dtype, const DecayArgs &a, bool grads);
hipError_t launch_decay_forward(int dtype, const DecayArgs &a, void *O, float *state_out, void *ws, hipStream_t s);
hipError_t launch_decay_backward(int dtype, const DecayArgs &a, const DecayGrads &g, void *ws, hipStream_t s);

}  // namespace seq
}  // namespace stl
