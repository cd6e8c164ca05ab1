// Attention with decay: fp32 storage.
#include "seq_decay.h"

namespace stl {
namespace seq {

hipError_t decay_pass_f32(const DecayPass &p, hipStream_t s) { return decay_pass<float>(p, s); }

}  // namespace seq
}  // namespace stl
