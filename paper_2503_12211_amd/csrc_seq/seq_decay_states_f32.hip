// Attention with decay: what segments add to the state, fp32 storage.
#include "seq_decay.h"

namespace stl {
namespace seq {

hipError_t decay_states_f32(const DecaySweeps &sw, hipStream_t s) { return decay_sweeps<float, false>(sw, s); }

}  // namespace seq
}  // namespace stl
