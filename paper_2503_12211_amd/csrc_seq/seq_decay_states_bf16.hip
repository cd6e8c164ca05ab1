// Attention with decay: what segments add to the state, bf16 storage.
#include "seq_decay.h"

namespace stl {
namespace seq {

hipError_t decay_states_bf16(const DecaySweeps &sw, hipStream_t s) { return decay_sweeps<bf16_t, false>(sw, s); }

}  // namespace seq
}  // namespace stl
