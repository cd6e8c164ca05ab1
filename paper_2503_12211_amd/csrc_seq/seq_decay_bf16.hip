// Attention with decay: sweeps in bf16 storage.
#include "seq_decay.h"

namespace stl {
namespace seq {

hipError_t decay_sweeps_bf16(const DecaySweeps &sw, hipStream_t s) { return decay_sweeps<bf16_t, true>(sw, s); }

}  // namespace seq
}  // namespace stl
