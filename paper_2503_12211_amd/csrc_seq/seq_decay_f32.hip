// Attention with decay: sweeps in fp32 storage.
#include "seq_decay.h"

namespace stl {
namespace seq {

hipError_t decay_sweeps_f32(const DecaySweeps &sw, hipStream_t s) { return decay_sweeps<float, true>(sw, s); }

}  // namespace seq
}  // namespace stl
