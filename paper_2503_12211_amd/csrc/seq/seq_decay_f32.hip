// Attention with decay: sweeps in fp32 storage.
#include "seq_decay.h"

namespace stl {
namespace seq {

hipError_t decay_sweeps_f32(const DecaySweeps &sw, bool outputs, hipStream_t s) { return decay_sweeps<float>(sw, outputs, s); }

}  // namespace seq
}  // namespace stl
