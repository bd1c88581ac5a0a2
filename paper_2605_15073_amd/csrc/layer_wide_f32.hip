// Layers with short inputs and wide outputs, in fp32.
#include "layer_wide.h"

namespace cgtp {

hipError_t launch_layer_wide_f32(const RowOrder &o, const RowProduct &p, hipStream_t s) { return rows::launch_wide_layer<float>(o, p, s); }

}  // namespace cgtp
