// Layers with short inputs and wide outputs, in bf16.
#include "layer_wide.h"

namespace cgtp {

hipError_t launch_layer_wide_bf16(const RowOrder &o, const RowProduct &p, hipStream_t s) { return rows::launch_wide_layer<rows::bf16_t>(o, p, s); }

}  // namespace cgtp
