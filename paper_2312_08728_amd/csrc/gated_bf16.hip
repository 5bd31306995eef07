// The products of the gated block in bfloat16.
#include "gated_tile.h"

namespace bmgd {

hipError_t gated_prepare_bf16() { return prepare_all<__bf16>(); }
hipError_t gated_launch_bf16(const GatedProduct& q, GatedOp op, hipStream_t stream) { return launch_any<__bf16>(q, op, stream); }

}  // namespace bmgd
