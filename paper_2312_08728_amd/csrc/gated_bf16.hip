// The products of the gated block in bfloat16.
#include "gated_tile.h"

namespace bmgd {

hipError_t gated_prepare_bf16() { return prepare_all<__bf16>(); }
hipError_t gated_launch_bf16(const GatedProduct& q, GatedOp op, hipStream_t stream) { return launch_any<__bf16>(q, op, stream); }
hipError_t gated_launch_grads_bf16(const GatedProduct* input, const GatedProduct* down, const GatedProduct* gate, hipStream_t stream)
{
    return launch_grads<__bf16>(input, down, gate, stream);
}

}  // namespace bmgd
