// The products of the gated block in half precision.
#include "gated_tile.h"

namespace bmgd {

hipError_t gated_prepare_f16() { return prepare_all<_Float16>(); }
hipError_t gated_launch_f16(const GatedProduct& q, GatedOp op, hipStream_t stream) { return launch_any<_Float16>(q, op, stream); }
hipError_t gated_launch_grads_f16(const GatedProduct* input, const GatedProduct* down, const GatedProduct* gate, hipStream_t stream)
{
    return launch_grads<_Float16>(input, down, gate, stream);
}

}  // namespace bmgd
