// The routing kernels for bfloat16 logits.
#include "moe_backward.hpp"
#include "moe_route.hpp"

namespace nimble::moe {

hipError_t route_bf16(const RouteArgs &a, hipStream_t stream) { return route_rows<BF16>(a, stream); }
hipError_t backward_bf16(const BackwardArgs &a, hipStream_t stream) { return backward_rows<BF16>(a, stream); }

}  // namespace nimble::moe
