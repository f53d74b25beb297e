// The routing kernels for binary16 logits.
#include "moe_backward.hpp"
#include "moe_route.hpp"

namespace nimble::moe {

hipError_t route_f16(const RouteArgs &a, hipStream_t stream) { return route_rows<F16>(a, stream); }
hipError_t backward_f16(const BackwardArgs &a, hipStream_t stream) { return backward_rows<F16>(a, stream); }

}  // namespace nimble::moe
