// The routing kernels for binary32 logits.
#include "moe_backward.hpp"
#include "moe_route.hpp"

namespace nimble::moe {

hipError_t route_f32(const RouteArgs &a, hipStream_t stream) { return route_rows<F32>(a, stream); }
hipError_t backward_f32(const BackwardArgs &a, hipStream_t stream) { return backward_rows<F32>(a, stream); }

}  // namespace nimble::moe
