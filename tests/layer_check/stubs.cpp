// Launchers of the recurrence and the norms replaced by stubs that report "no device",
// for the host sanitizer build of api_layer.cpp (see ../host_check/stubs.cpp).
#include "layer.h"

namespace hagdn {
hipError_t launch_glr_forward(const GlrArgs &, const GlrForm &, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_glr_backward(const GlrArgs &, const GlrForm &, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_glr_step(const GlrStepArgs &, const GlrForm &, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_add_norm(const AddNormArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_add_norm_backward(const AddNormArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_gate_norm(const GateNormArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_gate_norm_backward(const GateNormArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
}  // namespace hagdn
