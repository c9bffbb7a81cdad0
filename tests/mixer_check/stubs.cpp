// Launchers of the convolution, the scan and the pools replaced by stubs that report "no
// device", for the host sanitizer build of api_mixer.cpp (see ../host_check/stubs.cpp).
#include "mixer.h"

namespace hagdn {
hipError_t launch_conv_forward(const ConvArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_conv_backward(const ConvArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_conv_step(const ConvStepArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_ssm_forward(const SsmArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_ssm_backward(const SsmArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_ssm_step(const SsmStepArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_pool_copy(const PoolCopyArgs &, bool, int, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_pool_fork_plan(const PoolPlanArgs &, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_pool_compact_plan(const PoolPlanArgs &, hipStream_t) { return hipErrorNoDevice; }
}  // namespace hagdn
