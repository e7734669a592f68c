#include "sfda_delta.h"
namespace sfda { hipError_t launch_delta_bwd(const DeltaLaunch&, hipStream_t) { return hipErrorNotSupported; } }
