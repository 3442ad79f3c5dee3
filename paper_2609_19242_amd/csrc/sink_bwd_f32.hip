// The kernels of bwd_f32.hip for packed calls with a window and sinks (packed.hpp).
#define BDLM_PACKED_CALLS
#define BDLM_SINK_CALLS
#include "bwd_f32.hip"
