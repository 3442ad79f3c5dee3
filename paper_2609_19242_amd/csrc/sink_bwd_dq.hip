// The kernels of bwd_dq.hip for packed calls with a window and sinks (packed.hpp).
#define BDLM_PACKED_CALLS
#define BDLM_SINK_CALLS
#include "bwd_dq.hip"
