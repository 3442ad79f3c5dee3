// The kernels of bwd_dq.hip for packed calls (packed.hpp).
#define BDLM_PACKED_CALLS
#include "bwd_dq.hip"
