// The kernels of fwd_bf16.hip for packed calls (packed.hpp).
#define BDLM_PACKED_CALLS
#include "fwd_bf16.hip"
