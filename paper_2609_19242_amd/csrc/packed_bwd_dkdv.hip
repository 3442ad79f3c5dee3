// The kernels of bwd_dkdv.hip for packed calls (packed.hpp).
#define BDLM_PACKED_CALLS
#include "bwd_dkdv.hip"
