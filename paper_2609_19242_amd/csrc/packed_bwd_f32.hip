// The kernels of bwd_f32.hip for packed calls (packed.hpp).
#define BDLM_PACKED_CALLS
#include "bwd_f32.hip"
