// The kernels of fwd_f32.hip for packed calls (packed.hpp).
#define BDLM_PACKED_CALLS
#include "fwd_f32.hip"
