// The kernels of prefix_f32.hip for chunks of new tokens (chunk.hpp).
#define BDLM_CHUNK_CALLS
#include "prefix_f32.hip"
