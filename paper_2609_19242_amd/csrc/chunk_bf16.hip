// The kernels of prefix_bf16.hip for chunks of new tokens (chunk.hpp).
#define BDLM_CHUNK_CALLS
#include "prefix_bf16.hip"
