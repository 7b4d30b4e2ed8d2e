// libdybit, third translation unit: the key-value cache in 8-bit codes and the attention that reads it.
#include <string.h>

#include <algorithm>

#include "dybit_cache_api.cuh"

namespace dybit {
cudaError_t take_cache_status_word(cudaStream_t s, unsigned *word) { return take_status_word(s, word); }
}  // namespace dybit
