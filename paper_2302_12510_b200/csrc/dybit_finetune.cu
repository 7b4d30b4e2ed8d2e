// libdybit, second translation unit: the operators that fine-tune and adapt coded layers.
#include <string.h>

#include "dybit_adapters.cuh"
#include "dybit_checkpoint.cuh"
#include "dybit_wgrad.cuh"

namespace dybit {
cudaError_t take_finetune_status_word(cudaStream_t s, unsigned *word) { return take_status_word(s, word); }
}  // namespace dybit
