// Barriers that the blocks of a half's keys take in turn.  (Nothing of CUDA but the qualifiers: tests compile it for the host.)
#pragma once

namespace dybit {

// Block n of a half (counted over all parts of a block's share) completes phase n / 2 of barrier n % 2.  One barrier for all blocks
// would not do: a waiting warp sees no more of it than the parity of the current phase, and the products of two blocks can end
// before a slow warp has looked for the first.  With two, whoever waits for block n knows that block n - 2 is done, and block
// n + 2 is not begun before every softmax warp is past block n: the barrier is at block n's phase or the next one.
struct Turn { unsigned bar, parity; };
__host__ __device__ __forceinline__ Turn turn_of(unsigned n) { return {n & 1u, (n >> 1) & 1u}; }

}  // namespace dybit
