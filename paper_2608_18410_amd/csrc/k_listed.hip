// Attention over listed pages of the paged cache: the kernels of decode.hpp, which find a
// tile's pages through the list first, and compare a token's place in the sequence with
// what its row sees. Bound by memory: 32 of 64 tokens for each of 32 sequences and 8 key heads
// of 4 rows (180 MB) 39.5 us, 4.6 TB/s; 128 for each of 8 (210 MB) 42, 5.0 TB/s. One of 24 pages of
// 16 and 32 heads 13: a chain of loads.
#include "decode.hpp"

namespace rolesub {

hipError_t launch_decode_listed(const DecodeParams& p, bool bf16, hipStream_t s) { return launch_any<kListed>(p, bf16, s); }

}  // namespace rolesub
