// Attention over listed pages of the paged cache: the kernels of decode.hpp.
#include "decode.hpp"

namespace rolesub {

hipError_t launch_decode_listed(const DecodeParams& p, bool bf16, hipStream_t s) { return launch_any<kListed>(p, bf16, s); }

}  // namespace rolesub
