// Attention of drafted tokens that form a tree, over the paged cache: the kernels of
// decode.hpp.
#include "decode.hpp"

namespace rolesub {

hipError_t launch_decode_tree(const DecodeParams& p, bool bf16, hipStream_t s) { return launch_any<kTree>(p, bf16, s); }

}  // namespace rolesub
