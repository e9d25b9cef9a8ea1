// Chunk attention and scores for page layout 2 (kLayoutFmts[2]).
#include "chunk_kernels.hpp"

namespace dkv {
DKV_CHUNK_KERNELS(2)
}  // namespace dkv
