// Chunk attention and scores for page layout 1 (kLayoutFmts[1]).
#include "chunk_kernels.hpp"

namespace dkv {
DKV_CHUNK_KERNELS(1)
}  // namespace dkv
