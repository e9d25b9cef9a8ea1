// Chunk attention and scores for page layout 3 (kLayoutFmts[3]).
#include "chunk_kernels.hpp"

namespace dkv {
DKV_CHUNK_KERNELS(3)
}  // namespace dkv
