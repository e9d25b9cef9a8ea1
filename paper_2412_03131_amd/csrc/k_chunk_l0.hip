// Chunk attention and scores for page layout 0 (kLayoutFmts[0]).
#include "chunk_kernels.hpp"

namespace dkv {
DKV_CHUNK_KERNELS(0)
}  // namespace dkv
