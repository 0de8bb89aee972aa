// Chunk attention over quantized tiers of several formats, beside fp16 or bf16 ones.
#include "ttkv_chunk_kernels.h"

namespace ttkv {

void start_chunk_mixed(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream) { chunk::start_quantized<kInt8 | kInt4 | kInt84>(a, s, stream); }

}  // namespace ttkv
