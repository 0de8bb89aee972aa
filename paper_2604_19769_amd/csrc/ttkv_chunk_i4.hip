// Chunk attention over int4 tiers, beside fp16 or bf16 ones.
#include "ttkv_chunk_kernels.h"

namespace ttkv {

void start_chunk_i4(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream) { chunk::start_quantized<kInt4>(a, s, stream); }

}  // namespace ttkv
