// Chunk attention over tiers of int8 keys and int4 values, beside fp16 or bf16 ones.
#include "ttkv_chunk_kernels.h"

namespace ttkv {

void start_chunk_k8v4(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream) { chunk::start_quantized<kInt84>(a, s, stream); }

}  // namespace ttkv
