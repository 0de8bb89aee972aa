// Chunk attention over fp16 and bf16 tiers, the join of a row tile's items, and which kernel a launch takes.
#include "ttkv_chunk_kernels.h"

namespace ttkv {

namespace {

using namespace chunk;

// The items of a row tile joined: a wave per query row, two channels per lane.  Bound: the parts' way from the L2s (512 rows of 32 parts 7.0 us; one part after
// the other 11.1).
__global__ __launch_bounds__(256) void chunk_merge_kernel(const ChunkMergeArgs a, int n_rows) {
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (id >= n_rows) return;
  const int row_all = a.Hkv == 1 ? id : id / a.Hkv, hkv = id - row_all * a.Hkv;
  const int slot = __popcll(__ballot(a.row_base[lane] <= row_all)) - 1;
  const int row = row_all - a.row_base[slot], token = token_of(a, row), hq = hkv * a.G + row - token * a.G;
  const int n = a.n_split[slot], entry = a.entry[slot];
  const int64_t at = a.part_base[slot] + ((int64_t)row * a.Hkv + hkv) * n;
  float top = -INFINITY;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, a.pm[at + i]);
  top = wave_max(top);
  float l = 0.0f, x = 0.0f, y = 0.0f;
  for (int i = 0; i < n; i += 8) {   // eight asked for at once
    float m[8], ls[8];
    float2 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t k = at + min(i + j, n - 1);
      m[j] = a.pm[k];
      ls[j] = a.pl[k];
      v[j] = *(const float2 *)(a.pacc + k * 128 + 2 * lane);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i + j >= n) continue;
      const float by = m[j] == -INFINITY ? (ls[j] != 0.0f ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f(m[j] - top);
      l = fmaf(ls[j], by, l);
      x = fmaf(v[j].x, by, x);
      y = fmaf(v[j].y, by, y);
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  *(uint32_t *)(a.out + entry * a.o_seq + token * a.o_token + hq * a.o_head + 4 * lane) =
      a.out_fmt == TTKV_BF16 ? pack2<true>(x * inv, y * inv) : pack2<false>(x * inv, y * inv);
  if (a.lse && lane == 0) a.lse[((int64_t)entry * a.n_tokens + token) * a.Hq + hq] = l == 0.0f ? -INFINITY : (__builtin_amdgcn_logf(l) + top) * kLn2;
}

}  // namespace

// Rows per workgroup, each up to what it holds.  Measured beside its neighbour, 32 / 8 fp16 heads, us: 64 rows x 8 sequences of 8192 tokens 48 with 64, 47 with 128, one
// sequence of 16384 21 and 21 (and 64 divide by the rounded weights' sum, which costs the others more than it helps them); 128 rows 54 with 128, 69
// with 256, one sequence 24 and 25.
ChunkShape chunk_shape(int64_t most_rows, bool bf, int quantized) {
  return ChunkShape{most_rows <= 64 ? 64 : most_rows <= 128 ? 128 : 256, bf, quantized};
}

// (four for 64 rows: five drafted tokens 15.7 instead of 16.0 us, int4 histories slower)
int64_t chunk_least_steps(const ChunkShape &s) { return s.rows == 256 ? 4 : 8; }
int64_t chunk_resident(const ChunkShape &s) { return s.rows == 64 && s.quantized ? 512 : 256; }

hipError_t launch_chunk(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream) {
  switch (s.quantized) {
    case 0: s.bf ? chunk::start<true, 0, false>(a, s.rows, stream) : chunk::start<false, 0, false>(a, s.rows, stream); break;
    case kInt8: start_chunk_i8(a, s, stream); break;
    case kInt4: start_chunk_i4(a, s, stream); break;
    case kInt84: start_chunk_k8v4(a, s, stream); break;
    default: start_chunk_mixed(a, s, stream);
  }
  return hipGetLastError();
}

hipError_t launch_chunk_merge(const ChunkMergeArgs &a, int64_t n_rows, hipStream_t stream) {
  hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)((n_rows + 3) / 4)), dim3(256), 0, stream, a, (int)n_rows);
  return hipGetLastError();
}

}  // namespace ttkv
