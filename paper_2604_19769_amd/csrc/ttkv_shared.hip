// Attention of many query rows over the same tokens: a batch whose sequences share a prefix reads it once.  The rows of a KV
// head are the query heads that it serves in every sequence that takes part, R = sequences x heads per KV head, so both
// contractions are matrix products:
//       S^T[token][row] = sum_d K[token][d] Q[row][d],     O^T[d][row] += sum_token V[token][d] P[token][row]
// with the running maximum and sum of the softmax in between, and the un-normalised partial (m, l, O) of each part of the
// tokens at the end, in the form that merge_kernel joins.
//
// Both products are v_mfma_f32_32x32x16 with tokens (channels) as rows and query rows as columns.  A lane then holds 16 scores
// of ONE query row (lane % 32; its two halves share the row's 32 tokens), so the softmax needs one exchange between the
// halves, and the scores' registers are the second product's right operand as they lie: lane half h has tokens 16 b + 4 h + 0 .. 3
// and 16 b + 8 + 4 h + 0 .. 3 in registers 8 b .. 8 b + 7, and the value operand is read from LDS in that order of tokens
// (ds_read_b64_tr_b16: four tokens of one channel per lane).
//
// A workgroup's four waves are RW along the rows (32 each) times TW along the tokens of a tile; K and V tiles go global ->
// registers -> LDS, the next tile's loads in flight while one is computed.  LDS rows keep their sixteen 16-byte pieces in the
// order p ^ swz(row), which spreads both products' reads over the banks.
//
// The weights p carry 2^14 and meet fp16 values as an fp16 number and its remainder (22 bits), bf16 values as three bf16
// numbers (24 bits): the outputs are fp32.
#include "ttkv_attn_dev.h"

#include <algorithm>

namespace ttkv {

namespace {

using namespace dev;

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s4 *las_s4;

template <bool BF>
__device__ __forceinline__ f16v mma(const u32x4 &a, const u32x4 &b, const f16v &c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float x, float y) {   // nearest even
  const f2 v = {x, y};
  if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
}
template <bool BF>
__device__ __forceinline__ f2 unpack2(uint32_t w) {
  if constexpr (BF) return f2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  else return f2{(float)as_h2(w).x, (float)as_h2(w).y};
}
// Sixteen rows that differ in their low four bits keep a piece in sixteen places; rows 4 r .. 4 r + 3 in four pairs of places.
__device__ __forceinline__ int swz(int row) { return ((row & 3) << 1) | ((row >> 2) & 1) | (row & 8); }

constexpr int kTile(int tw) { return tw == 4 ? 128 : 64; }   // tokens in LDS at a time

template <bool BF, int RW, int TW>
__global__ __launch_bounds__(256, 2) void shared_kernel(const SharedArgs a) {
  static_assert(RW * TW == 4, "four waves");
  constexpr int TILE = kTile(TW), SUB = TILE / (32 * TW), NL = TILE / 16;   // 32-token steps of a wave per tile; 16-byte loads of K (V) per thread
  constexpr int NP = BF ? 3 : 2;                                            // numbers that hold a weight
  __shared__ __align__(16) char s_tile[2 * TILE * 256];   // K rows, V rows; at the end partial outputs, 16 KiB per row block
  char *const s_k = s_tile, *const s_v = s_tile + TILE * 256;
  static_assert(2 * TILE * 256 >= RW * 64 * 64 * 4 || TW == 1, "room for the partial outputs");
  __shared__ float s_m[4][32], s_l[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave % RW, tw = wave / RW;
  const int c = lane & 31, hh = lane >> 5;
  // workgroups that read the same tokens of a KV head lie on one XCD, one behind the other
  const int x8 = blockIdx.x >> 3, unit = x8 / a.row_tiles * 8 + (blockIdx.x & 7), rt = x8 % a.row_tiles;
  if (unit >= a.n_split * a.Hkv) return;
  const int split = unit / a.Hkv, hkv = unit - split * a.Hkv;
  const int t_begin = split * a.chunk, n_tok = min(a.chunk, a.len - t_begin);   // at least 1

  // ---- queries: the lane's row, channels 16 kb + 8 hh .. + 7 per step
  const int row = (rt * RW + rw) * 32 + c;
  const bool row_on = row < a.rows;
  const int row_in = min(row, a.rows - 1);
  const int n = row_in / a.G, seq = a.listed ? a.member[n] : n, hq = hkv * a.G + row_in - n * a.G;
  u32x4 qf[8];
  {
    const u32x4 *qp = (const u32x4 *)((const uint16_t *)a.q + ((int64_t)seq * a.Hq + hq) * 128);
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) qf[kb] = qp[2 * kb + hh];
    if (!BF && a.q_fmt == TTKV_BF16) {   // bf16 -> fp16 (exact inside the fp16 normal range, clamped outside)
#pragma unroll
      for (int kb = 0; kb < 8; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f2 v = unpack2<true>(qf[kb][i]);
          qf[kb][i] = pack2<false>(fminf(fmaxf(v.x, -65504.0f), 65504.0f), fminf(fmaxf(v.y, -65504.0f), 65504.0f));
        }
    }
  }
  const float cs = a.scale * kLog2e;   // scores are kept in the log2 domain

  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = -INFINITY, l = 0.0f, mcs = 0.0f, f = 0.0f;   // a token's weight: exp2(score cs + mcs) = 2^f e^(score - m)

  // ---- tiles: thread -> row (threadIdx / 16) + 16 i, piece threadIdx % 16
  const int ring = a.tv.ring_blocks * a.tv.bt, lr = threadIdx.x >> 4, lp = threadIdx.x & 15;
  u32x4 kr[NL], vr[NL];
  auto load = [&](int t0) {   // tokens t0 .. of the item; rows behind its end repeat its last one
#pragma unroll
    for (int g = 0; g < TILE / 64; ++g) {
      const int live0 = (n_tok - 1) & ~63;
      const int at = min(t0 + 64 * g, live0);
      const int last = n_tok - 1 - at;
      int tok = a.first_tok + t_begin + at;
      if (tok >= ring) tok -= ring;
      const int rb = div_bt(tok, a.tv.bt, a.tv.bt_magic), row0 = tok - rb * a.tv.bt;
      const int64_t rec = a.tv.table ? (int64_t)a.tv.table[rb] : (int64_t)rb;
      const uint8_t *head = a.tv.base + rec * a.tv.rec_bytes + (int64_t)hkv * a.tv.head_bytes + row0 * 256;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = min(lr + 16 * i, last);
        const uint8_t *p = head + r * 256 + lp * 16;
        kr[4 * g + i] = *(const u32x4 *)p;
        vr[4 * g + i] = *(const u32x4 *)(p + a.tv.v_off);
      }
    }
  };
  const int n_tiles = (n_tok + TILE - 1) / TILE;
  load(0);
  for (int t = 0; t < n_tiles; ++t) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = lr + 16 * i, at = r * 256 + ((lp ^ swz(r)) << 4);
      *(u32x4 *)(s_k + at) = kr[i];
      *(u32x4 *)(s_v + at) = vr[i];
    }
    __syncthreads();
    if (t + 1 < n_tiles) load((t + 1) * TILE);
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
      const int t0 = (tw * SUB + s) * 32;                 // the step's first token in the tile
      const int left = n_tok - t * TILE - t0;             // live tokens from it on
      if (left <= 0) break;                               // (wave-uniform)
      f16v sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
      for (int kb = 0; kb < 8; ++kb) {
        const int r = t0 + c;
        sc = mma<BF>(*(const u32x4 *)(s_k + r * 256 + (((2 * kb + hh) ^ swz(r)) << 4)), qf[kb], sc);
      }
      if (left < 32) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i / 4) + 4 * hh + i % 4 >= left) sc[i] = -INFINITY;
      }
      float mt = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mt = fmaxf(mt, sc[i]);
      const f2 both = both32(mt);
      mt = fmaxf(both.x, both.y);
      if (__any(mt > m)) {
#pragma clang fp contract(off)
        const float mn = fmaxf(m, mt), r = mn * cs, was = mcs;
        f = fabsf(r) < 4194304.0f ? 14.0f : 0.0f;   // beyond, f - mcs would not be exact
        mcs = mn == -INFINITY ? 0.0f : f - r;
        const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mcs - was);
        l *= alpha;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= alpha;
        m = mn;
      }
      u32x4 p[NP][2];   // [part of the weight][16 tokens]
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float w0 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i], cs, mcs)), w1 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i + 1], cs, mcs));
        l += w0 + w1;
#pragma unroll
        for (int u = 0; u < NP; ++u) {
          const uint32_t w = pack2<BF>(w0, w1);
          p[u][i / 4][i % 4] = w;
          const f2 x = unpack2<BF>(w);
          w0 -= x.x;
          w1 -= x.y;
        }
      }
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          u32x4 va;
#pragma unroll
          for (int jb = 0; jb < 2; ++jb) {
            const int r = t0 + 16 * b + 8 * jb + 4 * hh + ((lane & 15) >> 2);
            const int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((las_s4)(s_v + r * 256 + ((piece ^ swz(r)) << 4) + (lane & 1) * 8));
            const u32x2 y = __builtin_bit_cast(u32x2, x);
            va[2 * jb] = y.x;
            va[2 * jb + 1] = y.y;
          }
#pragma unroll
          for (int u = 0; u < NP; ++u) o[d] = mma<BF>(va, p[u][b], o[d]);
        }
    }
  }
  {   // the halves' sums, without the power of two
    const f2 both = both32(l);
    const float unit = f == 0.0f ? 1.0f : 0x1p-14f;
    l = (both.x + both.y) * unit;
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] *= unit;
  }

  // ---- the waves of one row block join
  float ref = m == -INFINITY ? -INFINITY : f - mcs;   // the weights are exp2(score cs - ref) ...
  if constexpr (TW > 1) {
    float *const s_o = (float *)s_tile;   // [row block][channel register][lane]
    __syncthreads();
    if (hh == 0) {
      s_m[wave][c] = ref;
      s_l[wave][c] = l;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < TW; ++u) top = fmaxf(top, s_m[u * RW + rw][c]);
    const float mine = ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref - top);
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < TW; ++u) {
      const float mu = s_m[u * RW + rw][c];
      sum += mu == -INFINITY ? 0.0f : s_l[u * RW + rw][c] * __builtin_amdgcn_exp2f(mu - top);
    }
    l = sum;
    ref = top;
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] *= mine;
    for (int u = 1; u < TW; ++u) {
      __syncthreads();
      if (tw == u) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) s_o[(rw * 64 + d * 16 + i) * 64 + lane] = o[d][i];
      }
      __syncthreads();
      if (tw == 0) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] += s_o[(rw * 64 + d * 16 + i) * 64 + lane];
      }
    }
    if (tw > 0) return;
  }
  if (!row_on) return;
  const int64_t at = ((int64_t)seq * a.Hq + hq) * a.part_stride + a.part_base + split;
  if (hh == 0) {
    a.pm[at] = ref * kLn2;          // ... = e^(score scale - ref ln 2)
    a.pl[at] = l;
  }
  float *po = a.pacc + at * 128;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) po[32 * d + 8 * (i / 4) + 4 * hh + i % 4] = o[d][i];
}

struct Shape {
  int rw, row_tiles;
};
Shape shape_of(int rows) {
  if (rows <= 32) return Shape{1, 1};
  if (rows <= 64) return Shape{2, 1};
  return Shape{4, (rows + 127) / 128};
}

}  // namespace

int shared_chunk(int rows, int n_kv_heads, int64_t len) {
  const Shape s = shape_of(rows);
  const int64_t want = std::max<int64_t>(1, 512 / std::max<int64_t>(1, (int64_t)n_kv_heads * s.row_tiles));
  return (int)(((len + want - 1) / want + 127) / 128 * 128);
}

hipError_t launch_shared(SharedArgs &a, hipStream_t s) {
  const Shape sh = shape_of(a.rows);
  a.row_tiles = sh.row_tiles;
  const dim3 grid((unsigned)(((int64_t)a.n_split * a.Hkv + 7) / 8 * 8 * sh.row_tiles));
  const bool bf = a.tv.k_fmt == TTKV_BF16;
#define TTKV_SHARED(RW, TW)                                                                          \
  if (bf) hipLaunchKernelGGL((shared_kernel<true, RW, TW>), grid, dim3(256), 0, s, a);              \
  else hipLaunchKernelGGL((shared_kernel<false, RW, TW>), grid, dim3(256), 0, s, a)
  switch (sh.rw) {
    case 1: TTKV_SHARED(1, 4); break;
    case 2: TTKV_SHARED(2, 2); break;
    default: TTKV_SHARED(4, 1); break;
  }
#undef TTKV_SHARED
  return hipGetLastError();
}

}  // namespace ttkv
