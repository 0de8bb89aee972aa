// Device code that the chunk's attention and the tokens' weights have in common: rows of a tier as operands, places of tokens, masks.
#pragma once
#include "ttkv_shared_dev.h"

#include <type_traits>

namespace ttkv {
namespace chunk {

using namespace dev;
using namespace shared;

template <int N>
using num = std::integral_constant<int, N>;

// ---------------------------------------------------------------- rows of a tier on their way into LDS
// Eight channels of a token: fp as they are, codes with what decompresses them.
template <int F>
struct Piece {
  u32x4 w;
};
template <>
struct Piece<TTKV_I8_SYM_G32> {
  u32x2 w;
  uint16_t s;
};
template <>
struct Piece<TTKV_I4_ASYM_G64> {
  uint32_t w, sz;
};
typedef const __attribute__((address_space(1))) u32x2 *gas_u32x2;
typedef const __attribute__((address_space(1))) uint32_t *gas_u32;
typedef const __attribute__((address_space(1))) uint16_t *gas_u16;
// Channels 8 p .. 8 p + 7 of row `row` of a block's section; codes and meta: its addresses.
template <int F>
__device__ __forceinline__ Piece<F> load_piece(uint64_t codes, uint64_t meta, int row, int p) {
  Piece<F> x;
  if constexpr (F == TTKV_I8_SYM_G32) {
    x.w = *(gas_u32x2)(codes + (uint32_t)(row * 128 + p * 8));
    x.s = *(gas_u16)(meta + (uint32_t)(row * 8 + p / 4 * 2));
  } else if constexpr (F == TTKV_I4_ASYM_G64) {
    x.w = *(gas_u32)(codes + (uint32_t)(row * 64 + p * 4));
    x.sz = *(gas_u32)(meta + (uint32_t)(row * 8 + p / 8 * 4));
  } else {
    x.w = *(gas_u32x4)(codes + (uint32_t)(row * 256 + p * 16));
  }
  return x;
}
// v as the nearest number of the product's type and what that leaves.  fp16's first number ends at 65504: the second one has the rest.
template <bool BF>
__device__ __forceinline__ void two_parts(const float (&v)[8], u32x4 &hi, u32x4 &lo) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x = v[2 * i], y = v[2 * i + 1];
    if constexpr (!BF) {
      x = __builtin_amdgcn_fmed3f(x, -65504.0f, 65504.0f);
      y = __builtin_amdgcn_fmed3f(y, -65504.0f, 65504.0f);
    }
    hi[i] = pack2<BF>(x, y);
    const f2 h = unpack2<BF>(hi[i]);
    lo[i] = pack2<BF>(v[2 * i] - h.x, v[2 * i + 1] - h.y);
  }
}
// Which of eight numbers are infinite or none, a bit each; they become 0.
template <bool BF>
__device__ __forceinline__ uint32_t take_wild(u32x4 &w) {
  constexpr uint32_t exp1 = BF ? 0x7f80u : 0x7c00u;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool low = (w[i] & exp1) == exp1, high = (w[i] >> 16 & exp1) == exp1;
    bits |= (low ? 1u << 2 * i : 0u) | (high ? 2u << 2 * i : 0u);
    w[i] &= ~((low ? 0xffffu : 0u) | (high ? 0xffff0000u : 0u));
  }
  return bits;
}
// Eight decompressed channels as two numbers each.
template <bool BF, int F>
__device__ __forceinline__ void unpack_piece(const Piece<F> &x, u32x4 &hi, u32x4 &lo) {
  float v[8];
  if constexpr (F == TTKV_I8_SYM_G32) {
    const float s = h2f(x.s);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)((int)(x.w[i / 4] << (24 - 8 * (i % 4))) >> 24) * s;
  } else {
    const float s = (float)as_h2(x.sz).x, z = (float)as_h2(x.sz).y;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf((float)(x.w >> (4 * i) & 15u), s, z);
  }
  two_parts<BF>(v, hi, lo);
}
template <bool BF, int F, bool CHECK = false>
__device__ __forceinline__ uint32_t put_piece(const Piece<F> &x, char *hi, char *lo) {
  uint32_t wild = 0;
  if constexpr (F == TTKV_I8_SYM_G32 || F == TTKV_I4_ASYM_G64) {
    u32x4 h, l;
    unpack_piece<BF, F>(x, h, l);
    if constexpr (CHECK) wild = take_wild<BF>(h) | take_wild<BF>(l);
    *(u32x4 *)hi = h;
    *(u32x4 *)lo = l;
  } else {
    u32x4 h = x.w;
    if constexpr (CHECK) wild = take_wild<BF>(h);
    *(u32x4 *)hi = h;
  }
  return wild;
}
// Queries of a bf16 model over fp16 tiers (exact inside the fp16 normal range, clamped outside; what is no number stays none).
__device__ __forceinline__ void to_fp16(u32x4 &x) {
  auto clamped = [](float v) { return v != v ? v : fminf(fmaxf(v, -65504.0f), 65504.0f); };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f2 v = unpack2<true>(x[i]);
    x[i] = pack2<false>(clamped(v.x), clamped(v.y));
  }
}

// New token of a query row.
template <typename A>
__device__ __forceinline__ int token_of(const A &a, int row) {
  return a.G == 1 ? row : a.g_magic ? (int)mul_high((uint32_t)row, a.g_magic) : row / a.G;
}
// A place in a run, kept in scalar registers: the KV head's part of a ring block, and a row of it.
struct Place {
  uint64_t base, head, table;
  int64_t rec_bytes;
  int bt, ring_blocks, block, row, seq;
  __device__ __forceinline__ int64_t record() const { return table ? (int64_t)((const_i32)table)[block] : (int64_t)seq * ring_blocks + block; }
  __device__ __forceinline__ void find() { head = base + (table ? (int64_t)((const_i32)table)[block] : (int64_t)block) * rec_bytes; }
  __device__ __forceinline__ Place(const TierView &tv, int seq_, int hkv, int tok) {
    seq = seq_;
    bt = tv.bt;
    ring_blocks = tv.ring_blocks;
    rec_bytes = tv.rec_bytes;
    table = (uint64_t)tv.table;
    base = (uint64_t)tv.base + (int64_t)hkv * tv.head_bytes;
    if (table) table += (uint64_t)((int64_t)seq * ring_blocks) * 4;
    else base += (uint64_t)((int64_t)seq * ring_blocks * rec_bytes);
    if (tok >= ring_blocks * bt) tok -= ring_blocks * bt;
    block = div_bt(tok, bt, tv.bt_magic);
    row = tok - block * bt;
    asm volatile("" : "+s"(bt), "+s"(ring_blocks), "+s"(rec_bytes), "+s"(table), "+s"(base));
    find();
  }
  __device__ __forceinline__ void advance(int rows) {
    row += rows;
    if (row < bt) return;
    do {
      row -= bt;
      block = block + 1 == ring_blocks ? 0 : block + 1;
    } while (row >= bt);
    find();
  }
};

// Tokens from `lim` on count nothing; lim by lane.
__device__ __forceinline__ void mask_from(f16v &sc, int lim, int hh) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (8 * (i / 4) + 4 * hh + i % 4 >= lim) sc[i] = -INFINITY;
    asm volatile("" : "+v"(sc[i]));   // stays a branch, not sixteen selects in every step
  }
}

}  // namespace chunk
}  // namespace ttkv
