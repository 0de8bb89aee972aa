// Device code that the chunk's attention and the tokens' weights have in common: rows of a tier as operands, places of tokens, masks.
#pragma once
#include "ttkv_shared_dev.h"

#include <type_traits>

namespace ttkv {
namespace chunk {

using namespace dev;
using namespace shared;

constexpr bool is_quant(int f) { return f != TTKV_F16 && f != TTKV_BF16; }

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
// Which of eight numbers are infinite or none, a bit each; they become 0.
template <bool BF>
__device__ __forceinline__ uint32_t take_wild(u32x4 &w) {
  constexpr uint32_t exps = BF ? 0x7f807f80u : 0x7c007c00u, one = BF ? 0x00800080u : 0x04000400u;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = ((w[i] & exps) + one) >> 15 & 0x10001u;   // an exponent of ones runs over into the sign's place
    bits |= (t | t >> 15) << 2 * i;
    w[i] &= ~(t * 0xffffu);
  }
  bits &= 0xffu;
  return bits;
}
// Eight decompressed channels as fp16 numbers and what those leave (22 bits; the first ones end at 65504, the others have the rest).  Codes
// are written into the mantissa of 1024 and are exact; code x scale (+ zero) in packed fp16 is rounded once, and the remainder comes from fused
// steps in fp32.
template <int F, bool TWO>
__device__ __forceinline__ void unpack_piece(const Piece<F> &x, u32x4 &hi, u32x4 &lo) {
  h2 s2, z2 = {};
  uint32_t n[4];
  float size;    // infinite where the scale is, or the zero point
  bool beyond;   // some value may
  if constexpr (F == TTKV_I8_SYM_G32) {
    const _Float16 s = __builtin_bit_cast(_Float16, x.s);
    s2 = h2{s, s};
    size = fabsf((float)s);
    beyond = !(size < 515.0f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w = x.w[i] ^ 0x80808080u;                                // code + 128
      n[2 * i] = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u);          // 1024 + that, two at a time
      n[2 * i + 1] = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = __builtin_bit_cast(uint32_t, as_h2(n[i]) - h2{(_Float16)1152, (_Float16)1152});
  } else {
    const h2 sz = as_h2(x.sz);
    s2 = h2{sz.x, sz.x};
    z2 = h2{sz.y, sz.y};
    size = fmaf(15.0f, fabsf((float)sz.x), fabsf((float)sz.y));
    beyond = !(size < 65504.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {                                             // nibbles 2 i and 2 i + 1
      const uint32_t w = x.w >> (8 * i);
      n[i] = __builtin_bit_cast(uint32_t, as_h2((w & 15u) | (w << 12 & 0xf0000u) | 0x64006400u) - h2{(_Float16)1024, (_Float16)1024});
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h2 h;
    if constexpr (F == TTKV_I8_SYM_G32) h = as_h2(n[i]) * s2;
    else h = __builtin_elementwise_fma(as_h2(n[i]), s2, z2);
    hi[i] = __builtin_bit_cast(uint32_t, h);
  }
  if (__any(beyond)) {
    // (what is infinite stays so: of two numbers the other one is)
    const float top = TWO || size < INFINITY ? 65504.0f : INFINITY;
    auto end = [&](_Float16 v) { return v != v ? v : (_Float16)fminf(fmaxf((float)v, -top), top); };
#pragma unroll
    for (int i = 0; i < 4; ++i) hi[i] = __builtin_bit_cast(uint32_t, h2{end(as_h2(hi[i]).x), end(as_h2(hi[i]).y)});
  }
  if constexpr (TWO) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float m1 = minus_one(), s = (float)s2.x;
      float a, b;
      if constexpr (F == TTKV_I8_SYM_G32) {
        a = fmaf((float)as_h2(n[i]).x, s, -(float)as_h2(hi[i]).x);
        b = fmaf((float)as_h2(n[i]).y, s, -(float)as_h2(hi[i]).y);
      } else {
        a = fmaf((float)as_h2(n[i]).x, s, fmaf((float)as_h2(hi[i]).x, m1, (float)z2.x));
        b = fmaf((float)as_h2(n[i]).y, s, fmaf((float)as_h2(hi[i]).y, m1, (float)z2.x));
      }
      lo[i] = pack2<false>(a, b);
    }
  }
}
template <bool BF, int F, bool TWO, bool CHECK = false>
__device__ __forceinline__ uint32_t put_piece(const Piece<F> &x, char *hi, char *lo) {
  uint32_t wild = 0;
  if constexpr (is_quant(F)) {
    u32x4 h, l;
    unpack_piece<F, TWO>(x, h, l);
    if constexpr (CHECK) wild = take_wild<false>(h);
    if constexpr (CHECK && TWO) wild |= take_wild<false>(l);
    *(u32x4 *)hi = h;
    if constexpr (TWO) *(u32x4 *)lo = l;
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
// A KV head's part of a sequence's ring, in scalar registers, and places in it.
struct Ring {
  uint64_t base, table;
  int64_t rec_bytes;
  int bt, blocks;
  __device__ __forceinline__ Ring(const TierView &tv, int seq, int hkv) {
    bt = tv.bt;
    blocks = tv.ring_blocks;
    rec_bytes = tv.rec_bytes;
    table = (uint64_t)tv.table;
    base = (uint64_t)tv.base + (int64_t)hkv * tv.head_bytes;
    if (table) table += (uint64_t)((int64_t)seq * blocks) * 4;
    else base += (uint64_t)((int64_t)seq * blocks * rec_bytes);
    asm volatile("" : "+s"(bt), "+s"(blocks), "+s"(rec_bytes), "+s"(table), "+s"(base));
  }
};
struct Place {
  uint64_t head;   // the block's part of the KV head
  int block, row;
  __device__ __forceinline__ void find(const Ring &g) {
    head = g.base + (g.table ? (int64_t)((const_i32)g.table)[block] : (int64_t)block) * g.rec_bytes;
  }
  __device__ __forceinline__ Place(const Ring &g, uint32_t magic, int tok) {
    if (tok >= g.blocks * g.bt) tok -= g.blocks * g.bt;
    block = div_bt(tok, g.bt, magic);
    row = tok - block * g.bt;
    find(g);
  }
  __device__ __forceinline__ void advance(const Ring &g, int rows) {
    row += rows;
    if (row < g.bt) return;
    do {
      row -= g.bt;
      block = block + 1 == g.blocks ? 0 : block + 1;
    } while (row >= g.bt);
    find(g);
  }
};
// Tokens from `lim` on count nothing; lim by lane.
__device__ __forceinline__ void mask_from(f16v &sc, int lim, int hh) {
  const int left = lim - 4 * hh;   // (against numbers that an instruction holds)
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (8 * (i / 4) + i % 4 >= left) sc[i] = -INFINITY;
    asm volatile("" : "+v"(sc[i]));   // stays a branch, not sixteen selects in every step
  }
}

}  // namespace chunk
}  // namespace ttkv
