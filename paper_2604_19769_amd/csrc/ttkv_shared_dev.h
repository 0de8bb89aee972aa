// Device code that the shared-prefix kernels have in common: the softmax of a wave's query rows, operands, the walk over the
// run, the join of a workgroup's waves.
#pragma once
#include "ttkv_attn_dev.h"

namespace ttkv {
namespace shared {

using namespace dev;

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s4 *las_s4;
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));   // the partials may start at any float

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
// x - the lower (upper) half of w, one instruction: -1 is kept from the compiler, which would convert and subtract otherwise.  (As inline
// assembly it would not be kept apart from matrix instructions that are still at its registers.)
__device__ __forceinline__ float minus_one() {
  float m = -1.0f;
  asm("" : "+s"(m));
  return m;
}
__device__ __forceinline__ float minus_low(uint32_t w, float x) { return fmaf((float)as_h2(w).x, minus_one(), x); }
__device__ __forceinline__ float minus_high(uint32_t w, float x) { return fmaf((float)as_h2(w).y, minus_one(), x); }
// LDS rows: eight rows' 16-byte pieces of one column fall into different banks (keys, 4 banks apart), and so do four rows' 32
// bytes (values, 8 banks apart); every address is one register and a constant.
constexpr int kRowK = 272, kRowV = 288;

// The weights carry 2^unit, and the reference moves only when a score is `room` (in powers of two) above it, so that a wave of 32 rows, some of
// whose maxima would grow in nearly every step, rescales its outputs now and then only.  Over bf16 values the two take each other back: no weight is
// above 1, and an average of values near bf16's largest stays finite on its way.  Over fp16 values weights stay below 2^16 and are good to
// 2^-25, half of fp16's smallest step: 22 bits down to 2^-17 of the reference and 2^-39 of it below, as in the decode kernels.  (2^8 and
// room for 2^7 took as long; results made of weights 2^-20 of the largest, whose values are 0, were 7e-5 off.  2^11 to 2^13 save 1-2 %
// of many rows' time.)
template <bool BF>
constexpr float unit_of() { return BF ? -7.0f : 14.0f; }
template <bool BF>
constexpr float room_of() { return BF ? 7.0f : 1.5f; }
constexpr float kFar = 1048576.0f;   // references beyond (in powers of two) carry no unit: f - mcs would not be exact, nor `far` to a fraction of one
template <bool BF>
constexpr int parts_of() { return BF ? 3 : 2; }   // numbers that hold a weight

// What a wave keeps of its 32 query rows beside the outputs: lane -> row lane % 32, both halves alike but for l.
struct Rows {
  float cs, inv_cs;                        // scores are kept in the log2 domain
  float m, l, mcs, f, far;                 // a token's weight: exp2(score cs + mcs) = 2^f e^(score - m); a score beyond `far` moves m
  int seq, hq;
  bool on;
};
// Row `row` of the KV head's rows (the last one again behind them) and its channels 16 kb + 8 hh .. + 7 in qf[kb].
template <bool BF>
__device__ __forceinline__ Rows begin_rows(const SharedArgs &a, int row, int hkv, int hh, u32x4 (&qf)[8]) {
  Rows r;
  r.on = row < a.rows;
  row = min(row, a.rows - 1);
  const int n = a.G == 1 ? row : a.g_magic ? (int)mul_high((uint32_t)row, a.g_magic) : row / a.G;
  r.seq = a.listed ? a.member[n] : n;
  r.hq = hkv * a.G + row - n * a.G;
  const u32x4 *qp = (const u32x4 *)((const uint16_t *)a.q + ((int64_t)r.seq * a.Hq + r.hq) * 128);
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) qf[kb] = qp[2 * kb + hh];
  if (!BF && a.q_fmt == TTKV_BF16) {   // bf16 -> fp16 (exact inside the fp16 normal range, clamped outside; what is no number stays none)
    auto clamped = [](float x) { return x != x ? x : fminf(fmaxf(x, -65504.0f), 65504.0f); };
#pragma unroll
    for (int kb = 0; kb < 8; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f2 v = unpack2<true>(qf[kb][i]);
        qf[kb][i] = pack2<false>(clamped(v.x), clamped(v.y));
      }
  }
  r.cs = a.scale * kLog2e;
  r.inv_cs = 1.0f / r.cs;
  r.m = r.far = -INFINITY;
  r.l = r.mcs = r.f = 0.0f;
  return r;
}
// The largest of a step's scores, in both halves.
__device__ __forceinline__ float step_max(const f16v &sc) {
  float mt = sc[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) mt = fmaxf(mt, sc[i]);
  const f2 both = both32(mt);
  return fmaxf(both.x, both.y);
}
__device__ __forceinline__ void rescale(f16v (&o)[4], float by) {
#pragma unroll
  for (int d = 0; d < 4; ++d) o[d] *= by;
}
// The reference moves up to the largest score so far, to the nearest power of two; what was added up by then counts 2^-k as much, exactly.
template <bool BF>
__device__ __forceinline__ float move_reference(Rows &r, float mt, f16v (&o)[4]) {
#pragma clang fp contract(off)
  const float mn = fmaxf(r.m, mt), at = __builtin_rintf(mn * r.cs), was = r.mcs;
  r.f = fabsf(at) < kFar ? unit_of<BF>() : 0.0f;
  r.mcs = mn == -INFINITY ? 0.0f : r.f - at;
  const float alpha = r.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.mcs - was);
  r.l *= alpha;
  rescale(o, alpha);
  r.m = mn;
  r.far = r.f == 0.0f ? mn : (at + room_of<BF>()) * r.inv_cs;
  return alpha;
}
// Scores of tokens from `left` on count nothing.
__device__ __forceinline__ void mask_step(f16v &sc, int left, int hh) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (8 * (i / 4) + 4 * hh + i % 4 >= left) sc[i] = -INFINITY;
    asm volatile("" : "+v"(sc[i]));   // stays a branch, not sixteen selects in every step
  }
}
// Weights 2 i and 2 i + 1 of a step as NP packed numbers each.
template <bool BF>
__device__ __forceinline__ void weigh(Rows &r, const f16v &sc, int i, u32x4 (&p)[parts_of<BF>()][2]) {
  float w0 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i], r.cs, r.mcs)), w1 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i + 1], r.cs, r.mcs));
  r.l += w0 + w1;
#pragma unroll
  for (int u = 0; u < parts_of<BF>(); ++u) {
    const uint32_t w = pack2<BF>(w0, w1);
    p[u][i / 4][i % 4] = w;
    if constexpr (BF) {
      const f2 x = unpack2<true>(w);
      w0 -= x.x;
      w1 -= x.y;
    } else {
      w0 = minus_low(w, w0);
      w1 = minus_high(w, w1);
    }
  }
}
// Value operand: channels 32 d .. + 31 (rows), tokens of half b in the order of the scores' registers.
__device__ __forceinline__ u32x4 value_operand(const char *v_at, int d, int b) {
  u32x4 va;
#pragma unroll
  for (int jb = 0; jb < 2; ++jb) {
    const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((las_s4)(v_at + (16 * b + 8 * jb) * kRowV + 64 * d));
    const u32x2 y = __builtin_bit_cast(u32x2, x);
    va[2 * jb] = y.x;
    va[2 * jb + 1] = y.y;
  }
  return va;
}
template <bool BF>
__device__ __forceinline__ void add_values(f16v &o, const u32x4 &va, const u32x4 (&p)[parts_of<BF>()][2], int b) {
#pragma unroll
  for (int u = 0; u < parts_of<BF>(); ++u) o = mma<BF>(va, p[u][b], o);
}
__device__ __forceinline__ void end_rows(Rows &r) {   // l over both halves
  const f2 both = both32(r.l);
  r.l = both.x + both.y;
}
// A place in the run: the KV head's part of a ring block and a row of it.  Everything a step further needs is kept in scalar
// registers, and the block table is read once per block: a scalar load in every step would be waited for together with the
// LDS reads that are in flight.
// Addresses are numbers until a load: a pointer that has been through a register constraint is loaded by flat instructions,
// which the LDS waits wait for as well.
typedef const __attribute__((address_space(1))) u32x4 *gas_u32x4;
typedef const __attribute__((address_space(4))) int32_t *const_i32;
struct Cursor {
  uint64_t base, head;   // the KV head's part of record 0, and of the block's
  uint64_t table;        // written before the launch: read through the constant address space
  int64_t rec_bytes;
  int bt, ring_blocks, block, row;
  __device__ __forceinline__ void find() { head = base + (table ? (int64_t)((const_i32)table)[block] : (int64_t)block) * rec_bytes; }
  __device__ __forceinline__ Cursor(const SharedArgs &a, int hkv, int token) {
    bt = a.tv.bt;
    ring_blocks = a.tv.ring_blocks;
    rec_bytes = a.tv.rec_bytes;
    table = (uint64_t)a.tv.table;
    base = (uint64_t)a.tv.base + (int64_t)hkv * a.tv.head_bytes;
    int tok = a.first_tok + token;
    if (tok >= ring_blocks * bt) tok -= ring_blocks * bt;
    block = div_bt(tok, bt, a.tv.bt_magic);
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
  __device__ __forceinline__ uint64_t rows() const { return head + row * 256; }
};
// workgroups that read the same tokens of a KV head lie on one XCD, one behind the other
struct Item {
  int row_tile, split, hkv, begin, n_tok;
};
__device__ __forceinline__ bool item_of(const SharedArgs &a, Item &it) {
  // all that the look-ups read, asked for at once: a launch's arguments are in no cache when its first workgroups start
  asm volatile("" ::"s"(a.row_tiles), "s"(a.Hkv), "s"(a.chunk), "s"(a.len), "s"(a.first_tok), "s"(a.G), "s"(a.q), "s"(a.rows), "s"(a.tv.base),
               "s"(a.tv.bt), "s"(a.part_stride), "s"(a.pm));
  const int x8 = blockIdx.x >> 3;
  const int x = a.row_tiles == 1 ? x8 : a.tiles_magic ? (int)mul_high((uint32_t)x8, a.tiles_magic) : x8 / a.row_tiles;
  const int unit = 8 * x + (blockIdx.x & 7);
  it.row_tile = x8 - x * a.row_tiles;
  it.split = a.Hkv == 1 ? unit : a.hkv_magic ? (int)mul_high((uint32_t)unit, a.hkv_magic) : unit / a.Hkv;
  it.hkv = unit - it.split * a.Hkv;
  it.begin = it.split * a.chunk;
  it.n_tok = min(a.chunk, a.len - it.begin);   // at least 1
  return unit < a.n_split * a.Hkv;
}
// the lane's place in a step's keys and values
__device__ __forceinline__ int k_lane(int lane) { return (lane & 31) * kRowK + 16 * (lane >> 5); }
__device__ __forceinline__ int v_lane(int lane) { return (4 * (lane >> 5) + ((lane & 15) >> 2)) * kRowV + 32 * ((lane >> 4) & 1) + 8 * (lane & 3); }

// The TW waves of one row block add up, each 128 / TW channels of the rows, and store them.  s_o: (16 - 16 / TW) KiB per wave; all
// waves of the workgroup take part.  Weights of a wave are exp2(score cs + mcs).
template <bool BF, int RW, int TW>
__device__ __forceinline__ void join_and_store(const SharedArgs &a, const Rows &r, const f16v (&o)[4], int rw, int tw, int lane, int split, char *s_o,
                                               float (*s_m)[32], float (*s_l)[32]) {
  constexpr int OWN = 16 / TW;   // pieces of 4 registers (channels 8 k + 4 hh .. + 3 of the block of 32) that a wave ends up with
  const int c = lane & 31, hh = lane >> 5;
  __syncthreads();   // everybody is done with the tiles
  if (hh == 0) {
    s_m[tw * RW + rw][c] = r.m == -INFINITY ? -INFINITY : -r.mcs;
    s_l[tw * RW + rw][c] = r.l;
  }
  // what the other waves of the row block need: [giver][taker, without the giver][piece][lane]
  auto place = [&](int giver, int taker, int e) __attribute__((always_inline)) -> float4 * {
    const int slot = taker - (taker > giver);
    return (float4 *)(s_o + ((((giver * RW + rw) * (TW - 1) + slot) * OWN + e) * 64 + lane) * 16);
  };
  auto piece = [&](int q) __attribute__((always_inline)) -> float4 {
    const f16v &x = o[q / 4];
    const int k = 4 * (q % 4);
    return float4{x[k], x[k + 1], x[k + 2], x[k + 3]};
  };
#pragma unroll
  for (int t = 0; t < TW; ++t)
    if (t != tw)   // (wave-uniform)
#pragma unroll
      for (int e = 0; e < OWN; ++e) *place(tw, t, e) = piece(t * OWN + e);
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < TW; ++u) top = fmaxf(top, s_m[u * RW + rw][c]);
  // the reference without the weights' power of two (exact: top is that of some wave)
  const float up = fabsf(top) < kFar ? unit_of<BF>() : 0.0f;
  float by[TW], l = 0.0f;
#pragma unroll
  for (int u = 0; u < TW; ++u) {
    const float mu = s_m[u * RW + rw][c];
    by[u] = mu == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mu - top) - up);
    l = fmaf(s_l[u * RW + rw][c], by[u], l);
  }
  const int64_t at = ((int64_t)r.seq * a.Hq + r.hq) * a.part_stride + a.part_base + split;
  float *const po = a.pacc + at * 128 + 4 * hh;
#pragma unroll
  for (int w = 0; w < TW; ++w) {
    if (w != tw) continue;
#pragma unroll
    for (int e = 0; e < OWN; ++e) {
      const int q = w * OWN + e;
      const float4 x = piece(q);
      float4 y = {x.x * by[w], x.y * by[w], x.z * by[w], x.w * by[w]};
#pragma unroll
      for (int u = 0; u < TW; ++u) {
        if (u == w) continue;
        const float4 z = *place(u, w, e);
        y.x = fmaf(z.x, by[u], y.x);
        y.y = fmaf(z.y, by[u], y.y);
        y.z = fmaf(z.z, by[u], y.z);
        y.w = fmaf(z.w, by[u], y.w);
      }
      if (r.on) *(float4_any *)(po + 8 * q) = float4_any{y.x, y.y, y.z, y.w};
    }
  }
  if (r.on && hh == 0 && tw == 0) {
    a.pm[at] = (top + up) * kLn2;   // the weights are e^(score scale - this)
    a.pl[at] = l;
  }
}

}  // namespace shared
}  // namespace ttkv
