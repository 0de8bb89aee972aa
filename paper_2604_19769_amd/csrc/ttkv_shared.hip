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
// registers -> LDS, the next tile's loads in flight while one is computed.
//
// The weights p meet fp16 values as an fp16 number and its remainder (22 bits), bf16 values as three bf16
// numbers (24 bits): the outputs are fp32.
#include "ttkv_attn_dev.h"

#include <algorithm>
#include <type_traits>

namespace ttkv {

namespace {

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
// x - the lower (upper) half of w
__device__ __forceinline__ float minus_low(uint32_t w, float x) {
  float r;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(w), "v"(x));
  return r;
}
__device__ __forceinline__ float minus_high(uint32_t w, float x) {
  float r;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(w), "v"(x));
  return r;
}
// LDS rows: eight rows' 16-byte pieces of one column fall into different banks (keys, 4 banks apart), and so do four rows' 32
// bytes (values, 8 banks apart); every address is one register and a constant.
constexpr int kRowK = 272, kRowV = 288;

// The weights carry 2^kUnit, and the reference moves only when a score is kRoom (in powers of two) above it: the weights stay below
// 2^15, and a wave of 32 rows, some of whose maxima would grow in nearly every step, hardly ever rescales its outputs.
constexpr float kUnit = 8.0f, kRoom = 7.0f;
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
  if (!BF && a.q_fmt == TTKV_BF16) {   // bf16 -> fp16 (exact inside the fp16 normal range, clamped outside)
#pragma unroll
    for (int kb = 0; kb < 8; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f2 v = unpack2<true>(qf[kb][i]);
        qf[kb][i] = pack2<false>(fminf(fmaxf(v.x, -65504.0f), 65504.0f), fminf(fmaxf(v.y, -65504.0f), 65504.0f));
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
// The reference moves up to the largest score so far.
__device__ __forceinline__ void move_reference(Rows &r, float mt, f16v (&o)[4]) {
#pragma clang fp contract(off)
  const float mn = fmaxf(r.m, mt), at = mn * r.cs, was = r.mcs;
  r.f = fabsf(at) < 4194304.0f ? kUnit : 0.0f;   // beyond, f - mcs would not be exact
  r.mcs = mn == -INFINITY ? 0.0f : r.f - at;
  const float alpha = r.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.mcs - was);
  r.l *= alpha;
  rescale(o, alpha);
  r.m = mn;
  r.far = r.f == 0.0f ? mn : (at + kRoom) * r.inv_cs;
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
template <int RW, int TW>
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
  const float up = fabsf(top) < 4194304.0f ? kUnit : 0.0f;
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

// ---------------------------------------------------------------- up to 64 rows per KV head
// Bound: memory.  One workgroup of eight waves per CU: TW teams of RW waves (32 rows each) take the item's steps of 32 tokens
// in turn (with a run of its own for each team, 2048 tokens of 256 items, the streams a power of two apart took 59.7 us instead of
// 49.8).  A team loads its steps' rows itself and needs no other; K of one step and V of the step before
// are always on their way, and leave their registers for LDS where the step before has been read.
template <bool BF, int RW, int TW>
__global__ __launch_bounds__(512, 1) void shared_kernel(const SharedArgs a) {
  static_assert(RW * TW == 8 && (RW == 1 || RW == 2), "eight waves");
  constexpr bool ALONE = RW == 1;   // a team of one waits for nobody: LDS takes a wave's stores and reads in order
  constexpr int NL = 8 / RW, LR = 4 * RW;                        // 16-byte loads of K (V) per thread; rows apart
  constexpr int kKeys = 32 * kRowK, kStep = 32 * (kRowK + kRowV), NBUF = ALONE ? 1 : 2;
  __shared__ __align__(16) char s_tile[TW * NBUF * kStep];       // per team: keys and values of one step (two); at the end what the waves exchange
  static_assert(TW * NBUF * kStep >= 8 * (16 - 16 / TW) * 1024, "room for what the waves exchange");
  __shared__ float s_m[8][32], s_l[8][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tw = wave / RW, rw = wave % RW;
  const int c = lane & 31, hh = lane >> 5;
  Item it;
  if (!item_of(a, it)) return;
  const int mine = it.n_tok - 32 * tw;                           // tokens from the team's first step on; it takes every TW-th
  Cursor keys(a, it.hkv, it.begin + (mine > 0 ? 32 * tw : 0)), values = keys;
  values.base += a.tv.v_off;
  values.head += a.tv.v_off;
  int k_left = mine, v_left = mine;                              // tokens from the cursors on
  const int lr = (threadIdx.x & (64 * RW - 1)) >> 4, lp = threadIdx.x & 15;
  u32x4 kr[NL], vr[NL];
  auto load = [&](Cursor &at, int &left, u32x4 (&x)[NL]) __attribute__((always_inline)) {   // the team's next step, if there is one; rows behind the item's end: its last one
    if (left <= 0) return;
    const int len = min(left, 32);
    const uint64_t head = at.rows();
#pragma unroll
    for (int i = 0; i < NL; ++i) x[i] = __builtin_nontemporal_load((gas_u32x4)(head + (uint32_t)(min(lr + LR * i, len - 1) * 256 + lp * 16)));
    left -= 32 * TW;
    if (left > 0) at.advance(32 * TW);
  };
  char *const team = s_tile + tw * NBUF * kStep;
  const char *const k_at = team + k_lane(lane), *const v_at = team + kKeys + v_lane(lane);
  char *const k_put = team + lr * kRowK + lp * 16, *const v_put = team + kKeys + lr * kRowV + lp * 16;
  auto put = [&](char *to, int row_bytes, const u32x4 (&x)[NL]) __attribute__((always_inline)) {
    if constexpr (ALONE) asm volatile("" ::: "memory");          // (the compiler has to leave the order as it is)
#pragma unroll
    for (int i = 0; i < NL; ++i) *(u32x4 *)(to + i * LR * row_bytes) = x[i];
    if constexpr (ALONE) asm volatile("" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < NL; ++i) kr[i] = vr[i] = u32x4{0, 0, 0, 0};
  load(keys, k_left, kr);
  load(values, v_left, vr);
  u32x4 qf[8];
  Rows r = begin_rows<BF>(a, (it.row_tile * RW + rw) * 32 + c, it.hkv, hh, qf);
  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  put(k_put, kRowK, kr);
  load(keys, k_left, kr);
  put(v_put, kRowV, vr);
  load(values, v_left, vr);
  // (with barriers all teams take as many steps as the first)
  const int n_steps = ((ALONE ? max(mine, 0) : it.n_tok) + 32 * TW - 1) / (32 * TW);
  int now = 0;   // buffer of the step
  for (int t = 0; t < n_steps; ++t) {
    if (!ALONE) __syncthreads();   // the step is in its buffer; everybody is done with the other one
    const int next = ALONE ? 0 : kStep - now, len = mine - 32 * TW * t;
    f16v sc = {};
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) sc = mma<BF>(*(const u32x4 *)(k_at + now + 32 * kb), qf[kb], sc);
    put(k_put + next, kRowK, kr);
    load(keys, k_left, kr);
    if (len > 0) {   // (wave-uniform)
      if (len < 32) mask_step(sc, len, hh);
      const float mt = step_max(sc);
      if (__any(mt > r.far)) move_reference(r, mt, o);
      u32x4 p[parts_of<BF>()][2];
#pragma unroll
      for (int i = 0; i < 8; ++i) weigh<BF>(r, sc, i, p);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int b = 0; b < 2; ++b) add_values<BF>(o[d], value_operand(v_at + now, d, b), p, b);
    }
    put(v_put + next, kRowV, vr);
    load(values, v_left, vr);
    now = next;
  }
  end_rows(r);
  join_and_store<RW, TW>(a, r, o, rw, tw, lane, it.split, s_tile, s_m, s_l);
}

// ---------------------------------------------------------------- more rows: 128 per workgroup
// Bound: the matrix cores.  The steps of 32 tokens overlap inside a wave: while the softmax of step s runs on the vector unit, the
// matrix cores work on the values of step s - 1 and the scores of step s + 1, none of which depends on it.  LDS holds two
// steps' keys and values each (s + 1 and s + 2; s - 1 and s), one barrier per step.
template <bool BF>
__global__ __launch_bounds__(512, 1) void shared_rows_kernel(const SharedArgs a) {
  constexpr int NP = parts_of<BF>(), kKeys = 32 * kRowK, kValues = 32 * kRowV, kHalf = 2 * (kKeys + kValues);
  __shared__ __align__(16) char s_tile[2 * kHalf];   // per half: keys of even and odd steps, values of even and odd steps
  static_assert(2 * kHalf >= 8 * 8 * 1024, "room for what the waves exchange");
  __shared__ float s_m[8][32], s_l[8][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hh = lane >> 5, rw = wave & 3, half = wave >> 2;
  Item it;
  if (!item_of(a, it)) return;
  // Four waves take the item's first half, four the second; one without tokens looks at a live one that counts nothing.
  const int n_half = a.chunk / 2, n_steps = ((min(it.n_tok, n_half) + 31) / 32 + 1) & ~1;   // in pairs: the last ones may have no live token
  const int n_tok = half ? max(it.n_tok - n_half, 0) : min(it.n_tok, n_half);
  const bool idle = (it.row_tile * 4 + rw) * 32 >= a.rows;   // a wave without rows only helps with the tiles
  if (half && n_tok) it.begin += n_half;
  const int lr = threadIdx.x >> 4 & 15, lp = threadIdx.x & 15;
  char *const s_half = s_tile + half * kHalf;
  const char *const k_at = s_half + k_lane(lane), *const v_at = s_half + 2 * kKeys + v_lane(lane);
  char *const k_put = s_half + lr * kRowK + lp * 16, *const v_put = s_half + 2 * kKeys + lr * kRowV + lp * 16;
  u32x4 kr[2], vr[2];
  // rows lr and lr + 16 of the next step; behind the item's end rows of its last one again
  Cursor keys(a, it.hkv, it.begin), values = keys;
  values.base += a.tv.v_off;
  values.head += a.tv.v_off;
  int k_left = max(n_tok, 1), v_left = k_left;   // tokens from the cursors on
  auto load = [&](Cursor &at, int &left, u32x4 (&x)[2]) __attribute__((always_inline)) {
    const uint64_t head = at.rows();
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = *(gas_u32x4)(head + (uint32_t)(min(lr + 16 * i, left - 1) * 256 + lp * 16));
    if (left > 32) {
      left -= 32;
      at.advance(32);
    }
  };
  auto load_keys = [&]() __attribute__((always_inline)) { load(keys, k_left, kr); };
  auto load_values = [&]() __attribute__((always_inline)) { load(values, v_left, vr); };
  auto put_keys = [&](int odd) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *(u32x4 *)(k_put + odd * kKeys + i * 16 * kRowK) = kr[i];
  };
  auto put_values = [&](int odd) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *(u32x4 *)(v_put + odd * kValues + i * 16 * kRowV) = vr[i];
  };
  // everything that the first steps need is asked for at once
  u32x4 first[2][2];
  load(keys, k_left, first[0]);
  load(keys, k_left, first[1]);
  load_keys();
  load_values();
  u32x4 qf[8];
  Rows r = begin_rows<BF>(a, (it.row_tile * 4 + rw) * 32 + c, it.hkv, hh, qf);
  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  // Step s (of parity ODD): sc its scores, p the weights of step s - 1; next, pn receive the scores of s + 1 and its own weights.
  auto body = [&](int s, auto odd_tag, f16v &sc, f16v &next, u32x4 (&p)[NP][2], u32x4 (&pn)[NP][2]) __attribute__((always_inline)) {
    constexpr int ODD = decltype(odd_tag)::value;
    __syncthreads();   // keys of s + 1 and values of s - 1 are there; everybody is done with those of s and s - 2
    const char *const v_old = v_at + (1 - ODD) * kValues, *const k_next = k_at + (1 - ODD) * kKeys;
    if (idle) {
      put_keys(ODD);
      put_values(ODD);
      load_keys();
      load_values();
      return;
    }
    const float mt = step_max(sc);
    if (__any(mt > r.far)) {
      if (s) {   // the outputs take the weights of the old reference first; what is added below is then nothing
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int b = 0; b < 2; ++b) add_values<BF>(o[d], value_operand(v_old, d, b), p, b);
#pragma unroll
        for (int u = 0; u < NP; ++u) p[u][0] = p[u][1] = u32x4{0, 0, 0, 0};
      }
      move_reference(r, mt, o);
    }
    put_keys(ODD);       // of s + 2
    put_values(ODD);     // of s
    load_keys();         // of s + 3
    load_values();       // of s + 1
    f16v nx = {};
#pragma unroll
    for (int g = 0; g < 8; ++g) {   // a product of the scores, two or three of the values, an eighth of the softmax
      add_values<BF>(o[g / 2], value_operand(v_old, g / 2, g % 2), p, g % 2);
      nx = mma<BF>(*(const u32x4 *)(k_next + 32 * g), qf[g], nx);
      weigh<BF>(r, sc, g, pn);
    }
    const int left = n_tok - 32 * (s + 1);
    if (left < 32) mask_step(nx, left, hh);
    next = nx;
  };
  u32x4 p0[NP][2], p1[NP][2];
#pragma unroll
  for (int u = 0; u < NP; ++u) p0[u][0] = p0[u][1] = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int odd = 0; odd < 2; ++odd)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      *(u32x4 *)(k_put + odd * kKeys + i * 16 * kRowK) = first[odd][i];
      if (odd) *(u32x4 *)(v_put + kValues + i * 16 * kRowV) = u32x4{0, 0, 0, 0};   // there is no step before the first: weights of zero meet zeros
    }
  __syncthreads();
  f16v s0 = {}, s1;
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) s0 = mma<BF>(*(const u32x4 *)(k_at + 32 * kb), qf[kb], s0);
  if (n_tok < 32) mask_step(s0, n_tok, hh);
  for (int s = 0; s < n_steps; s += 2) {
    body(s, std::integral_constant<int, 0>{}, s0, s1, p0, p1);
    body(s + 1, std::integral_constant<int, 1>{}, s1, s0, p1, p0);
  }
  __syncthreads();
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int b = 0; b < 2; ++b) add_values<BF>(o[d], value_operand(v_at + kValues, d, b), p0, b);
  end_rows(r);
  join_and_store<4, 2>(a, r, o, rw, half, lane, it.split, s_tile, s_m, s_l);
}

// Query rows per workgroup, workgroups along the rows.
struct Shape {
  int rows, row_tiles, resident, tokens;   // resident: workgroups on the chip at once; tokens of an item: a multiple of this
};
Shape shape_of(int rows) {
  if (rows <= 32) return Shape{32, 1, 256, 32};
  if (rows <= 64) return Shape{64, 1, 256, 32};
  return Shape{128, (rows + 127) / 128, 256, 128};
}

}  // namespace

int shared_chunk(int rows, int n_kv_heads, int64_t len) {
  const Shape s = shape_of(rows);
  const int64_t most = std::max<int64_t>(1, s.resident / std::max<int64_t>(1, (int64_t)n_kv_heads * s.row_tiles));
  const int64_t want = std::min(most, (len + 63) / 64);
  return (int)(((len + want - 1) / want + s.tokens - 1) / s.tokens * s.tokens);
}

hipError_t launch_shared(SharedArgs &a, hipStream_t s) {
  const Shape sh = shape_of(a.rows);
  a.row_tiles = sh.row_tiles;
  const int64_t units = ((int64_t)a.n_split * a.Hkv + 7) / 8 * 8;
  a.g_magic = a.rows < 1 << 20 ? magic_heads(1 << 20, a.G) : 0;
  auto magic = [](int64_t most, int d) { return d > 1 && most * d < (1ll << 32) ? (uint32_t)(((1ll << 32) + d - 1) / d) : 0u; };
  a.hkv_magic = magic(units, a.Hkv);
  a.tiles_magic = magic(units / 8 * sh.row_tiles, sh.row_tiles);
  const dim3 grid((unsigned)(units * sh.row_tiles)), block(512);
  const bool bf = a.tv.k_fmt == TTKV_BF16;
  switch (sh.rows) {
    case 32:
      if (bf) hipLaunchKernelGGL((shared_kernel<true, 1, 8>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((shared_kernel<false, 1, 8>), grid, block, 0, s, a);
      break;
    case 64:
      if (bf) hipLaunchKernelGGL((shared_kernel<true, 2, 4>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((shared_kernel<false, 2, 4>), grid, block, 0, s, a);
      break;
    default:
      if (bf) hipLaunchKernelGGL(shared_rows_kernel<true>, grid, block, 0, s, a);
      else hipLaunchKernelGGL(shared_rows_kernel<false>, grid, block, 0, s, a);
      break;
  }
  return hipGetLastError();
}

}  // namespace ttkv
