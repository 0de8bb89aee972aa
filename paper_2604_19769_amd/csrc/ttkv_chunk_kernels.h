// Attention of a chunk of new tokens over the tiers that hold them and everything before them: what a prompt, a part of one, or a few
// drafted tokens ask of the cache.  The query rows of a KV head are its G query heads in every new token, row r = (token r / G, head r % G),
// and a row sees the tokens up to its own:
//       S^T[token][row] = sum_d K[token][d] Q[row][d],     O^T[d][row] += sum_token V[token][d] P[token][row]
// with the running maximum and sum of the softmax in between.  Both products are v_mfma_f32_32x32x16 with tokens (channels) as rows and query
// rows as columns, so a lane has 16 scores of ONE row and the scores' registers are the second product's operand as they lie.
//
// Outputs are 16 bits wide, so the weights are rounded once to the product's type; their sum, the maximum and the log-sum-exp stay fp32.
// Quantized tiers are worked on in fp16 whatever the others' type, in front of them.  Their rows are decompressed on their way into LDS, keys
// into two numbers each (22 bits: the log-sum-exp is an fp32 number), values into two where the outputs are fp16, into one where bf16 outputs
// end far above what that rounds.  (fp16 outputs over bf16 tiers: the weights have bf16's 8 bits there too.)
//
// A kernel knows the formats that it meets (Q: none, one, or all of the quantized ones): with the loops of all of them in every kernel, registers end in
// scratch (20001 int8 tokens 1423 us instead of 1193, int4 turns 106 instead of 95).  Where a launch's tiers have several quantized formats it takes the
// kernels of all of them, and there 14 to 60 registers do end in scratch: 2048 new tokens of 32 / 8 fp16 heads over 10000 int8 and 10000 int4 tokens
// 1405 us, over each of the two alone 665; 16 x 12 new ones over 4096 and 4096 142, alone 78 and 85.
#pragma once
#include "ttkv_chunk_dev.h"

#include <algorithm>

namespace ttkv {
namespace chunk {

// Weights are 2^unit times e^(score - reference), and the reference moves only when a score is `room` above it (powers of two): over
// bf16 values no weight is above 1, over fp16 values they stay below 2^16 and keep 11 bits down to 2^-22 of the reference.
template <bool BF>
constexpr float unit16() { return BF ? -7.0f : 8.0f; }
constexpr float kRoom16 = 7.0f;

typedef __attribute__((address_space(3))) char *las_char;

// ---------------------------------------------------------------- items
struct ChunkItem {
  int slot, entry, seq, hkv, row_tile, split, n_split;
  int count, rows;   // new tokens, query rows
};
__device__ __forceinline__ ChunkItem chunk_item(const ChunkArgs &a, int rows_per_tile) {
  // all that the look-ups read, asked for at once: a launch's arguments are in no cache when its first workgroups start
  asm volatile("" ::"s"(a.Hkv), "s"(a.n_tiers), "s"(a.q), "s"(a.q_seq), "s"(a.tv[0].base), "s"(a.tv[0].bt), "s"(a.first_item[0]), "s"(a.count[0]),
               "s"(a.part_base[0]), "s"(a.n_split[0]), "s"(a.entry[0]), "s"(a.first_tok[0][0]), "s"(a.len[0][0]), "s"(a.prefix_len[0]));
  ChunkItem it;
  const uint32_t id = blockIdx.x;
  const int item = a.Hkv == 1 ? id : a.hkv_magic ? (int)mul_high(id, a.hkv_magic) : (int)(id / (uint32_t)a.Hkv);
  it.hkv = id - item * a.Hkv;
  it.slot = __popcll(__ballot(a.first_item[threadIdx.x & 63] <= item)) - 1;
  it.entry = a.entry[it.slot];
  it.seq = a.first_seq + it.entry;
  it.count = a.count[it.slot];
  it.rows = it.count * a.G;
  it.n_split = a.n_split[it.slot];
  const int local = item - a.first_item[it.slot], x = local / it.n_split;
  it.split = local - x * it.n_split;
  it.row_tile = (it.rows + rows_per_tile - 1) / rows_per_tile - 1 - x;   // those that see most first
  return it;
}
struct ChunkTier {
  int tok, len;
};
__device__ __forceinline__ ChunkTier chunk_tier(const ChunkArgs &a, const ChunkItem &it, int t) {
  if (t < a.n_prefix) return {a.prefix_tok[t], a.members >> it.seq & 1 ? a.prefix_len[t] : 0};
  return {a.first_tok[t - a.n_prefix][it.slot], a.len[t - a.n_prefix][it.slot]};
}
// ---------------------------------------------------------------- rows
struct ChunkRows {
  float cs, inv_cs;
  float m, l, mcs, far;   // as in Rows
  float rounded;          // l of the rounded weights, where it is kept (0: it is not)
  int token, hq, pos;     // new token, query head, place behind the oldest token
  bool on;
};
__device__ __forceinline__ ChunkRows begin_chunk_rows(const ChunkArgs &a, const ChunkItem &it, int total, int row) {
  ChunkRows r;
  r.on = row < it.rows;
  row = min(row, it.rows - 1);
  r.token = token_of(a, row);
  r.hq = it.hkv * a.G + row - r.token * a.G;
  r.pos = total - it.count + r.token;
  r.cs = a.scale * kLog2e;
  r.inv_cs = 1.0f / r.cs;
  r.m = r.far = -INFINITY;
  r.l = r.mcs = r.rounded = 0.0f;
  return r;
}
// The row's channels 16 kb + 8 hh .. + 7 in qf[kb], in the product's type.
template <bool BF>
__device__ __forceinline__ void load_query(const ChunkArgs &a, const ChunkItem &it, const ChunkRows &r, int hh, u32x4 (&qf)[8]) {
  const u32x4 *qp = (const u32x4 *)(a.q + it.entry * a.q_seq + r.token * a.q_token + r.hq * a.q_head);
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) qf[kb] = qp[2 * kb + hh];
  if (!BF && a.q_fmt == TTKV_BF16)
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) to_fp16(qf[kb]);
}
template <bool BF>
__device__ __forceinline__ void move_chunk_reference(ChunkRows &r, float mt, f16v (&o)[4]) {
#pragma clang fp contract(off)
  const float mn = fmaxf(r.m, mt), at = __builtin_rintf(mn * r.cs), was = r.mcs;
  const bool unit = fabsf(at) < kFar;
  r.mcs = mn == -INFINITY ? 0.0f : (unit ? unit16<BF>() : 0.0f) - at;
  const float alpha = r.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.mcs - was);
  r.l *= alpha;
  r.rounded *= alpha;
  rescale(o, alpha);
  r.m = mn;
  r.far = unit ? (at + kRoom16) * r.inv_cs : mn;
}
// Where a row is kept from a token whose value is infinite or no number, a weight of 0 would still make a NaN of it.  So in steps that not every row
// of a tile sees such values go into LDS as 0 and into a list of bits, a byte for eight channels of a token, and a row that does see one gets
// a NaN in that channel.
struct Wild {
  int step[2];                 // per buffer: the last step with such a value
  __align__(16) uint8_t bits[2][32][16];
};
// Step's tokens below lim, by lane.
__device__ __forceinline__ void spoil(f16v (&o)[4], const uint8_t (&bits)[32][16], int lim, int hh) {
  u32x4 all = {0, 0, 0, 0};
#pragma unroll 1
  for (int t = 0; t < 32; ++t) {
    const u32x4 w = *(const u32x4 *)bits[t];
    if (t < lim) all |= w;
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) {   // (without comparisons: 64 conditions at once took the loop's scalar registers, 7-10 % of the time)
    const uint32_t w = all[d] >> 4 * hh;
    f16v x = o[d];
#pragma unroll
    for (int i = 0; i < 16; ++i)   // channel 32 d + 8 (i / 4) + 4 hh + i % 4
      x[i] = __uint_as_float(__float_as_uint(x[i]) | ((uint32_t)__builtin_amdgcn_sbfe(w, 8 * (i / 4) + i % 4, 1) & 0x7fc00000u));
    o[d] = x;
  }
}

// ---------------------------------------------------------------- a workgroup's part
// RW waves of 32 rows each share the tokens' tiles, TW such teams take the steps of 32 tokens in turn.
template <int RW, int TW>
struct Share {
  ChunkItem it;
  int lane, tw, rw, c, hh, tid;      // tid: of the team
  int row0;                          // of the wave
  bool idle;                         // a wave without rows only helps with the tiles
  int total, base;                   // tokens that the sequence attends; place of the first new one
  int sees, tile_sees;               // tokens that the tile's last row sees, its first one
  int first_sees, last_sees;         // of the wave's rows
  int s0, s1;                        // this item's steps, tiers one behind the other
  __device__ __forceinline__ explicit Share(const ChunkArgs &a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63;
    tw = wave / RW;
    rw = wave % RW;
    c = lane & 31;
    hh = lane >> 5;
    tid = threadIdx.x & (64 * RW - 1);
    it = chunk_item(a, 32 * RW);
    total = 0;
    for (int t = 0; t < a.n_tiers; ++t) total += chunk_tier(a, it, t).len;
    row0 = it.row_tile * 32 * RW + rw * 32;
    idle = row0 >= it.rows;
    base = total - it.count;
    sees = max(0, base + 1 + token_of(a, min(it.row_tile * 32 * RW + 32 * RW, it.rows) - 1));
    tile_sees = base + 1 + token_of(a, it.row_tile * 32 * RW);
    first_sees = base + 1 + token_of(a, min(row0, it.rows - 1));
    last_sees = base + 1 + token_of(a, min(row0 + 31, it.rows - 1));
    int n_steps = 0, before = 0;
    for (int t = 0; t < a.n_tiers; ++t) {
      const int len = chunk_tier(a, it, t).len, n = min(max(sees - before, 0), len);
      n_steps += (n + 31) / 32;
      before += len;
    }
    const int per = ((n_steps + it.n_split - 1) / it.n_split + TW - 1) / TW * TW;
    s0 = min(it.split * per, n_steps);
    s1 = min(s0 + per, n_steps);
  }
  // f(tier, its run, its sequence, steps lo .. hi - 1 of it, tokens before it) for every quantized (or every other) tier that the item has
  // steps of
  template <typename F>
  __device__ __forceinline__ void tiers(const ChunkArgs &a, bool quantized, F &&f) const {
    int at = 0, before = 0;
    for (int t = 0; t < a.n_tiers; ++t) {
      const ChunkTier T = chunk_tier(a, it, t);
      const int n = (min(max(sees - before, 0), T.len) + 31) / 32;
      const int lo = max(s0 - at, 0), hi = min(s1 - at, n);
      if (lo < hi && quantized == is_quant(a.tv[t].k_fmt)) f(a.tv[t], T, t < a.n_prefix ? 0 : it.seq, lo, hi, before);
      at += n;
      before += T.len;
    }
  }
};

// Where piece p (16 bytes) of a step's row lies in LDS.  Padded: rows begin in other banks each.  Swizzled: rows of 256 bytes whose pieces are exchanged
// by the row, so that sixteen rows' pieces (four rows' blocks of 64 bytes, for the transposed reads) lie in banks of their own; what the loads
// without registers ask for, which write 1024 bytes in order.
struct Padded {
  static __device__ __forceinline__ int key(int row, int p) { return row * kRowK + 16 * p; }
  static __device__ __forceinline__ int value(int row, int p) { return row * kRowV + 16 * p; }
};
struct Swizzled {
  static __device__ __forceinline__ int key(int row, int p) { return row * 256 + 16 * (p ^ (row & 15)); }
  static __device__ __forceinline__ int value(int row, int p) { return row * 256 + 16 * (p ^ (row & 3) << 2); }
};
constexpr int kSlot = 32 * 256;   // a step's keys or values there

// A team's rows of one tier on their way: steps mine, mine + TW, .. below hi; keys and values apart.
template <int F, typename AT, int RW, int TW>
struct Stream {
  static constexpr int NL = 8 / RW;   // pieces per thread and step
  const Ring &ring;
  Place at;
  int step, hi, len, tid;
  uint32_t codes, meta;               // offsets of the sections in the head's part
  Piece<F> x[NL];
  __device__ __forceinline__ Stream(const Ring &g, const Place &from, int mine, int hi_, int len_, int tid_, uint32_t codes_, uint32_t meta_)
      : ring(g), at(from), step(mine), hi(hi_), len(len_), tid(tid_), codes(codes_), meta(meta_) {
#pragma unroll
    for (int i = 0; i < NL; ++i) x[i] = Piece<F>{};
  }
  __device__ __forceinline__ void load() {   // the next step, if there is one; behind the tier's end its last row
    if (step >= hi) return;
    const int last = min(31, len - 32 * step - 1);
#pragma unroll
    for (int i = 0; i < NL; ++i) x[i] = load_piece<F>(at.head + codes, at.head + meta, at.row + min((tid >> 4) + 4 * RW * i, last), tid & 15);
    step += TW;
    if (step < hi) at.advance(ring, 32 * TW);
  }
  template <bool BF, bool TWO>
  __device__ __forceinline__ void put_keys(char *to, int part_bytes) const {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      char *const p = to + AT::key((tid >> 4) + 4 * RW * i, tid & 15);
      put_piece<BF, F, TWO>(x[i], p, p + part_bytes);
    }
  }
  // Values of step `of`; all_see: tokens of the tier that every row of the tile sees.
  template <bool BF, bool TWO>
  __device__ __forceinline__ void put_values(char *to, int part_bytes, int of, int all_see, Wild &wild, int buffer) const {
    const bool all = 32 * of + 32 <= all_see;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = (tid >> 4) + 4 * RW * i;
      char *const p = to + AT::value(row, tid & 15);
      if (all) {
        put_piece<BF, F, TWO>(x[i], p, p + part_bytes);
        continue;
      }
      const uint32_t bits = put_piece<BF, F, TWO, true>(x[i], p, p + part_bytes);
      wild.bits[buffer][row][tid & 15] = (uint8_t)bits;
      if (bits) wild.step[buffer] = of;
    }
  }
};

// fp rows of one tier on their way into LDS without registers: a wave's four rows at a time, 1024 bytes in order.
template <int RW, int TW>
struct Direct {
  static constexpr int NL = 8 / RW;   // per wave and step
  const Ring &ring;
  Place at;
  int step, hi, len;
  uint32_t codes;
  __device__ __forceinline__ Direct(const Ring &g, const Place &from, int mine, int lo, int hi_, int len_, uint32_t codes_)
      : ring(g), at(from), step(mine < hi_ ? mine : lo), hi(hi_), len(len_), codes(codes_) {}
  // The next step's rows (behind the last step: its own again, so that as many loads are always under way); to: LDS address of the step, piece_of: the
  // lane's piece in row 4 rw + lane / 16, which is the same in every fourth row and, of keys, exchanged by 4 RW i too.
  template <bool KEYS>
  __device__ __forceinline__ void issue(uint32_t to, int rw, int lane) {
    const int last = min(31, len - 32 * step - 1);
    const uint64_t base = at.head + codes + (uint64_t)((int64_t)at.row * 256);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = 4 * (rw + RW * i) + (lane >> 4), p = (lane & 15) ^ (KEYS ? row & 15 : (row & 3) << 2);
      const uint32_t off = min(row, last) * 256 + 16 * p, m0 = to + 1024 * (rw + RW * i);
      // (not the builtin: the compiler waits for every such load of its own in front of every read of LDS.  Five wait states: the vector unit may have
      // written the base just before.)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(m0), "v"(off), "s"(base) : "memory", "m0");
    }
    if (step + TW < hi) {
      step += TW;
      at.advance(ring, 32 * TW);
    }
  }
};
template <int N>
__device__ __forceinline__ void wait_loads() {   // until N at most are under way
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// The rounded weights 2 i and 2 i + 1 of a step.
template <bool BF>
__device__ __forceinline__ void weigh2(ChunkRows &r, const f16v &sc, int i, u32x4 (&p)[2]) {
  const float w0 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i], r.cs, r.mcs)), w1 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i + 1], r.cs, r.mcs));
  r.l += w0 + w1;
  p[i / 4][i % 4] = pack2<BF>(w0, w1);
}

// The sum of a step's weights as the values meet them.
template <bool BF>
__device__ __forceinline__ float rounded_sum(const u32x4 (&p)[2], float sum) {
  constexpr uint32_t ones = BF ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (BF) sum = __builtin_amdgcn_fdot2_f32_bf16(as_b2(p[i / 4][i % 4]), as_b2(ones), sum, false);
    else sum = __builtin_amdgcn_fdot2(as_h2(p[i / 4][i % 4]), as_h2(ones), sum, false);
  }
  return sum;
}

// What the workgroup's rows come to: the teams' results meet, each wave ends with 128 / TW channels of its rows and stores them.
template <bool ROUNDED, int RW, int TW>
__device__ __forceinline__ void finish(const ChunkArgs &a, const Share<RW, TW> &w, ChunkRows &r, f16v (&o)[4], char *s_tile, float (*s_m)[32], float (*s_l)[32]) {
  const int lane = w.lane, tw = w.tw, rw = w.rw, c = w.c, hh = w.hh;
  const ChunkItem &it = w.it;
  const int row0 = w.row0;
  const f2 both = both32(r.l);
  r.l = both.x + both.y;
  float top = r.m == -INFINITY ? -INFINITY : -r.mcs, l = r.l;
  if constexpr (ROUNDED) {
    const f2 halves = both32(r.rounded);
    if (halves.x + halves.y > 0.0f) rescale(o, l / (halves.x + halves.y));
  }
  constexpr int OWN = 4 / TW > 0 ? 4 / TW : 1;                   // blocks of 32 channels that a wave stores (TW <= 4)
  if constexpr (TW > 1) {
    __syncthreads();
    if (hh == 0) {
      s_m[tw * RW + rw][c] = top;
      s_l[tw * RW + rw][c] = l;
    }
    auto place = [&](int giver, int taker, int e, int k) __attribute__((always_inline)) -> float4 * {   // [giver][taker but the giver][block][piece][lane]
      const int slot = taker - (taker > giver);
      return (float4 *)(s_tile + (((((giver * RW + rw) * (TW - 1) + slot) * OWN + e) * 4 + k) * 64 + lane) * 16);
    };
#pragma unroll
    for (int t = 0; t < TW; ++t)
      if (t != tw)
#pragma unroll
        for (int e = 0; e < OWN; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) *place(tw, t, e, k) = float4{o[t * OWN + e][4 * k], o[t * OWN + e][4 * k + 1], o[t * OWN + e][4 * k + 2], o[t * OWN + e][4 * k + 3]};
    __syncthreads();
    top = -INFINITY;
#pragma unroll
    for (int u = 0; u < TW; ++u) top = fmaxf(top, s_m[u * RW + rw][c]);
    float by[TW];
    l = 0.0f;
#pragma unroll
    for (int u = 0; u < TW; ++u) {
      const float mu = s_m[u * RW + rw][c];
      by[u] = mu == -INFINITY ? (s_l[u * RW + rw][c] != 0.0f ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f(mu - top);   // (a sum that is no number stays none)
      l = fmaf(s_l[u * RW + rw][c], by[u], l);
    }
#pragma unroll
    for (int w = 0; w < TW; ++w) {
      if (w != tw) continue;
#pragma unroll
      for (int e = 0; e < OWN; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          f16v &x = o[w * OWN + e];
          float y[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = x[4 * k + j] * by[w];
#pragma unroll
          for (int u = 0; u < TW; ++u) {
            if (u == w) continue;
            const float4 z = *place(u, w, e, k);
            y[0] = fmaf(z.x, by[u], y[0]);
            y[1] = fmaf(z.y, by[u], y[1]);
            y[2] = fmaf(z.z, by[u], y[2]);
            y[3] = fmaf(z.w, by[u], y[3]);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) x[4 * k + j] = y[j];
        }
    }
  }
  if (!r.on) return;
  // channels 32 d + 8 k + 4 hh .. + 3 of the row lie in registers 4 k .. + 3 of block d
  if (it.n_split > 1) {
    const int64_t at_part = a.part_base[it.slot] + ((int64_t)(row0 + c) * a.Hkv + it.hkv) * it.n_split + it.split;
    float *const po = a.pacc + at_part * 128 + 4 * hh;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if (TW > 1 && d / OWN != tw) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k) *(float4 *)(po + 32 * d + 8 * k) = float4{o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]};
    }
    if (hh == 0 && tw == 0) {
      a.pm[at_part] = top;     // weights are exp2(score cs - this)
      a.pl[at_part] = l;
    }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint8_t *const out = a.out + it.entry * a.o_seq + r.token * a.o_token + r.hq * a.o_head + 8 * hh;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if (TW > 1 && d / OWN != tw) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u32x2 w;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float x = o[d][4 * k + 2 * j] * inv, y = o[d][4 * k + 2 * j + 1] * inv;
        w[j] = a.out_fmt == TTKV_BF16 ? pack2<true>(x, y) : pack2<false>(x, y);
      }
      *(u32x2 *)(out + 64 * d + 16 * k) = w;
    }
  }
  if (a.lse && hh == 0 && tw == 0)
    a.lse[((int64_t)it.entry * a.n_tokens + r.token) * a.Hq + r.hq] = l == 0.0f ? -INFINITY : (__builtin_amdgcn_logf(l) + top) * kLn2;
}

// run(key format, value format, ..) for every tier that the item has steps of, the quantized ones first.  Their weights are fp16 numbers and carry that
// type's power of two; beside bf16 tiers it changes in between.
template <bool BF, int Q, int RW, int TW, typename R>
__device__ __forceinline__ void each_tier(const ChunkArgs &a, const Share<RW, TW> &w, ChunkRows &r, f16v (&o)[4], u32x4 (&qf)[8], R &run) {
  constexpr int FP = BF ? TTKV_BF16 : TTKV_F16;
  if constexpr (Q != 0) {
    load_query<false>(a, w.it, r, w.hh, qf);
    w.tiers(a, true, [&](const TierView &tv, const ChunkTier &T, int seq, int lo, int hi, int ahead) __attribute__((always_inline)) {
      if constexpr ((Q & kInt4) != 0)
        if (Q == kInt4 || tv.k_fmt == TTKV_I4_ASYM_G64) return run(num<TTKV_I4_ASYM_G64>{}, num<TTKV_I4_ASYM_G64>{}, tv, T, seq, lo, hi, ahead);
      if constexpr ((Q & kInt84) != 0)
        if (Q == kInt84 || tv.v_fmt == TTKV_I4_ASYM_G64) return run(num<TTKV_I8_SYM_G32>{}, num<TTKV_I4_ASYM_G64>{}, tv, T, seq, lo, hi, ahead);
      if constexpr ((Q & kInt8) != 0) run(num<TTKV_I8_SYM_G32>{}, num<TTKV_I8_SYM_G32>{}, tv, T, seq, lo, hi, ahead);
    });
    if constexpr (BF) {
      constexpr float step = unit16<true>() - unit16<false>();
      if (fabsf(r.mcs) < kFar) {   // (a reference beyond carries none)
        const float by = __builtin_amdgcn_exp2f(step);
        if (r.m != -INFINITY) r.mcs += step;
        r.l *= by;
        rescale(o, by);
      }
    }
  }
  if constexpr (BF || Q == 0) load_query<BF>(a, w.it, r, w.hh, qf);
  w.tiers(a, false, [&](const TierView &tv, const ChunkTier &T, int seq, int lo, int hi, int ahead) __attribute__((always_inline)) {
    run(num<FP>{}, num<FP>{}, tv, T, seq, lo, hi, ahead);
  });
}

// ---------------------------------------------------------------- few rows
// Bound: memory, not at its best (32 sequences of 4000 to 6000 bf16 tokens, 32 / 8 heads, 16 rows per KV head: 522 MB in 107 us, 4.9 TB/s; a decode step reads
// such rows at 6.2, a kernel that only loads at 6.9): one step's rows are on their way at a time, through registers.  A workgroup has all rows of a KV
// head and a part of its tokens, four teams of two waves; keys of one step and values of the one before are on their way while one is computed.  The
// outputs are divided by the sum of the weights as they were rounded: where a token or two have most of the weight, their rounding then cancels.  With
// quantized tiers LDS holds one step only, so that a CU has two workgroups: one decompresses while the other computes (int4 histories of 8192 tokens,
// 48 rows: 89 us; with one workgroup of eight waves 250).
template <bool BF, int Q, bool V2, int RW, int TW>
__global__ __launch_bounds__(64 * RW * TW, Q ? 2 : 1) void chunk_kernel(const ChunkArgs a) {
  constexpr int kKeys = 32 * kRowK, kValues = 32 * kRowV, kPartsK = Q ? 2 : 1, kPartsV = V2 ? 2 : 1, kStep = kPartsK * kKeys + kPartsV * kValues;
  constexpr int kBuffers = Q ? 1 : 2;
  __shared__ __align__(16) char s_tile[TW * kBuffers * kStep];   // per team: keys and values of two steps (one); at the end what the waves exchange
  static_assert(TW * kBuffers * kStep >= TW * RW * (16 - 16 / TW) * 1024, "room for what the waves exchange");
  __shared__ float s_m[TW * RW][32], s_l[TW * RW][32];
  __shared__ Wild s_wild[TW];
  const Share<RW, TW> w(a);
  u32x4 qf[8];
  ChunkRows r = begin_chunk_rows(a, w.it, w.total, w.row0 + w.c);
  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) o[d] = f16v{};
  char *const team = s_tile + w.tw * kBuffers * kStep;
  const char *const k_at = team + k_lane(w.lane), *const v_at = team + kPartsK * kKeys + v_lane(w.lane);

  auto run = [&](auto kf, auto vf, const TierView &tv, const ChunkTier &T, int seq, int lo, int hi, int ahead) __attribute__((always_inline)) {
    constexpr int KF = decltype(kf)::value, VF = decltype(vf)::value;
    constexpr bool two_k = is_quant(KF), two_v = is_quant(VF) && V2, BT = BF && !is_quant(KF);   // the product's type: quantized tiers in fp16
    const int mine = lo + w.tw;
    const Ring ring(tv, seq, w.it.hkv);
    const Place from(ring, tv.bt_magic, T.tok + 32 * (mine < hi ? mine : lo));
    Stream<KF, Padded, RW, TW> keys(ring, from, mine, hi, T.len, w.tid, 0, tv.k_meta_off);
    Stream<VF, Padded, RW, TW> values(ring, from, mine, hi, T.len, w.tid, tv.v_off, tv.v_meta_off);
    Wild &wild = s_wild[w.tw];
    auto put_values = [&](int at, int step) __attribute__((always_inline)) {
      values.template put_values<BT, two_v>(team + at + kPartsK * kKeys, kValues, step, w.tile_sees - ahead, wild, at != 0);
    };
    auto put_keys = [&](int at) __attribute__((always_inline)) { keys.template put_keys<BT, two_k>(team + at, kKeys); };
    auto works = [&](int s) __attribute__((always_inline)) { return s < hi && !w.idle && 32 * s < w.last_sees - ahead; };   // (wave-uniform)
    auto scores = [&](int at, f16v &sc) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 8; ++kb) {
        sc = mma<BT>(*(const u32x4 *)(k_at + at + 32 * kb), qf[kb], sc);
        if constexpr (two_k) sc = mma<BT>(*(const u32x4 *)(k_at + at + kKeys + 32 * kb), qf[kb], sc);
      }
    };
    auto attend = [&](int at, int s, f16v &sc) __attribute__((always_inline)) {
      const int lim = min(r.pos + 1 - ahead, T.len) - 32 * s;
      if (32 * s + 32 > min(w.first_sees - ahead, T.len)) mask_from(sc, lim, w.hh);
      const float mt = step_max(sc);
      if (__any(mt > r.far)) move_chunk_reference<BT>(r, mt, o);
      u32x4 p[2];
#pragma unroll
      for (int i = 0; i < 8; ++i) weigh2<BT>(r, sc, i, p);
      if constexpr (Q == 0) r.rounded = rounded_sum<BT>(p, r.rounded);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          o[d] = mma<BT>(value_operand(v_at + at, d, b), p[b], o[d]);
          if constexpr (two_v) o[d] = mma<BT>(value_operand(v_at + at + kValues, d, b), p[b], o[d]);
        }
      if (32 * s + 32 > w.tile_sees - ahead && wild.step[at != 0] == s) spoil(o, wild.bits[at != 0], lim, w.hh);
    };
    __syncthreads();   // everybody is done with the tier before
    keys.load();
    values.load();
    if (w.tid == 0) wild.step[0] = wild.step[1] = -1;
    __syncthreads();
    const int n_it = (hi - lo + TW - 1) / TW;      // of the first team: all take as many barriers
    if constexpr (Q != 0) {
      for (int t = 0; t < n_it; ++t) {
        const int s = mine + TW * t;
        put_keys(0);
        put_values(0, s);
        keys.load();
        values.load();
        __syncthreads();
        if (works(s)) {
          f16v sc = {};
          scores(0, sc);
          attend(0, s, sc);
        }
        __syncthreads();
      }
    } else {
      put_keys(0);
      keys.load();
      put_values(0, mine);
      values.load();
      int now = 0;
      for (int t = 0; t < n_it; ++t) {
        __syncthreads();   // the step is in its buffer; everybody is done with the other one
        const int next = kStep - now, s = mine + TW * t;
        const bool on = works(s);
        f16v sc = {};
        if (on) scores(now, sc);
        put_keys(next);
        keys.load();
        if (on) attend(now, s, sc);
        put_values(next, s + TW);
        values.load();
        now = next;
      }
    }
  };
  each_tier<BF, Q>(a, w, r, o, qf, run);
  finish<Q == 0>(a, w, r, o, s_tile, s_m, s_l);
}

// Keeps a step's products and its softmax side by side: after every product some vector instructions and the next operands' loads.
template <bool TWO_K, bool TWO_V>
__device__ __forceinline__ void interleave() {
  constexpr int pairs = 1 + (TWO_K && TWO_V), vector = 6 / (2 * pairs);
  __builtin_amdgcn_sched_group_barrier(0x100, 9, 0);
#pragma unroll
  for (int i = 0; i < 8 * pairs; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, vector, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, vector, 0);
  }
}

// ---------------------------------------------------------------- many rows
// Bound: the matrix cores and the power limit, then what the rows' way into LDS costs: 2048 new fp16 tokens (8192 rows per KV head) of 32 / 8 heads behind 32768 1085 to 1125 us, 1.0
// PFLOP/s where a large library product reaches 1.36.  Builds for the measurement, beside this one at 1150 us (the clock goes with the card's power): 980 without the loads, 870 with the
// products alone.  The steps overlap inside a wave: while the softmax of step s runs on the vector unit, the matrix cores work on the values of step s - 1 and
// the scores of step s + 1.  One barrier per step.  fp rows come into LDS without registers, three steps ahead, into four slots each of keys and values
// (through registers, one step ahead: 1205); codes through registers, into two.  256 rows per workgroup, so that the CUs read an XCD's KV head
// from its L2 half as often as with 128; two workgroups of four waves per CU 1356 where this took 1268.
template <bool BF, int Q, bool V2, int RW, int TW>
__global__ __launch_bounds__(64 * RW * TW, 1) void chunk_rows_kernel(const ChunkArgs a) {
  constexpr int kPartsK = Q ? 2 : 1, kPartsV = V2 ? 2 : 1, kTeam = 8 * kSlot;
  __shared__ __align__(1024) char s_tile[TW * kTeam];            // per team: four slots of keys, four of values
  __shared__ float s_m[TW * RW][32], s_l[TW * RW][32];
  __shared__ Wild s_wild[TW];
  const Share<RW, TW> w(a);
  u32x4 qf[8];
  ChunkRows r = begin_chunk_rows(a, w.it, w.total, w.row0 + w.c);
  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) o[d] = f16v{};
  char *const team = s_tile + w.tw * kTeam, *const team_v = team + 4 * kSlot;
  const uint32_t team_at = (uint32_t)(uintptr_t)(las_char)team;
  const int k_at = w.tw * kTeam + Swizzled::key(w.c, w.hh);                      // in s_tile; block kb of 16 channels: ^ 32 kb
  const int v_row = 4 * w.hh + ((w.lane & 15) >> 2);
  const int v_at = w.tw * kTeam + 4 * kSlot + Swizzled::value(v_row, 2 * (w.lane >> 4 & 1) + (w.lane >> 1 & 1)) + 8 * (w.lane & 1);   // block d of 32 channels: ^ 64 d

  auto run = [&](auto kf, auto vf, const TierView &tv, const ChunkTier &T, int seq, int lo, int hi, int ahead) __attribute__((always_inline)) {
    constexpr int KF = decltype(kf)::value, VF = decltype(vf)::value;
    constexpr bool two_k = is_quant(KF), two_v = is_quant(VF) && V2, BT = BF && !is_quant(KF);   // the product's type: quantized tiers in fp16
    constexpr bool direct = !is_quant(KF);
    constexpr int kSlots = direct ? 4 : 2, kKeys = direct ? kSlot : kPartsK * kSlot, kValues = direct ? kSlot : kPartsV * kSlot;
    const int mine = lo + w.tw;
    const Ring ring(tv, seq, w.it.hkv);
    const Place from(ring, tv.bt_magic, T.tok + 32 * (mine < hi ? mine : lo));
    auto keys = [&] __attribute__((always_inline)) {
      if constexpr (direct) return Direct<RW, TW>(ring, from, mine, lo, hi, T.len, 0);
      else return Stream<KF, Swizzled, RW, TW>(ring, from, mine, hi, T.len, w.tid, 0, tv.k_meta_off);
    }();
    auto values = [&] __attribute__((always_inline)) {
      if constexpr (direct) return Direct<RW, TW>(ring, from, mine, lo, hi, T.len, tv.v_off);
      else return Stream<VF, Swizzled, RW, TW>(ring, from, mine, hi, T.len, w.tid, tv.v_off, tv.v_meta_off);
    }();
    const int seen_by_all = min(w.first_sees - ahead, T.len), seen = w.idle ? 0 : min(32 * hi, w.last_sees - ahead);   // by the wave's rows
    const int lim = min(r.pos + 1 - ahead, T.len);
    Wild &wild = s_wild[w.tw];
    auto bring_keys = [&](int slot) __attribute__((always_inline)) {
      if constexpr (direct) keys.template issue<true>(team_at + slot * kKeys, w.rw, w.lane);
      else {
        keys.template put_keys<BT, two_k>(team + slot * kKeys, kSlot);
        keys.load();
      }
    };
    auto bring_values = [&](int slot, int step) __attribute__((always_inline)) {
      if constexpr (direct) values.template issue<false>(team_at + 4 * kSlot + slot * kValues, w.rw, w.lane);
      else {
        values.template put_values<BT, two_v>(team_v + slot * kValues, kSlot, step, w.tile_sees - ahead, wild, slot);
        values.load();
      }
    };
    // The wave's own part of a step's values, when it has come: see Wild.
    auto check_values = [&](int slot, int step) __attribute__((always_inline)) {
      if (32 * step + 32 <= w.tile_sees - ahead) return;
#pragma unroll
      for (int i = 0; i < 8 / RW; ++i) {
        const int row = 4 * (w.rw + RW * i) + (w.lane >> 4), p = w.lane & 15;
        u32x4 *const at = (u32x4 *)(team_v + slot * kValues + Swizzled::value(row, p));
        u32x4 x = *at;
        const uint32_t bits = take_wild<BT>(x);
        if (bits) *at = x;
        wild.bits[slot & 1][row][p] = (uint8_t)bits;
        if (bits) wild.step[slot & 1] = step;
      }
    };
    auto score = [&](f16v &x, int slot, int kb) __attribute__((always_inline)) {
      const char *const k = s_tile + (k_at ^ 32 * kb) + slot * kKeys;
      x = mma<BT>(*(const u32x4 *)k, qf[kb], x);
      if constexpr (two_k) x = mma<BT>(*(const u32x4 *)(k + kSlot), qf[kb], x);
    };
    auto operand = [&](const char *v, int b) __attribute__((always_inline)) -> u32x4 {
      u32x4 va;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((las_s4)(v + (16 * b + 8 * j) * 256)));
        va[2 * j] = y.x;
        va[2 * j + 1] = y.y;
      }
      return va;
    };
    auto value = [&](int slot, int d, int b, const u32x4 (&p)[2]) __attribute__((always_inline)) {
      const char *const v = s_tile + (v_at ^ 64 * d) + slot * kValues;
      o[d] = mma<BT>(operand(v, b), p[b], o[d]);
      if constexpr (two_v) o[d] = mma<BT>(operand(v + kSlot, b), p[b], o[d]);
    };
    // The weights of step s meet its values, by themselves.
    auto flush = [&](int slot, const u32x4 (&p)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int b = 0; b < 2; ++b) value(slot, d, b, p);
    };
    auto spoil_by = [&](int slot, int s) __attribute__((always_inline)) {
      if (32 * s + 32 > w.tile_sees - ahead && wild.step[slot & 1] == s) spoil(o, wild.bits[slot & 1], lim - 32 * s, w.hh);
    };
    // Step s, in slot NOW: sc its scores, p the weights of the step before (zeros where its values are added already); next and pn receive
    // the next step's scores and its own weights.
    auto body = [&](int s, auto slot_tag, f16v &sc, f16v &next, u32x4 (&p)[2], u32x4 (&pn)[2], bool &pending) __attribute__((always_inline)) {
      constexpr int NOW = decltype(slot_tag)::value, BEFORE = (NOW + kSlots - 1) % kSlots, NEXT = (NOW + 1) % kSlots;
      if constexpr (direct) {
        wait_loads<4 * (8 / RW)>();   // all but those of the last two steps
        check_values(BEFORE, s - TW);
      }
      __syncthreads();   // keys of the next step and values of the one before are there; everybody is done with those of this one and the one before that
      if (pending) spoil_by(BEFORE, s - TW);
      const bool works = 32 * s < seen;   // (wave-uniform)
      const float mt = step_max(sc);
      const bool moves = works && __any(mt > r.far);
      if (moves || !works) {
        if (pending) flush(BEFORE, p);
        p[0] = p[1] = u32x4{0, 0, 0, 0};
        if (moves) move_chunk_reference<BT>(r, mt, o);
      }
      bring_keys(NOW);                                     // (of the fourth step behind this one; of the second)
      bring_values(direct ? (NOW + 2) % kSlots : NOW, s);  // (of the second behind it; its own)
      if (works) {
        f16v nx = {};
#pragma unroll
        for (int g = 0; g < 8; ++g) {   // a product of the values, one of the scores, an eighth of the softmax
          value(BEFORE, g / 2, g % 2, p);
          score(nx, NEXT, g);
          weigh2<BT>(r, sc, g, pn);
        }
        // (kept here: the weights are wanted in the next step only, and would be worked out there, behind the products)
        asm volatile("" : "+v"(pn[0]), "+v"(pn[1]), "+v"(r.l));
        interleave<two_k, two_v>();
        if (32 * (s + TW) + 32 > seen_by_all) mask_from(nx, lim - 32 * (s + TW), w.hh);
        next = nx;
      }
      pending = works;
    };
    u32x4 p0[2], p1[2];
    p0[0] = p0[1] = u32x4{0, 0, 0, 0};
    __syncthreads();   // everybody is done with the tier before
    // there is no step before the first: weights of zero meet zeros
    for (int i = w.tid; i < kValues / 16; i += 64 * RW) ((u32x4 *)(team_v + (kSlots - 1) * kValues))[i] = u32x4{0, 0, 0, 0};
    if (w.tid == 0) wild.step[0] = wild.step[1] = -1;
    if constexpr (direct) {
      bring_keys(0);
      bring_keys(1);
      bring_keys(2);
      bring_values(0, 0);
      bring_keys(3);
      bring_values(1, 0);
      wait_loads<5 * (8 / RW)>();
    } else {
      keys.load();
      bring_keys(0);
      bring_keys(1);
      values.load();
    }
    __syncthreads();
    f16v s0 = {}, s1 = {};
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) score(s0, 0, kb);
    if (32 * mine + 32 > seen_by_all) mask_from(s0, lim - 32 * mine, w.hh);
    bool pending = false;
    const int n_it = (hi - lo + TW - 1) / TW;      // of the first team: all take as many barriers
    int t = 0;
    for (; t < n_it; t += kSlots) {
      body(mine + TW * t, num<0>{}, s0, s1, p0, p1, pending);
      body(mine + TW * (t + 1), num<1>{}, s1, s0, p1, p0, pending);
      if constexpr (direct) {
        body(mine + TW * (t + 2), num<2>{}, s0, s1, p0, p1, pending);
        body(mine + TW * (t + 3), num<3>{}, s1, s0, p1, p0, pending);
      }
    }
    const int last = mine + TW * (t - 1);
    if constexpr (direct) {
      wait_loads<0>();
      check_values(kSlots - 1, last);
    }
    __syncthreads();
    if (pending) {
      spoil_by(kSlots - 1, last);
      flush(kSlots - 1, p0);
    }
  };
  each_tier<BF, Q>(a, w, r, o, qf, run);
  finish<false>(a, w, r, o, s_tile, s_m, s_l);
}

template <bool BF, int Q, bool V2>
void start(const ChunkArgs &a, int rows, hipStream_t s) {
  const dim3 grid((unsigned)a.n_items * (unsigned)a.Hkv);
  if (rows == 256) hipLaunchKernelGGL((chunk_rows_kernel<BF, Q, V2, 8, 1>), grid, dim3(512), 0, s, a);
  else if (rows == 128) hipLaunchKernelGGL((chunk_rows_kernel<BF, Q, V2, 4, 2>), grid, dim3(512), 0, s, a);
  else if constexpr (Q != 0) hipLaunchKernelGGL((chunk_kernel<BF, Q, V2, 2, 2>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((chunk_kernel<BF, Q, V2, 2, 4>), grid, dim3(512), 0, s, a);
}
// Values in two numbers for fp16 outputs.
template <int Q>
void start_quantized(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream) {
  const bool fine = a.out_fmt == TTKV_F16;
  if (s.bf) fine ? start<true, Q, true>(a, s.rows, stream) : start<true, Q, false>(a, s.rows, stream);
  else fine ? start<false, Q, true>(a, s.rows, stream) : start<false, Q, false>(a, s.rows, stream);
}

}  // namespace chunk
}  // namespace ttkv
