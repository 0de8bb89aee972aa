// What a cache's tokens have been worth: the attention weight that queries give every token of a tier, added up, and the eviction of
// the tokens that received least.
#include "ttkv_chunk_dev.h"

#include <algorithm>

namespace ttkv {

namespace {

using namespace dev;
using namespace shared;
using namespace chunk;

// ---------------------------------------------------------------- weights
// weight[token] += sum over rows that see it of e^(scale q.k - lse): the score product of the chunk's attention with the roles turned.  A
// wave keeps the keys of 32 tokens in registers and takes the chunk's query rows 32 at a time from LDS; a lane has 16 scores of one row,
// and adds the weights of its rows up by itself until the lanes meet at the end.  No two waves add to one place, so
// the order of a sum is fixed.
constexpr int kWaves = 8, kTile = 32 * kWaves;   // tokens that a workgroup's waves take together
constexpr int kFewRows = 256;

// What an item works on.
struct WeighItem {
  int slot, entry, seq, hkv, rows, sees, len, t0, split;   // t0: the item's first token
};
__device__ __forceinline__ WeighItem weigh_item(const WeighArgs &a) {
  // all that the look-ups read, asked for at once: a launch's arguments are in no cache when its first workgroups start
  asm volatile("" ::"s"(a.Hkv), "s"(a.q), "s"(a.sums), "s"(a.tv.base), "s"(a.tv.bt), "s"(a.first_item[0]), "s"(a.count[0]), "s"(a.sees[0]),
               "s"(a.first_tok[0]), "s"(a.len[0]), "s"(a.first_fresh[0]), "s"(a.entry[0]));
  WeighItem w;
  const int lane = threadIdx.x & 63;
  uint32_t id = blockIdx.x;
  w.split = 0;
  if (a.n_split > 1) {
    w.split = id % (uint32_t)a.n_split;
    id /= (uint32_t)a.n_split;
  }
  const int item = a.Hkv == 1 ? id : a.hkv_magic ? (int)mul_high(id, a.hkv_magic) : (int)(id / (uint32_t)a.Hkv);
  w.hkv = id - item * a.Hkv;
  w.slot = __popcll(__ballot(a.first_item[lane] <= item)) - 1;
  w.entry = a.entry[w.slot];
  w.seq = a.first_seq + w.entry;
  w.rows = a.count[w.slot] * a.G;
  w.sees = a.sees[w.slot];
  w.len = a.len[w.slot];
  w.t0 = (item - a.first_item[w.slot]) * a.chunk;
  return w;
}
// Keys of 32 tokens as left operands: lane -> token c, channels 16 kb + 8 hh .. + 7.
template <int KF>
struct Operands {
  static constexpr bool two = is_quant(KF);
  u32x4 hi[8], lo[two ? 8 : 1];
  __device__ __forceinline__ void load(const Place &at, uint32_t meta, int left, int c, int hh) {   // left: live tokens from `at` on
    const int row = at.row + min(c, left - 1);
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) {
      const Piece<KF> x = load_piece<KF>(at.head, at.head + meta, row, 2 * kb + hh);
      if constexpr (two) unpack_piece<KF, true>(x, hi[kb], lo[kb]);
      else hi[kb] = x.w;
    }
  }
};
// Scores of 32 rows (right operands at q_at) and the wave's 32 tokens.
template <bool BF, int KF>
__device__ __forceinline__ f16v score_rows(const Operands<KF> &k, const char *q_at) {
  f16v sc = {};
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) {
    const u32x4 q = *(const u32x4 *)(q_at + 32 * kb);
    sc = mma<BF>(k.hi[kb], q, sc);
    if constexpr (is_quant(KF)) sc = mma<BF>(k.lo[kb], q, sc);
  }
  return sc;
}
// lim: tokens of the wave's that the lane's row sees.
__device__ __forceinline__ f16v mask_rows(f16v sc, int lim, int hh) {
  if (!__all(lim >= 32)) mask_from(sc, lim, hh);
  return sc;
}
// Their weights; off: -lse in the log2 domain.
__device__ __forceinline__ f16v add_rows(f16v acc, const f16v sc, float cs, float off) {
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] += __builtin_amdgcn_exp2f(fmaf(sc[i], cs, off));
  return acc;
}
// The next step's products and this one's exponentials side by side: products of one chain wait for each other, and what stands behind a waiting one waits
// as well.
template <bool BF, int KF>
__device__ __forceinline__ f16v side_by_side(const Operands<KF> &k, const char *q_at, f16v &sums, const f16v now, float cs, float off) {
  constexpr bool two = is_quant(KF);
  f16v then = {}, acc = sums;   // (elements are written of local variables only: of ones that a lambda holds they end in scratch)
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) {
    const u32x4 q = *(const u32x4 *)(q_at + 32 * kb);
    then = mma<BF>(k.hi[kb], q, then);
    if constexpr (two) then = mma<BF>(k.lo[kb], q, then);
    acc[2 * kb] += __builtin_amdgcn_exp2f(fmaf(now[2 * kb], cs, off));
    acc[2 * kb + 1] += __builtin_amdgcn_exp2f(fmaf(now[2 * kb + 1], cs, off));
  }
  asm volatile("" : "+v"(acc));   // (kept here: wanted in the next step only, the sums would be worked out there)
  __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, two ? 3 : 6, 0);
    if constexpr (two) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
    }
  }
  sums = acc;
  return then;
}
// Over the 32 lanes of a half; lane c < 16 of half hh then has token 8 (c / 4) + 4 hh + c % 4.
__device__ __forceinline__ float gather(const f16v &acc, int c) {
  float mine = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v = group_sum<16>(acc[i]);
    const f2 both = both16(v);
    v = both.x + both.y;
    if (c == i) mine = v;
  }
  return mine;
}
__device__ __forceinline__ void store_weights(const WeighArgs &a, const WeighItem &w, const Ring &ring, const Place &at, int t0, float mine, int c, int hh) {
  const int t = 8 * (c / 4) + 4 * hh + c % 4;
  if (c >= 16 || t0 + t >= w.len) return;
  const int64_t r = (int64_t)w.seq * ring.blocks + at.block, rec = a.tv.table ? (int64_t)a.tv.table[r] : r;
  float *const x = a.weights + (rec * a.Hkv + w.hkv) * ring.bt + at.row + t;
  *x = t0 + t >= a.first_fresh[w.slot] ? mine : *x + mine;
}
// A row's log-sum-exp as it lies, and the tokens of the tier that the row sees (rows behind the last: none).
struct RawRow {
  float lse;
  int sees;
};
__device__ __forceinline__ RawRow raw_row(const WeighArgs &a, const WeighItem &w, int row) {
  const int r = min(row, w.rows - 1), token = token_of(a, r), hq = w.hkv * a.G + r - token * a.G;
  return {a.lse[((int64_t)w.entry * a.n_tokens + token) * a.Hq + hq], row < w.rows ? min(w.sees + token, w.len) : 0};
}
// The exponent's summand, and the tokens again: none where the log-sum-exp is not finite.
struct RowOf {
  float off;
  int sees;
};
__device__ __forceinline__ RowOf row_of(const RawRow &x) {
  const bool on = fabsf(x.lse) < INFINITY;
  return {on ? -x.lse * kLog2e : 0.0f, on ? x.sees : 0};
}
template <bool BF>
__device__ __forceinline__ u32x4 query_piece(const WeighArgs &a, const WeighItem &w, int row, int p) {
  const int r = min(row, w.rows - 1), token = token_of(a, r), hq = w.hkv * a.G + r - token * a.G;
  u32x4 x = *(const u32x4 *)(a.q + w.entry * a.q_seq + token * a.q_token + hq * a.q_head + 16 * p);
  if (!BF && a.q_fmt == TTKV_BF16) to_fp16(x);
  return x;
}

// Steps s .. n - 1 of rows that lie in LDS: the next one's products beside this one's exponentials.  row_at: the lane's of step 0; t: the wave's first token.
template <bool BF, int KF>
__device__ __forceinline__ f16v sum_steps(f16v acc, const Operands<KF> &ops, const char *q_at, const RowOf *row_at, int s, int n, int t, float cs, int hh) {
  constexpr int kStep = 32 * kRowK;
  if (s >= n) return acc;
  f16v sc, nx;
  RowOf r = row_at[32 * s], rn;
  auto one = [&](f16v &now, f16v &then, const RowOf &of, RowOf &of_next) __attribute__((always_inline)) {
    of_next = row_at[32 * s + 32];
    then = mask_rows(side_by_side<BF, KF>(ops, q_at + (s + 1) * kStep, acc, now, cs, of.off), of_next.sees - t, hh);
  };
  sc = mask_rows(score_rows<BF, KF>(ops, q_at + s * kStep), r.sees - t, hh);
  for (; s + 2 < n; ++s) {
    one(sc, nx, r, rn);
    ++s;
    one(nx, sc, rn, r);
  }
  if (s + 1 == n) return add_rows(acc, sc, cs, r.off);
  one(sc, nx, r, rn);
  return add_rows(acc, nx, cs, rn.off);
}

// Few rows (a step's, the last queries of a prompt).  Bound: memory, not at its best (a step of 48 sequences of 2000 to 4000 fp16 tokens, 32 / 8 heads: 305 MB in 57-65 us, 4.7 to 5.3
// TB/s; a decode step reads fp16 rows at 5.9), and from some 200 rows on the vector unit's exponentials (256 rows x 4 x 16384 bf16 tokens 51 us; its bytes
// alone 28).  All rows lie in LDS; the waves take an item's tokens 32 at a time, the
// next ones' keys on their way, and meet nobody.  Keys are loaded as whole lines and turned into operands through LDS of the wave's own (as
// operands they are pieces of 32 bytes of 32 rows per instruction: a step of 48 x 4000 tokens of 32 / 8 heads 86 us).
template <bool BF, int KF, int ROWS, int NW>
__global__ __launch_bounds__(64 * NW, 1) void weigh_few_kernel(const WeighArgs a) {
  constexpr int kPart = 32 * kRowK, kOwn = (is_quant(KF) ? 2 : 1) * kPart;
  __shared__ __align__(16) char s_all[ROWS * kRowK + NW * kOwn];
  __shared__ RowOf s_row[ROWS];
  char *const s_q = s_all, *const s_k = s_all + ROWS * kRowK;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, hh = lane >> 5;
  const WeighItem w = weigh_item(a);
  const int end = min(w.t0 + a.chunk, w.len), steps = (w.rows + 31) / 32;
  const Ring ring(a.tv, w.seq, w.hkv);
  int t = w.t0 + 32 * wave;
  Place next(ring, a.tv.bt_magic, a.first_tok[w.slot] + (t < end ? t : w.t0)), at = next;
  Piece<KF> x[8];   // rows lane / 16 + 4 i, piece lane % 16
  auto load = [&](int left) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = load_piece<KF>(next.head, next.head + a.tv.k_meta_off, next.row + min((lane >> 4) + 4 * i, min(31, left - 1)), lane & 15);
  };
  if (t < end) load(w.len - t);
  for (int i = threadIdx.x; i < steps * 512; i += 64 * NW) *(u32x4 *)(s_q + (i >> 4) * kRowK + 16 * (i & 15)) = query_piece<BF>(a, w, i >> 4, i & 15);
  for (int i = threadIdx.x; i < steps * 32; i += 64 * NW) s_row[i] = row_of(raw_row(a, w, i));
  __syncthreads();
  char *const own = s_k + wave * kOwn;
  const char *const q_at = s_q + k_lane(lane);
  const float cs = a.scale * kLog2e;
  for (; t < end; t += 32 * NW) {
    // (LDS takes a wave's stores and reads in order; the compiler has to leave them so)
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      char *const to = own + ((lane >> 4) + 4 * i) * kRowK + 16 * (lane & 15);
      put_piece<BF, KF, true>(x[i], to, to + kPart);
    }
    asm volatile("" ::: "memory");
    at = next;
    if (t + 32 * NW < end) {
      next.advance(ring, 32 * NW);
      load(w.len - t - 32 * NW);
    }
    Operands<KF> ops;
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) {
      ops.hi[kb] = *(const u32x4 *)(own + k_lane(lane) + 32 * kb);
      if constexpr (is_quant(KF)) ops.lo[kb] = *(const u32x4 *)(own + kPart + k_lane(lane) + 32 * kb);
    }
    // from the first row that sees one of the tokens on
    const f16v acc = sum_steps<BF, KF>(f16v{}, ops, q_at, s_row + c, max(0, t - w.sees + 1) * a.G / 32, steps, t, cs, hh);
    store_weights(a, w, ring, at, t, gather(acc, c), c, hh);
  }
}

// Many rows (a prompt's).  Bound: the vector unit's exponentials, and in short prompts the launch's start (2047 queries of 28 / 4 heads 33 us, the sums 4).  A wave keeps its tokens, the rows come through LDS; where there are few tokens, several
// items share a tile's rows, and weigh_sum_kernel adds their sums in order.
// (128 rows between two barriers: with 32 a step's rows were asked for one step ahead, less than they take; 2047 queries of 28 / 4 heads 52 us.)
template <bool BF, int KF>
__global__ __launch_bounds__(64 * kWaves, 1) void weigh_kernel(const WeighArgs a) {
  constexpr int kRows = 128, kSteps = kRows / 32, kStage = kRows * kRowK, NL = kRows * 16 / (64 * kWaves);
  __shared__ __align__(16) char s_q[2 * kStage];   // two stages' rows
  __shared__ RowOf s_row[2 * kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, hh = lane >> 5;
  const WeighItem w = weigh_item(a);
  const int t0 = w.t0 + 32 * wave;
  const bool idle = t0 >= w.len;
  const Ring ring(a.tv, w.seq, w.hkv);
  const Place at(ring, a.tv.bt_magic, a.first_tok[w.slot] + (idle ? w.t0 : t0));
  // rows in steps of 32, from the first that sees a token of the tile on; this item's share of them
  const int all1 = (w.rows + 31) / 32, all0 = min(max(0, w.t0 - w.sees + 1) * a.G / 32, all1);
  const int per = (all1 - all0 + a.n_split - 1) / a.n_split;
  const int s0 = min(all0 + w.split * per, all1), s1 = min(s0 + per, all1);
  const int qrow = threadIdx.x >> 4, qp = threadIdx.x & 15;
  u32x4 qr[NL];
  RawRow raw = {};
  auto load = [&](int s) __attribute__((always_inline)) {   // rows of the stage that begins with step s
#pragma unroll
    for (int i = 0; i < NL; ++i) qr[i] = query_piece<BF>(a, w, 32 * s + qrow + 4 * kWaves * i, qp);
    if (threadIdx.x < kRows) raw = raw_row(a, w, 32 * s + threadIdx.x);
  };
  auto put = [&](int buffer) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) *(u32x4 *)(s_q + buffer * kStage + (qrow + 4 * kWaves * i) * kRowK + 16 * qp) = qr[i];
    if (threadIdx.x < kRows) s_row[buffer * kRows + threadIdx.x] = row_of(raw);
  };
  if (s0 < s1) load(s0);
  Operands<KF> ops;
  ops.load(at, a.tv.k_meta_off, max(w.len - t0, 1), c, hh);
  f16v acc = {};
  const float cs = a.scale * kLog2e;
  if (s0 < s1) put(0);
  if (s0 + kSteps < s1) load(s0 + kSteps);
  int now = 0;
  for (int s = s0; s < s1; s += kSteps) {
    __syncthreads();   // the stage's rows are there; everybody is done with those of the one before
    if (s + kSteps < s1) put(1 - now);
    if (s + 2 * kSteps < s1) load(s + 2 * kSteps);
    if (!idle)
      acc = sum_steps<BF, KF>(acc, ops, s_q + now * kStage + k_lane(lane), s_row + now * kRows + c, 0, min(kSteps, s1 - s), t0, cs, hh);
    now = 1 - now;
  }
  if (idle) return;
  const float mine = gather(acc, c);
  if (a.n_split == 1) return store_weights(a, w, ring, at, t0, mine, c, hh);
  if (c < 16) a.sums[((int64_t)w.split * a.Hkv + w.hkv) * a.n_sums + (int64_t)a.first_item[w.slot] * kTile + t0 + 8 * (c / 4) + 4 * hh + c % 4] = mine;
}
// The sums of a tile's items, a thread per token.
__global__ __launch_bounds__(kTile) void weigh_sum_kernel(const WeighArgs a) {
  const int item = blockIdx.x, hkv = blockIdx.y;
  const int slot = __popcll(__ballot(a.first_item[threadIdx.x & 63] <= item)) - 1;
  const int t = (item - a.first_item[slot]) * kTile + threadIdx.x;
  if (t >= a.len[slot]) return;
  const float *const sums = a.sums + (int64_t)hkv * a.n_sums + (int64_t)a.first_item[slot] * kTile + t;
  float v = 0.0f;
  const int64_t stride = (int64_t)a.Hkv * a.n_sums;
  for (int i = 0; i < a.n_split; i += 8) {   // eight asked for at once
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = i + j < a.n_split ? sums[(i + j) * stride] : 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) v += x[j];
  }
  int tok = a.first_tok[slot] + t;
  if (tok >= a.tv.ring_blocks * a.tv.bt) tok -= a.tv.ring_blocks * a.tv.bt;
  const int block = div_bt(tok, a.tv.bt, a.tv.bt_magic);
  const int64_t r = (int64_t)(a.first_seq + a.entry[slot]) * a.tv.ring_blocks + block, rec = a.tv.table ? (int64_t)a.tv.table[r] : r;
  float *const x = a.weights + (rec * a.Hkv + hkv) * a.tv.bt + tok - block * a.tv.bt;
  *x = t >= a.first_fresh[slot] ? v : *x + v;
}

// ---------------------------------------------------------------- the lightest tokens go
// Weights in an order of unsigned numbers: what is no number counts as the least.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.0f);   // -0 is 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
struct TokenPlace {
  int64_t rec;
  int row;
};
__device__ __forceinline__ TokenPlace token_place(const TierView &tv, int seq, int tok) {
  if (tok >= tv.ring_blocks * tv.bt) tok -= tv.ring_blocks * tv.bt;
  const int block = div_bt(tok, tv.bt, tv.bt_magic);
  const int64_t r = (int64_t)seq * tv.ring_blocks + block;
  return {tv.table ? (int64_t)tv.table[r] : r, tok - block * tv.bt};
}
// What a lane of 32 has to do with a row that moves: lanes 0 .. 15 its keys, 16 .. 31 its values (16 bytes each), lanes 0 and 16 what decompresses
// them, lane 1 the weight.
struct RowMove {
  u32x4 *x, *y;       // from, to
  u32x2 *mx, *my;
  float *wx, *wy;
  u32x4 v, u;
  u32x2 mv, mu;
  float wv, wu;
  bool on, meta, weight;
  __device__ __forceinline__ void begin(const LightArgs &a, int slot, int hkv, int from, int to, int lane, bool valid) {   // asks for what moves
    const TokenPlace f = token_place(a.tv, a.seq[slot], a.first_tok[slot] + from), t = token_place(a.tv, a.seq[slot], a.first_tok[slot] + to);
    const int64_t head = (int64_t)hkv * a.tv.head_bytes;
    uint8_t *const fh = a.tv.base + f.rec * a.tv.rec_bytes + head, *const th = a.tv.base + t.rec * a.tv.rec_bytes + head;
    const int side = lane >> 4, p = lane & 15, width = side ? a.vc : a.kc, off = side ? a.tv.v_off : 0, m = side ? a.tv.v_meta_off : a.tv.k_meta_off;
    on = valid && 16 * p < width;
    meta = valid && p == 0 && (side ? a.vm : a.km);
    weight = valid && lane == 1;
    x = (u32x4 *)(fh + off + (int64_t)f.row * width + 16 * p);
    y = (u32x4 *)(th + off + (int64_t)t.row * width + 16 * p);
    mx = (u32x2 *)(fh + m + (int64_t)f.row * 8);
    my = (u32x2 *)(th + m + (int64_t)t.row * 8);
    wx = a.weights + (f.rec * a.Hkv + hkv) * a.tv.bt + f.row;
    wy = a.weights + (t.rec * a.Hkv + hkv) * a.tv.bt + t.row;
    if (on) v = *x;
    if (meta) mv = *mx;
    if (weight) wv = *wx;
    if (!a.swap) return;
    if (on) u = *y;
    if (meta) mu = *my;
    if (weight) wu = *wy;
  }
  __device__ __forceinline__ void end(const LightArgs &a) const {
    if (on) *y = v;
    if (meta) *my = mv;
    if (weight) *wy = wv;
    if (!a.swap) return;
    if (on) *x = u;
    if (meta) *mx = mu;
    if (weight) *wx = wu;
  }
};

typedef int i32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ int row_sum(int v) {   // over 16 lanes, in each of them
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);
  return v;
}
// A workgroup per (sequence, KV head), each of its 16 waves a stretch of the tokens, 64 at a time; up to 64 IPT of them a wave keeps their orders in
// registers, beyond (IPT 0) it reads the weights again.  The (old - gone)-th largest order is found by a radix select, 11, 11 and 10 bits of it at a time:
// the first ones are exponent and two bits of the mantissa, so that tokens whose weights share an exponent do not all count on one of
// LDS's counters.  (Counting the tokens above three candidates by ballots, two bits at a time: 4 x 32768 tokens 76 us.)  Then each wave
// knows the places of its tokens from the counts of the waves before it: the i-th token that stays among the first `gone` moves to the i-th
// place behind them whose token goes.
// Bound: the instructions of the CUs that work, for an item is a sequence's KV head (32 heads of up to 32768 tokens 37 us, 384 heads of 4096 16; orders read again
// instead of kept 91 and 28; registers for 32768 tokens where 4096 are 27).
// Moves that the selecting workgroup makes by itself: a launch less (384 heads of 4096 tokens that free a block 16.4 us, in two launches 16.7 + 3.9).
constexpr int kInPlace = 256;
template <int IPT>
__global__ __launch_bounds__(1024, IPT > 12 ? 1 : 2) void light_select_kernel(const LightArgs a, int in_place) {
  __shared__ i32x2 s_count[2][16];
  __shared__ int s_hist[2][2048], s_total[16], s_pick[2];
  __shared__ int32_t s_list[2 * kInPlace];
  const int hkv = blockIdx.x % a.Hkv, slot = blockIdx.x / a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int old = a.old[slot], gone = a.gone[slot], keep = old - gone, seq = a.seq[slot], first = a.first_tok[slot];
  const int steps = (old + 1023) / 1024;            // of 64 tokens, of each wave
  const int begin = wave * steps * 64;
  int32_t *const list = in_place ? s_list : a.moves + 2 * (a.move_base[slot] + (int64_t)hkv * a.most_moves[slot]);
  // 64 tokens lie in one block: the weights of the wave's c-th ones; behind the last token: what lies beside it, or its own 64 again
  auto weights_at = [&](int c) __attribute__((always_inline)) -> const float * {
    const TokenPlace p = token_place(a.tv, seq, first + min(begin + 64 * c, (old - 1) & ~63));
    return a.weights + (p.rec * a.Hkv + hkv) * a.tv.bt + p.row;
  };
  auto order_at = [&](int c, float w) __attribute__((always_inline)) { return begin + 64 * c + lane < old ? order_of(w) : 0u; };
  uint32_t u[IPT ? IPT : 1];
  if constexpr (IPT > 0) {   // each lane looks one up, then all are asked for at once
    const uint64_t at = (uint64_t)weights_at(lane);
    const int lo = (int)at, hi = (int)(at >> 32);
    float x[IPT];
#pragma unroll
    for (int c = 0; c < IPT; ++c) {
      const uint64_t p = (uint32_t)__builtin_amdgcn_readlane(lo, c) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, c) << 32;
      x[c] = ((const __attribute__((address_space(1))) float *)p)[lane];
    }
#pragma unroll
    for (int c = 0; c < IPT; ++c) u[c] = order_at(c, x[c]);
  }
  auto each = [&](auto f) __attribute__((always_inline)) {   // f(step, order), tokens behind the last one's: order 0
    if constexpr (IPT > 0) {
#pragma unroll
      for (int c = 0; c < IPT; ++c)
        if (c < steps) f(c, u[c]);   // (what follows is the next wave's)
    } else {
      for (int c = 0; c < steps; c += 4) {   // four asked for at once
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = weights_at(c + j)[lane];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + j < steps) f(c + j, order_at(c + j, x[j]));
      }
    }
  };
  int buffer = 0;
  // Counts of the wave for everybody: lane v < 16 then has wave v's, and the sums over all waves (before: over the waves before this one) come
  // from lanes 0 .. 15 of each row.
  auto meet = [&](const int (&n)[2], int (&before)[2], int (&all)[2]) __attribute__((always_inline)) {
    if (lane == 0) s_count[buffer][wave] = i32x2{n[0], n[1]};
    __syncthreads();
    const i32x2 x = s_count[buffer][lane & 15];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      all[j] = __builtin_amdgcn_readfirstlane(row_sum(x[j]));
      before[j] = __builtin_amdgcn_readfirstlane(row_sum((lane & 15) < wave ? x[j] : 0));
    }
    buffer ^= 1;   // written again after the next meeting only
  };
  int before[2], all[2];
  uint32_t least = 0;   // the largest order that `keep` tokens have at least
  int left = keep;      // of the tokens that begin like it so many stay (the oldest)
  if (keep > 0) {
    for (int i = threadIdx.x; i < 2048; i += 1024) s_hist[0][i] = 0;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      int *const hist = s_hist[pass & 1];
      each([&](int c, uint32_t x) __attribute__((always_inline)) {
        const bool on = begin + 64 * c + lane < old && (pass == 0 || (pass == 1 ? x >> 21 == least >> 21 : x >> 10 == least >> 10));
        const int digit = x >> shift & 2047;
        const uint64_t who = __ballot(on);
        if (!who) return;
        const int one = __builtin_amdgcn_readlane(digit, __builtin_ctzll(who));
        if (__ballot(on && digit != one) == 0) {   // one counter: added to once
          if (lane == 0) atomicAdd(&hist[one], __popcll(who));
        } else if (on) {
          atomicAdd(&hist[digit], 1);
        }
      });
      __syncthreads();
      if (pass < 2)
        for (int i = threadIdx.x; i < 2048; i += 1024) s_hist[1 - (pass & 1)][i] = 0;
      // thread t: counters 2047 - 2 t and 2046 - 2 t
      const int h1 = hist[2047 - 2 * threadIdx.x], h0 = hist[2046 - 2 * threadIdx.x];
      int sum = h1 + h0;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(sum, d);
        if (lane >= d) sum += x;
      }
      if (lane == 63) s_total[wave] = sum;
      __syncthreads();
      const int mine = s_total[lane & 15];
      const int above = sum - h1 - h0 + __builtin_amdgcn_readfirstlane(row_sum((lane & 15) < wave ? mine : 0));   // counted in higher counters
      if (above < left && above + h1 + h0 >= left) {
        const bool upper = above + h1 >= left;
        s_pick[0] = 2047 - 2 * threadIdx.x - !upper;
        s_pick[1] = left - above - (upper ? 0 : h1);
      }
      __syncthreads();
      least |= (uint32_t)s_pick[0] << shift;
      left = s_pick[1];
    }
  }
  // 64 tokens in order stay or go together before or behind `gone`, which is whole blocks.  f(step, is in front of it, bits of those that stay, of
  // those that are live)
  const uint64_t lower = (1ull << lane) - 1;
  int n[2] = {0, 0};
  each([&](int c, uint32_t x) __attribute__((always_inline)) { n[0] += __popcll(__ballot(x == least && begin + 64 * c + lane < old)); });
  meet(n, before, all);
  const int equal_before = before[0];
  auto each_group = [&](auto f) __attribute__((always_inline)) {
    int rank = equal_before;
    each([&](int c, uint32_t x) __attribute__((always_inline)) {
      const int i0 = begin + 64 * c;
      const uint64_t live = old - i0 >= 64 ? ~0ull : old > i0 ? (1ull << (old - i0)) - 1 : 0;
      const uint64_t equal = __ballot(x == least) & live;
      uint64_t stays = __ballot(x > least) & live;
      if (equal) {
        const bool me = equal >> lane & 1;
        stays |= __ballot(me && rank + __popcll(equal & lower) < left);
        rank += __popcll(equal);
      }
      if (keep == 0) stays = 0;
      f(c, i0 < gone, stays, live);
    });
  };
  n[0] = n[1] = 0;
  each_group([&](int, bool front, uint64_t stays, uint64_t live) __attribute__((always_inline)) {
    if (front) n[0] += __popcll(stays);
    else n[1] += __popcll(live & ~stays);
  });
  meet(n, before, all);
  int rank[2] = {before[0], before[1]};
  each_group([&](int c, bool front, uint64_t stays, uint64_t live) __attribute__((always_inline)) {
    const uint64_t who = front ? stays : live & ~stays;
    int &at = front ? rank[0] : rank[1];
    if (who >> lane & 1) list[2 * (at + __popcll(who & lower)) + !front] = begin + 64 * c + lane;
    at += __popcll(who);
  });
  if (threadIdx.x == 0) a.count[slot * a.Hkv + hkv] = all[0];
  if (!in_place) return;
  __syncthreads();
  const int moves = all[0], group = threadIdx.x >> 5;
  for (int i = group; i < moves; i += 32) {
    RowMove m;
    m.begin(a, slot, hkv, s_list[2 * i], s_list[2 * i + 1], threadIdx.x & 31, true);
    m.end(a);
  }
}
// Two rows per 32 lanes.  Bound: memory's latency and rate (32 heads, up to 1800 rows of 516 bytes each: 11 us).
__global__ __launch_bounds__(256) void light_move_kernel(const LightArgs a) {
  const int hkv = blockIdx.y % a.Hkv, slot = blockIdx.y / a.Hkv;
  const int moves = a.count[slot * a.Hkv + hkv], i = blockIdx.x * 16 + (threadIdx.x >> 5);
  if (i >= moves) return;
  const int32_t *const list = a.moves + 2 * (a.move_base[slot] + (int64_t)hkv * a.most_moves[slot]);
  RowMove m[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int k = min(i + 8 * j, moves - 1);
    m[j].begin(a, slot, hkv, list[2 * k], list[2 * k + 1], threadIdx.x & 31, i + 8 * j < moves);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) m[j].end(a);
}

}  // namespace

void weigh_shape(int64_t most_rows, int64_t tiles, int32_t Hkv, int32_t &chunk, int32_t &n_split) {
  n_split = 1;
  chunk = kTile;
  const int64_t resident = 256;
  // Up to 256 rows, all in LDS: 256 rows x 4 x 16384 tokens 54 us, 75 in the kernel for many; 256 x 4096 tokens 10.5 and 10.9.  fp keys: one round of the workgroups that a CU
  // holds, three with 64 rows (8 x 8192 fp16 tokens 24.8 us, 28.5 with 2048 items; in the kernel for 256 rows 24.9, but 48 x 4000 98 instead of 82), one with 256.
  // int8 and int4 keys, in two numbers each, leave room for one workgroup per CU either way; 768 items instead of 256, us with some 6 of the timing's own: a query of
  // 48 x 4000 tokens int8 133 and 166, int4 145 and 183; of 8 x 8192 60 and 52, 63 and 56 (fp16 88 and 101, 33 and 38); 64 queries of 4 x 16384 have 256: 100, 102 (60).
  if (most_rows <= kFewRows) {
    const int64_t want = most_rows <= 64 ? 768 : 256;
    chunk = (int32_t)(kTile * std::max<int64_t>(1, std::min<int64_t>(64, (tiles * Hkv + want - 1) / want)));
    return;
  }
  // several items per tile where the tiles alone leave CUs idle: steps of 32 rows, eight at least
  n_split = (int32_t)std::max<int64_t>(1, std::min((2 * resident + tiles * Hkv - 1) / (tiles * Hkv), (most_rows + 255) / 256));
  if (tiles * Hkv >= resident) n_split = 1;
}

template <bool BF, int KF>
hipError_t start_weigh(const WeighArgs &a, int64_t most_rows, hipStream_t s) {
  const dim3 grid((unsigned)a.n_items * (unsigned)a.Hkv * (unsigned)a.n_split);
  constexpr int mid = is_quant(KF) ? 4 : 8;
  if (most_rows <= 64) hipLaunchKernelGGL((weigh_few_kernel<BF, KF, 64, 4>), grid, dim3(256), 0, s, a);
  else if (most_rows <= kFewRows) hipLaunchKernelGGL((weigh_few_kernel<BF, KF, kFewRows, mid>), grid, dim3(64 * mid), 0, s, a);
  else hipLaunchKernelGGL((weigh_kernel<BF, KF>), grid, dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_weigh(const WeighArgs &a, int64_t most_rows, hipStream_t s, int *n_kernels) {
  hipError_t e;
  switch (a.tv.k_fmt) {
    case TTKV_F16: e = start_weigh<false, TTKV_F16>(a, most_rows, s); break;
    case TTKV_BF16: e = start_weigh<true, TTKV_BF16>(a, most_rows, s); break;
    case TTKV_I8_SYM_G32: e = start_weigh<false, TTKV_I8_SYM_G32>(a, most_rows, s); break;
    default: e = start_weigh<false, TTKV_I4_ASYM_G64>(a, most_rows, s);
  }
  *n_kernels += 1;
  if (e != hipSuccess || a.n_split == 1) return e;
  hipLaunchKernelGGL(weigh_sum_kernel, dim3((unsigned)a.n_items, (unsigned)a.Hkv), dim3(kTile), 0, s, a);
  *n_kernels += 1;
  return hipGetLastError();
}

hipError_t launch_light(const LightArgs &a, int32_t most_moves, hipStream_t s, int *n_kernels) {
  const bool in_place = most_moves <= kInPlace;
  const dim3 grid((unsigned)(a.n_slots * a.Hkv)), block(1024);
  const int most_old = *std::max_element(a.old, a.old + a.n_slots);
  if (most_old <= 4 * 1024) hipLaunchKernelGGL(light_select_kernel<4>, grid, block, 0, s, a, (int)in_place);
  else if (most_old <= 12 * 1024) hipLaunchKernelGGL(light_select_kernel<12>, grid, block, 0, s, a, (int)in_place);
  else if (most_old <= 32 * 1024) hipLaunchKernelGGL(light_select_kernel<32>, grid, block, 0, s, a, (int)in_place);
  else hipLaunchKernelGGL(light_select_kernel<0>, grid, block, 0, s, a, (int)in_place);
  *n_kernels += 1;
  hipError_t e = hipGetLastError();
  if (in_place || e != hipSuccess) return e;
  hipLaunchKernelGGL(light_move_kernel, dim3((unsigned)((most_moves + 15) / 16), (unsigned)(a.n_slots * a.Hkv)), dim3(256), 0, s, a);
  *n_kernels += 1;
  return hipGetLastError();
}

}  // namespace ttkv
