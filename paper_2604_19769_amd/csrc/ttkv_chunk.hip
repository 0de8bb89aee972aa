// Attention of a chunk of new tokens over the tiers that hold them and everything before them: what a prompt, a part of one, or a few
// drafted tokens ask of the cache.  The query rows of a KV head are its G query heads in every new token, row r = (token r / G, head r % G),
// and a row sees the tokens up to its own:
//       S^T[token][row] = sum_d K[token][d] Q[row][d],     O^T[d][row] += sum_token V[token][d] P[token][row]
// with the running maximum and sum of the softmax in between.  Both products are v_mfma_f32_32x32x16 with tokens (channels) as rows and query
// rows as columns, so a lane has 16 scores of ONE row and the scores' registers are the second product's operand as they lie.
//
// Outputs are 16 bits wide, so the weights are rounded once to the product's type; their sum, the maximum and the log-sum-exp stay fp32.
// A quantized tier's rows are decompressed on their way into LDS, into two numbers of the product's type each (22 or 16 bits), and
// every product is made of both.
#include "ttkv_chunk_dev.h"

#include <algorithm>

namespace ttkv {

namespace {

using namespace dev;
using namespace shared;
using namespace chunk;

// Weights are 2^unit times e^(score - reference), and the reference moves only when a score is `room` above it (powers of two): over
// bf16 values no weight is above 1, over fp16 values they stay below 2^16 and keep 11 bits down to 2^-22 of the reference.
template <bool BF>
constexpr float unit16() { return BF ? -7.0f : 8.0f; }
constexpr float kRoom16 = 7.0f;

// ---------------------------------------------------------------- items
struct ChunkItem {
  int slot, entry, seq, hkv, row_tile, split, n_split;
  int count, rows;   // new tokens, query rows
};
__device__ __forceinline__ ChunkItem chunk_item(const ChunkArgs &a, int rows_per_tile) {
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
  int token, hq, pos;     // new token, query head, place behind the oldest token
  bool on;
};
template <bool BF>
__device__ __forceinline__ ChunkRows begin_chunk_rows(const ChunkArgs &a, const ChunkItem &it, int total, int row, int hh, u32x4 (&qf)[8]) {
  ChunkRows r;
  r.on = row < it.rows;
  row = min(row, it.rows - 1);
  r.token = token_of(a, row);
  r.hq = it.hkv * a.G + row - r.token * a.G;
  r.pos = total - it.count + r.token;
  const u32x4 *qp = (const u32x4 *)(a.q + it.entry * a.q_seq + r.token * a.q_token + r.hq * a.q_head);
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) qf[kb] = qp[2 * kb + hh];
  if (!BF && a.q_fmt == TTKV_BF16)
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) to_fp16(qf[kb]);
  r.cs = a.scale * kLog2e;
  r.inv_cs = 1.0f / r.cs;
  r.m = r.far = -INFINITY;
  r.l = r.mcs = 0.0f;
  return r;
}
template <bool BF>
__device__ __forceinline__ void move_chunk_reference(ChunkRows &r, float mt, f16v (&o)[4]) {
#pragma clang fp contract(off)
  const float mn = fmaxf(r.m, mt), at = __builtin_rintf(mn * r.cs), was = r.mcs;
  const bool unit = fabsf(at) < kFar;
  r.mcs = mn == -INFINITY ? 0.0f : (unit ? unit16<BF>() : 0.0f) - at;
  const float alpha = r.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.mcs - was);
  r.l *= alpha;
  rescale(o, alpha);
  r.m = mn;
  r.far = unit ? (at + kRoom16) * r.inv_cs : mn;
}
// Where a row is kept from a token whose value is infinite or no number, a weight of 0 would still make a NaN of it.  So such values meet
// the product as 0, and a row that does see one (its weight's operand `seen` is 1) gets NaN in that channel.
template <bool BF>
__device__ __forceinline__ void add_guarded(f16v &o, u32x4 va, const u32x4 &p, const u32x4 &seen) {
  constexpr uint32_t exp1 = BF ? 0x7f80u : 0x7c00u, one = BF ? 0x3f80u : 0x3c00u;
  u32x4 bad;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool low = (va[i] & exp1) == exp1, high = (va[i] >> 16 & exp1) == exp1;
    va[i] &= ~((low ? 0xffffu : 0u) | (high ? 0xffff0000u : 0u));
    bad[i] = (low ? one : 0u) | (high ? one << 16 : 0u);
  }
  o = mma<BF>(va, p, o);
  const f16v n = mma<BF>(bad, seen, f16v{});
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (n[i] > 0.0f) o[i] = __builtin_nanf("");
  __builtin_amdgcn_sched_barrier(0);   // one at a time: this is rare, and registers are dear
}

// ---------------------------------------------------------------- the kernel
// RW waves of 32 rows each share the tokens' tiles, TW such teams take the steps of 32 tokens in turn.
template <bool BF, bool QUANT, int RW, int TW>
__global__ __launch_bounds__(64 * RW * TW, 1) void chunk_kernel(const ChunkArgs a) {
  constexpr int NL = 8 / RW;                                     // pieces per thread of a step's keys (values)
  constexpr int kKeys = 32 * kRowK, kValues = 32 * kRowV, kParts = QUANT ? 2 : 1, kStep = kParts * (kKeys + kValues);
  __shared__ __align__(16) char s_tile[TW * 2 * kStep];          // per team: keys and values of two steps; at the end what the waves exchange
  __shared__ float s_m[TW * RW][32], s_l[TW * RW][32];
  __shared__ int s_wild[TW][2];                                  // per buffer: the last step with a value that is infinite or none
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tw = wave / RW, rw = wave % RW, c = lane & 31, hh = lane >> 5;
  const int tid = threadIdx.x & (64 * RW - 1);
  const ChunkItem it = chunk_item(a, 32 * RW);
  int total = 0;
  for (int t = 0; t < a.n_tiers; ++t) total += chunk_tier(a, it, t).len;
  const int row0 = it.row_tile * 32 * RW + rw * 32;
  const bool idle = row0 >= it.rows;                             // a wave without rows only helps with the tiles
  u32x4 qf[8];
  ChunkRows r = begin_chunk_rows<BF>(a, it, total, row0 + c, hh, qf);
  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) o[d] = f16v{};
  // what the tile's rows see together, what this wave's first row and its last one see
  const int base = total - it.count;
  const int sees = max(0, base + 1 + token_of(a, min(it.row_tile * 32 * RW + 32 * RW, it.rows) - 1));
  const int tile_sees = base + 1 + token_of(a, it.row_tile * 32 * RW);   // its first row
  const int first_sees = base + 1 + token_of(a, min(row0, it.rows - 1)), last_sees = base + 1 + token_of(a, min(row0 + 31, it.rows - 1));
  // this item's share of the steps, tiers one behind the other
  int n_steps = 0, before = 0;
  for (int t = 0; t < a.n_tiers; ++t) {
    const int len = chunk_tier(a, it, t).len, n = min(max(sees - before, 0), len);
    n_steps += (n + 31) / 32;
    before += len;
  }
  const int per = ((n_steps + it.n_split - 1) / it.n_split + TW - 1) / TW * TW;
  const int s0 = min(it.split * per, n_steps), s1 = min(s0 + per, n_steps);
  char *const team = s_tile + tw * 2 * kStep;
  const char *const k_at = team + k_lane(lane), *const v_at = team + kParts * kKeys + v_lane(lane);

  auto run = [&](auto kf, auto vf, const TierView &tv, int seq, int tok, int len, int lo, int hi, int ahead) __attribute__((always_inline)) {
    // steps lo .. hi - 1 of a tier of len tokens; `ahead`: tokens in the tiers before it
    constexpr int KF = decltype(kf)::value, VF = decltype(vf)::value;
    const int mine = lo + tw;
    Place keys(tv, seq, it.hkv, tok + 32 * (mine < hi ? mine : lo)), values = keys;
    int ks = mine, vs = mine;
    Piece<KF> kr[NL];
    Piece<VF> vr[NL];
    auto load_keys = [&]() __attribute__((always_inline)) {   // the team's next step, if there is one; behind the tier's end its last row
      if (ks >= hi) return;
      const int last = min(31, len - 32 * ks - 1);
      const uint64_t codes = keys.head, meta = keys.head + tv.k_meta_off;
#pragma unroll
      for (int i = 0; i < NL; ++i) kr[i] = load_piece<KF>(codes, meta, keys.row + min((tid >> 4) + 4 * RW * i, last), tid & 15);
      ks += TW;
      if (ks < hi) keys.advance(32 * TW);
    };
    auto load_values = [&]() __attribute__((always_inline)) {
      if (vs >= hi) return;
      const int last = min(31, len - 32 * vs - 1);
      const uint64_t codes = values.head + tv.v_off, meta = values.head + tv.v_meta_off;
#pragma unroll
      for (int i = 0; i < NL; ++i) vr[i] = load_piece<VF>(codes, meta, values.row + min((tid >> 4) + 4 * RW * i, last), tid & 15);
      vs += TW;
      if (vs < hi) values.advance(32 * TW);
    };
    auto put_keys = [&](int at) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        char *const to = team + at + ((tid >> 4) + 4 * RW * i) * kRowK + (tid & 15) * 16;
        put_piece<BF, KF>(kr[i], to, to + kKeys);
      }
    };
    auto put_values = [&](int at, int step) __attribute__((always_inline)) {
      if (32 * step + 32 <= tile_sees - ahead) {   // every row of the tile sees the step
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          char *const to = team + at + kParts * kKeys + ((tid >> 4) + 4 * RW * i) * kRowV + (tid & 15) * 16;
          put_piece<BF, VF>(vr[i], to, to + kValues);
        }
      } else {
        bool wild = false;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          char *const to = team + at + kParts * kKeys + ((tid >> 4) + 4 * RW * i) * kRowV + (tid & 15) * 16;
          wild |= put_piece<BF, VF, true>(vr[i], to, to + kValues);
        }
        if (wild) s_wild[tw][at != 0] = step;
      }
    };
    constexpr bool two_k = QUANT && KF != TTKV_F16 && KF != TTKV_BF16, two_v = QUANT && VF != TTKV_F16 && VF != TTKV_BF16;
#pragma unroll
    for (int i = 0; i < NL; ++i) kr[i] = Piece<KF>{}, vr[i] = Piece<VF>{};
    __syncthreads();   // everybody is done with the tier before
    load_keys();
    load_values();
    put_keys(0);
    load_keys();
    if (tid == 0) s_wild[tw][0] = s_wild[tw][1] = -1;
    __syncthreads();
    put_values(0, mine);
    load_values();
    const int n_it = (hi - lo + TW - 1) / TW;      // of the first team: all take as many barriers
    int now = 0;
    for (int t = 0; t < n_it; ++t) {
      __syncthreads();   // the step is in its buffer; everybody is done with the other one
      const int next = kStep - now, s = mine + TW * t;
      const bool works = s < hi && !idle && 32 * s < last_sees - ahead;   // (wave-uniform)
      f16v sc = {};
      if (works) {
#pragma unroll
        for (int kb = 0; kb < 8; ++kb) {
          sc = mma<BF>(*(const u32x4 *)(k_at + now + 32 * kb), qf[kb], sc);
          if constexpr (two_k) sc = mma<BF>(*(const u32x4 *)(k_at + now + kKeys + 32 * kb), qf[kb], sc);
        }
      }
      put_keys(next);
      load_keys();
      if (works) {
        const bool masked = 32 * s + 32 > min(first_sees - ahead, len), wild = masked && s_wild[tw][now != 0] == s;
        if (masked) mask_from(sc, min(r.pos + 1 - ahead, len) - 32 * s, hh);
        const float mt = step_max(sc);
        if (__any(mt > r.far)) move_chunk_reference<BF>(r, mt, o);
        u32x4 p[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float w0 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i], r.cs, r.mcs)), w1 = __builtin_amdgcn_exp2f(fmaf(sc[2 * i + 1], r.cs, r.mcs));
          r.l += w0 + w1;
          p[i / 4][i % 4] = pack2<BF>(w0, w1);
        }
        if (wild) {
          constexpr uint32_t one = BF ? 0x3f80u : 0x3c00u;
          u32x4 seen[2];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            seen[i / 4][i % 4] = (sc[2 * i] == -INFINITY ? 0u : one) | (sc[2 * i + 1] == -INFINITY ? 0u : one << 16);
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              add_guarded<BF>(o[d], value_operand(v_at + now, d, b), p[b], seen[b]);
              if constexpr (two_v) add_guarded<BF>(o[d], value_operand(v_at + now + kValues, d, b), p[b], seen[b]);
            }
        } else {
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              o[d] = mma<BF>(value_operand(v_at + now, d, b), p[b], o[d]);
              if constexpr (two_v) o[d] = mma<BF>(value_operand(v_at + now + kValues, d, b), p[b], o[d]);
            }
        }
      }
      put_values(next, s + TW);
      load_values();
      now = next;
    }
  };

  int at = 0;
  before = 0;
  for (int t = 0; t < a.n_tiers; ++t) {
    const ChunkTier T = chunk_tier(a, it, t);
    const int n = (min(max(sees - before, 0), T.len) + 31) / 32;
    const int lo = max(s0 - at, 0), hi = min(s1 - at, n);
    if (lo < hi) {
      const TierView &tv = a.tv[t];
      const int seq = t < a.n_prefix ? 0 : it.seq;
      constexpr int FP = BF ? TTKV_BF16 : TTKV_F16;
      if constexpr (QUANT) {
        if (tv.k_fmt == FP) run(num<FP>{}, num<FP>{}, tv, seq, T.tok, T.len, lo, hi, before);
        else if (tv.k_fmt == TTKV_I4_ASYM_G64) run(num<TTKV_I4_ASYM_G64>{}, num<TTKV_I4_ASYM_G64>{}, tv, seq, T.tok, T.len, lo, hi, before);
        else if (tv.v_fmt == TTKV_I4_ASYM_G64) run(num<TTKV_I8_SYM_G32>{}, num<TTKV_I4_ASYM_G64>{}, tv, seq, T.tok, T.len, lo, hi, before);
        else run(num<TTKV_I8_SYM_G32>{}, num<TTKV_I8_SYM_G32>{}, tv, seq, T.tok, T.len, lo, hi, before);
      } else {
        run(num<FP>{}, num<FP>{}, tv, seq, T.tok, T.len, lo, hi, before);
      }
    }
    at += n;
    before += T.len;
  }

  // The teams' results meet: each wave ends with 128 / TW channels of its rows.
  const f2 both = both32(r.l);
  r.l = both.x + both.y;
  float top = r.m == -INFINITY ? -INFINITY : -r.mcs, l = r.l;
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
  if (a.part_stride) {
    const int64_t at_part = (((int64_t)a.row_base[it.slot] + row0 + c) * a.Hkv + it.hkv) * a.part_stride + it.split;
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

// The items of a row tile joined: a wave per query row, two channels per lane.
__global__ __launch_bounds__(256) void chunk_merge_kernel(const ChunkArgs a, int n_rows) {
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (id >= n_rows) return;
  const int row_all = a.Hkv == 1 ? id : id / a.Hkv, hkv = id - row_all * a.Hkv;
  const int slot = __popcll(__ballot(a.row_base[lane] <= row_all)) - 1;
  const int row = row_all - a.row_base[slot], token = token_of(a, row), hq = hkv * a.G + row - token * a.G;
  const int n = a.n_split[slot], entry = a.entry[slot];
  const int64_t at = (int64_t)id * a.part_stride;
  float top = -INFINITY;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, a.pm[at + i]);
  top = wave_max(top);
  float l = 0.0f, x = 0.0f, y = 0.0f;
  for (int i = 0; i < n; ++i) {
    const float m = a.pm[at + i], li = a.pl[at + i];
    const float by = m == -INFINITY ? (li != 0.0f ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f(m - top);
    const float2 v = *(const float2 *)(a.pacc + (at + i) * 128 + 2 * lane);
    l = fmaf(li, by, l);
    x = fmaf(v.x, by, x);
    y = fmaf(v.y, by, y);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  *(uint32_t *)(a.out + entry * a.o_seq + token * a.o_token + hq * a.o_head + 4 * lane) =
      a.out_fmt == TTKV_BF16 ? pack2<true>(x * inv, y * inv) : pack2<false>(x * inv, y * inv);
  if (a.lse && lane == 0) a.lse[((int64_t)entry * a.n_tokens + token) * a.Hq + hq] = l == 0.0f ? -INFINITY : (__builtin_amdgcn_logf(l) + top) * kLn2;
}

template <bool BF, bool QUANT>
void start(const ChunkArgs &a, int rows, hipStream_t s) {
  const dim3 grid((unsigned)a.n_items * (unsigned)a.Hkv);
  if (rows == 256) hipLaunchKernelGGL((chunk_kernel<BF, QUANT, 8, 1>), grid, dim3(512), 0, s, a);
  else if (rows == 128) hipLaunchKernelGGL((chunk_kernel<BF, QUANT, 4, 2>), grid, dim3(512), 0, s, a);
  else if constexpr (!QUANT) hipLaunchKernelGGL((chunk_kernel<BF, QUANT, 2, 4>), grid, dim3(512), 0, s, a);
}

}  // namespace

ChunkShape chunk_shape(int64_t most_rows, bool bf, bool quantized) {
  return ChunkShape{most_rows <= 64 && !quantized ? 64 : most_rows <= 128 ? 128 : 256, bf, quantized};
}

int64_t chunk_least_steps(const ChunkShape &s) { return s.rows == 256 ? 4 : s.rows == 128 ? 8 : 8; }
int64_t chunk_resident(const ChunkShape &) { return 256; }

hipError_t launch_chunk(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream) {
  if (s.bf) s.quantized ? start<true, true>(a, s.rows, stream) : start<true, false>(a, s.rows, stream);
  else s.quantized ? start<false, true>(a, s.rows, stream) : start<false, false>(a, s.rows, stream);
  return hipGetLastError();
}

hipError_t launch_chunk_merge(const ChunkArgs &a, int64_t n_rows, hipStream_t stream) {
  hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)((n_rows + 3) / 4)), dim3(256), 0, stream, a, (int)n_rows);
  return hipGetLastError();
}

}  // namespace ttkv
