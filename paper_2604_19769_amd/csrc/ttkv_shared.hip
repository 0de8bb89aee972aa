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
// Rows of K and V go global -> registers -> LDS, those of the next steps on their way while one is computed.  The run is cut
// into as many items as fill the 256 CUs with one workgroup of eight waves each: the partials, 520 bytes per row and item, are what
// more items cost (four waves and two workgroups per CU: 128 rows x 32K tokens 57.7 us, now 45-47; 4 x 131072 tokens, 28 / 4 heads, 55.6
// and 50).
//
// The weights p meet fp16 values as an fp16 number and its remainder (22 bits), bf16 values as three bf16 numbers (24 bits): the
// outputs are fp32, and against 64 bits they are 2e-7 to 1.2e-6 off (2-norm, 1000 to 131072 tokens).
#include "ttkv_shared_dev.h"

#include <algorithm>
#include <type_traits>

namespace ttkv {

namespace {

using namespace dev;
using namespace shared;

// ---------------------------------------------------------------- up to 64 rows per KV head
// Bound: memory.  24 sequences x 8229 bf16 tokens, 32 / 32 heads (135 MB): 27.0 us, 5.0 TB/s; 5 x 131072, 28 / 4 (268 MB): 45-55 us
// as the clock allows, 4.9-6.0.  With everything but the copies taken out the first takes 24.5 (a load-only kernel 6.5-7.0 TB/s).  Four teams of two waves, 32 rows each, take the item's steps of
// 32 tokens in turn (with a run of its own for each team, 2048 tokens of 256 items, the streams a power of two apart took 59.7 us instead
// of 49.8).  A team loads its steps' rows itself; K of one step and V of the step before are always on their way, and leave their
// registers for LDS where the step before has been read (both together, once per step: 5 x 131072 58.9 us with the merge, 51.9 so).
// Up to 32 rows the teams' second waves only help with the copies (eight waves with rows and tokens of their own, and no barrier,
// were 1-3 % faster on long runs and 6-14 % slower on short ones).
template <bool BF>
__global__ __launch_bounds__(512, 1) void shared_kernel(const SharedArgs a) {
  constexpr int RW = 2, TW = 4, NL = 4;                          // 16-byte loads of K (V) per thread and step
  constexpr int kKeys = 32 * kRowK, kStep = 32 * (kRowK + kRowV);
  __shared__ __align__(16) char s_tile[TW * 2 * kStep];          // per team: keys and values of two steps; at the end what the waves exchange
  static_assert(TW * 2 * kStep >= 8 * (16 - 16 / TW) * 1024, "room for what the waves exchange");
  __shared__ float s_m[8][32], s_l[8][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tw = wave / RW, rw = wave % RW;
  const int c = lane & 31, hh = lane >> 5;
  Item it;
  if (!item_of(a, it)) return;
  const bool idle = rw * 32 >= a.rows;
  const int mine = it.n_tok - 32 * tw;                           // tokens from the team's first step on; it takes every TW-th
  Cursor keys(a, it.hkv, it.begin + (mine > 0 ? 32 * tw : 0)), values = keys;
  values.base += a.tv.v_off;
  values.head += a.tv.v_off;
  int k_left = mine, v_left = mine;                              // tokens from the cursors on
  const int lr = (threadIdx.x & 127) >> 4, lp = threadIdx.x & 15;
  u32x4 kr[NL], vr[NL];
  auto load = [&](Cursor &at, int &left, u32x4 (&x)[NL]) __attribute__((always_inline)) {   // the team's next step, if there is one; rows behind the item's end: its last one
    if (left <= 0) return;
    const int len = min(left, 32);
    const uint64_t head = at.rows();
#pragma unroll
    for (int i = 0; i < NL; ++i) x[i] = __builtin_nontemporal_load((gas_u32x4)(head + (uint32_t)(min(lr + 8 * i, len - 1) * 256 + lp * 16)));
    left -= 32 * TW;
    if (left > 0) at.advance(32 * TW);
  };
  char *const team = s_tile + tw * 2 * kStep;
  const char *const k_at = team + k_lane(lane), *const v_at = team + kKeys + v_lane(lane);
  char *const k_put = team + lr * kRowK + lp * 16, *const v_put = team + kKeys + lr * kRowV + lp * 16;
  auto put = [&](char *to, int row_bytes, const u32x4 (&x)[NL]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) *(u32x4 *)(to + i * 8 * row_bytes) = x[i];
  };
#pragma unroll
  for (int i = 0; i < NL; ++i) kr[i] = vr[i] = u32x4{0, 0, 0, 0};
  load(keys, k_left, kr);
  load(values, v_left, vr);
  u32x4 qf[8];
  Rows r = begin_rows<BF>(a, rw * 32 + c, it.hkv, hh, qf);
  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  put(k_put, kRowK, kr);
  load(keys, k_left, kr);
  put(v_put, kRowV, vr);
  load(values, v_left, vr);
  const int n_steps = (it.n_tok + 32 * TW - 1) / (32 * TW);      // of the first team: all take as many barriers
  int now = 0;   // buffer of the step
  for (int t = 0; t < n_steps; ++t) {
    __syncthreads();   // the step is in its buffer; everybody is done with the other one
    const int next = kStep - now, len = mine - 32 * TW * t;
    const bool works = len > 0 && !idle;   // (wave-uniform)
    f16v sc = {};
    if (works) {
#pragma unroll
      for (int kb = 0; kb < 8; ++kb) sc = mma<BF>(*(const u32x4 *)(k_at + now + 32 * kb), qf[kb], sc);
    }
    put(k_put + next, kRowK, kr);
    load(keys, k_left, kr);
    if (works) {
      if (len < 32) mask_step(sc, len, hh);
      const float mt = step_max(sc);
      if (__any(mt > r.far)) move_reference<BF>(r, mt, o);
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
  join_and_store<BF, RW, TW>(a, r, o, rw, tw, lane, it.split, s_tile, s_m, s_l);
}

// ---------------------------------------------------------------- more rows: 128 per workgroup
// Bound: the matrix cores, and what they may draw: 256 rows x 32K fp16 tokens of 8 KV heads 67-79 us (52 more for every 32K tokens beyond),
// where the core clock falls from 2.4 to 1.55 GHz within the launch; 660 TFLOP/s of products that count once and 990 with the
// remainders' against the 1170-1230 of a large library product (matrix cores busy in 40 % of the kernel's cycles, the vector unit in 37).  Without loads 42, without the softmax 45 of the 52: each part's
// share of the power.  64 rows per wave (half the LDS reads, accumulators in the AGPRs) came out alike, 53.  The steps of 32 tokens overlap inside a wave: while the softmax of step s runs on the vector unit, the
// matrix cores work on the values of step s - 1 and the scores of step s + 1, none of which depends on it.  LDS holds two
// steps' keys and values each (s + 1 and s + 2; s - 1 and s), one barrier per step.  Two halves of the item's tokens per workgroup meet
// at its end: half the partials of a workgroup for each.
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
      if constexpr (BF) {
        if (s) {   // the outputs take the weights of the old reference first; what is added below is then nothing
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int b = 0; b < 2; ++b) add_values<BF>(o[d], value_operand(v_old, d, b), p, b);
#pragma unroll
          for (int u = 0; u < NP; ++u) p[u][0] = p[u][1] = u32x4{0, 0, 0, 0};
        }
        move_reference<BF>(r, mt, o);
      } else {     // weights of the old reference: times the power of two as well
        const float alpha = move_reference<BF>(r, mt, o);
        const h2 by = {(_Float16)alpha, (_Float16)alpha};
#pragma unroll
        for (int u = 0; u < NP; ++u)
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) p[u][b][i] = __builtin_bit_cast(uint32_t, as_h2(p[u][b][i]) * by);
      }
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
  join_and_store<BF, 4, 2>(a, r, o, rw, half, lane, it.split, s_tile, s_m, s_l);
}

// Query rows per workgroup, workgroups along the rows.  32 / 8 heads x 32K fp16 tokens, us with blocks of 64 and of 128 rows: 32 rows 30.8 and
// 36.6, 64 rows 34.5 and 39.4, 96 rows 47.5 and 43.0, 128 rows 46.6 and 47.8; 48 rows of 32 KV heads x 8192 tokens 33.2 and 43.9.
constexpr int kWorkgroups = 256;   // on the chip at once, one per CU
struct Shape {
  int rows, row_tiles, tokens;   // tokens of an item: a multiple of this
};
Shape shape_of(int rows, bool quantized) {
  if (quantized) return Shape{32, (rows + 31) / 32, 32};
  if (rows <= 64) return Shape{64, 1, 32};
  return Shape{128, (rows + 127) / 128, 128};
}

}  // namespace

int shared_chunk(int rows, int n_kv_heads, int64_t len, bool quantized) {
  const Shape s = shape_of(rows, quantized);
  const int64_t most = std::max<int64_t>(1, kWorkgroups / std::max<int64_t>(1, (int64_t)n_kv_heads * s.row_tiles));
  const int64_t want = std::min(most, (len + 63) / 64);   // (at least 128 or 256 tokens: the same within 3 % at 1000 to 8000 tokens)
  return (int)(((len + want - 1) / want + s.tokens - 1) / s.tokens * s.tokens);
}

hipError_t launch_shared(SharedArgs &a, hipStream_t s) {
  const bool quantized = !is_fp(a.tv.k_fmt);
  const Shape sh = shape_of(a.rows, quantized);
  a.row_tiles = sh.row_tiles;
  const int64_t units = ((int64_t)a.n_split * a.Hkv + 7) / 8 * 8;
  a.g_magic = a.rows < 1 << 20 ? magic_heads(1 << 20, a.G) : 0;
  auto magic = [](int64_t most, int d) { return d > 1 && most * d < (1ll << 32) ? (uint32_t)(((1ll << 32) + d - 1) / d) : 0u; };
  a.hkv_magic = magic(units, a.Hkv);
  a.tiles_magic = magic(units / 8 * sh.row_tiles, sh.row_tiles);
  const dim3 grid((unsigned)(units * sh.row_tiles)), block(512);
  if (quantized) return launch_shared_quant(a, grid, s);
  const bool bf = a.tv.k_fmt == TTKV_BF16;
  if (sh.rows == 64) {
    if (bf) hipLaunchKernelGGL(shared_kernel<true>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(shared_kernel<false>, grid, block, 0, s, a);
  } else {
    if (bf) hipLaunchKernelGGL(shared_rows_kernel<true>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(shared_rows_kernel<false>, grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace ttkv
