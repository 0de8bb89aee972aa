// Between the projections and the cache: RMS norm of queries and keys per head, position rotation, and the rows' way into
// a tier, in one pass over them.
//
//   y = x rsqrt(mean(x^2) + eps) w         over one head's 128 channels (optional per side)
//   angle_i = pos freq_i;  c_i = magnitude cos, s_i = magnitude sin
//   (a, b) -> (a c - b s, b c + a s)       for the pairs (i, i + R/2), or (2 i, 2 i + 1); channels from R on pass
//
// A wave takes one token and eight heads at a time, eight lanes per head.  Lane j of a head holds two of the row's sixteen 16-byte pieces
// (of 16-bit channels): j and j + 8, so that the lanes of one instruction cover whole lines, where pairs are side by side or all 128
// channels turn; pieces j and j + R/16 where fewer turn half a rotation apart, lanes from R/16 on then hold pieces that pass.  From fp32 to
// fp32, with whole lines, the lane's sixteen channels are four pieces of four, j + 8 k, for the same reason.  Either way
// a rotation needs no exchange between lanes.  Stores carry the streaming hint, which pays where the lanes of one instruction fill whole lines of
// 128 bytes (2 x 4096 tokens of 32 / 8 bf16 heads 40.4 -> 33.9 us) and costs where they do not (6000 tokens of 32 / 32 fp32 heads to bf16, 96
// channels turning, 88 -> 110): where a lane's pieces are no whole lines the head's lanes exchange them through LDS first (82).  The wave's 64 lanes work out one angle each and hand them to the eight heads through
// LDS.  Angles are counted in turns: pos x (freq / 2 pi) with the factor in two 64-bit numbers and the product's rounding taken back, so
// what is left after the whole turns is right at any position (one 64-bit product alone would be 1e-4 off at 2^40); everything else is
// fp32, rounded once to the destination's type.
//
// Bound: memory.  2 x 4096 tokens of 32 / 8 bf16 heads (168 MB) 34.4 us, 4.9 TB/s of read + write; seven prompts of up to 4999 tokens into fp16
// pages (600 MB) 112 us, 5.4; 3 x 1021 tokens of 28 / 4 fp32 heads (100 MB) 18.0 us, 5.6 (with pieces of eight channels 23.2); a copy of 2 GiB reaches
// 4.9.  A single token 3.6 us, a launch.
#include "ttkv_internal.h"

#include <hip/hip_fp16.h>

#include <algorithm>

namespace ttkv {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

template <int F>
constexpr int elem_bytes() { return F == TTKV_F32 ? 4 : 2; }

// Eight channels as they lie.
template <int F>
struct Piece {
  u32x4 w[F == TTKV_F32 ? 2 : 1];
};
// STEP: 16-byte units between an fp32 piece's halves.
template <int F, int STEP>
__device__ __forceinline__ Piece<F> load_piece(const uint8_t *row, int channel) {
  Piece<F> p;
  const u32x4 *s = (const u32x4 *)(row + channel * elem_bytes<F>());
#pragma unroll
  for (int i = 0; i < elem_bytes<F>() / 2; ++i) p.w[i] = s[i * STEP];
  return p;
}
template <int F>
__device__ __forceinline__ void expand(const Piece<F> &p, float (&x)[8]) {
  if constexpr (F == TTKV_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(p.w[i / 4][i % 4]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = p.w[0][i];
      if constexpr (F == TTKV_F16) {
        const h2 v = __builtin_bit_cast(h2, u);
        x[2 * i] = (float)v.x;
        x[2 * i + 1] = (float)v.y;
      } else {
        x[2 * i] = __uint_as_float(u << 16);
        x[2 * i + 1] = __uint_as_float(u & 0xffff0000u);
      }
    }
  }
}
template <int F>
__device__ __forceinline__ Piece<F> pack(const float (&x)[8]) {   // nearest even
  Piece<F> p;
#pragma unroll
  for (int i = 0; i < 4 * elem_bytes<F>() / 2; ++i) {
    const f2 v = {x[2 * i % 8], x[(2 * i + 1) % 8]};
    if constexpr (F == TTKV_F32) p.w[i / 4][i % 4] = __float_as_uint(x[i]);
    else if constexpr (F == TTKV_F16) p.w[0][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
    else p.w[0][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  }
  return p;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_of_eight_lanes(float v) {
  v += dpp<0xB1>(v);            // quad_perm [1,0,3,2]
  v += dpp<0x4E>(v);            // quad_perm [2,3,0,1]
  return v + dpp<0x141>(v);     // row_half_mirror
}

// WHOLE: pairs are side by side, or all channels turn, or none; QUADS: pieces of four channels (see above).
template <int SRC, int DST, bool WHOLE>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a) {
  constexpr bool QUADS = WHOLE && SRC == TTKV_F32 && DST == TTKV_F32;
  constexpr int STEP = QUADS ? 8 : 1;
  constexpr int UNITS = elem_bytes<DST>() / 2;   // of 16 bytes in a piece that is stored
  constexpr bool EXCHANGE = !WHOLE || (DST == TTKV_F32 && !QUADS);
  __shared__ f2 s_turn[4][64];
  __shared__ u32x4 s_row[EXCHANGE ? 4 : 1][8][16 * UNITS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.y;
  const int64_t w = (int64_t)blockIdx.x * 4 + wave;
  const int64_t token = w >> a.wave_shift;
  const int part = (int)(w - (token << a.wave_shift)), parts = 1 << a.wave_shift;
  if (token >= a.count[j]) return;    // whole waves leave together; no barriers

  const int l8 = lane & 7, slot = lane >> 3;
  // The lane's two pieces and which of them turn.
  const int p0 = !WHOLE && l8 >= a.turning ? 2 * l8 : l8, p1 = WHOLE ? l8 + 8 : l8 < a.turning ? l8 + a.turning : 2 * l8 + 1;
  int at[4];                          // first channel of each four that the lane holds
  bool turn[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    at[k] = QUADS ? 32 * k + 4 * l8 : 8 * (k < 2 ? p0 : p1) + 4 * (k & 1);
    turn[k] = !a.interleaved ? l8 < a.turning : QUADS ? at[k] < 16 * a.turning : (k < 2 ? p0 : p1) < 2 * a.turning;
  }
  // A batch: eight heads of the queries, the keys or the values.  The next one is asked for before one is worked on.
  struct Batch {
    Piece<SRC> w0, w1;
    int side, h;
  };
  auto ask = [&](int b) __attribute__((always_inline)) -> Batch {
    Batch t;
    t.side = b >= a.first_batch[2] ? 2 : b >= a.first_batch[1] ? 1 : 0;
    const RopeSide &s = a.side[t.side];
    t.h = (b - a.first_batch[t.side]) * 8 + slot;
    const uint8_t *src = s.src + j * s.src_seq + token * s.src_token + (t.h < s.n_heads ? t.h : 0) * s.src_head;
    t.w0 = load_piece<SRC, STEP>(src, t.side == 2 ? 8 * l8 : at[0]);     // values do not turn (and go to a tier, never an fp32 one)
    t.w1 = load_piece<SRC, STEP>(src, t.side == 2 ? 8 * l8 + 64 : at[2]);
    return t;
  };
  const Batch first = ask(min(part, a.n_batches - 1));

  if (lane < 8 * a.turning) {
#pragma clang fp contract(off)
    const int64_t pos = a.positions ? a.positions[(int64_t)j * a.pos_stride + token] : a.first_pos[j] + token;
    const double x = (double)pos, turns = x * a.turns[lane];
    const double t = (turns - __builtin_rint(turns)) + (__builtin_fma(x, a.turns[lane], -turns) + x * a.turns_rest[lane]);
    const float r = (float)(t - __builtin_rint(t));   // (beyond 2^53 turns the product's rounding is whole turns itself)
    float s, c;
    sincospif(2.0f * r, &s, &c);
    s_turn[wave][lane] = f2{c * a.magnitude, s * a.magnitude};
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  f2 cs[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    cs[i] = a.interleaved ? turn[i / 2] ? s_turn[wave][at[i / 2] / 2 + i % 2] : f2{1.0f, 0.0f}
                          : turn[0] ? s_turn[wave][at[i / 4] + i % 4] : f2{1.0f, 0.0f};

  uint8_t *head0 = nullptr;   // the token's place in the tier
  int64_t head_step = 0;
  int64_t v_off = 0;
  if (a.in_tier) {
    const TierView &tv = a.tier;
    int64_t tok = a.dst_first_tok[j] + token;
    const int64_t ring = (int64_t)tv.ring_blocks * tv.bt;
    if (tok >= ring) tok -= ring;
    const int r = div_bt((int)tok, tv.bt, tv.bt_magic), row = (int)tok - r * tv.bt;
    const int64_t at = (int64_t)a.seq_id[j] * tv.ring_blocks + r;
    const int64_t rec = tv.table ? (int64_t)tv.table[at] : at;
    head0 = tv.base + rec * tv.rec_bytes + row * 256;
    head_step = tv.head_bytes;
    v_off = tv.v_off;
  }

  auto work = [&](const Batch &t) __attribute__((always_inline)) {
    const RopeSide &s = a.side[t.side];
    float x[8], y[8];
    expand<SRC>(t.w0, x);
    expand<SRC>(t.w1, y);
    if (t.side < 2) {
      if (s.norm) {
        auto mean_square = [&]() __attribute__((always_inline)) {
          float sq = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], fmaf(y[i], y[i], sq));
          return sum_of_eight_lanes(sq) * (1.0f / 128.0f);
        };
        float ms = mean_square() + a.eps;
        // squares outside fp32's range, or near its end: those of the row times a power of two (the check takes 1.5 % of 8192 tokens of 32 / 8
        // bf16 heads, nothing of fp32 rows; fp16 ones stay inside)
        if (SRC != TTKV_F16 && __builtin_expect(!(ms >= 0x1p-100f && ms <= 0x1p120f), 0)) {
          const float by = ms < 1.0f ? 0x1p100f : 0x1p-70f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] *= by;
            y[i] *= by;
          }
          ms = mean_square() + a.eps * by * by;
        }
        const float inv = 1.0f / sqrtf(ms);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] *= inv;
          y[i] *= inv;
        }
        if (s.weight) {
          const float4 *w0 = (const float4 *)(s.weight + at[0]), *w1 = (const float4 *)(s.weight + at[2]);
          const float4 u0 = w0[0], u1 = w0[STEP], v0 = w1[0], v1 = w1[STEP];
          const float u[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w}, v[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] *= u[i];
            y[i] *= v[i];
          }
        }
      }
      if (a.interleaved) {
        auto pairs = [&](float (&z)[8], int from, int to, const f2 *t) __attribute__((always_inline)) {
#pragma unroll
          for (int i = from; i < to; ++i) {
            const float u = z[2 * i], v = z[2 * i + 1];
            z[2 * i] = u * t[i].x - v * t[i].y;
            z[2 * i + 1] = v * t[i].x + u * t[i].y;
          }
        };
        if constexpr (QUADS) {
          if (turn[0]) pairs(x, 0, 2, cs);
          if (turn[1]) pairs(x, 2, 4, cs);
          if (turn[2]) pairs(y, 0, 2, cs + 4);
          if (turn[3]) pairs(y, 2, 4, cs + 4);
        } else {
          if (turn[0]) pairs(x, 0, 4, cs);
          if (turn[2]) pairs(y, 0, 4, cs + 4);
        }
      } else if (turn[0]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = x[i], v = y[i];
          x[i] = u * cs[i].x - v * cs[i].y;
          y[i] = v * cs[i].x + u * cs[i].y;
        }
      }
    }
    if (t.h >= s.n_heads) return;
    uint8_t *dst = a.in_tier && t.side ? head0 + t.h * head_step + (t.side == 2 ? v_off : 0)
                                       : s.dst + j * s.dst_seq + token * s.dst_token + t.h * s.dst_head;
    Piece<DST> o[2] = {pack<DST>(x), pack<DST>(y)};
    if constexpr (EXCHANGE)
      if (t.side != 2) {   // the head's eight lanes hand their pieces over, for whole lines per store
        u32x4 *row = s_row[wave][slot];
#pragma unroll
        for (int i = 0; i < 2 * UNITS; ++i) row[at[i / UNITS * 2] / 8 * UNITS + i % UNITS] = o[i / UNITS].w[i % UNITS];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 2 * UNITS; ++i) o[i / UNITS].w[i % UNITS] = row[l8 + 8 * i];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
    for (int i = 0; i < 2 * UNITS; ++i) __builtin_nontemporal_store(o[i / UNITS].w[i % UNITS], (u32x4 *)dst + l8 + 8 * i);
  };
  Batch now = first;
  for (int b = part; b < a.n_batches; b += parts) {
    Batch next = now;
    if (b + parts < a.n_batches) next = ask(b + parts);
    work(now);
    now = next;
  }
}

template <int SRC, int DST>
void launch_kernel(const RopeArgs &a, dim3 grid, hipStream_t s) {
  if (a.interleaved || a.turning == 0 || a.turning == 8) hipLaunchKernelGGL((rope_kernel<SRC, DST, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rope_kernel<SRC, DST, false>), grid, dim3(256), 0, s, a);
}
template <int SRC>
void launch_from(const RopeArgs &a, int dst, dim3 grid, hipStream_t s) {
  switch (dst) {
    case TTKV_F16: launch_kernel<SRC, TTKV_F16>(a, grid, s); break;
    case TTKV_BF16: launch_kernel<SRC, TTKV_BF16>(a, grid, s); break;
    default: launch_kernel<SRC, TTKV_F32>(a, grid, s); break;
  }
}

}  // namespace

// a.count: tokens per entry, at most n_tokens.
hipError_t launch_rope(RopeArgs &a, int n_seq, int64_t n_tokens, int src_fmt, int dst_fmt, hipStream_t s) {
  int n = 0;
  for (int i = 0; i < 3; ++i) {
    a.first_batch[i] = n;
    n += (a.side[i].n_heads + 7) / 8;
  }
  a.n_batches = n;
  // A wave works its angles out once for all its heads; where there are too few tokens to fill the chip (eight waves per
  // CU's four SIMDs) they are shared out over more waves.
  a.wave_shift = 0;
  while ((1 << a.wave_shift) < n && ((n_tokens * n_seq) << a.wave_shift) < 8192) ++a.wave_shift;
  const dim3 grid((unsigned)(((n_tokens << a.wave_shift) + 3) / 4), n_seq);
  switch (src_fmt) {
    case TTKV_F16: launch_from<TTKV_F16>(a, dst_fmt, grid, s); break;
    case TTKV_BF16: launch_from<TTKV_BF16>(a, dst_fmt, grid, s); break;
    default: launch_from<TTKV_F32>(a, dst_fmt, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace ttkv
