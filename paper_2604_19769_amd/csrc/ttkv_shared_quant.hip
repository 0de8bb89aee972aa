// Attention over a shared prefix in quantized tiers (K int8 or int4, V int8 or int4): 32 query rows per workgroup, eight waves that take
// its steps of 32 tokens in turn, each with its own rows in LDS.  A wave decompresses nothing: the codes are small integers, exact as fp16
// (keys) and bf16 (values), and the scales and zero points s, z of a token's channel group g enter in fp32:
//       score = sum_g s_{t,g} (q . code)_g + z_{t,g} sum_{c in g} q_c
//       O[c] = sum_t (p_t s_{t,g}) code_{t,c} + sum_t p_t z_{t,g}              (g the group of channel c)
// with one product chain per group for the scores, and for the values one right operand per group, p s as three bf16 numbers (24 bits of
// any size).  The two sums of O cancel (16 codes of one sign against their zero point), so they meet in every step of 32 tokens: the step's sum of
// p z, three bf16 numbers too, is a product with ones between the step's two.  Apart until the end, their error grew with
// the tokens (of the result, 512 / 2048 / 8192 tokens per wave: 2.3e-5 / 1.1e-4 / 4e-4, now 1.6e-6 / 1.9e-6 / 3.5e-6) for 1-5 % less time.
// Bound: the vector unit (codes into operands, 16 weights per group), busy in 67-75 % of the kernel's cycles, beside memory: with the merge, us, fp16 / int8 / int4 / K int8 V int4:
// 4 x 131072 tokens, 28 / 4 heads 49 / 47 / 40 / 41; 24 x 8229, 32 / 32 heads 30 / 28 / 24 / 25; 64 x 16384, 32 / 8 heads (eight blocks of 32 rows, each
// over the codes for itself) 41 / 68 / 60 / 63.  Codes converted by instructions for it instead of written into mantissas: 8-10 % more.
#include "ttkv_shared_dev.h"

namespace ttkv {

namespace {

using namespace dev;
using namespace shared;

template <int F>
constexpr int groups_of() { return F == TTKV_I8_SYM_G32 ? 4 : 2; }
template <int F>
constexpr int row_of() { return F == TTKV_I8_SYM_G32 ? 128 : 64; }   // bytes of a row's codes

// A step's codes and meta words of one wave, as loaded: 16 bytes of row lane / LPR + (64 / LPR) i, word lane % 2 of row lane / 2.
template <int F>
struct Codes {
  static constexpr int LPR = row_of<F>() / 16, N = LPR / 2;
  u32x4 w[N];
  uint32_t meta;
};
typedef const __attribute__((address_space(1))) uint32_t *gas_u32;
template <int F>
__device__ __forceinline__ Codes<F> load_codes(uint64_t codes, uint64_t meta, int len, int lane) {   // rows behind len: its last one
  using C = Codes<F>;
  C c;
#pragma unroll
  for (int i = 0; i < C::N; ++i)
    c.w[i] = *(gas_u32x4)(codes + (uint32_t)(min(lane / C::LPR + 64 / C::LPR * i, len - 1) * row_of<F>() + lane % C::LPR * 16));
  c.meta = *(gas_u32)(meta + (uint32_t)(min(lane >> 1, len - 1) * 8 + (lane & 1) * 4));
  return c;
}
__device__ __forceinline__ uint32_t low_halves(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); }
// Eight channels' codes as packed fp16 (keys; in the order of the queries' `paired`) or bf16 numbers (values; ascending).  A nibble n is
// written into the mantissa of 1.0, 1 + n / 16: two instructions for two codes, where converting them takes five to seven.
__device__ __forceinline__ u32x4 key_nibbles(uint32_t x) {   // channels (i, i + 4)
  constexpr uint32_t m = 0x03c003c0u, one = 0x3c003c00u;
  return u32x4{(x << 6 & m) | one, (x << 2 & m) | one, (x >> 2 & m) | one, (x >> 6 & m) | one};
}
__device__ __forceinline__ u32x4 value_nibbles(uint32_t x) {
  constexpr uint32_t m = 0x00780078u, one = 0x3f803f80u;
  const uint32_t a = (x << 3 & m) | one, b = (x >> 1 & m) | one, c = (x >> 5 & m) | one, d = (x >> 9 & m) | one;
  return u32x4{low_halves(a, b), low_halves(c, d), high_halves(a, b), high_halves(c, d)};
}
__device__ __forceinline__ uint2 key_bytes(uint32_t x) {     // channels (0, 2), (1, 3)
  constexpr uint32_t m = 0x00ff00ffu, big = 0x64006400u;     // 1024 + (code + 128), exact; so is the difference
  const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
  x ^= 0x80808080u;
  return uint2{__builtin_bit_cast(uint32_t, as_h2((x & m) | big) - off), __builtin_bit_cast(uint32_t, as_h2((x >> 8 & m) | big) - off)};
}
__device__ __forceinline__ uint2 value_bytes(uint32_t x) {
  const float a = (float)(int8_t)x, b = (float)(int8_t)(x >> 8), c = (float)(int8_t)(x >> 16), d = (float)(int8_t)(x >> 24);
  return uint2{pack2<true>(a, b), pack2<true>(c, d)};         // exact: eight bits
}
template <int F>
__device__ __forceinline__ u32x4 paired(const u32x4 &q) {
  if constexpr (F == TTKV_I8_SYM_G32) return u32x4{low_halves(q[0], q[1]), high_halves(q[0], q[1]), low_halves(q[2], q[3]), high_halves(q[2], q[3])};
  else return u32x4{low_halves(q[0], q[2]), high_halves(q[0], q[2]), low_halves(q[1], q[3]), high_halves(q[1], q[3])};
}
// Codes to rows of packed numbers in LDS, meta words to fp32: scale of group g and token t at sz[32 g + t], zero points 64 behind.  Of
// nibbles, whose rows hold 1 + n / 16: s n + z = 16 s (1 + n / 16) + (z - 16 s).
template <int F, bool VALUES>
__device__ __forceinline__ void put_codes(const Codes<F> &c, char *rows, int row_bytes, float *sz, int lane) {
  using C = Codes<F>;
#pragma unroll
  for (int i = 0; i < C::N; ++i) {
    char *at = rows + (lane / C::LPR + 64 / C::LPR * i) * row_bytes + lane % C::LPR * (256 / C::LPR);
    if constexpr (F == TTKV_I8_SYM_G32) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint2 x = VALUES ? value_bytes(c.w[i][2 * k]) : key_bytes(c.w[i][2 * k]);
        const uint2 y = VALUES ? value_bytes(c.w[i][2 * k + 1]) : key_bytes(c.w[i][2 * k + 1]);
        *(u32x4 *)(at + 16 * k) = u32x4{x.x, x.y, y.x, y.y};
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) *(u32x4 *)(at + 16 * k) = VALUES ? value_nibbles(c.w[i][k]) : key_nibbles(c.w[i][k]);
    }
  }
  const float lo = (float)as_h2(c.meta).x, hi = (float)as_h2(c.meta).y;
  const int t = lane >> 1, w = lane & 1;
  if constexpr (F == TTKV_I8_SYM_G32) {
    sz[32 * (2 * w) + t] = lo;
    sz[32 * (2 * w + 1) + t] = hi;
  } else {
    sz[32 * w + t] = 16.0f * lo;
    sz[64 + 32 * w + t] = fmaf(-16.0f, lo, hi);
  }
}
// The lane's sixteen tokens' numbers of a row of 32, in the order of the scores' registers.
__device__ __forceinline__ f16v of_tokens(const float *x, int hh) {
  f16v y;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float4 v = *(const float4 *)(x + 8 * k + 4 * hh);
    y[4 * k] = v.x;
    y[4 * k + 1] = v.y;
    y[4 * k + 2] = v.z;
    y[4 * k + 3] = v.w;
  }
  return y;
}

template <int KF, int VF>
__global__ __launch_bounds__(512, 1) void shared_quant_kernel(const SharedArgs a) {
  constexpr int TW = 8, GK = groups_of<KF>(), GV = groups_of<VF>();
  constexpr int kKeys = 32 * kRowK, kRows = kKeys + 32 * kRowV, kStep = kRows + 2 * 512;   // rows of K and V, their scales and zero points
  __shared__ __align__(16) char s_tile[TW * kStep];
  static_assert(TW * kStep >= 8 * (16 - 16 / TW) * 1024, "room for what the waves exchange");
  __shared__ float s_m[8][32], s_l[8][32];
  const int lane = threadIdx.x & 63, tw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hh = lane >> 5;
  Item it;
  if (!item_of(a, it)) return;
  const int mine = it.n_tok - 32 * tw;                           // tokens from the wave's first step on; it takes every TW-th
  Cursor at(a, it.hkv, it.begin + (mine > 0 ? 32 * tw : 0));
  int to_load = mine;
  const int k_meta = a.tv.k_meta_off, v_off = a.tv.v_off, v_meta = a.tv.v_meta_off;
  Codes<KF> kc{};
  Codes<VF> vc{};
  auto load = [&]() __attribute__((always_inline)) {   // the wave's next step, if there is one
    if (to_load <= 0) return;
    const int len = min(to_load, 32);
    kc = load_codes<KF>(at.head + (uint32_t)(at.row * row_of<KF>()), at.head + k_meta + (uint32_t)(at.row * 8), len, lane);
    vc = load_codes<VF>(at.head + v_off + (uint32_t)(at.row * row_of<VF>()), at.head + v_meta + (uint32_t)(at.row * 8), len, lane);
    to_load -= 32 * TW;
    if (to_load > 0) at.advance(32 * TW);
  };
  load();
  u32x4 qf[8];
  Rows r = begin_rows<false>(a, it.row_tile * 32 + c, it.hkv, hh, qf);
  float q_sum[2] = {};   // of a group of 64 channels
  if constexpr (KF == TTKV_I4_ASYM_G64) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
#pragma unroll
      for (int kb = 4 * g; kb < 4 * g + 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f2 v = unpack2<false>(qf[kb][i]);
          q_sum[g] += v.x + v.y;
        }
      const f2 both = both32(q_sum[g]);
      q_sum[g] = both.x + both.y;
    }
  }
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) qf[kb] = paired<KF>(qf[kb]);
  f16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  char *const team = s_tile + tw * kStep;
  float *const k_sz = (float *)(team + kRows), *const v_sz = k_sz + 128;
  const char *const k_at = team + k_lane(lane), *const v_at = team + kKeys + v_lane(lane);
  constexpr uint32_t one = 0x3f803f80u;
  const u32x4 ones = {one, one, one, one};
  const int n_steps = (max(mine, 0) + 32 * TW - 1) / (32 * TW);
  for (int t = 0; t < n_steps; ++t) {
    // (LDS takes a wave's stores and reads in order; the compiler has to leave them so)
    asm volatile("" ::: "memory");
    put_codes<KF, false>(kc, team, kRowK, k_sz, lane);
    put_codes<VF, true>(vc, team + kKeys, kRowV, v_sz, lane);
    asm volatile("" ::: "memory");
    load();
    f16v sc = {};
#pragma unroll
    for (int g = 0; g < GK; ++g) {
      f16v x = {};
#pragma unroll
      for (int kb = g * (8 / GK); kb < (g + 1) * (8 / GK); ++kb) x = mma<false>(*(const u32x4 *)(k_at + 32 * kb), qf[kb], x);
      const f16v s = of_tokens(k_sz + 32 * g, hh);
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = fmaf(x[i], s[i], sc[i]);
      if constexpr (KF == TTKV_I4_ASYM_G64) {
        const f16v z = of_tokens(k_sz + 64 + 32 * g, hh);
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = fmaf(z[i], q_sum[g], sc[i]);
      }
    }
    const int len = mine - 32 * TW * t;
    if (len < 32) mask_step(sc, len, hh);
    const float mt = step_max(sc);
    if (__any(mt > r.far)) move_reference<true>(r, mt, o);
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], r.cs, r.mcs));
      r.l += p[i];
    }
    u32x4 zero[2] = {};   // the sum of p z over the lane's tokens, per group of 64 channels: right operand of a product with ones
    if constexpr (VF == TTKV_I4_ASYM_G64) {
      float pz[2] = {};
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const f16v z = of_tokens(v_sz + 64 + 32 * g, hh);
#pragma unroll
        for (int i = 0; i < 16; ++i) pz[g] = fmaf(p[i], z[i], pz[g]);
      }
      uint32_t x[3];
#pragma unroll
      for (int u = 0; u < 3; ++u) {
        x[u] = pack2<true>(pz[0], pz[1]);
        const f2 y = unpack2<true>(x[u]);
        pz[0] -= y.x;
        pz[1] -= y.y;
      }
      zero[0] = u32x4{low_halves(x[0], x[1]), x[2] & 0xffffu, 0, 0};
      zero[1] = u32x4{high_halves(x[0], x[1]), x[2] >> 16, 0, 0};
    }
#pragma unroll
    for (int g = 0; g < GV; ++g) {
      const f16v s = of_tokens(v_sz + 32 * g, hh);
      u32x4 w[3][2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float w0 = p[2 * i] * s[2 * i], w1 = p[2 * i + 1] * s[2 * i + 1];
#pragma unroll
        for (int u = 0; u < 3; ++u) {
          const uint32_t x = pack2<true>(w0, w1);
          w[u][i / 4][i % 4] = x;
          const f2 y = unpack2<true>(x);
          w0 -= y.x;
          w1 -= y.y;
        }
      }
#pragma unroll
      for (int d = g * (4 / GV); d < (g + 1) * (4 / GV); ++d) {
        add_values<true>(o[d], value_operand(v_at, d, 0), w, 0);
        if constexpr (VF == TTKV_I4_ASYM_G64) o[d] = mma<true>(ones, zero[g], o[d]);   // in between: the sum on the way is half as large
        add_values<true>(o[d], value_operand(v_at, d, 1), w, 1);
      }
    }
  }
  end_rows(r);
  join_and_store<true, 1, TW>(a, r, o, 0, tw, lane, it.split, s_tile, s_m, s_l);
}

}  // namespace

bool shared_quant_fits(int k_fmt, int v_fmt) {
  const bool k8 = k_fmt == TTKV_I8_SYM_G32, k4 = k_fmt == TTKV_I4_ASYM_G64, v8 = v_fmt == TTKV_I8_SYM_G32, v4 = v_fmt == TTKV_I4_ASYM_G64;
  return (k8 && (v8 || v4)) || (k4 && v4);
}

hipError_t launch_shared_quant(const SharedArgs &a, dim3 grid, hipStream_t s) {
  if (a.tv.k_fmt == TTKV_I4_ASYM_G64)
    hipLaunchKernelGGL((shared_quant_kernel<TTKV_I4_ASYM_G64, TTKV_I4_ASYM_G64>), grid, dim3(512), 0, s, a);
  else if (a.tv.v_fmt == TTKV_I4_ASYM_G64)
    hipLaunchKernelGGL((shared_quant_kernel<TTKV_I8_SYM_G32, TTKV_I4_ASYM_G64>), grid, dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((shared_quant_kernel<TTKV_I8_SYM_G32, TTKV_I8_SYM_G32>), grid, dim3(512), 0, s, a);
  return hipGetLastError();
}

}  // namespace ttkv
