// What a cache's tokens have been worth: the attention weight that queries give every token of a tier, added up, and the eviction of
// the tokens that received least.
#include "ttkv_shared_dev.h"
#include "ttkv_chunk_dev.h"

namespace ttkv {

namespace {

using namespace dev;
using namespace shared;
using namespace chunk;

// ---------------------------------------------------------------- weights
// weight[token] += sum over rows that see it of e^(scale q.k - lse): the score product of the chunk's attention with the roles turned.  A
// wave keeps the keys of 64 tokens in registers and takes the chunk's query rows 32 at a time from LDS; a lane has 16 scores of one row
// from each 32 tokens, and adds the weights of its rows up by itself until the lanes meet at the end.  No two waves add to one token, so
// the order of a sum is fixed.
constexpr int kWaves = 4, kTokens = 64 * kWaves;   // of a workgroup
template <bool BF, int KF>
__global__ __launch_bounds__(64 * kWaves, 1) void weigh_kernel(const WeighArgs a) {
  constexpr bool two = is_quant(KF);
  __shared__ __align__(16) char s_q[2][32 * kRowK];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, hh = lane >> 5;
  const uint32_t id = blockIdx.x;
  const int item = a.Hkv == 1 ? id : a.hkv_magic ? (int)mul_high(id, a.hkv_magic) : (int)(id / (uint32_t)a.Hkv);
  const int hkv = id - item * a.Hkv;
  const int slot = __popcll(__ballot(a.first_item[lane] <= item)) - 1;
  const int entry = a.entry[slot], seq = a.first_seq + entry, rows = a.count[slot] * a.G, sees = a.sees[slot], len = a.len[slot];
  const int tile = (item - a.first_item[slot]) * kTokens, t0 = tile + 64 * wave;
  const bool idle = t0 >= len;
  const Ring ring(a.tv, seq, hkv);
  const Place at(ring, a.tv.bt_magic, a.first_tok[slot] + (idle ? tile : t0));
  // keys as left operands: lane -> token 32 g + c, channels 16 kb + 8 hh .. + 7
  u32x4 kf[2][8], kl[two ? 2 : 1][two ? 8 : 1];
  const int last = max(min(63, len - t0 - 1), 0);
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) {
      const Piece<KF> x = load_piece<KF>(at.head, at.head + a.tv.k_meta_off, at.row + min(32 * g + c, last), 2 * kb + hh);
      if constexpr (two) unpack_piece<KF, true>(x, kf[g][kb], kl[g][kb]);
      else kf[g][kb] = x.w;
    }
  float acc[2][16];
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[g][i] = 0.0f;
  const float cs = a.scale * kLog2e;
  // rows in steps of 32, from the first that sees a token of the tile on
  const int first_row = max(0, tile - sees + 1) * a.G;
  const int s0 = min(first_row, rows) / 32, s1 = (rows + 31) / 32;
  u32x4 qr[2];
  const int qrow = threadIdx.x >> 4, qp = threadIdx.x & 15;
  auto load = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = min(32 * s + qrow + 16 * i, rows - 1), token = token_of(a, row), hq = hkv * a.G + row - token * a.G;
      qr[i] = *(const u32x4 *)(a.q + entry * a.q_seq + token * a.q_token + hq * a.q_head + 16 * qp);
      if (!BF && a.q_fmt == TTKV_BF16) to_fp16(qr[i]);
    }
  };
  auto put = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *(u32x4 *)(s_q[s & 1] + (qrow + 16 * i) * kRowK + 16 * qp) = qr[i];
  };
  if (s0 < s1) {
    load(s0);
    put(s0);
    if (s0 + 1 < s1) load(s0 + 1);
  }
  for (int s = s0; s < s1; ++s) {
    __syncthreads();   // the step's rows are there; everybody is done with those of the step before
    if (s + 1 < s1) {
      put(s + 1);
      if (s + 2 < s1) load(s + 2);
    }
    if (idle) continue;
    const int row = 32 * s + c, token = token_of(a, min(row, rows - 1)), hq = hkv * a.G + min(row, rows - 1) - token * a.G;
    const float lse = a.lse[((int64_t)entry * a.n_tokens + token) * a.Hq + hq];
    // tokens of the wave's that the row sees; a row whose log-sum-exp is not finite gives nothing
    const int lim = row < rows && fabsf(lse) < INFINITY ? min(sees + token, len) - t0 : 0;
    const float off = fabsf(lse) < INFINITY ? -lse * kLog2e : 0.0f;
    u32x4 qf[8];
    const char *const q_at = s_q[s & 1] + k_lane(lane);
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) qf[kb] = *(const u32x4 *)(q_at + 32 * kb);
    const bool whole = __all(lim >= 64);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      f16v sc = {};
#pragma unroll
      for (int kb = 0; kb < 8; ++kb) {
        sc = mma<BF>(kf[g][kb], qf[kb], sc);
        if constexpr (two) sc = mma<BF>(kl[g][kb], qf[kb], sc);
      }
      if (!whole) mask_from(sc, lim - 32 * g, hh);
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[g][i] += __builtin_amdgcn_exp2f(fmaf(sc[i], cs, off));
    }
  }
  if (idle) return;
  // over the 32 lanes of a half; lane c of half hh then stores token 32 g + 8 (c / 4) + 4 hh + c % 4 (c < 16)
  float mine[2] = {0.0f, 0.0f};
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = group_sum<16>(acc[g][i]);
      const f2 both = both16(v);
      v = both.x + both.y;
      if (c == i) mine[g] = v;
    }
  if (c >= 16) return;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int t = 32 * g + 8 * (c / 4) + 4 * hh + c % 4;
    if (t0 + t >= len) continue;
    const int64_t r = (int64_t)seq * ring.blocks + at.block, rec = a.tv.table ? (int64_t)a.tv.table[r] : r;
    float *const w = a.weights + (rec * a.Hkv + hkv) * ring.bt + at.row + t;
    *w = t0 + t >= a.first_fresh[slot] ? mine[g] : *w + mine[g];
  }
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
// One row, by 32 lanes: keys (lanes 0 .. 15), values, what decompresses them, the weight.
__device__ __forceinline__ void move_row(const LightArgs &a, int slot, int hkv, int from, int to, int lane) {
  const TokenPlace f = token_place(a.tv, a.seq[slot], a.first_tok[slot] + from), t = token_place(a.tv, a.seq[slot], a.first_tok[slot] + to);
  uint8_t *const fh = a.tv.base + f.rec * a.tv.rec_bytes + (int64_t)hkv * a.tv.head_bytes, *const th = a.tv.base + t.rec * a.tv.rec_bytes + (int64_t)hkv * a.tv.head_bytes;
  const int side = lane >> 4, p = lane & 15;
  const int width = side ? a.vc : a.kc, off = side ? a.tv.v_off : 0;
  if (16 * p < width) {
    u32x4 *const x = (u32x4 *)(fh + off + (int64_t)f.row * width + 16 * p), *const y = (u32x4 *)(th + off + (int64_t)t.row * width + 16 * p);
    const u32x4 v = *x;
    if (a.swap) *x = *y;
    *y = v;
  }
  if (p == 0 && (side ? a.vm : a.km)) {
    const int meta = side ? a.tv.v_meta_off : a.tv.k_meta_off;
    u32x2 *const x = (u32x2 *)(fh + meta + (int64_t)f.row * 8), *const y = (u32x2 *)(th + meta + (int64_t)t.row * 8);
    const u32x2 v = *x;
    if (a.swap) *x = *y;
    *y = v;
  }
  if (lane == 1) {
    const int Hkv = a.Hkv, bt = a.tv.bt;
    float *const x = a.weights + (f.rec * Hkv + hkv) * bt + f.row, *const y = a.weights + (t.rec * Hkv + hkv) * bt + t.row;
    const float v = *x;
    if (a.swap) *x = *y;
    *y = v;
  }
}

// A workgroup per (sequence, KV head): the (old - gone)-th largest weight by a radix select of its order, four passes of 8 bits; equal ones
// stay from the oldest on.  Then the tokens in order, 1024 at a time: the i-th that stays among the first `gone` moves to the i-th place
// behind them whose token goes.
constexpr int kInPlace = 64;   // moves that the selecting workgroup makes by itself
__global__ __launch_bounds__(1024) void light_select_kernel(const LightArgs a, int in_place) {
  __shared__ uint32_t s_hist[256];
  __shared__ int s_wave[16][3];
  __shared__ uint32_t s_prefix;
  __shared__ int s_left;
  const int hkv = blockIdx.x % a.Hkv, slot = blockIdx.x / a.Hkv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int old = a.old[slot], gone = a.gone[slot], keep = old - gone, seq = a.seq[slot], first = a.first_tok[slot];
  int32_t *const list = a.moves + 2 * (a.move_base[slot] + (int64_t)hkv * a.most_moves[slot]);
  auto weight = [&](int i) __attribute__((always_inline)) {
    const TokenPlace p = token_place(a.tv, seq, first + i);
    return order_of(a.weights[(p.rec * a.Hkv + hkv) * a.tv.bt + p.row]);
  };
  uint32_t prefix = 0;
  int left = keep;   // of the tokens whose order begins with the prefix, so many stay
  for (int shift = 24; shift >= 0 && keep > 0; shift -= 8) {
    if (threadIdx.x < 256) s_hist[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < old; i += 1024) {
      const uint32_t u = weight(i);
      if (shift == 24 || u >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&s_hist[u >> shift & 255], 1u);
    }
    __syncthreads();
    if (threadIdx.x < 64) {   // lane -> bins 255 - 4 lane .. 252 - 4 lane
      int n[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += n[j] = s_hist[255 - 4 * lane - j];
      int before = sum;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(before, d);
        if (lane >= d) before += x;
      }
      before -= sum;
      if (before < left && before + sum >= left) {
        int j = 0;
        while (before + n[j] < left) before += n[j++];
        s_prefix = prefix | (uint32_t)(255 - 4 * lane - j) << shift;
        s_left = left - before;
      }
    }
    __syncthreads();
    prefix = s_prefix;
    left = s_left;
  }
  int n_equal = 0, n_from = 0, n_to = 0;   // of the tokens before
  for (int i0 = 0; i0 < old; i0 += 1024) {
    const int i = i0 + threadIdx.x;
    const uint32_t u = i < old ? weight(i) : 0;
    const bool equal = keep > 0 && i < old && u == prefix;
    const uint64_t me = (1ull << lane) - 1, be = __ballot(equal);
    if (lane == 0) s_wave[wave][0] = __popcll(be);
    __syncthreads();
    int rank = n_equal + __popcll(be & me);
    for (int w = 0; w < wave; ++w) rank += s_wave[w][0];
    for (int w = 0; w < 16; ++w) n_equal += s_wave[w][0];
    const bool stays = keep > 0 && i < old && (u > prefix || (equal && rank < left));
    const bool from = stays && i < gone, to = !stays && i >= gone && i < old;
    const uint64_t bf = __ballot(from), bt = __ballot(to);
    if (lane == 0) {
      s_wave[wave][1] = __popcll(bf);
      s_wave[wave][2] = __popcll(bt);
    }
    __syncthreads();
    int rf = n_from + __popcll(bf & me), rt = n_to + __popcll(bt & me);
    for (int w = 0; w < wave; ++w) {
      rf += s_wave[w][1];
      rt += s_wave[w][2];
    }
    for (int w = 0; w < 16; ++w) {
      n_from += s_wave[w][1];
      n_to += s_wave[w][2];
    }
    if (from) list[2 * rf] = i;
    if (to) list[2 * rt + 1] = i;
  }
  if (threadIdx.x == 0) a.count[slot * a.Hkv + hkv] = n_from;
  if (!in_place) return;
  __threadfence_block();
  __syncthreads();
  for (int i = threadIdx.x >> 5; i < n_from; i += 32) move_row(a, slot, hkv, list[2 * i], list[2 * i + 1], threadIdx.x & 31);
}
__global__ __launch_bounds__(256) void light_move_kernel(const LightArgs a) {
  const int hkv = blockIdx.y % a.Hkv, slot = blockIdx.y / a.Hkv;
  const int i = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (i >= a.count[slot * a.Hkv + hkv]) return;
  const int32_t *const list = a.moves + 2 * (a.move_base[slot] + (int64_t)hkv * a.most_moves[slot]);
  move_row(a, slot, hkv, list[2 * i], list[2 * i + 1], threadIdx.x & 31);
}

}  // namespace

hipError_t launch_weigh(const WeighArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.n_items * (unsigned)a.Hkv), block(64 * kWaves);
  switch (a.tv.k_fmt) {
    case TTKV_F16: hipLaunchKernelGGL((weigh_kernel<false, TTKV_F16>), grid, block, 0, s, a); break;
    case TTKV_BF16: hipLaunchKernelGGL((weigh_kernel<true, TTKV_BF16>), grid, block, 0, s, a); break;
    case TTKV_I8_SYM_G32: hipLaunchKernelGGL((weigh_kernel<false, TTKV_I8_SYM_G32>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((weigh_kernel<false, TTKV_I4_ASYM_G64>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_light(const LightArgs &a, int32_t most_moves, hipStream_t s, int *n_kernels) {
  const bool in_place = most_moves <= kInPlace;
  hipLaunchKernelGGL(light_select_kernel, dim3((unsigned)(a.n_slots * a.Hkv)), dim3(1024), 0, s, a, (int)in_place);
  *n_kernels += 1;
  hipError_t e = hipGetLastError();
  if (in_place || e != hipSuccess) return e;
  hipLaunchKernelGGL(light_move_kernel, dim3((unsigned)((most_moves + 7) / 8), (unsigned)(a.n_slots * a.Hkv)), dim3(256), 0, s, a);
  *n_kernels += 1;
  return hipGetLastError();
}

}  // namespace ttkv
