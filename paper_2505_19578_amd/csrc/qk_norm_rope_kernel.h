// Norms of queries and keys per head with the rotation of their positions, and the cache's write, in one pass.
#ifndef SP_QK_NORM_ROPE_KERNEL_H
#define SP_QK_NORM_ROPE_KERNEL_H
#include "cache_common.h"

namespace {

// y = x / sqrt(mean(x^2) + eps) * w over a head's D elements, then each pair (a, b) of the rotated part becomes
// (a cos - b sin, a sin + b cos) with the angle position * inv_freq[pair].  All of it in 32 bits, rounded to bf16 once.
// The angle is formed in 64 bits, in whole turns, and reduced there: at position 2^20 a 32-bit product is off by 0.06 rad.
// A workgroup takes TB tokens: it forms the TB * rotary / 2 sines and cosines once, in LDS, and every head of the token uses
// them.  D / 8 lanes hold a row, four pairs each, as two 8-byte pieces that hold the pairs' halves, so that a pair never
// crosses lanes whichever way the pairs are laid out.
// WHOLE: every element of a head is rotated (rotary == D).  Otherwise (rotary is a multiple of 8) a lane's four pairs are all
// rotated or none is, and elements that are not keep their value: the turn (1, 0) would give them 0 times a partner that may be
// infinite.  Of its own, as the eight choices cost 1.5 % of a long prompt whose heads are rotated whole (176 us and 173).
// Bound by HBM (each row read once, written once, keys and values twice: output and cache): 32768 tokens of 32 + 8 heads of 128 172 us
// = 5.1 TB/s, what a large copy reaches; 1952 tokens 16.7 us = 5.0; one token 4.6 us.
constexpr int ROPE_THREADS = 256;
constexpr int ROPE_LAUNCH = 1 << 22;  // tokens of a launch: a grid's threads (here up to 2^30) have to stay below 2^32

struct RopeParams {
  const uint16_t *q, *k, *v, *qw, *kw;
  const float *inv_freq;
  const int32_t *positions, *slots;
  uint16_t *q_out, *k_out, *k_cache, *v_cache;
  int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh, qo_st, qo_sh, ko_st, ko_sh, c_sp, c_st, c_sh;
  int first, tokens, hq, hk, rotary, interleaved, page_shift;  // tokens first .. of all `tokens`, as many as the launch has
  int64_t n_slots;  // slots of the cache; 0: no cache
  float eps;
};

// where lane j's two pieces of four elements lie, and its first pair (pair numbers from rotary / 2 on are not rotated)
template <int D>
__device__ __forceinline__ void rope_pieces(int j, int rotary, int interleaved, int &a, int &b) {
  if (interleaved) {
    a = 8 * j;
    b = a + 4;
  } else if (8 * j < rotary) {
    a = 4 * j;
    b = a + rotary / 2;
  } else {
    a = rotary / 2 + 4 * j;
    b = a + (D - rotary) / 2;
  }
}

template <int D, int TB, bool WHOLE>
__global__ __launch_bounds__(ROPE_THREADS) void qk_norm_rope_kernel(RopeParams p) {
  constexpr int L = D / 8, GROUPS = ROPE_THREADS / L;  // lanes of a row, rows at a time
  __shared__ float2 turn[TB][D / 2];                   // cos, sin of a token's pairs; (1, 0) where nothing is rotated
  const int tid = threadIdx.x, j = tid % L, group = tid / L;
  const int t0 = p.first + blockIdx.x * TB, nt = min(TB, p.tokens - t0);
  for (int x = tid; x < nt * (D / 2); x += ROPE_THREADS) {
    const int t = x / (D / 2), pair = x % (D / 2);
    float2 cs = {1.f, 0.f};
    if (pair < p.rotary / 2) {
      const double turns = (double)p.positions[t0 + t] * (double)p.inv_freq[pair] * 0.15915494309189533577;  // 1 / 2 pi
      const float part = (float)(turns - __builtin_rint(turns));  // [-1/2, 1/2]
      sincospif(2.f * part, &cs.y, &cs.x);
    }
    turn[t][pair] = cs;
  }
  __syncthreads();
  const bool turned = WHOLE || 8 * j < p.rotary;
  int a, b;
  rope_pieces<D>(j, p.rotary, p.interleaved, a, b);
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.f;
  if (p.qw) {
    const u32x2 x = *(const u32x2 *)(p.qw + a), y = *(const u32x2 *)(p.qw + b);
    wq[0] = bf_lo(x[0]), wq[1] = bf_hi(x[0]), wq[2] = bf_lo(x[1]), wq[3] = bf_hi(x[1]);
    wq[4] = bf_lo(y[0]), wq[5] = bf_hi(y[0]), wq[6] = bf_lo(y[1]), wq[7] = bf_hi(y[1]);
  }
  if (p.kw) {
    const u32x2 x = *(const u32x2 *)(p.kw + a), y = *(const u32x2 *)(p.kw + b);
    wk[0] = bf_lo(x[0]), wk[1] = bf_hi(x[0]), wk[2] = bf_lo(x[1]), wk[3] = bf_hi(x[1]);
    wk[4] = bf_lo(y[0]), wk[5] = bf_hi(y[0]), wk[6] = bf_lo(y[1]), wk[7] = bf_hi(y[1]);
  }
  const int rows = p.hq + p.hk + (p.n_slots ? p.hk : 0);
  for (int x = group; x < nt * rows; x += GROUPS) {
    const int t = x / rows, row = x - t * rows, tok = t0 + t;
    int64_t cache = -1;  // element offset of the token's slot
    if (row >= p.hq && p.n_slots) {
      const int s = p.slots[tok];
      if (s >= 0 && s < p.n_slots)
        cache = (int64_t)(s >> p.page_shift) * p.c_sp + (int64_t)(s & ((1 << p.page_shift) - 1)) * p.c_st;
    }
    if (row >= p.hq + p.hk) {  // a value goes to its slot as it is
      const int h = row - p.hq - p.hk;
      const u32x4 y = *(const u32x4 *)(p.v + (int64_t)tok * p.v_st + (int64_t)h * p.v_sh + 8 * j);
      if (cache >= 0) *(u32x4 *)(p.v_cache + cache + (int64_t)h * p.c_sh + 8 * j) = y;
      continue;
    }
    const bool is_q = row < p.hq;
    const int h = is_q ? row : row - p.hq;
    const uint16_t *src = is_q ? p.q + (int64_t)tok * p.q_st + (int64_t)h * p.q_sh : p.k + (int64_t)tok * p.k_st + (int64_t)h * p.k_sh;
    const u32x2 xa = *(const u32x2 *)(src + a), xb = *(const u32x2 *)(src + b);
    float f[8] = {bf_lo(xa[0]), bf_hi(xa[0]), bf_lo(xa[1]), bf_hi(xa[1]), bf_lo(xb[0]), bf_hi(xb[0]), bf_lo(xb[1]), bf_hi(xb[1])};
    if (is_q ? p.qw != nullptr : p.kw != nullptr) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += f[e] * f[e];
#pragma unroll
      for (int d = 1; d < L; d *= 2) ss += __shfl_xor(ss, d);
      const float r = 1.f / sqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= r * (is_q ? wq[e] : wk[e]);
    }
    float2 cs[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) cs[e] = turn[t][4 * j + e];
    float y[8];
    if (p.interleaved) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[2 * e] = f[2 * e] * cs[e].x - f[2 * e + 1] * cs[e].y;
        y[2 * e + 1] = f[2 * e] * cs[e].y + f[2 * e + 1] * cs[e].x;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = f[e] * cs[e].x - f[e + 4] * cs[e].y;
        y[e + 4] = f[e] * cs[e].y + f[e + 4] * cs[e].x;
      }
    }
    if (!WHOLE && !turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = f[e];
    }
    const u32x2 ya = {pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])}, yb = {pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
    uint16_t *dst = is_q ? p.q_out + (int64_t)tok * p.qo_st + (int64_t)h * p.qo_sh
                         : p.k_out ? p.k_out + (int64_t)tok * p.ko_st + (int64_t)h * p.ko_sh : nullptr;
    if (dst) {
      *(u32x2 *)(dst + a) = ya;
      *(u32x2 *)(dst + b) = yb;
    }
    if (!is_q && cache >= 0) {
      uint16_t *c = p.k_cache + cache + (int64_t)h * p.c_sh;
      *(u32x2 *)(c + a) = ya;
      *(u32x2 *)(c + b) = yb;
    }
  }
}

}  // namespace

#endif
