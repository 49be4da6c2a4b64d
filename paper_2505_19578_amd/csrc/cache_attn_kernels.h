// Attention of the requests' new tokens (one, a chain or a drafted tree) over the paged key/value cache.
#ifndef SP_CACHE_ATTN_KERNELS_H
#define SP_CACHE_ATTN_KERNELS_H
#include "cache_common.h"

namespace {

// Per query row (token, head): x = scale q.k over the keys it sees, o = sum 2^(x c - m) v / sum 2^(x c - m), one pass with a running
// reference m, in fp32.  The query rows of a request that share a KV head (group * tokens) are one matrix: a tile of them meets
// each key once.
//
// Products (v_mfma_f32_16x16x32_bf16; lane = 16 g + i): A (16 x 32) row i, k = 8g .. 8g+7; B (32 x 16) column i, the same k;
// D (16 x 16) column i, rows 4g .. 4g+3.  S^T = K Q^T puts a query into one column of lanes; its weights, rounded to bf16, are the
// B operand of O^T = V^T P^T if k slot (g, e) stands for key 4g + e (e < 4) and 16 + 4g + e - 4 (e >= 4) of the step's 32 keys.
// V comes from LDS transposed (ds_read_b64_tr_b16: 16 lanes read four rows of 16 elements, lane i gets column i).
//
// Two kernels.  cache_attn_narrow_kernel (few rows: decoding, small trees; bound by HBM): every wavefront takes steps of 32 keys by
// itself.  cache_attn_wide_kernel (many rows; bound by the matrix pipe and the softmax): the four wavefronts share K and V in LDS and
// split the rows.
//
// Long contexts are cut into chunks (cache_chunk_units), which cache_join_kernel joins in their order: no atomics, and the bits of
// a request do not depend on what else the call holds.
constexpr int CA_THREADS = 256, CA_WAVES = 4;
constexpr float CA_SLACK = 8.0f;  // how far (log2) a row's maximum may outgrow its reference before the reference moves
constexpr float CA_LEAST = 1.17549435e-38f;  // 2^-126: what stands for a factor that 32 bits do not hold, where O is infinite
constexpr float CA_NONE = -3.0e38f;  // the reference of a row that has seen nothing: finite, so that 2^(-infinity - it) is 0

struct CacheAttnParams {
  const uint16_t *q, *k, *v;
  uint16_t *o;
  float *lse;
  const int32_t *table, *seq, *start;
  const uint64_t *mask;
  float *part_o, *part_ml;  // [partial rows][D], [partial rows][4]: reference, sum, sum of rounded weights
  int64_t q_st, q_sh, o_st, o_sh, c_sp, c_st, c_sh;
  int most_keys;
  int n_req, n_tok, hq, hk, group, page_shift, n_pages, width, words, many_split;
  float c;  // softmax scale * log2(e)
};

// The kernel's parameters once more from where they lie, for code that is rarely run: held in registers through the loops for its
// sake they were spilled, and the loops reloaded others.  (Every kernel here has the struct as its only parameter.)
__device__ __forceinline__ const CacheAttnParams &reloaded(const CacheAttnParams &) {
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const CacheAttnParams *)(const __attribute__((address_space(4))) CacheAttnParams *)at;
}

// A request as the workgroups of a call see it.
struct CacheRequest {
  CacheShare s;
  int r;
  int items_before;  // workgroups' items of the requests before it
  int rows_before;   // rows of partial results of the requests before it
  int joins_before;  // rows to join of the requests before it
};

// How far a walk has come: requests, items, rows of partial results and rows to join (of chunked requests, all KV heads) before the
// present 64 requests.
struct CacheBefore {
  int r0 = 0, items = 0, rows = 0, joins = 0;
};
// Walks the requests of a call forward, 64 at a time, one to a lane.  (Made anew for each item, from the place where the last one was:
// kept whole, it would take registers from the loops, and begun at the first request each time, the lookups of a call would grow with
// the square of its requests: 1024 of one token over up to 40, 8 KV heads, 89 us and 145, 65536 5.2 ms and 262.)
template <int TILE>
struct CacheWalk : CacheBefore {
  const CacheAttnParams &p;
  const int lane;
  int first, end, keys;  // of this lane's request, as the arrays hold them
  int upto, parts, joint;  // items, rows and rows to join up to and with it
  bool good;
  __device__ __forceinline__ CacheWalk(const CacheAttnParams &params, int l, const CacheBefore &from = {}) : CacheBefore(from), p(reloaded(params)), lane(l) {
    look();
  }
  __device__ __forceinline__ void look() {
    const int r = r0 + lane;
    const bool live = r < p.n_req;
    first = live ? p.start[r] : 0, end = live ? p.start[r + 1] : 0, keys = live ? p.seq[r] : 0;
    const CacheShare s = cache_share(first, end, keys, p.n_tok, p.most_keys, p.group, TILE, p.hk, p.many_split);
    good = !any_lane(end < first);  // otherwise this is no tok_start: nothing is done for these 64 and all behind, so that no index leaves its buffer
    upto = items + (int)wave_prefix((uint32_t)(s.tiles * p.hk * s.chunks));
    parts = rows + (int)wave_prefix((uint32_t)(s.chunks > 1 ? s.rows * p.hk * s.chunks : 0));
    joint = joins + (int)wave_prefix((uint32_t)(s.chunks > 1 ? s.rows * p.hk : 0));
  }
  template <class Test>
  __device__ __forceinline__ bool seek(Test &&test, CacheRequest &out) {
    for (;;) {
      if (!good) return false;
      const uint64_t hit = __builtin_amdgcn_ballot_w64(test(*this));
      if (hit) {
        const int at = __builtin_ctzll(hit);
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
        out.s = cache_share(of(first), of(end), of(keys), p.n_tok, p.most_keys, p.group, TILE, p.hk, p.many_split);
        out.r = r0 + at;
        out.items_before = of(upto) - out.s.tiles * p.hk * out.s.chunks;
        out.rows_before = of(parts) - (out.s.chunks > 1 ? out.s.rows * p.hk * out.s.chunks : 0);
        out.joins_before = of(joint) - (out.s.chunks > 1 ? out.s.rows * p.hk : 0);
        return true;
      }
      if (r0 + 64 >= p.n_req) return false;
      items = __builtin_amdgcn_readlane(upto, 63);
      rows = __builtin_amdgcn_readlane(parts, 63);
      joins = __builtin_amdgcn_readlane(joint, 63);
      r0 += 64;
      look();
    }
  }
  __device__ __forceinline__ bool item(int index, CacheRequest &out, CacheBefore &before) {
    const bool found = seek([index](const CacheWalk &w) { return w.upto > index; }, out);
    before = *this;
    return found;
  }
  __device__ __forceinline__ bool join(int index, CacheRequest &out) {
    return seek([index](const CacheWalk &w) { return w.joint > index; }, out);
  }
};

// One workgroup's item: a tile of a request's rows under one KV head, and a chunk of its keys.
struct CacheItem {
  int kvh, tile, chunk;
  int k_begin, k_end;  // keys
  int ctx;             // the request's new tokens begin here (negative without keys: nothing is walked then)
};
__device__ __forceinline__ CacheItem item_of(const CacheRequest &rq, int index, int hk) {
  const CachePlace place = cache_place(index - rq.items_before, rq.s.chunks * hk, rq.s.tiles);
  CacheItem it;
  it.chunk = (int)((uint32_t)place.pair / (uint32_t)hk);
  it.kvh = place.pair - it.chunk * hk;
  it.tile = place.tile;
  const CacheKeys keys = cache_chunk_keys(rq.s, it.chunk);
  it.k_begin = keys.begin, it.k_end = keys.end;
  it.ctx = rq.s.keys - rq.s.fresh;
  return it;
}
// where a row's partial result of a chunk lies: a row's chunks side by side
__device__ __forceinline__ int64_t partial_row(const CacheRequest &rq, int kvh, int row, int chunk) {
  return rq.rows_before + ((int64_t)kvh * rq.s.rows + row) * rq.s.chunks + chunk;
}

__device__ __forceinline__ bool odd_bf16x2(uint32_t x) {  // an infinity or NaN in either half
  return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t without_odd(uint32_t x) {
  return ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
}
// 1.0 where the half is of this kind: infinity, -infinity, NaN
constexpr int ODD_KINDS = 3;
__device__ __forceinline__ uint32_t ones_of_kind(uint32_t x, int kind) {
  uint32_t y = 0;
#pragma unroll
  for (int half = 0; half < 32; half += 16) {
    const uint32_t z = (x >> half) & 0xffffu;
    const bool hit = kind == 0 ? z == 0x7f80u : kind == 1 ? z == 0xff80u : (z & 0x7fffu) > 0x7f80u;
    y |= hit ? 0x3f80u << half : 0u;
  }
  return y;
}
__device__ __forceinline__ float value_of_kind(int kind) {
  return kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __builtin_nanf("");
}

typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4;
__device__ __forceinline__ bf16x8 read_transposed(char *low, char *high) {
  const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)low);
  const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)high);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The rows of a wavefront: NC column groups of 16 queries, and what a step of 32 keys does to them.
template <int D, int NC>
struct CacheRows {
  static constexpr int KS = D / 32, DT = D / 16;  // k-steps of S^T, row tiles of O^T
  bf16x8 q[NC][KS];
  f32x4 o[NC][DT], ones[NC];
  // reference (log2), what a product has to exceed to move it, sum of the weights
  float m[NC], limit[NC], l[NC];
  // CA_LEAST where this lane's part of O got something infinite: O's factors, 2^(difference of references), are no less than that, as
  // 0 times an infinite element would be NaN, and it is not to be left out either.  (0 in all other rows: their bits do not change.)
  float least[NC];
  int tok[NC];  // the column's new token

  __device__ __forceinline__ void begin(const CacheAttnParams &p, const CacheRequest &rq, int kvh, int row0, int g, int i) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int row = row0 + 16 * c + i;
      const bool live = row < rq.s.rows;
      const int t = live ? (int)((uint32_t)row / (uint32_t)p.group) : 0, hq = kvh * p.group + (live ? row - t * p.group : 0);
      tok[c] = t;
      const uint16_t *src = p.q + (int64_t)(rq.s.first + t) * p.q_st + (int64_t)hq * p.q_sh + 8 * g;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        u32x4 x = *(const u32x4 *)(src + 32 * s);
        if (!live) x = u32x4{0, 0, 0, 0};
        q[c][s] = __builtin_bit_cast(bf16x8, x);
      }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int d = 0; d < DT; ++d) o[c][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      ones[c] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[c] = CA_NONE;
      limit[c] = -INFINITY;
      l[c] = 0.f;
      least[c] = 0.f;
    }
  }
  // Bits of the step's keys that column c's query sees, from key 4 g of each half on (bits 0 .. 3 and 16 .. 19).  mask: the words of
  // its token, if there are any.
  __device__ __forceinline__ uint32_t sees(const CacheRequest &rq, const CacheItem &it, int c, int kb, uint32_t there, int g, int words,
                                           const uint64_t *mask) const {
    const uint32_t see = words == 0   ? cache_visible_chain(kb, it.ctx, rq.s.fresh, tok[c])
                         : words == 1 ? cache_visible_word(kb, it.ctx, rq.s.fresh, mask[0])
                                      : cache_visible_words(kb, it.ctx, rq.s.fresh, mask, words);
    return (see & there) >> (4 * g);
  }
  // A step's products x (keys that are not seen: -infinity) in three parts: the largest of each column's, ..
  __device__ __forceinline__ void largest(const f32x4 (&x)[2][NC], float (&top)[NC]) const {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float t = fmaxf(fmaxf(x[0][c][0], x[0][c][1]), fmaxf(x[0][c][2], x[0][c][3]));
      top[c] = fmaxf(t, fmaxf(fmaxf(x[1][c][0], x[1][c][1]), fmaxf(x[1][c][2], x[1][c][3])));
    }
  }
  // .. the references, which only have to stay within 2^SLACK of the largest weight, so that they rarely move, ..
  __device__ __forceinline__ void follow(const float (&top)[NC], float scale) {
    bool grow = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) grow |= top[c] > limit[c];
    if (!any_lane(grow)) return;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float t = top[c];
      t = fmaxf(t, __shfl_xor(t, 16));
      t = fmaxf(t, __shfl_xor(t, 32));
      if (t > limit[c]) {
        const float to = t * scale, f = __builtin_amdgcn_exp2f(m[c] - to);
        m[c] = to;
        limit[c] = t + CA_SLACK / scale;
        l[c] *= f;
        ones[c] *= f;
        const float fo = fmaxf(f, least[c]);
#pragma unroll
        for (int d = 0; d < DT; ++d) o[c][d] *= fo;
      }
    }
  }
  // .. and the weights, as the B operand of the next product.  They are rounded to bf16 for it (relative 2^-8 at most each).
  // O is divided by the sum of the rounded ones, which the matrix pipe forms with a row of ones (add_ones), so a row that few
  // keys dominate keeps no error of its sum; lse is that of the unrounded sum.
  // (pairs of them: pairs[c][n] are weights 2 n and 2 n + 1 of column group c)
  template <int FROM, int TO>
  __device__ __forceinline__ void weigh_part(const f32x4 (&x)[2][NC], float scale, uint32_t (&pairs)[NC][4]) {
    static_assert(FROM % 2 == 0 && TO % 2 == 0, "pairs");
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int e = FROM; e < TO; e += 2) {
        const float y = __builtin_amdgcn_exp2f(x[e / 4][c][e % 4] * scale - m[c]);
        const float z = __builtin_amdgcn_exp2f(x[e / 4][c][e % 4 + 1] * scale - m[c]);
        l[c] += y;
        l[c] += z;
        pairs[c][e / 2] = pack_bf16(y, z);
      }
    }
  }
  static __device__ __forceinline__ bf16x8 weights_of(const uint32_t (&pairs)[4]) {
    return __builtin_bit_cast(bf16x8, (u32x4{pairs[0], pairs[1], pairs[2], pairs[3]}));
  }
  __device__ __forceinline__ void add_ones(const bf16x8 (&pf)[NC]) {
    const uint32_t one2 = 0x3f803f80u;
    const bf16x8 all_ones = __builtin_bit_cast(bf16x8, (u32x4{one2, one2, one2, one2}));
#pragma unroll
    for (int c = 0; c < NC; ++c) ones[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(all_ones, pf[c], ones[c], 0, 0, 0);
  }
  // O += V P, V's fragments as read(d) gives them
  template <class Read>
  __device__ __forceinline__ void add_values(const bf16x8 (&pf)[NC], Read &&read) {
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const bf16x8 a = read(d);
#pragma unroll
      for (int c = 0; c < NC; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[c], o[c][d], 0, 0, 0);
    }
  }
  // what `see` of a step's columns says, as a B operand of ones and zeros
  static __device__ __forceinline__ bf16x8 as_ones(uint32_t see) {
    u32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int bit = 16 * (e >> 1) + 2 * (e & 1);
      y[e] = ((see >> bit) & 1 ? 0x3f80u : 0u) | ((see >> (bit + 1)) & 1 ? 0x3f800000u : 0u);
    }
    return __builtin_bit_cast(bf16x8, y);
  }
  // O += the kind's value where a row sees a value of this kind: V's fragments are 1 where a value is of the kind
  template <class Read>
  __device__ __forceinline__ void add_kind(const bf16x8 (&seen)[NC], int kind, Read &&read) {
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const bf16x8 a = read(d);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, seen[c], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n[r] > 0.f) o[c][d][r] += value_of_kind(kind), least[c] = CA_LEAST;
      }
    }
  }
  __device__ __forceinline__ bool any_odd() const {
    uint32_t high = 0;  // an exponent of ones stays the largest
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const u32x4 bits = __builtin_bit_cast(u32x4, o[c][d]);  // (of a vector's element the compiler takes the first one's bits)
#pragma unroll
        for (int r = 0; r < 4; ++r) high = max(high, bits[r] & 0x7fffffffu);
      }
    return any_lane(high >= 0x7f800000u);
  }
  // row sums over the lanes that share a column
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      l[c] += __shfl_xor(l[c], 16);
      l[c] += __shfl_xor(l[c], 32);
    }
  }
};

__device__ __forceinline__ float lse_of(float ref, float sum) {
  return sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}
__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

// ---------------------------------------------------------------------------------------------------------------- narrow
// A wavefront has its own registers and its own piece of LDS (V on its way to the transposed read), and no barrier until the
// workgroup's four wavefronts add up at the end.  K goes from memory to the A registers as it lies.  K of the next step is asked
// for as soon as the products have read this one's, V as soon as it lies in LDS; two workgroups on a compute unit keep 128 KiB in flight.
// 64 contexts of up to 16384 under 8 KV heads, one token each: 505 us = 5.2 TB/s, the rate of a large copy.  One of 4000: 9.1 us
// and 4.5 in the join, a chain of dependent loads (lengths, pages, keys) and of launches.
template <int D>
__global__ __launch_bounds__(CA_THREADS, 2) void cache_attn_narrow_kernel(CacheAttnParams p) {
  constexpr int NC = 1, ROWS = 16 * NC;  // one column group: with two, 17 to 32 rows took 9 to 20 % longer than in the wide kernel
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int NV = D / 16;           // 16-byte loads of a lane for a step's V
  constexpr int VL = D / 8;            // lanes of a V row
  constexpr int VROW = 2 * D + 32;     // bytes of a V row in LDS: 16 lanes' reads of four rows, and writes, meet no bank twice
  constexpr int OROW = D + 4;          // floats of an O row in LDS
  constexpr int V_BYTES = CACHE_STEP * VROW, SUM_BYTES = CA_WAVES * 16 * OROW * 4;
  constexpr int LDS = CA_WAVES * V_BYTES > SUM_BYTES ? CA_WAVES * V_BYTES : SUM_BYTES;
  __shared__ __attribute__((aligned(16))) char smem[LDS];
  __shared__ float sm[CA_WAVES][ROWS], sl[CA_WAVES][ROWS], sr[CA_WAVES][ROWS];

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, i = lane & 15;
  const int w = uniform(tid >> 6);
  char *const v_lds = smem + w * V_BYTES;
  auto v_fragment = [&](int d) -> bf16x8 {
    char *at = v_lds + (4 * g + (i >> 2)) * VROW + d * 32 + (i & 3) * 8;
    return read_transposed(at, at + 16 * VROW);
  };
  auto store_v = [&](const u32x4 *x) {
#pragma unroll
    for (int n = 0; n < NV; ++n) *(u32x4 *)(v_lds + ((64 / VL) * n + lane / VL) * VROW + (lane % VL) * 16) = x[n];
  };
  const uint32_t k_lane = 2u * (uint32_t)(i * (int)p.c_st + 8 * g);  // bytes
  const uint32_t v_lane = 2u * (uint32_t)((lane / VL) * (int)p.c_st + 8 * (lane % VL));

  CacheRequest rq;
  CacheBefore before;
  for (int index = blockIdx.x; CacheWalk<ROWS>(p, lane, before).item(index, rq, before); index += gridDim.x) {
    const CacheItem it = item_of(rq, index, reloaded(p).hk);
    CacheRows<D, NC> rows;
    const int row0 = it.tile * ROWS;
    rows.begin(reloaded(p), rq, it.kvh, row0, g, i);

    // Pages of 32 of the wavefront's steps at a time: lane 2 s + half holds that of step s, keys 16 half .. 16 half + 15 (a page
    // holds 16 keys and more, and begins at a multiple of them); -1: no such key, or a page that the cache does not have.
    const int32_t *row_pages = p.table + (int64_t)rq.r * p.width;
    const int first = it.k_begin + CACHE_STEP * w;
    const int steps = first < it.k_end ? (it.k_end - first + CACHE_UNIT - 1) / CACHE_UNIT : 0;
    auto step_key = [&](int s) { return first + CACHE_UNIT * s; };
    int pages = -1, pages_from = 0;
    auto load_pages = [&](int s0) {
      const int s = s0 + (lane >> 1), key = step_key(s) + 16 * (lane & 1);
      pages = -1;
      if (s < steps && key < it.k_end) {
        const int id = row_pages[key >> p.page_shift];
        pages = id >= 0 && id < p.n_pages ? id : -1;
      }
      pages_from = s0;
    };
    const int64_t head_off = (int64_t)it.kvh * p.c_sh;
    auto group_base = [&](int id, int key) -> int64_t {
      return (int64_t)(id < 0 ? 0 : id) * p.c_sp + (int64_t)(key & ((1 << p.page_shift) - 1)) * p.c_st + head_off;
    };
    u32x4 kr[2][KS], vr[NV];
    auto load_k = [&](int key, int id0, int id1) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint16_t *base = p.k + group_base(j ? id1 : id0, key + 16 * j);
#pragma unroll
        for (int x = 0; x < KS; ++x) kr[j][x] = *(const u32x4 *)((const char *)base + k_lane + 64 * x);
      }
    };
    auto load_v = [&](int key, int id0, int id1) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint16_t *base = p.v + group_base(j ? id1 : id0, key + 16 * j);
#pragma unroll
        for (int x = 0; x < NV / 2; ++x)
          vr[j * (NV / 2) + x] = *(const u32x4 *)((const char *)(base + (int64_t)(64 / VL) * x * p.c_st) + v_lane);
      }
    };
    int id0 = -1, id1 = -1;  // pages of the step whose keys are being loaded
    auto take_ids = [&](int s) {
      if (s - pages_from >= 32) load_pages(s);
      id0 = __builtin_amdgcn_readlane(pages, 2 * (s - pages_from));
      id1 = __builtin_amdgcn_readlane(pages, 2 * (s - pages_from) + 1);
    };

    // A second time, with care, if anything of O is not finite: a product of weight zero with an infinite value is NaN.  With care
    // values that are not finite are kept out of the products and added to the rows that see them.
    for (bool careful = false;; careful = true) {
      rows.clear();
      if (steps > 0) {
        load_pages(0);
        take_ids(0);
        load_k(step_key(0), id0, id1);
        load_v(step_key(0), id0, id1);
      }
      for (int s = 0; s < steps; ++s) {
        const int kb = step_key(s), was0 = id0, was1 = id1;
        f32x4 x[2][NC];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < KS; ++y)
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[j][y]), rows.q[c][y], acc, 0, 0, 0);
            x[j][c] = acc;
          }
        if (s + 1 < steps) {
          take_ids(s + 1);
          load_k(step_key(s + 1), id0, id1);
        }
        // all keys of a step in the context are seen by every row
        const bool exist = was0 >= 0 && was1 >= 0;
        const uint32_t there = (was0 < 0 ? 0u : 0xffffu) | (was1 < 0 ? 0u : 0xffff0000u);
        auto no_value = [&](int n) { return kb + (64 / VL) * n + lane / VL >= it.k_end || (n < NV / 2 ? was0 : was1) < 0; };
        const CacheAttnParams &cp = reloaded(p);
        auto mask_of = [&](int c) { return cp.mask + (int64_t)(rq.s.first + rows.tok[c]) * cp.words; };
        if (kb + CACHE_STEP > it.ctx || !exist) {
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const uint32_t see = rows.sees(rq, it, c, kb, there, g, cp.words, mask_of(c));
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (!((see >> (16 * j + r)) & 1)) x[j][c][r] = -INFINITY;
          }
        }
        if (kb + CACHE_STEP > it.k_end || !exist)  // values of keys that do not exist count as zeros
#pragma unroll
          for (int n = 0; n < NV; ++n)
            if (no_value(n)) vr[n] = u32x4{0, 0, 0, 0};
        if (careful)
#pragma unroll
          for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) vr[n][e] = without_odd(vr[n][e]);
        store_v(vr);
        if (!careful && s + 1 < steps) load_v(step_key(s + 1), id0, id1);
        float top[NC];
        rows.largest(x, top);
        rows.follow(top, p.c);
        uint32_t pairs[NC][4];
        rows.template weigh_part<0, 8>(x, p.c, pairs);
        bf16x8 pf[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) pf[c] = rows.weights_of(pairs[c]);
        rows.add_ones(pf);
        rows.add_values(pf, v_fragment);
        if (careful) {
          bf16x8 seen[NC];
#pragma unroll
          for (int c = 0; c < NC; ++c) seen[c] = rows.as_ones(rows.sees(rq, it, c, kb, there, g, cp.words, mask_of(c)));
#pragma unroll 1
          for (int kind = 0; kind < ODD_KINDS; ++kind) {
            load_v(kb, was0, was1);
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) vr[n][e] = no_value(n) ? 0u : ones_of_kind(vr[n][e], kind);
            store_v(vr);
            rows.add_kind(seen, kind, v_fragment);
          }
          if (s + 1 < steps) load_v(step_key(s + 1), id0, id1);
        }
      }
      if (careful || !rows.any_odd()) break;
    }

    // the four wavefronts add up, sixteen rows at a time
    rows.finish();
    const CacheAttnParams &q = reloaded(p);
    __syncthreads();  // (the last item's sums are read)
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (g == 0) {
        sm[w][16 * c + i] = rows.m[c];
        sl[w][16 * c + i] = rows.l[c];
        sr[w][16 * c + i] = rows.ones[c][0];
      }
    const int orow = tid >> 4, piece = tid & 15;  // this thread's row and its D / 16 elements of it
    float *const sum = (float *)smem;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      __syncthreads();
      {
        float top = sm[0][16 * c + i];
#pragma unroll
        for (int x = 1; x < CA_WAVES; ++x) top = fmaxf(top, sm[x][16 * c + i]);
        const float f = fmaxf(rows.m[c] == CA_NONE ? 0.f : __builtin_amdgcn_exp2f(rows.m[c] - top), rows.least[c]);
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4 *)(sum + (w * 16 + i) * OROW + 16 * d + 4 * g) = rows.o[c][d] * f;
      }
      __syncthreads();
      const int row = it.tile * ROWS + 16 * c + orow;
      float top = CA_NONE, ls = 0.f, lr = 0.f;
#pragma unroll
      for (int x = 0; x < CA_WAVES; ++x) top = fmaxf(top, sm[x][16 * c + orow]);
#pragma unroll
      for (int x = 0; x < CA_WAVES; ++x) {
        const float f = sm[x][16 * c + orow] == CA_NONE ? 0.f : __builtin_amdgcn_exp2f(sm[x][16 * c + orow] - top);
        ls += f * sl[x][16 * c + orow];
        lr += f * sr[x][16 * c + orow];
      }
      constexpr int E = D / 16;
      float y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = 0.f;
#pragma unroll
      for (int x = 0; x < CA_WAVES; ++x)
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const f32x4 z = *(const f32x4 *)(sum + (x * 16 + orow) * OROW + E * piece + e);
          y[e] += z[0], y[e + 1] += z[1], y[e + 2] += z[2], y[e + 3] += z[3];
        }
      if (row >= rq.s.rows) continue;
      if (rq.s.chunks > 1) {
        const int64_t at = partial_row(rq, it.kvh, row, it.chunk);
#pragma unroll
        for (int e = 0; e < E; e += 4) *(f32x4 *)(q.part_o + at * D + E * piece + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
        if (piece == 0) *(f32x4 *)(q.part_ml + at * 4) = f32x4{top, ls, lr, 0.f};
      } else {
        const int t = (int)((uint32_t)row / (uint32_t)q.group), hq = it.kvh * q.group + row - t * q.group;
        const float inv = inverse(lr);
        uint16_t *dst = q.o + (int64_t)(rq.s.first + t) * q.o_st + (int64_t)hq * q.o_sh + E * piece;
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *(u32x2 *)(dst + e) = u32x2{pack_bf16(y[e] * inv, y[e + 1] * inv), pack_bf16(y[e + 2] * inv, y[e + 3] * inv)};
        if (q.lse && piece == 0) q.lse[(int64_t)(rq.s.first + t) * q.hq + hq] = lse_of(top, ls);
      }
    }
    __syncthreads();  // the sums lie where V of the next item will
  }
}

// ------------------------------------------------------------------------------------------------------------------ wide
// N wavefront-wide copies of 1 KiB from memory to LDS, lds_base and on: lane l of copy n moves 16 bytes at g_uniform + lane_off[n] +
// 1024 n to LDS byte address lds_base + 1024 n + 16 l (the instruction's own offset moves both addresses).
// From inline assembly, so that the compiler does not wait for them at the next LDS read: the kernel counts these loads itself
// (wait_copies), and the compiler's own waits, which count in order, only become stricter by them.
template <int N>
__device__ __forceinline__ void copy_to_lds(const void *g_uniform, const uint32_t (&lane_off)[N], uint32_t lds_base) {
  static_assert(N == 1 || N == 2, "one setting of M0");
  if constexpr (N == 1)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_base), "v"(lane_off[0]), "s"(g_uniform)
                 : "memory", "m0");
  else
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024" ::"s"(lds_base),
        "v"(lane_off[0]), "v"(lane_off[1]), "s"(g_uniform)
        : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Steps of 32 keys lie in LDS, four of K and four of V in rings, filled two steps ahead by copies that pass no registers; one
// barrier for two steps.  A row's 16-byte pieces lie XOR-swizzled by the row number, so that K's fragments (16 rows at a time) meet no
// bank twice, V's (four rows, two neighbouring pieces of each) no more than twice; the copies' lanes fetch the pieces in that order.
// (An order in which V's meet none twice either measured the same: LDS is busy a quarter of the time.)
//
// Step s: the matrix pipe takes S of step s + 1, then O += V P of step s; beside it the vector unit makes the weights of step s,
// then the largest of S of step s + 1.
//
// A tree of 64 tokens over 131000, 64 query heads: 328 to 359 us on different cards (the clock falls under the load) = 840 to 766
// TFLOP/s next to 1184 of a large library product; the matrix pipe is busy 37 % of the cycles, the vector unit 46 %, and what is
// left is their waiting for each other and, after each pair's barrier, for three registers that come back from scratch: with two
// column groups of 128 the kernel holds 256 and spills 56, most of them for the careful pass and the rare branches.  Twelve trees of 21
// over up to 6150, 28 query heads (one column group, nothing spilled): 36 us for 87 MB of keys and values: start and end of the
// workgroups, about 8 us, and 40 steps.  A tile walks every key of its chunk, in a chain also those behind its last token, which
// it hides: a prompt over no context does twice the products that it needs.
//
// N products groups, group n with the fragment that read(n) names: use(n, fragment) issues it and its share of the vector work.
// AHEAD fragments are on their way before the first group and one more goes out with each, in this order (the fences): left to
// itself the compiler keeps one fragment at a time and has every group wait for a read of its own.
template <int N, class Read, class Use>
__device__ __forceinline__ void groups_read_ahead(Read &&read, Use &&use) {
  constexpr int AHEAD = N < 4 ? N : 4;
  bf16x8 fr[AHEAD + 1];
  static_for<0, AHEAD>([&](auto nc) __attribute__((always_inline)) { fr[decltype(nc)::value] = read(decltype(nc)::value); });
  __builtin_amdgcn_sched_barrier(0);
  static_for<0, N>([&](auto nc) __attribute__((always_inline)) {
    constexpr int n = decltype(nc)::value;
    if constexpr (n + AHEAD < N) fr[(n + AHEAD) % (AHEAD + 1)] = read(n + AHEAD);
    use(nc, fr[n % (AHEAD + 1)]);
    __builtin_amdgcn_sched_barrier(0);
  });
}

template <int D, int NC>
__global__ __launch_bounds__(CA_THREADS, 2) void cache_attn_wide_kernel(CacheAttnParams p) {
  constexpr int WROWS = 16 * NC, ROWS = CA_WAVES * WROWS;
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int RING = 4;
  constexpr int ROWB = 2 * D;                   // bytes of a K or V row
  constexpr int TILE = CACHE_STEP * ROWB;       // of a step's K (or V)
  constexpr int PIECES = ROWB / 16;             // 16-byte pieces of a row
  constexpr int COPY_ROWS = 1024 / ROWB;        // rows that one copy moves
  constexpr int COPIES = CACHE_STEP / CA_WAVES / COPY_ROWS;  // copies of a wavefront for its 8 rows of K (and as many for V)
  __shared__ __attribute__((aligned(1024))) char smem[RING * 2 * TILE];  // slot n: K of a step, then V of a step
  __shared__ uint64_t words[ROWS * CACHE_MAX_WORDS];  // mask words of the tile's rows
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) char *)smem;

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, i = lane & 15;
  const int w = uniform(tid >> 6);
  auto swizzle = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
  // this lane's part of copy n: row and piece (the LDS side is lane after lane)
  uint32_t copy_off[COPIES];
#pragma unroll
  for (int n = 0; n < COPIES; ++n) {
    const int r = (CACHE_STEP / CA_WAVES) * w + COPY_ROWS * n + lane / PIECES;
    // (rows are at least D elements apart, so 1024 n, which the instruction adds, never exceeds row COPY_ROWS * n's begin)
    copy_off[n] = 2u * (uint32_t)((r & 15) * (int)p.c_st + 8 * ((lane % PIECES) ^ swizzle(r))) - 1024u * n;
  }
  // byte of this lane's part of the first fragments (in slot 0); the others' are XORs of it, as pieces are numbered from 0 in a row
  const uint32_t k_lane = lds0 + (uint32_t)(i * ROWB + 16 * (g ^ swizzle(i)));
  const int v_row = 4 * g + (i >> 2);
  const uint32_t v_lane = lds0 + (uint32_t)(v_row * ROWB + 16 * (((i & 3) >> 1) ^ swizzle(v_row)) + 8 * (i & 1));
  typedef __attribute__((address_space(3))) const bf16x8 *lds_bf16x8;
  auto k_fragment = [&](uint32_t slot, int j, int y) -> bf16x8 {
    return *(lds_bf16x8)(((slot + k_lane) ^ (64 * y)) + 16 * ROWB * j);
  };
  auto v_fragment = [&](uint32_t slot, int d) -> bf16x8 {
    const uint32_t at = ((slot + v_lane) ^ (32 * d)) + TILE;
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)at);
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(at + 16 * ROWB));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto slot_of = [](int s) { return (uint32_t)(s % RING) * (2 * TILE); };

  CacheRequest rq;
  CacheBefore before;
  for (int index = blockIdx.x; CacheWalk<ROWS>(p, lane, before).item(index, rq, before); index += gridDim.x) {
    const CacheItem it = item_of(rq, index, reloaded(p).hk);
    CacheRows<D, NC> rows;
    const int row0 = it.tile * ROWS + w * WROWS;
    const bool idle = row0 >= rq.s.rows;  // no rows are left for this wavefront
    rows.begin(reloaded(p), rq, it.kvh, row0, g, i);
    if (const CacheAttnParams &cp = reloaded(p); cp.words)  // (the ring's first barrier lies before their use)
      for (int n = tid; n < ROWS * cp.words; n += CA_THREADS) {
        const int r = (int)((uint32_t)n / (uint32_t)cp.words), row = it.tile * ROWS + r;
        if (row < rq.s.rows)
          words[n] = cp.mask[(int64_t)(rq.s.first + (int)((uint32_t)row / (uint32_t)cp.group)) * cp.words + (n - r * cp.words)];
      }
    const int steps = it.k_begin < it.k_end ? (it.k_end - it.k_begin + CACHE_STEP - 1) / CACHE_STEP : 0;
    // All keys of a step before `soft` lie in the context and on pages that exist: every row sees them.  All keys of a step before
    // `holes` exist.
    int soft = it.ctx > it.k_begin ? (it.ctx - it.k_begin) / CACHE_STEP : 0, holes = (it.k_end - it.k_begin) / CACHE_STEP;
    auto page_at = [&](const CacheAttnParams &c, int key) {
      if (key >= it.k_end) return -1;
      const int id = c.table[(int64_t)rq.r * c.width + (key >> c.page_shift)];
      return id >= 0 && id < c.n_pages ? id : -1;
    };
    // Places of this wavefront's half of 64 steps at a time, lane s those of step s, in bytes from the cache's begin.  Keys that do
    // not exist or lie on no page are read from page 0; they count for nothing.
    uint32_t from_low = 0, from_high = 0;
    int from_step = 0;
    auto load_places = [&](int s0) {
      const CacheAttnParams &c = reloaded(p);
      const int key = it.k_begin + CACHE_STEP * (s0 + lane), mine = key + 16 * (w >> 1);
      const int a = page_at(c, key), b = page_at(c, key + 16), id = w >> 1 ? b : a;
      const uint64_t none = __builtin_amdgcn_ballot_w64(key < it.k_end && (a < 0 || (b < 0 && key + 16 < it.k_end)));
      if (none) {
        const int first = s0 + (int)__builtin_ctzll(none);
        soft = min(soft, first);
        holes = min(holes, first);
      }
      const uint64_t at = 2 * ((uint64_t)(id < 0 ? 0 : id) * (uint64_t)c.c_sp +
                               (uint64_t)(mine & ((1 << c.page_shift) - 1)) * (uint64_t)c.c_st + (uint64_t)it.kvh * (uint64_t)c.c_sh);
      from_low = (uint32_t)at, from_high = (uint32_t)(at >> 32);
      from_step = s0;
    };
    auto place_of = [&](int s) {
      return (uint32_t)__builtin_amdgcn_readlane(from_low, s - from_step) |
             (uint64_t)(uint32_t)__builtin_amdgcn_readlane(from_high, s - from_step) << 32;
    };
    const uint32_t own_rows = lds0 + (uint32_t)((CACHE_STEP / CA_WAVES) * w * ROWB);
    auto fetch_k = [&](int s) { copy_to_lds<COPIES>((const char *)p.k + place_of(s), copy_off, own_rows + slot_of(s)); };
    auto fetch_v = [&](int s) { copy_to_lds<COPIES>((const char *)p.v + place_of(s), copy_off, own_rows + slot_of(s) + TILE); };
    // S^T of a step into `next`, and beside it beside(n) for n = 0 .. 2 KS - 1
    auto products = [&](uint32_t slot, f32x4 (&next)[2][NC], auto &&beside) __attribute__((always_inline)) {
      groups_read_ahead<2 * KS>([&](int n) { return k_fragment(slot, n / KS, n % KS); },
                                [&](auto nc, const bf16x8 &a) __attribute__((always_inline)) {
        constexpr int n = decltype(nc)::value, j = n / KS, y = n % KS;
#pragma unroll
        for (int c = 0; c < NC; ++c)
          next[j][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, rows.q[c][y], y ? next[j][c] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        beside(nc);
      });
    };
    // what the rows see of step s that is not before `soft`
    auto there = [&](const CacheAttnParams &c, int kb) {
      return (page_at(c, kb) < 0 ? 0u : 0xffffu) | (page_at(c, kb + 16) < 0 ? 0u : 0xffff0000u);
    };
    auto hide = [&](int s, f32x4 (&x)[2][NC]) __attribute__((always_inline)) {
      const CacheAttnParams &cp = reloaded(p);
      const int kb = it.k_begin + CACHE_STEP * s;
      const uint32_t exist = there(cp, kb);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint32_t see = rows.sees(rq, it, c, kb, exist, g, cp.words, words + (w * WROWS + 16 * c + i) * cp.words);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!((see >> (16 * j + r)) & 1)) x[j][c][r] = -INFINITY;
      }
    };
    constexpr int OWN = TILE / 16 / CA_THREADS;  // pieces of a step's V that are this thread's to look at
    auto own_piece = [&](int s, int n) { return smem + slot_of(s) + TILE + (n * CA_THREADS + tid) * 16; };
    auto exists = [&](int s, int n, uint32_t exist) {  // the key of such a piece
      const int r = (n * CA_THREADS + tid) * 16 / ROWB;
      return it.k_begin + CACHE_STEP * s + r < it.k_end && ((exist >> r) & 1);
    };
    // values of keys that do not exist become zeros
    auto clear_holes = [&](int s) {
      const uint32_t exist = there(reloaded(p), it.k_begin + CACHE_STEP * s);
#pragma unroll
      for (int n = 0; n < OWN; ++n)
        if (!exists(s, n, exist)) *(u32x4 *)own_piece(s, n) = u32x4{0, 0, 0, 0};
    };
    float top[NC];
    auto step = [&](int s, f32x4 (&x)[2][NC], f32x4 (&next)[2][NC]) __attribute__((always_inline)) {
      rows.follow(top, p.c);
      uint32_t pairs[NC][4];
      // (behind the last step: the products of whatever lies there, for nobody)
      products(slot_of(s + 1), next, [&](auto nc) __attribute__((always_inline)) {
        constexpr int n = decltype(nc)::value, each = 16 / (2 * KS);  // of 8 weights, an even number every other group
        if constexpr (each >= 4)
          rows.template weigh_part<each / 2 * n, each / 2 *(n + 1)>(x, p.c, pairs);
        else if constexpr (n % 2 == 0)
          rows.template weigh_part<n, n + 2>(x, p.c, pairs);
      });
      bf16x8 pf[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        asm volatile("" : "+v"(pairs[c][0]), "+v"(pairs[c][1]), "+v"(pairs[c][2]), "+v"(pairs[c][3]));  // made here, not where they are used
        pf[c] = rows.weights_of(pairs[c]);
      }
      if (s + 1 >= soft) hide(s + 1, next);
      __builtin_amdgcn_s_setprio(1);  // the other workgroup's vector work goes beside it: 3 % of a tree over 128K
      rows.add_ones(pf);
      groups_read_ahead<DT>([&](int d) { return v_fragment(slot_of(s), d); },
                            [&](auto dc, const bf16x8 &a) __attribute__((always_inline)) {
        constexpr int d = decltype(dc)::value;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          rows.o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[c], rows.o[c][d], 0, 0, 0);
#pragma unroll
          for (int e = 8 / DT * d; e < 8 / DT * (d + 1); ++e) top[c] = e ? fmaxf(top[c], next[e / 4][c][e % 4]) : next[0][c][0];
        }
      });
      __builtin_amdgcn_s_setprio(0);
    };
    rows.clear();
    if (steps > 0) {
      // (steps behind the last are fetched from page 0 like keys that do not exist)
      load_places(0);
      fetch_k(0);
      fetch_v(0);
      fetch_k(1);
      fetch_v(1);
      fetch_k(2);
      f32x4 even[2][NC], odd[2][NC];
      wait_copies<0>();
      __syncthreads();
      if (!idle) {
        products(0, even, [](auto) {});
        if (0 >= soft) hide(0, even);
        rows.largest(even, top);
      }
      for (int s = 0; s < steps; s += 2) {
        // K of steps s + 1 and s + 2 and V of steps s and s + 1 have arrived, and nobody reads what came before (the first time: K
        // of step 0, in whose place that of step 4 goes)
        wait_copies<0>();
        __syncthreads();
        if (s + 2 < steps) {
          if (s + 4 - from_step >= 64) load_places(s + 2);
          fetch_k(s + 3);
          fetch_v(s + 2);
          fetch_k(s + 4);
          fetch_v(s + 3);
        }
        if (s + 1 >= holes) {
          clear_holes(s);
          clear_holes(s + 1);
          __syncthreads();
        }
        if (!idle) {
          step(s, even, odd);
          if (s + 1 < steps) step(s + 1, odd, even);
        }
      }
    }
    // (with this barrier nobody reads the ring any more)
    if (__syncthreads_or(rows.any_odd())) {
      // Something of O is not finite, and a product of weight zero with an infinite value is NaN: once more, step by step, with
      // the values that are not finite kept out of the product and added to the rows that see them.
      rows.clear();
#pragma unroll 1
      for (int s = 0; s < steps; ++s) {
        if (s == 0 || s - from_step >= 64 || s < from_step) load_places(s);
        fetch_k(s);
        fetch_v(s);
        wait_copies<0>();
        __syncthreads();
        f32x4 x[2][NC];
        products(slot_of(s), x, [](auto) {});
        hide(s, x);
        rows.largest(x, top);
        rows.follow(top, p.c);
        uint32_t pairs[NC][4];
        rows.template weigh_part<0, 8>(x, p.c, pairs);
        bf16x8 pf[NC], seen[NC];
        const int kb = it.k_begin + CACHE_STEP * s;
        const CacheAttnParams &cp = reloaded(p);
        const uint32_t exist = there(cp, kb);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          pf[c] = rows.weights_of(pairs[c]);
          seen[c] = rows.as_ones(rows.sees(rq, it, c, kb, exist, g, cp.words, words + (w * WROWS + 16 * c + i) * cp.words));
        }
        rows.add_ones(pf);
        u32x4 keep[OWN];
#pragma unroll
        for (int n = 0; n < OWN; ++n) keep[n] = exists(s, n, exist) ? *(const u32x4 *)own_piece(s, n) : u32x4{0, 0, 0, 0};
#pragma unroll 1
        for (int kind = 0; kind <= ODD_KINDS; ++kind) {  // the last round is of the finite values
#pragma unroll
          for (int n = 0; n < OWN; ++n) {
            u32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = kind == ODD_KINDS ? without_odd(keep[n][e]) : ones_of_kind(keep[n][e], kind);
            *(u32x4 *)own_piece(s, n) = y;
          }
          __syncthreads();
          if (kind < ODD_KINDS)
            rows.add_kind(seen, kind, [&](int d) { return v_fragment(slot_of(s), d); });
          else
            rows.add_values(pf, [&](int d) { return v_fragment(slot_of(s), d); });
          __syncthreads();
        }
      }
    }
    rows.finish();
    const CacheAttnParams &e = reloaded(p);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int row = row0 + 16 * c + i;
      if (row >= rq.s.rows) continue;
      const float lr = rows.ones[c][0];
      if (rq.s.chunks > 1) {
        const int64_t at = partial_row(rq, it.kvh, row, it.chunk);
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4 *)(e.part_o + at * D + 16 * d + 4 * g) = rows.o[c][d];
        if (g == 0) *(f32x4 *)(e.part_ml + at * 4) = f32x4{rows.m[c], rows.l[c], lr, 0.f};
      } else {
        const int t = (int)((uint32_t)row / (uint32_t)e.group), hq = it.kvh * e.group + row - t * e.group;
        const float inv = inverse(lr);
        uint16_t *dst = e.o + (int64_t)(rq.s.first + t) * e.o_st + (int64_t)hq * e.o_sh + 4 * g;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const f32x4 y = rows.o[c][d] * inv;
          *(u32x2 *)(dst + 16 * d) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
        }
        if (e.lse && g == 0) e.lse[(int64_t)(rq.s.first + t) * e.hq + hq] = lse_of(rows.m[c], rows.l[c]);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------ join
// Joins the chunks of the rows that have several, in their order: a wavefront per row, and on to the row as many wavefronts as the
// launch has further on.  Bound by latency: 4.5 us for the 32 rows of one token over 4000, 9.6 for 4096 rows of 16 chunks (34 MB).
template <int D>
__global__ __launch_bounds__(CA_THREADS) void cache_join_kernel(CacheAttnParams p) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  CacheWalk<16> walk(p, lane);  // (nothing here depends on the tiles; rows are short work: it is kept)
  CacheRequest rq;
  for (int index = (int)blockIdx.x * CA_WAVES + uniform(threadIdx.x >> 6); walk.join(index, rq); index += (int)gridDim.x * CA_WAVES) {
    const int in = index - rq.joins_before, kvh = (int)((uint32_t)in / (uint32_t)rq.s.rows), row = in - kvh * rq.s.rows;
    const int t = (int)((uint32_t)row / (uint32_t)p.group), token = rq.s.first + t, hq = kvh * p.group + row - t * p.group;
    const int64_t from = partial_row(rq, kvh, row, 0);
    const int chunks = rq.s.chunks;
    constexpr int AHEAD = 8;
    // the sums, 64 chunks to a wavefront, and the first results before anything waits for them
    auto sums = [&](int c) { return c < chunks ? *(const f32x4 *)(p.part_ml + (from + c) * 4) : f32x4{CA_NONE, 0.f, 0.f, 0.f}; };
    auto results = [&](int c, float (&z)[AHEAD][E]) {
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
#pragma unroll
        for (int e = 0; e < E; ++e) z[a][e] = p.part_o[(from + min(c + a, chunks - 1)) * D + E * lane + e];
    };
    f32x4 ml = sums(lane);
    float z[AHEAD][E];
    results(0, z);
    float top = ml[0];
    for (int c = lane + 64; c < chunks; c += 64) top = fmaxf(top, sums(c)[0]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    float ls = 0.f, lr = 0.f, y[E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = 0.f;
    for (int c0 = 0; c0 < chunks; c0 += 64) {
      if (c0) ml = sums(c0 + lane);
      const float f = ml[0] == CA_NONE ? 0.f : __builtin_amdgcn_exp2f(ml[0] - top);
      ls += f * ml[1];
      lr += f * ml[2];
      const int n = min(64, chunks - c0);
      for (int c = 0; c < n; c += AHEAD) {
        if (c0 + c) results(c0 + c, z);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
          const float fc = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), (c + a) & 63));
          if (c + a < n && fc != 0.f)
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] += fc * z[a][e];
        }
      }
      // a chunk whose factor 32 bits do not hold still gives what is not finite in it
      uint64_t far = __builtin_amdgcn_ballot_w64(f == 0.f && ml[0] != CA_NONE);
      while (__builtin_expect(far != 0, 0)) {
        const int c = c0 + __builtin_ctzll(far);
        far &= far - 1;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float x = p.part_o[(from + c) * D + E * lane + e];
          if ((__builtin_bit_cast(uint32_t, x) & 0x7f800000u) == 0x7f800000u) y[e] += x;
        }
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      ls += __shfl_xor(ls, d);
      lr += __shfl_xor(lr, d);
    }
    const float inv = inverse(lr);
    uint16_t *dst = p.o + (int64_t)token * p.o_st + (int64_t)hq * p.o_sh + E * lane;
    if constexpr (E == 2)
      *(uint32_t *)dst = pack_bf16(y[0] * inv, y[1] * inv);
    else
      *dst = (uint16_t)pack_bf16(y[0] * inv, 0.f);
    if (p.lse && lane == 0) p.lse[(int64_t)token * p.hq + hq] = lse_of(top, ls);
  }
}

}  // namespace

#endif
