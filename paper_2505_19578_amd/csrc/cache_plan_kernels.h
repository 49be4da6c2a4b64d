// The plan of a step over the paged cache: which pages the new tokens get, where each of them goes, what a drafted one sees.
#ifndef SP_CACHE_PLAN_KERNELS_H
#define SP_CACHE_PLAN_KERNELS_H
#include "cache_common.h"

namespace {

// Two parts.  plan_requests: one workgroup walks the requests in order (two prefix sums: tokens, then pages of the requests
// that are not refused) and writes what there is one of per request.  plan_tokens: every new token finds its request by
// bisection in tok_start and writes its slot; the token that opens a fresh page also writes that page into the request's row.
// Page entries that are read are those the request held before, the ones that are written come after them, so tokens need no
// order among each other.  A token's ancestors are walked up from it, in LDS, where a workgroup lays the parents of its tokens and
// of the PLAN_MAX_TREE before them, which is as far as a tree with masks reaches.
// Bound by latency: a few dependent loads and two scans; 256 requests of one token 4.3 us (an empty launch: about 2).  Three ways:
//   spread       up to PLAN_THREADS requests: every workgroup does the first part for itself, in LDS, and PLAN_THREADS tokens of the
//                second; the first one writes what there is per request.  One launch of any number of tokens, but what the first
//                part reads may not be what it writes: not for n_held and n_free that are updated in place.
//   one          otherwise, up to PLAN_ONE_LAUNCH tokens: one workgroup does both parts
//   two launches otherwise: the second part is spread over the chip.
// Spread and what it would be otherwise (us on the device; a second launch takes its caller 2.5 more): 256 requests of one token 4.7 and
// 4.5, 96 trees of 32 tokens 5.9 and 9.4, 250 6.0 and 9.4, 4000 tokens of chains 4.7 and 6.8, 1000 requests of 8 tokens 5.5 and 9.4, 40
// of 8192 8.8 and 8.3, 400 trees of 256 16.2 and 14.8.  One and two launches: 256 requests of one token 4.5 and 6.6, 60 trees of 32
// 7.4 and 8.6, 120 10.3 and 8.9, 8000 trees' tokens 18.7 and 9.2.
constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64;
constexpr int PLAN_ONE_LAUNCH = 4096;           // tokens
constexpr int PLAN_PART_THREADS = 256;          // and tokens of a workgroup, of the second part's own launch
constexpr int PLAN_MAX_TREE = 64 * CACHE_MAX_WORDS;

struct PlanParams {
  const int32_t *ctx, *fresh, *held, *free_pages, *n_free, *parents;
  int32_t *table, *held_out, *n_free_out, *tok_start, *seq_len, *positions, *slots, *status;
  uint64_t *mask;
  int32_t *old_held, *page_start;  // workspace: [n] each; page_start < 0: a refused request
  int32_t *free_count;             // workspace: [1], pages that were free before the call
  int n, max_tokens, page_shift, width, words, free_capacity;
};

// One request as its tokens see it.  (16 bytes: one load)
struct alignas(16) PlanRequest {
  int32_t ctx, held, page_start, pad;
};

// inclusive prefix sum over the workgroup; `total` gets the sum of all.  `room`: of this call alone
__device__ __forceinline__ uint64_t block_scan(uint64_t x, uint64_t *room, uint64_t &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  x = wave_prefix(x);
  if (lane == 63) room[w] = x;
  __syncthreads();
  const uint64_t y = wave_prefix(lane < PLAN_WAVES ? room[lane] : 0);
  auto at = [&](int l) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)y, l) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(y >> 32), l) << 32;
  };
  total = at(PLAN_WAVES - 1);
  return x + (w > 0 ? at(uniform(w) - 1) : 0);
}

// Keep: called with (request, start of the next one, PlanRequest) for every request.  lead: this workgroup writes the outputs.
// Returns the number of free pages before the call.
template <class Keep>
__device__ __forceinline__ int plan_requests(const PlanParams &p, bool lead, uint64_t (&room)[4][PLAN_WAVES], Keep &&keep) {
  uint64_t tokens = 0, pages = 0;  // before this round's requests
  int n_free = p.n_free[0];
  n_free = n_free < 0 ? 0 : n_free > p.free_capacity ? p.free_capacity : n_free;
  const int64_t most = p.words ? 64 * p.words : 0x7fffffff;
  for (int r0 = 0, round = 0; r0 < p.n; r0 += PLAN_THREADS, round ^= 1) {  // (two rounds' rooms: a barrier lies between their uses)
    const int r = r0 + threadIdx.x;
    const bool live = r < p.n;
    const int ctx = live ? p.ctx[r] : 0, fresh = live ? p.fresh[r] : 0, held = live ? p.held[r] : 0;
    uint64_t total;
    const uint64_t end = tokens + block_scan(fresh > 0 ? fresh : 0, room[2 * round], total);
    tokens += total;
    int st = plan_length_status(ctx, fresh, held, p.width, 1 << p.page_shift, most);
    if (st == PLAN_OK && end > (uint64_t)p.max_tokens) st = PLAN_NO_ROOM;
    const uint64_t lack = live && st == PLAN_OK ? plan_lacking((int64_t)ctx + fresh, held, 1 << p.page_shift) : 0;
    const uint64_t last = pages + block_scan(lack, room[2 * round + 1], total);
    // the first request for which the pages do not suffice knows how many were given out: all those before it
    if (lead && lack > 0 && last > (uint64_t)n_free && last - lack <= (uint64_t)n_free) p.n_free_out[0] = n_free - (int)(last - lack);
    pages += total;
    if (st == PLAN_OK && lack > 0 && last > (uint64_t)n_free) st = PLAN_NO_PAGES;
    const bool ok = st == PLAN_OK;
    if (live) {
      const int start = (int)(end < (uint64_t)p.max_tokens ? end : p.max_tokens);
      if (lead) {
        p.tok_start[r + 1] = start;
        p.seq_len[r] = ok ? ctx + fresh : 0;
        p.status[r] = st;
        p.held_out[r] = ok ? held + (int)lack : held;
      }
      keep(r, start, PlanRequest{ctx, held, ok ? (int)(last - lack) : -1, 0});
    }
  }
  if (lead && threadIdx.x == 0) {
    p.tok_start[0] = 0;
    p.free_count[0] = n_free;
    if (pages <= (uint64_t)n_free) p.n_free_out[0] = n_free - (int)pages;
  }
  return n_free;
}

// Tokens t0 + threadIdx, + threads, .. below t1.  start(r) and request(r): of the requests; up: parents of tokens up0 .. in LDS.
template <class Start, class Request>
__device__ __forceinline__ void plan_tokens(const PlanParams &p, int n_free, int t0, int t1, int threads, Start &&start, Request &&request,
                                            const int16_t *up, int up0) {
  const int used = p.n ? start(p.n) : 0;
  for (int t = t0 + (int)threadIdx.x; t < t1; t += threads) {
    int slot = -1, pos = 0, depth = 0;
    uint64_t m[CACHE_MAX_WORDS] = {0, 0, 0, 0};
    if (t < used) {
      int lo = 0, hi = p.n - 1;  // the first request whose tokens end behind t
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start(mid + 1) > t)
          hi = mid;
        else
          lo = mid + 1;
      }
      const PlanRequest q = request(lo);
      if (q.page_start >= 0) {
        const int first = start(lo), i = t - first;
        pos = q.ctx + i;
        const int entry = pos >> p.page_shift, off = pos & ((1 << p.page_shift) - 1);
        const int64_t at = (int64_t)lo * p.width + entry;
        int id;
        if (entry < q.held) {
          id = p.table[at];
        } else {
          id = p.free_pages[n_free - 1 - (q.page_start + entry - q.held)];
          if (off == 0) p.table[at] = id;
        }
        slot = cache_slot(id, 1 << p.page_shift, off);
        if (!p.parents) {
          depth = i;
#pragma unroll
          for (int w = 0; w < CACHE_MAX_WORDS; ++w) {
            const int n = i - 64 * w;  // bits 0 .. i
            m[w] = n < 0 ? 0ull : n >= 63 ? ~0ull : (2ull << n) - 1;
          }
        } else if (p.words) {
          const int16_t *mine = up + (first - up0);
          depth = -1;
          auto walk = [&](auto &&mark) {
            for (int a = i; a >= 0; ++depth) {
              const int q2 = mine[a];
              mark(a);
              a = q2 < a ? q2 : -1;  // no earlier token of the request: a root
            }
          };
          if (p.words == 1)
            walk([&](int a) { m[0] |= 1ull << a; });
          else
            walk([&](int a) {
#pragma unroll
              for (int w = 0; w < CACHE_MAX_WORDS; ++w) m[w] |= (a >> 6) == w ? 1ull << (a & 63) : 0ull;
            });
        } else {  // positions alone: a tree of any size, by its own memory
          for (int a = i;; ++depth) {
            const int q2 = p.parents[first + a];
            if (q2 < 0 || q2 >= a) break;
            a = q2;
          }
        }
        pos = q.ctx + depth;
      }
    }
    p.slots[t] = slot;
    p.positions[t] = pos;
#pragma unroll
    for (int w = 0; w < CACHE_MAX_WORDS; ++w)
      if (w < p.words) p.mask[(int64_t)t * p.words + w] = m[w];
  }
}
// parents as they are laid in LDS: what no tree with masks can hold is no parent
__device__ __forceinline__ int16_t short_parent(int x) { return x < 0 || x >= PLAN_MAX_TREE ? -1 : (int16_t)x; }

// each: tokens of a workgroup, at most PLAN_ONE_LAUNCH; 0: the tokens are another launch's
__global__ __launch_bounds__(PLAN_THREADS) void plan_kernel(PlanParams p, int each) {
  __shared__ uint64_t room[4][PLAN_WAVES];
  __shared__ int16_t up[PLAN_MAX_TREE + PLAN_ONE_LAUNCH];
  __shared__ int32_t starts[PLAN_THREADS + 1];
  __shared__ PlanRequest requests[PLAN_THREADS];
  const int tid = threadIdx.x;
  const bool lead = blockIdx.x == 0;
  const int t0 = (int)blockIdx.x * each, t1 = min(p.max_tokens, t0 + each), up0 = max(0, t0 - PLAN_MAX_TREE);
  if (each && p.parents && p.words)
    for (int t = up0 + tid; t < t1; t += PLAN_THREADS) up[t - up0] = short_parent(p.parents[t]);
  if (tid == 0) starts[0] = 0;
  if (each && p.n <= PLAN_THREADS) {
    const int n_free = plan_requests(p, lead, room, [&](int r, int start, const PlanRequest &q) {
      starts[r + 1] = start;
      requests[r] = q;
    });
    __syncthreads();
    plan_tokens(p, n_free, t0, t1, PLAN_THREADS, [&](int r) { return starts[r]; }, [&](int r) { return requests[r]; }, up, up0);
    return;
  }
  const int n_free = plan_requests(p, lead, room, [&](int r, int, const PlanRequest &q) {
    p.old_held[r] = q.held;
    p.page_start[r] = q.page_start;
  });
  if (!each) return;
  __syncthreads();
  plan_tokens(p, n_free, t0, t1, PLAN_THREADS, [&](int r) { return p.tok_start[r]; },
              [&](int r) { return PlanRequest{p.ctx[r], p.old_held[r], p.page_start[r], 0}; }, up, up0);
}

__global__ __launch_bounds__(PLAN_PART_THREADS) void plan_tokens_kernel(PlanParams p) {
  __shared__ int16_t up[PLAN_PART_THREADS + PLAN_MAX_TREE];
  const int t0 = blockIdx.x * PLAN_PART_THREADS, t1 = min(p.max_tokens, t0 + PLAN_PART_THREADS), up0 = max(0, t0 - PLAN_MAX_TREE);
  if (p.parents && p.words) {
    for (int t = up0 + (int)threadIdx.x; t < t1; t += PLAN_PART_THREADS) up[t - up0] = short_parent(p.parents[t]);
    __syncthreads();
  }
  plan_tokens(p, p.free_count[0], t0, t1, PLAN_PART_THREADS, [&](int r) { return p.tok_start[r]; },
              [&](int r) { return PlanRequest{p.ctx[r], p.old_held[r], p.page_start[r], 0}; }, up, up0);
}

}  // namespace

#endif
