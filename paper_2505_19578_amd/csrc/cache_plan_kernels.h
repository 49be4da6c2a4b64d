// The plan of a step over the paged cache: which pages the new tokens get, where each of them goes, what a drafted one sees.
#ifndef SP_CACHE_PLAN_KERNELS_H
#define SP_CACHE_PLAN_KERNELS_H
#include "cache_common.h"

namespace {

// Two parts.  plan_requests: one workgroup walks the requests in order (two prefix sums: tokens, then pages of the requests
// that are not refused) and writes what there is one of per request.  plan_tokens: every new token finds its request by
// bisection in tok_start and writes its slot; the token that opens a fresh page also writes that page into the request's row.
// Page entries that are read are those the request held before, the ones that are written come after them, so tokens need no
// order among each other.  A wavefront per request walks the drafted trees.
// Bound by latency: a few dependent loads and two scans.  Up to SP_PLAN_ONE_LAUNCH tokens one workgroup does both parts in one
// launch; beyond, the second part is spread over the chip.
constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64;
constexpr int PLAN_PART_THREADS = 256;          // of the second part's own launch
constexpr int PLAN_MAX_TREE = 64 * CACHE_MAX_WORDS;

struct PlanParams {
  const int32_t *ctx, *fresh, *held, *free_pages, *n_free, *parents;
  int32_t *table, *held_out, *n_free_out, *tok_start, *seq_len, *positions, *slots, *status;
  uint64_t *mask;
  int32_t *old_held, *page_start;  // workspace: [n] each
  int32_t *free_count;             // workspace: [1], pages that were free before the call
  int n, max_tokens, page, width, words, free_capacity;
};

__device__ __forceinline__ int64_t wave_scan(int64_t x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// inclusive prefix sum over the workgroup; `total` gets the sum of all
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t *room, int64_t &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  x = wave_scan(x, lane);
  __syncthreads();
  if (lane == 63) room[w] = x;
  __syncthreads();
  const int64_t y = wave_scan(lane < PLAN_WAVES ? room[lane] : 0, lane);
  total = __shfl(y, PLAN_WAVES - 1);
  const int64_t before = __shfl(y, w > 0 ? w - 1 : 0);
  return w > 0 ? x + before : x;
}

__device__ void plan_requests(const PlanParams &p, int64_t *room) {
  int64_t tokens = 0, pages = 0, taken = 0;  // before this round's requests
  int n_free = p.n_free[0];
  n_free = n_free < 0 ? 0 : n_free > p.free_capacity ? p.free_capacity : n_free;
  const int64_t most = p.words ? 64 * p.words : 0x7fffffff;
  for (int r0 = 0; r0 < p.n; r0 += PLAN_THREADS) {
    const int r = r0 + threadIdx.x;
    const bool live = r < p.n;
    const int ctx = live ? p.ctx[r] : 0, fresh = live ? p.fresh[r] : 0, held = live ? p.held[r] : 0;
    int64_t total;
    const int64_t end = tokens + block_scan(fresh > 0 ? fresh : 0, room, total);
    tokens += total;
    int st = plan_length_status(ctx, fresh, held, p.width, p.page, most);
    if (st == PLAN_OK && end > p.max_tokens) st = PLAN_NO_ROOM;
    const int64_t lack = live && st == PLAN_OK ? plan_lacking((int64_t)ctx + fresh, held, p.page) : 0;
    const int64_t last = pages + block_scan(lack, room, total);
    pages += total;
    if (st == PLAN_OK && lack > 0 && last > n_free) st = PLAN_NO_PAGES;
    const bool ok = st == PLAN_OK;
    (void)block_scan(ok ? lack : 0, room, total);
    taken += total;
    if (live) {
      p.tok_start[r + 1] = (int)(end < p.max_tokens ? end : p.max_tokens);
      p.seq_len[r] = ok ? ctx + fresh : 0;
      p.status[r] = st;
      p.old_held[r] = held;
      p.page_start[r] = (int)(last - lack);
      p.held_out[r] = ok ? held + (int)lack : held;
    }
  }
  if (threadIdx.x == 0) {
    p.tok_start[0] = 0;
    p.free_count[0] = n_free;
    p.n_free_out[0] = n_free - (int)taken;
  }
}

// slots (and, where no tree says otherwise, positions and chain masks) of tokens t0, t0 + stride, ..
__device__ void plan_tokens(const PlanParams &p, int t0, int stride) {
  const int n_free = p.free_count[0], used = p.tok_start[p.n];
  for (int t = t0; t < p.max_tokens; t += stride) {
    int slot = -1, pos = 0, i = 0;
    bool ok = false;
    if (t < used) {
      int lo = 0, hi = p.n - 1;  // the first request whose tokens end behind t
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.tok_start[mid + 1] > t)
          hi = mid;
        else
          lo = mid + 1;
      }
      const int r = lo;
      ok = p.status[r] == PLAN_OK;
      if (ok) {
        i = t - p.tok_start[r];
        pos = p.ctx[r] + i;
        const int entry = pos / p.page, off = pos - entry * p.page, held = p.old_held[r];
        int64_t at = (int64_t)r * p.width + entry;
        int id;
        if (entry < held) {
          id = p.table[at];
        } else {
          id = p.free_pages[n_free - 1 - (p.page_start[r] + entry - held)];
          if (off == 0) p.table[at] = id;
        }
        slot = cache_slot(id, p.page, off);
      }
    }
    p.slots[t] = slot;
    if (!p.parents || !ok) p.positions[t] = pos;
    if (p.words && (!p.parents || !ok))
      for (int w = 0; w < p.words; ++w) {
        const int n = i - 64 * w;  // bits 0 .. i
        p.mask[(int64_t)t * p.words + w] = !ok || n < 0 ? 0ull : n >= 63 ? ~0ull : (2ull << n) - 1;
      }
  }
}

// depth and ancestors of one request's drafted tokens, by one wavefront.  `up`: PLAN_MAX_TREE ints of its own in LDS.
__device__ void plan_tree(const PlanParams &p, int r, int32_t *up) {
  const int lane = threadIdx.x & 63;
  if (p.status[r] != PLAN_OK) return;
  const int first = p.tok_start[r], n = p.tok_start[r + 1] - first, ctx = p.ctx[r];
  for (int i = lane; i < n && i < PLAN_MAX_TREE; i += 64) {
    const int q = p.parents[first + i];
    up[i] = q < 0 || q >= i ? -1 : q;  // no earlier token of the request: a root
  }
  __builtin_amdgcn_wave_barrier();
  for (int i = lane; i < n; i += 64) {
    if (!p.words) {  // positions alone: a tree of any size, by its own memory
      int depth = 0;
      for (int q = i; (q = [&](int x) { const int y = p.parents[first + x]; return y < 0 || y >= x ? -1 : y; }(q)) >= 0;) ++depth;
      p.positions[first + i] = ctx + depth;
      continue;
    }
    uint64_t m[CACHE_MAX_WORDS] = {0, 0, 0, 0};
    int depth = -1;
    for (int q = i; q >= 0; q = up[q]) {
#pragma unroll
      for (int w = 0; w < CACHE_MAX_WORDS; ++w) m[w] |= (q >> 6) == w ? 1ull << (q & 63) : 0ull;
      ++depth;
    }
    p.positions[first + i] = ctx + depth;
#pragma unroll
    for (int w = 0; w < CACHE_MAX_WORDS; ++w)
      if (w < p.words) p.mask[(int64_t)(first + i) * p.words + w] = m[w];
  }
  __builtin_amdgcn_wave_barrier();
}

__global__ __launch_bounds__(PLAN_THREADS) void plan_kernel(PlanParams p, int with_tokens) {
  __shared__ int64_t room[PLAN_WAVES];
  __shared__ int32_t up[PLAN_WAVES][PLAN_MAX_TREE];
  plan_requests(p, room);
  if (!with_tokens) return;
  __syncthreads();
  plan_tokens(p, threadIdx.x, PLAN_THREADS);
  if (p.parents)
    for (int r = threadIdx.x >> 6; r < p.n; r += PLAN_WAVES) plan_tree(p, r, up[threadIdx.x >> 6]);
}

__global__ __launch_bounds__(PLAN_PART_THREADS) void plan_tokens_kernel(PlanParams p, int token_blocks) {
  __shared__ int32_t up[PLAN_PART_THREADS / 64][PLAN_MAX_TREE];
  const int b = blockIdx.x, w = threadIdx.x >> 6;
  if (b < token_blocks) {
    plan_tokens(p, b * PLAN_PART_THREADS + threadIdx.x, token_blocks * PLAN_PART_THREADS);
  } else {
    const int r = (b - token_blocks) * (PLAN_PART_THREADS / 64) + w;
    if (r < p.n) plan_tree(p, r, up[w]);
  }
}

}  // namespace

#endif
