// Accepted drafted tokens close up behind the context.
#ifndef SP_CACHE_ACCEPT_KERNEL_H
#define SP_CACHE_ACCEPT_KERNEL_H
#include "cache_common.h"

namespace {

// Row ctx + i of a request takes row ctx + path[i], i = 0, 1, ..; path ascends, so path[i] >= i, and the rows that move i
// reads lie at or behind the one it writes.  Row ctx + i may itself be the source of a move before i only, so a column's owner that
// loads a run of sources before it stores the run keeps the order of the definition, and runs follow one another.
// A thread owns 16 bytes of the row (K and V of every KV head of one layer) through all moves of a request: no two threads meet.
// Bound by latency for few layers (table, then sources), by HBM for many: one request's 5 rows in 32 layers 4.9 us, 48 requests' up to
// 8 rows in 16 layers of 8 heads 11.9 us.
constexpr int ACCEPT_THREADS = 256, ACCEPT_RUN = 8, ACCEPT_MAX = 256;

struct AcceptParams {
  uint16_t *k, *v;
  const int32_t *table, *ctx, *seq, *path, *count;
  int32_t *ctx_out;
  int64_t c_sl, c_sp, c_st, c_sh;
  int n_pages, page_shift, width, max_accept, hk, d8;  // d8: pieces of 16 bytes in a head
};

__global__ __launch_bounds__(ACCEPT_THREADS) void cache_accept_kernel(AcceptParams p) {
  __shared__ int32_t path[ACCEPT_MAX];
  __shared__ int32_t found;
  const int r = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x;
  const int ctx = p.ctx[r];
  // the path ends at the first entry that does not ascend or is no new token of the request
  if (tid < 64) {
    const int seq = p.seq[r], fresh = ctx < 0 || seq < ctx ? 0 : seq - ctx;
    int n = p.count[r], prev = -1;
    n = n < 0 ? 0 : n > p.max_accept ? p.max_accept : n;
    int len = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const int i = i0 + tid, x = i < n ? p.path[(int64_t)r * p.max_accept + i] : -1;
      int before = __shfl_up(x, 1);
      if (tid == 0) before = prev;
      const bool fine = i < n && x > before && x < fresh;
      const uint64_t bad = ~__builtin_amdgcn_ballot_w64(fine);
      const int run = bad ? __builtin_ctzll(bad) : 64;
      if (i < ACCEPT_MAX) path[i] = x;
      len += run;
      prev = __shfl(x, 63);
      if (run < 64) break;
    }
    if (tid == 0) {
      found = len;
      if (p.ctx_out && layer == 0 && blockIdx.z == 0) p.ctx_out[r] = ctx + len;
    }
  }
  __syncthreads();
  const int n = found;
  const int piece = blockIdx.z * ACCEPT_THREADS + tid, half = p.hk * p.d8;
  if (piece >= 2 * half) return;
  const int x = piece < half ? piece : piece - half, h = x / p.d8, e = x - h * p.d8;
  uint16_t *base = (piece < half ? p.k : p.v) + layer * p.c_sl + h * p.c_sh + 8 * e;
  const int32_t *row = p.table + (int64_t)r * p.width;
  auto place = [&](int64_t pos) -> uint16_t * {
    const int64_t entry = pos >> p.page_shift;
    if (entry >= p.width) return nullptr;
    const int id = row[entry];
    if (id < 0 || id >= p.n_pages) return nullptr;
    return base + (int64_t)id * p.c_sp + (pos & ((1 << p.page_shift) - 1)) * p.c_st;
  };
  for (int i0 = 0; i0 < n; i0 += ACCEPT_RUN) {
    u32x4 val[ACCEPT_RUN];
    uint16_t *to[ACCEPT_RUN];
#pragma unroll
    for (int e2 = 0; e2 < ACCEPT_RUN; ++e2) {
      const int i = i0 + e2;
      to[e2] = nullptr;
      if (i < n && path[i] != i) {
        const uint16_t *from = place((int64_t)ctx + path[i]);
        to[e2] = place((int64_t)ctx + i);
        if (!from) to[e2] = nullptr;
        if (to[e2]) val[e2] = *(const u32x4 *)from;
      }
    }
#pragma unroll
    for (int e2 = 0; e2 < ACCEPT_RUN; ++e2)
      if (to[e2]) *(u32x4 *)to[e2] = val[e2];
  }
}

}  // namespace

#endif
