// Index arithmetic of the paged key/value cache: what a step sees of a page, of a drafted tree and of the split of long contexts.
// Plain C++ (constexpr functions also run on the device), so that a test can compile it for the CPU.
#ifndef SP_CACHE_INDEX_H
#define SP_CACHE_INDEX_H
#include <cstddef>
#include <cstdint>

constexpr int CACHE_MAX_WORDS = 4;        // mask words of a drafted token
constexpr int CACHE_MIN_PAGE = 16, CACHE_MAX_PAGE = 4096;
constexpr int CACHE_STEP = 32;            // keys of a wavefront's step
constexpr int CACHE_UNIT = 4 * CACHE_STEP;  // keys that the four wavefronts of a workgroup take at once

// Refusals of sp_cache_plan, in the order in which they are tested.
enum CachePlanStatus { PLAN_OK = 0, PLAN_BAD_LENGTH = 1, PLAN_TOO_LONG = 2, PLAN_NO_ROOM = 3, PLAN_NO_PAGES = 4 };

// What the lengths of one request alone say.  `width` pages of `page` tokens a row, at most `most` new tokens.
constexpr int plan_length_status(int64_t ctx, int64_t fresh, int64_t held, int64_t width, int64_t page, int64_t most) {
  if (fresh < 0 || ctx < 0 || held < 0 || held > width || held * page < ctx) return PLAN_BAD_LENGTH;
  if (ctx + fresh > width * page || fresh > most) return PLAN_TOO_LONG;
  return PLAN_OK;
}
// Pages a request lacks for `tokens` tokens when it holds `held`.
constexpr int64_t plan_lacking(int64_t tokens, int64_t held, int64_t page) {
  const int64_t need = (tokens + page - 1) / page;
  return need > held ? need - held : 0;
}
// The slot of position `offset` of page `page_id`, -1 where there is none that 32 bits hold.
constexpr int32_t cache_slot(int64_t page_id, int64_t page, int64_t offset) {
  const int64_t s = page_id * page + offset;
  return page_id < 0 || s > 0x7fffffff ? -1 : (int32_t)s;
}

// Keys kb .. kb + 31 that a new token of a request sees, as bits.  The request has `ctx` tokens in the cache before its `fresh`
// new ones; new token j lies at position ctx + j.  kb may lie anywhere, also behind the last key.
//
// `seen`: bits of new tokens kb - ctx, .. that it sees (of those before the context's end, none count)
constexpr uint32_t cache_with_context(uint64_t seen, int64_t kb, int64_t ctx) {
  const int64_t before = ctx - kb;  // keys from kb on that lie in the context
  const uint64_t old = before <= 0 ? 0 : before >= 32 ? 0xffffffffu : (1ull << before) - 1;
  return (uint32_t)((seen & ~old) | old);
}
constexpr uint64_t cache_low_bits(int64_t n) { return n <= 0 ? 0 : n >= 32 ? 0xffffffffu : (1ull << n) - 1; }
// New token i of a chain sees tokens 0 .. i.
constexpr uint32_t cache_visible_chain(int64_t kb, int64_t ctx, int fresh, int i) {
  const int64_t last = i < fresh ? i : fresh - 1;  // the last new token that is seen
  return cache_with_context(cache_low_bits(last - (kb - ctx) + 1), kb, ctx);
}
// One mask word: bit j says whether the token sees new token j.
constexpr uint32_t cache_visible_word(int64_t kb, int64_t ctx, int fresh, uint64_t word) {
  const int64_t j0 = kb - ctx;
  uint64_t seen = j0 >= 64 || j0 <= -32 ? 0 : j0 >= 0 ? word >> j0 : word << -j0;
  seen &= cache_low_bits(fresh - j0);  // keys from kb on that exist
  return cache_with_context(seen, kb, ctx);
}
// Several: bit j % 64 of word j / 64.
constexpr uint32_t cache_visible_words(int64_t kb, int64_t ctx, int fresh, const uint64_t *mask, int words) {
  const int64_t j0 = kb - ctx;
  uint64_t seen = 0;
  if (j0 < 64 * (int64_t)words && j0 > -32) {
    if (j0 >= 0) {
      const int w = (int)(j0 >> 6), sh = (int)(j0 & 63);
      seen = mask[w] >> sh;
      if (sh && w + 1 < words) seen |= mask[w + 1] << (64 - sh);
    } else {
      seen = mask[0] << -j0;
    }
    seen &= cache_low_bits(fresh - j0);
  }
  return cache_with_context(seen, kb, ctx);
}

// One request's share of an attention call: `rows` query rows per KV head in `tiles` tiles, `units` of CACHE_UNIT keys in
// `chunks` chunks.
struct CacheShare {
  int32_t first, fresh, keys, rows, tiles, units, chunks;
};
// Units of a chunk.  It goes by the request's own sizes and the cache's heads alone, so that a request's result is the same bits
// whatever else the call holds.  t = rows / 64 counts the rows; a chunk takes 2 units and more, as its partial results are written
// and read, 1 KiB a row, next to 64 KiB of keys and values a unit, and at most 8 t, so that a long context makes more chunks still.
//   up to 192 rows   about 16 / t chunks of at least 2 t units
//   more             a KV head has work for many workgroups, and a chunk's own costs are small next to it: 256 / t chunks over all KV
//                    heads (at least 16 / t a head), of at least t hk / 8 units.  Against the rule above, 32 query heads: one request
//                    of 64 tokens over 8000 under 4 KV heads 43 us and 109, four 66 and 115, eight 130 and 134, sixteen 239 and 197;
//                    of 56 tokens under 8 KV heads 45 and 66, 70 and 79, 135 and 123, 258 and 234.  Batches that fill
//                    the chip lose, most where contexts are short: sixteen of 64 tokens over 1200 under 4 KV heads 88 and 57.  (From 65
//                    rows on: 12 requests of 21 tokens over 6150, 28 query and 4 KV heads, 90 and 73, one 33 and 45.)
constexpr uint32_t CACHE_FEW_SPLIT = 16;
constexpr int32_t cache_many_split(int32_t hk) { return 256 / hk > (int32_t)CACHE_FEW_SPLIT ? 256 / hk : (int32_t)CACHE_FEW_SPLIT; }
constexpr uint32_t cache_chunk_units(uint32_t units, uint32_t rows, uint32_t hk, uint32_t many_split) {
  const uint32_t t = rows > 64 ? (rows + 63) / 64 : 1, n = t < 4 ? CACHE_FEW_SPLIT : many_split, most = 8 * t;
  // (32 bits hold the product below up to t = 2^21; from there on `least` exceeds the units, of which there are fewer than 2048: one chunk)
  if (units >= 8 * n) return most;
  uint32_t least = t < 4 ? 2 * t : t * hk / 8;
  least = least < 2 ? 2 : least > most ? most : least;
  const uint32_t u = (units * t + n - 1) / n;
  return u < least ? least : u;
}
// Tokens and keys come from device memory: whatever is in it, a share is a share of rows and keys that exist.
constexpr CacheShare cache_share(int32_t first, int32_t end, int32_t keys, int32_t n_tokens, int32_t most_keys, int32_t group,
                                 int32_t tile_rows, int32_t hk, int32_t many_split) {
  if (first < 0) first = 0;
  if (end > n_tokens) end = n_tokens;
  const int32_t fresh = end > first ? end - first : 0;
  if (keys > most_keys) keys = most_keys;
  if (keys < fresh) keys = 0;  // a request that the plan refused: no keys, its rows become zeros
  CacheShare s{};
  s.first = first, s.fresh = fresh, s.keys = keys;
  s.rows = fresh * group;  // (32 bits hold n_tokens * group)
  s.tiles = (int32_t)(((uint32_t)s.rows + tile_rows - 1) / (uint32_t)tile_rows);
  s.units = keys > 0 ? (int32_t)(((uint32_t)keys + CACHE_UNIT - 1) / CACHE_UNIT) : 1;
  const uint32_t u = cache_chunk_units((uint32_t)s.units, (uint32_t)s.rows, (uint32_t)hk, (uint32_t)many_split);
  s.chunks = (int32_t)(((uint32_t)s.units + u - 1) / u);
  return s;
}
// Keys of a chunk: as many units for each, and the last one ends with the request.
struct CacheKeys {
  int32_t begin, end;
};
constexpr CacheKeys cache_chunk_keys(const CacheShare &s, int32_t chunk) {
  const int32_t per = (int32_t)((uint32_t)(s.units + s.chunks - 1) / (uint32_t)s.chunks);
  const int32_t begin = chunk * per * CACHE_UNIT, left = s.keys - begin;  // (the last chunk's units may end behind what 32 bits number)
  return CacheKeys{begin, begin + (left < per * CACHE_UNIT ? left : per * CACHE_UNIT)};
}
// Upper bounds of what all requests of a call add up to, per KV head; the kernels' sums never pass them.
// chunks <= most / t + 1 with t = ceil(rows / 64) and `most` as follows; from 193 rows on with the larger split
constexpr int64_t cache_most_chunks(int64_t most_keys, int64_t split) {
  const int64_t units = (most_keys + CACHE_UNIT - 1) / CACHE_UNIT;
  return units <= 2 ? 1 : (units + 7) / 8 > split ? (units + 7) / 8 : split;
}
constexpr bool cache_any_chunks(int64_t most_keys) { return cache_most_chunks(most_keys, CACHE_FEW_SPLIT) > 1; }
// what the requests of 193 rows and more add to a bound with the smaller split: how many there can be, times the difference
constexpr int64_t cache_many_extra(int64_t n_requests, int64_t rows, int64_t most_keys, int hk) {
  const int64_t many = rows / 193 < n_requests ? rows / 193 : n_requests;
  return many * (cache_most_chunks(most_keys, cache_many_split(hk)) - cache_most_chunks(most_keys, CACHE_FEW_SPLIT));
}
// rows of partial results: rows * chunks
constexpr int64_t cache_partial_rows(int64_t n_requests, int64_t n_tokens, int group, int64_t most_keys, int hk) {
  if (!cache_any_chunks(most_keys)) return 0;
  const int64_t rows = n_tokens * group, wide = rows < 64 * n_requests ? rows : 64 * n_requests;
  return wide * cache_most_chunks(most_keys, CACHE_FEW_SPLIT) + 64 * cache_many_extra(n_requests, rows, most_keys, hk) + rows;
}
// workgroups: tiles * chunks
constexpr int64_t cache_grid(int64_t n_requests, int64_t n_tokens, int group, int64_t most_keys, int tile_rows, int hk) {
  const int64_t live = n_requests < n_tokens ? n_requests : n_tokens, rows = n_tokens * group;
  const int64_t tiles = rows / tile_rows + live, per = tile_rows < 64 ? 64 / tile_rows : 1;
  const int64_t wide = tiles < per * live ? tiles : per * live;
  return wide * cache_most_chunks(most_keys, CACHE_FEW_SPLIT) + per * cache_many_extra(n_requests, rows, most_keys, hk) + tiles;
}

// Place of a workgroup among a request's: `pairs` pairs (chunk, KV head), KV head first, times `tiles`.  Workgroups go round-robin
// to the 8 XCDs, so pairs are taken eight at a time and the tiles of a pair, which read the same keys, lie eight apart: one L2.
struct CachePlace {
  int32_t pair, tile;
};
constexpr CachePlace cache_place(uint32_t index, uint32_t pairs, uint32_t tiles) {
  if (tiles == 1) return CachePlace{(int32_t)index, 0};
  const uint32_t eight = index / (8 * tiles), rest = index - eight * 8 * tiles;
  const uint32_t wide = pairs - 8 * eight < 8 ? pairs - 8 * eight : 8;
  if (wide == 8) return CachePlace{(int32_t)(8 * eight + rest % 8), (int32_t)(rest / 8)};
  return CachePlace{(int32_t)(8 * eight + rest % wide), (int32_t)(rest / wide)};
}
#endif
