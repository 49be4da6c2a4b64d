"""Index arithmetic of the paged cache on the CPU: the plain C++ of csrc/cache_index.h compiled with g++, undefined behaviour an
error, against loops that say the same the long way."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2505_19578_amd", "csrc")


def _run(tmp_path, body):
    src, exe = tmp_path / "t.cc", tmp_path / "t"
    src.write_text('#include "cache_index.h"\n#include <cstdio>\n#include <cstdlib>\n#include <initializer_list>\n'
                   "int main() {\n" + body + "\nreturn 0;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I" + CSRC, str(src), "-o", str(exe)], check=True, timeout=120)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stderr + r.stdout)


@pytest.mark.parametrize("words", [0, 1, 2, 4])
def test_visible_keys_of_a_step(tmp_path, words):
    """Every step around the border of context and new tokens, at every border position, against a test per key."""
    _run(tmp_path, f"""
      const int words = {words};
      srand(7);
      for (int fresh : {{1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 256}}) {{
        if (words && fresh > 64 * words) continue;
        uint64_t mask[4] = {{0, 0, 0, 0}};
        for (int w = 0; w < words; ++w) mask[w] = (uint64_t)rand() << 42 ^ (uint64_t)rand() << 21 ^ (uint64_t)rand();
        for (int ctx : {{0, 1, 15, 31, 32, 33, 64, 100, 2147400000}})
          for (int i : {{0, 1, fresh / 2, fresh - 1}}) {{
            if (i >= fresh) continue;
            const int64_t from = ctx / 32 * 32 - 64;
            for (int64_t kb = from < 0 ? 0 : from; kb <= (int64_t)ctx + fresh + 64; kb += 32) {{
              const uint32_t got = words ? cache_visible_words(kb, ctx, fresh, mask, words) : cache_visible_chain(kb, ctx, fresh, i);
              if (words == 1 && got != cache_visible_word(kb, ctx, fresh, mask[0])) return 2;
              for (int b = 0; b < 32; ++b) {{
                const int64_t j = kb + b - ctx;
                const bool want = j < 0 || (j < fresh && (words ? (mask[j / 64] >> (j % 64)) & 1 : j <= i));
                if (((got >> b) & 1) != want) {{ std::printf("fresh %d ctx %d i %d kb %lld b %d\\n", fresh, ctx, i, (long long)kb, b); return 1; }}
              }}
            }}
          }}
      }}""")


def test_shares_stay_inside_their_bounds(tmp_path):
    """Chunks cover the keys and do not overlap; a call's partial rows and workgroups stay below what its workspace and grid are
    sized for, whatever the lengths are."""
    _run(tmp_path, """
      srand(11);
      for (int round = 0; round < 20000; ++round) {
        const int heads[] = {1, 2, 3, 4, 8, 16, 40, 1024};
        const int group = 1 + rand() % 16, n = 1 + rand() % 9, hk = heads[rand() % 8], split = cache_many_split(hk);
        const int64_t page = 16 << (rand() % 5), most = page * (1 + rand() % (rand() % 2 ? 9000 : 60));
        int64_t start[10] = {0}, keys[9];
        for (int r = 0; r < n; ++r) {
          start[r + 1] = start[r] + (round % 4 == 0 ? (193 + rand() % 70) / group : rand() % 3 ? rand() % 5 : rand() % 300);
          keys[r] = rand() % 7 ? (int64_t)rand() % (most + 1) : most;
        }
        const int64_t tokens = start[n];
        if (!tokens) continue;
        for (int tile : {16, 32, 64, 128, 192}) {
          int64_t rows = 0, items = 0;
          for (int r = 0; r < n; ++r) {
            const CacheShare s = cache_share(start[r], start[r + 1], keys[r], tokens, most, group, tile, hk, split);
            if (s.chunks < 1 || s.units < 1 || s.keys > most) return 2;
            const int per = (s.units + s.chunks - 1) / s.chunks;
            if ((int64_t)per * s.chunks < s.units || (int64_t)per * CACHE_UNIT * s.chunks < s.keys) return 3;
            if (s.tiles && s.chunks > cache_most_chunks(most, s.rows < 193 ? CACHE_FEW_SPLIT : split) / ((s.rows + 63) / 64) + 1) return 4;
            if (!cache_any_chunks(most) && s.chunks > 1) return 5;
            if (s.chunks > 1) rows += (int64_t)s.rows * s.chunks;
            items += (int64_t)s.tiles * s.chunks;
          }
          if (rows > cache_partial_rows(n, tokens, group, most, hk)) { std::printf("rows %lld\\n", (long long)rows); return 6; }
          if (items > cache_grid(n, tokens, group, most, tile, hk)) { std::printf("items %lld tile %d\\n", (long long)items, tile); return 7; }
        }
      }""")


def test_a_share_of_anything_is_a_share_of_what_exists(tmp_path):
    _run(tmp_path, """
      const int64_t wild[] = {-2147483647 - 1, -1, 0, 1, 7, 100, 2147483647};
      for (int64_t a : wild) for (int64_t b : wild) for (int64_t keys : wild) {
        const CacheShare s = cache_share(a, b, keys, 50, 4096, 8, 64, 4, cache_many_split(4));
        if (s.first < 0 || s.fresh < 0 || (s.fresh && s.first + s.fresh > 50) || s.keys < 0 || s.keys > 4096) return 1;
        if (s.keys && s.keys < s.fresh) return 2;
      }""")


@pytest.mark.parametrize("tiles", [1, 2, 5])
def test_places_of_workgroups(tmp_path, tiles):
    """Every (pair, tile) has one place, and tiles of a pair among eight pairs lie eight apart."""
    _run(tmp_path, f"""
      const int tiles = {tiles};
      for (int pairs : {{1, 2, 7, 8, 9, 16, 23, 128}}) {{
        static bool seen[1 << 12];
        for (bool &x : seen) x = false;
        for (int n = 0; n < pairs * tiles; ++n) {{
          const CachePlace at = cache_place(n, pairs, tiles);
          if (at.pair < 0 || at.pair >= pairs || at.tile < 0 || at.tile >= tiles || seen[at.pair * tiles + at.tile]) return 1;
          seen[at.pair * tiles + at.tile] = true;
          if (at.pair / 8 * 8 + 8 <= pairs && (n - at.pair) % 8) return 3;
        }}
      }}""")


def test_slots_and_pages(tmp_path):
    _run(tmp_path, """
      if (cache_slot(-1, 16, 3) != -1 || cache_slot(5, 16, 3) != 83) return 1;
      if (cache_slot(2147483647, 16, 0) != -1 || cache_slot(134217727, 16, 15) != 2147483647 || cache_slot(134217728, 16, 0) != -1) return 2;
      if (plan_lacking(0, 0, 16) || plan_lacking(1, 0, 16) != 1 || plan_lacking(16, 1, 16) || plan_lacking(17, 1, 16) != 1 || plan_lacking(17, 9, 16)) return 3;
      if (plan_length_status(0, -1, 0, 4, 16, 99) != PLAN_BAD_LENGTH || plan_length_status(-1, 0, 0, 4, 16, 99) != PLAN_BAD_LENGTH) return 4;
      if (plan_length_status(17, 0, 1, 4, 16, 99) != PLAN_BAD_LENGTH || plan_length_status(0, 0, 5, 4, 16, 99) != PLAN_BAD_LENGTH) return 5;
      if (plan_length_status(60, 5, 4, 4, 16, 99) != PLAN_TOO_LONG || plan_length_status(60, 4, 4, 4, 16, 99) != PLAN_OK) return 6;
      if (plan_length_status(2147483647, 2147483647, 2147483647, 2147483647, 1, 2147483647) != PLAN_TOO_LONG) return 7;""")
