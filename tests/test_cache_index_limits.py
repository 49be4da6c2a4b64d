"""The paged cache's index arithmetic at the ends of its envelope, on the CPU with undefined behaviour an error."""
from tests.test_cache_index import _run


def test_chunks_cover_the_keys_of_the_longest_requests(tmp_path):
    """Chunk after chunk without a gap up to the request's last key, with block tables as wide as 32 bits allow."""
    _run(tmp_path, """
      for (int hk : {1, 2, 8, 64, 1024})
        for (int64_t most : {2147479551ll, 2147479551ll - 127, 1ll << 30, 40000ll})   // max_pages * page_size
          for (int64_t keys : {most, most - 1, most / 2 + 1, most / 3})
            for (int64_t rows : {1, 16, 64, 65, 192, 193, 256, 512, 513, 1024, 2048, 65536, 1 << 20}) {
              if (rows > keys) continue;
              const CacheShare s = cache_share(0, (int32_t)rows, (int32_t)keys, (int32_t)rows, (int32_t)most, 1, 64, hk, cache_many_split(hk));
              if (s.keys != keys || s.rows != rows) return 1;
              int64_t at = 0;
              for (int c = 0; c < s.chunks; ++c) {
                const CacheKeys k = cache_chunk_keys(s, c);
                if (k.begin != at || k.end <= k.begin || k.begin % CACHE_UNIT) { std::printf("rows %lld chunk %d of %d: %d .. %d\\n", (long long)rows, c, s.chunks, k.begin, k.end); return 2; }
                at = k.end;
              }
              if (at != keys) { std::printf("hk %d rows %lld keys %lld: covered to %lld\\n", hk, (long long)rows, (long long)keys, (long long)at); return 3; }
            }""")


def test_units_of_a_chunk_against_64_bits(tmp_path):
    """The rule's product passes 32 bits only where its lower bound alone makes one chunk."""
    _run(tmp_path, """
      for (uint32_t hk : {1u, 2u, 4u, 16u, 40u, 1024u})
        for (uint32_t rows = 1; rows && (uint64_t)rows * hk <= 0x7fffffffu; rows = rows * 2 + (rows >> 3))
          for (uint32_t units : {1u, 2u, 15u, 16u, 127u, 128u, 1000u, 1024u, 2047u, 2048u, 100000u, 16777183u}) {
            const uint64_t n = rows > 64 && (rows + 63) / 64 >= 4 ? cache_many_split((int32_t)hk) : CACHE_FEW_SPLIT;
            const uint64_t t = rows > 64 ? (rows + 63) / 64 : 1, most = 8 * t;
            uint64_t least = t < 4 ? 2 * t : t * hk / 8, want = most;
            least = least < 2 ? 2 : least > most ? most : least;
            if (units < 8 * n) {
              want = (units * t + n - 1) / n;
              want = want < least ? least : want;
            }
            const uint32_t u = cache_chunk_units(units, rows, hk, (uint32_t)cache_many_split((int32_t)hk));
            if (u < 1 || (units + (uint64_t)u - 1) / u != (units + want - 1) / want) { std::printf("rows %u units %u hk %u: %u %llu\\n", rows, units, hk, u, (unsigned long long)want); return 1; }
          }""")
