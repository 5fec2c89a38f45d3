// How attention over the cache splits its work (plan_cache_attend), on the host: a batch a
// line on standard input, its plan a line on standard output (tests/test_cache_plan.py).
#include <stdio.h>

#include "sp_internal.h"

int main() {
  sp::CacheShape s{};
  sp::CacheRows rows{};
  sp::CacheRuns runs{}, prefix{};
  long long n;
  s.page_shift = 6;
  s.pages = 1 << 20;
  while (scanf("%d %d %d %d %lld %d %d %d %d %d", &s.dtype, &s.q_heads, &s.kv_heads, &s.head_dim, &n, &rows.max_rows,
               &runs.count, &runs.max_len, &prefix.count, &prefix.max_len) == 10) {
    rows.rows = n;
    const sp::AttendPlan p = sp::plan_cache_attend(s, rows, runs, prefix);
    printf("alone %d wide %d spread %d prefix_parts %d short_parts %d chunk_thin %d tall_parts %d chunk_tall %d tall_tiles %d tall_blocks %lld\n",
           p.alone, p.wide, p.spread, p.prefix_parts, p.short_parts, p.chunk_thin, p.tall_parts, p.chunk_tall, p.tall_tiles,
           (long long)p.tall_blocks);
  }
  return 0;
}
