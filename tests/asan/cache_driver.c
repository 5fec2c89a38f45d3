/*
 * Host driver for the sanitizer build of the cache's calls
 * (tests/test_asan_cache.py): the workspace query, which splits the work as a call
 * would, over bounds from nothing to the largest, and each entry point with
 * arguments that its validation refuses.  Nothing reaches the device; pointers are
 * fake (never dereferenced) and the stream is 0.
 */
#include <stdint.h>
#include <stdio.h>

#include "stepprune.h"

#define FAKE ((void*)0x10000)
#define FAKE_OUT ((void*)0x110000)

static int failures = 0;

static void expect(const char* what, sp_status got, sp_status want) {
  if (got != want) {
    printf("FAIL %s: got %d (%s), want %d\n", what, (int)got, stepprune_status_string(got), (int)want);
    ++failures;
  }
}

#define LEN(a) ((int)(sizeof(a) / sizeof((a)[0])))

static void plans(void) {
  static const int heads[][2] = {{1, 1}, {7, 1}, {32, 32}, {40, 8}, {1024, 1024}, {1024, 1}};
  static const int64_t rows[] = {0, 1, 5, 300, 4096, 1 << 15, 1 << 20, 1 << 25};
  static const int32_t counts[] = {0, 1, 3, 64, 65, 4096, 1 << 24};
  static const int32_t lens[] = {0, 1, 64, 257, 1025, 1 << 20, 1 << 30};
  long asked = 0, refused = 0;
  for (int dtype = 0; dtype < 2; ++dtype)
    for (int dim = 64; dim <= 128; dim += 64)
      for (int h = 0; h < LEN(heads); ++h)
        for (int r = 0; r < LEN(rows); ++r)
          for (int c = 0; c < LEN(counts); ++c)
            for (int l = 0; l < LEN(lens); ++l)
              for (int p = -1; p < LEN(lens); ++p)
                for (int most = 0; most < 3; ++most) {
                  sp_cache_dims d = {heads[h][0], heads[h][1], dim, dtype, 256, 1 << 22};
                  const int32_t max_rows = most == 0 ? 1 : most == 1 ? 60 : 1 << 30;
                  sp_cache_rows b = {rows[r], SP_LAYOUT_PACKED, 0, NULL, max_rows};
                  sp_cache_runs own = {NULL, NULL, counts[c], 1 << 22, lens[l]};
                  sp_cache_runs pre = {NULL, NULL, counts[c] > 4 ? 4 : counts[c], 1 << 22, p < 0 ? 0 : lens[p]};
                  const size_t n = stepprune_cache_workspace_bytes(&d, &b, &own, p < 0 ? NULL : &pre);
                  ++asked;
                  refused += n == 0;
                  if (n != 0 && (n < 256 || n > ((size_t)1 << 56))) {
                    printf("FAIL workspace of %zu bytes\n", n);
                    ++failures;
                  }
                }
  printf("%ld plans, %ld refused\n", asked, refused);
}

int main(void) {
  plans();
  const sp_cache_dims d = {8, 2, 128, SP_BF16, 16, 10};
  const sp_cache_rows b = {4, SP_LAYOUT_PACKED, 0, (const int32_t*)FAKE, 4};
  const sp_cache_runs own = {(const int32_t*)FAKE, (const int32_t*)FAKE, 2, 3, 48};
  const sp_cache_rotation rot = {(const float*)FAKE, 100, 128, 0, NULL, 1, {64, 0, 0}};
#define ATTEND(D, B, R, P, G, SCALE, FLAGS) \
  stepprune_cache_attend(D, FAKE, 1024, B, R, P, G, SCALE, FLAGS, FAKE, FAKE, FAKE_OUT, NULL, FAKE, 0, NULL, 0)
#define APPEND(D, B, R, T) \
  stepprune_cache_append(D, FAKE, 1024, FAKE, 256, FAKE, 256, B, R, T, FAKE_OUT, FAKE, FAKE, FAKE, 0, 0)
  expect("attend", ATTEND(&d, &b, &own, NULL, NULL, 0.1f, 0), SP_EWORKSPACE);
  expect("attend, prefix", ATTEND(&d, &b, &own, &own, (const int32_t*)FAKE, 0.1f, SP_ATTEND_ALL), SP_EWORKSPACE);
  expect("append", APPEND(&d, &b, &own, &rot), SP_EWORKSPACE);
  expect("attend without dims", ATTEND(NULL, &b, &own, NULL, NULL, 0.1f, 0), SP_EINVAL);
  expect("attend without rows", ATTEND(&d, NULL, &own, NULL, NULL, 0.1f, 0), SP_EINVAL);
  expect("attend without runs", ATTEND(&d, &b, NULL, NULL, NULL, 0.1f, 0), SP_EINVAL);
  expect("attend, groups only", ATTEND(&d, &b, &own, NULL, (const int32_t*)FAKE, 0.1f, 0), SP_EINVAL);
  expect("attend, scale", ATTEND(&d, &b, &own, NULL, NULL, -0.0f, 0), SP_EINVAL);
  expect("attend, flags", ATTEND(&d, &b, &own, NULL, NULL, 0.1f, 4), SP_EINVAL);
  expect("append without dims", APPEND(NULL, &b, &own, &rot), SP_EINVAL);
  const int32_t odd[] = {INT32_MIN, -1, 0, 1, 3, 24, 1 << 30, INT32_MAX};
  for (int i = 0; i < LEN(odd); ++i)
    for (int f = 0; f < 15; ++f) {
      sp_cache_dims dd = d;
      sp_cache_rows bb = b;
      sp_cache_runs rr = own;
      sp_cache_rotation tt = rot;
      int32_t* const field[] = {&dd.q_heads, &dd.kv_heads, &dd.head_dim, &dd.dtype, &dd.page_size, &dd.pages,
                                &bb.layout, &bb.rows_per_seq, &bb.max_rows, &rr.count, &rr.table_width,
                                &rr.max_len, &tt.positions, &tt.rot_dim, &tt.section[0]};
      *field[f] = odd[i];
      bb.rows = f == 14 ? odd[i] : bb.rows;
      const sp_status a = ATTEND(&dd, &bb, &rr, NULL, NULL, 0.1f, 0), p = APPEND(&dd, &bb, &rr, &tt);
      /* a workspace of no bytes: nothing comes further than that */
      if (a < SP_EINVAL || a > SP_EWORKSPACE || p < SP_EINVAL || p > SP_EWORKSPACE) {
        printf("FAIL field %d = %d: %d, %d\n", f, (int)odd[i], (int)a, (int)p);
        ++failures;
      }
      stepprune_cache_workspace_bytes(&dd, &bb, &rr, &rr);
    }
  expect("positions", stepprune_compact_positions((const int32_t*)FAKE, 10, (const int32_t*)FAKE, (const int32_t*)FAKE, 5,
                                                  (const int32_t*)FAKE, 4, (const int32_t*)FAKE, (const int32_t*)FAKE,
                                                  (const int32_t*)FAKE, 2, SP_LAYOUT_PACKED, 0, 15, (int32_t*)FAKE_OUT,
                                                  FAKE, 256, 0), SP_EINVAL);
  expect("positions, padded", stepprune_compact_positions((const int32_t*)FAKE, 10, (const int32_t*)FAKE,
                                                          (const int32_t*)FAKE, 5, (const int32_t*)FAKE, 1,
                                                          (const int32_t*)FAKE, (const int32_t*)FAKE, (const int32_t*)FAKE,
                                                          INT32_MAX, SP_LAYOUT_PADDED, INT32_MAX, 15, (int32_t*)FAKE_OUT,
                                                          FAKE, 256, 0), SP_EINVAL);
  printf("ok: %d failure(s)\n", failures);
  return failures != 0;
}
