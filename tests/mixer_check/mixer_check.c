/* Drives the C entry points of the convolution, the scan and the pools through their argument
 * checks, size computations and error paths over a grid of ordinary and extreme arguments, with
 * fake pointers that are never dereferenced.  Every valid call ends at the stub launchers
 * ("no device": HAGDN_EHIP). */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "hagdn.h"

#define P(i) ((void *)(((uintptr_t)(i) + 1) << 56)) /* far enough apart for any extent that counts */
#define CHECK(cond)                                                                        \
  do {                                                                                     \
    if (!(cond)) {                                                                         \
      fprintf(stderr, "line %d: %s (last error: %s)\n", __LINE__, #cond, hagdn_last_error()); \
      exit(1);                                                                             \
    }                                                                                      \
  } while (0)

static const int sizes[] = {INT32_MIN, -1, 0, 1, 2, 16, 63, 64, 65, 16384, 65536, INT32_MAX - 1, INT32_MAX};
#define NS (int)(sizeof sizes / sizeof *sizes)
static const int64_t strides[] = {INT64_MIN, -1, 0, 64, INT32_MAX, (int64_t)INT32_MAX + 1, INT64_MAX};
#define NT (int)(sizeof strides / sizeof *strides)

static int known(int rc) {
  CHECK(rc >= HAGDN_OK && rc <= HAGDN_EHIP);
  if (rc != HAGDN_OK) CHECK(strlen(hagdn_last_error()) > 0);
  return rc;
}

int main(void) {
  size_t all = SIZE_MAX;
  int reached = 0;
  for (int i = 0; i < NS; ++i)
    for (int j = 0; j < NS; ++j)
      for (int k = 0; k < NS; ++k) {
        const int N = sizes[i], T = sizes[j], D = sizes[k];
        for (int s = 0; s < NS; ++s) {
          hagdn_conv_workspace_size(T, D, sizes[s], 1);
          ssm_workspace_size(T, D, sizes[s], sizes[i], 1);
          ssm_checkpoints_size(T, D, sizes[s]);
          reached += HAGDN_EHIP == known(ssm_prefill(P(0), 64, P(1), 64, P(2), P(3), 64, P(4), 64, P(5), P(6), 64, P(7), P(8),
                                                     P(9), N, T, D, sizes[s], 1, 1, 0, 2, P(10), P(11), P(12), P(13), all, NULL));
          reached += HAGDN_EHIP == known(ssm_backward(P(0), 64, P(1), 64, P(2), 64, P(3), P(4), 64, P(5), 64, P(6), P(7), 64, P(8),
                                                      P(9), P(10), P(11), P(12), N, T, D, sizes[s], sizes[i], 0, 0, 2, P(13),
                                                      P(14), P(15), P(16), P(17), P(18), P(19), P(20), P(21), P(22), all, NULL));
          reached += HAGDN_EHIP == known(ssm_decode(P(0), 0, P(1), 0, P(2), P(3), 0, P(4), 0, NULL, NULL, 0, NULL, P(5), P(6), T, N,
                                                    D, sizes[s], 1, 1, 1, 0, P(7), NULL));
        }
        for (int W = -1; W < 11; ++W) {
          reached += HAGDN_EHIP == known(hagdn_conv_prefill(P(0), 64, P(1), P(2), P(3), P(4), N, T, D, W, 1, 0, P(5), P(6), P(7), all,
                                                            NULL));
          reached += HAGDN_EHIP == known(hagdn_conv_backward(P(0), 64, P(1), 64, P(2), P(3), P(4), P(5), P(6), N, T, D, W, 0, 2, P(7),
                                                             P(8), P(9), P(10), P(11), all, NULL));
          reached += HAGDN_EHIP == known(hagdn_conv_decode(P(0), 64, P(1), NULL, P(2), P(3), T, N, D, W, 1, 2, P(4), NULL));
        }
        void *pools[1] = {P(0)};
        const void *sources[1] = {P(1)};
        size_t row[1] = {(size_t)(uint32_t)D};
        reached += HAGDN_EHIP == known(hagdn_pool_copy(pools, NULL, row, 1, P(2), P(3), N, T, 0, NULL));
        reached += HAGDN_EHIP == known(hagdn_pool_copy(pools, sources, row, 1, P(2), NULL, N, T, T, NULL));
        hagdn_pool_workspace_size(T);
        reached += HAGDN_EHIP == known(hagdn_pool_fork(pools, row, 1, P(2), N, P(3), D, T, P(4), P(5), all, NULL));
        reached += HAGDN_EHIP == known(hagdn_pool_compact(pools, row, 1, P(2), N, T, P(2), P(5), all, NULL));
      }
  CHECK(reached > 1000);
  for (int i = 0; i < NT; ++i) {
    const int ok = strides[i] >= 0 && strides[i] <= INT32_MAX;
    CHECK((known(hagdn_conv_prefill(P(0), strides[i], P(1), NULL, NULL, NULL, 1, 5, 64, 4, 1, 0, P(5), NULL, P(7), all, NULL)) ==
           HAGDN_EHIP) == ok);
    CHECK((known(ssm_prefill(P(0), 64, P(1), 64, P(2), P(3), strides[i], P(4), strides[i], NULL, NULL, 0, NULL, NULL, NULL, 1, 5, 64,
                             16, 1, 1, 0, 0, P(10), NULL, NULL, P(13), all, NULL)) == HAGDN_EHIP) == ok);
  }
  /* as many pools as a call takes, of all alignments */
  enum { MOST = 1024 };
  static void *many[MOST];
  static size_t rows[MOST];
  for (int p = 0; p < MOST; ++p) {
    many[p] = (char *)P(0) + (size_t)((p * 7919) % MOST) * 4096;
    rows[p] = (size_t)(p % 64) + 1;
  }
  CHECK(known(hagdn_pool_copy(many, NULL, rows, MOST, P(2), P(3), 5, 64, 0, NULL)) == HAGDN_EHIP);
  CHECK(known(hagdn_pool_copy(many, NULL, rows, MOST, P(2), P(3), 5, 65, 0, NULL)) == HAGDN_EINVAL);
  CHECK(known(hagdn_pool_copy(many, NULL, rows, MOST + 1, P(2), P(3), 5, 64, 0, NULL)) == HAGDN_EINVAL);
  puts("mixer checks passed");
  return 0;
}
