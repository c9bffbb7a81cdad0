/* Drives the recurrence's and the norms' C entry points through their argument checks,
 * size computations and error paths over a grid of ordinary and extreme arguments, with
 * fake pointers that are never dereferenced.  Every valid call ends at the stub
 * launchers ("no device": HAGDN_EHIP). */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "hagdn.h"

#define P ((void *)0x100000)
#define CHECK(cond)                                                                        \
  do {                                                                                     \
    if (!(cond)) {                                                                         \
      fprintf(stderr, "line %d: %s (last error: %s)\n", __LINE__, #cond, hagdn_last_error()); \
      exit(1);                                                                             \
    }                                                                                      \
  } while (0)

static const int sizes[] = {INT32_MIN, -1, 0, 1, 2, 63, 64, 65, 16384, 16385, 65536, INT32_MAX - 1, INT32_MAX};
#define NS (int)(sizeof sizes / sizeof *sizes)
static const int64_t strides[] = {INT64_MIN, -1, 0, 64, INT32_MAX, (int64_t)INT32_MAX + 1, INT64_MAX};
#define NT (int)(sizeof strides / sizeof *strides)

static int known(int rc) {
  CHECK(rc >= HAGDN_OK && rc <= HAGDN_EHIP);
  if (rc != HAGDN_OK) CHECK(strlen(hagdn_last_error()) > 0);
  return rc;
}

int main(void) {
  float *f = P;
  const int32_t *cu = P;
  size_t all = SIZE_MAX;
  int reached = 0;
  for (int i = 0; i < NS; ++i)
    for (int j = 0; j < NS; ++j) {
      glr_workspace_size(sizes[i], sizes[j]);
      hagdn_add_norm_workspace_size(sizes[i], sizes[j], 1, 1);
      for (int k = 0; k < NS; ++k) {
        hagdn_gate_norm_workspace_size(sizes[i], sizes[j], sizes[k]);
        reached += HAGDN_EHIP == known(glr_prefill(P, 64, P, 64, f, cu, sizes[i], sizes[j], sizes[k], 1, 1, 1, 2, P, f, f, P,
                                                   all, NULL));
        reached += HAGDN_EHIP == known(glr_backward(P, 64, P, 64, P, 64, f, f, f, cu, sizes[i], sizes[j], sizes[k], 1, 0, 0,
                                                    0, P, P, f, P, all, NULL));
        reached += HAGDN_EHIP == known(glr_decode(P, 0, P, 0, f, cu, sizes[i], sizes[j], sizes[k], 0, 0, 0, 0, P, NULL));
        reached += HAGDN_EHIP == known(hagdn_gate_norm(P, 64, P, 64, f, 1e-6f, sizes[i], sizes[j], sizes[k], 1, 0, P, NULL));
        reached += HAGDN_EHIP == known(hagdn_gate_norm_backward(P, 64, P, 64, P, 64, f, 1e-6f, sizes[i], sizes[j], sizes[k],
                                                                0, 1, P, P, f, P, all, NULL));
      }
      reached += HAGDN_EHIP == known(hagdn_add_norm(P, 64, P, 64, f, f, f, 1.f, 1e-6f, sizes[i], sizes[j], 1, 0, P, NULL, NULL));
      reached += HAGDN_EHIP == known(hagdn_add_norm_backward(P, 64, NULL, 0, P, 64, P, 64, f, f, f, 1.f, 1e-6f, sizes[i],
                                                             sizes[j], 1, 1, P, P, f, f, f, P, all, NULL));
    }
  CHECK(reached > 100);
  for (int i = 0; i < NT; ++i) {
    int ok = strides[i] >= 0 && strides[i] <= INT32_MAX;
    CHECK((known(glr_prefill(P, strides[i], P, 64, NULL, NULL, 1, 5, 64, 1, 1, 0, 0, P, NULL, NULL, P, all, NULL)) ==
           HAGDN_EHIP) == ok);
    CHECK((known(hagdn_gate_norm(P, 64, P, strides[i], f, 0.f, 5, 1, 64, 1, 0, P, NULL)) == HAGDN_EHIP) == ok);
  }
  /* the workspace sizes are what the calls ask for */
  for (int T = 0; T < 400; T += 37)
    for (int D = 1; D < 300; D += 41) {
      size_t n = glr_workspace_size(T, D);
      CHECK(n > 0);
      CHECK(glr_prefill(P, D, P, D, NULL, NULL, 1, T, D, 0, 0, 0, 0, P, NULL, NULL, P, n - 1, NULL) == HAGDN_EWORKSPACE);
      CHECK(glr_prefill(P, D, P, D, NULL, NULL, 1, T, D, 0, 0, 0, 0, P, NULL, NULL, P, n, NULL) == HAGDN_EHIP);
      n = hagdn_add_norm_workspace_size(T, D, 1, 0);
      CHECK(hagdn_add_norm_backward(P, D, P, D, P, D, P, D, f, NULL, f, 1.f, 0.f, T, D, 0, 0, P, NULL, f, f, NULL, P, n - 1,
                                    NULL) == HAGDN_EWORKSPACE);
      CHECK(hagdn_add_norm_backward(P, D, P, D, P, D, P, D, f, NULL, f, 1.f, 0.f, T, D, 0, 0, P, NULL, f, f, NULL, P, n,
                                    NULL) == HAGDN_EHIP);
    }
  /* a long message is cut, not overrun */
  CHECK(known(hagdn_add_norm(P, 64, P, 64, f, f, f, 1.f, NAN, 5, 64, 1, 0, P, NULL, NULL)) == HAGDN_EINVAL);
  puts("layer checks passed");
  return 0;
}
