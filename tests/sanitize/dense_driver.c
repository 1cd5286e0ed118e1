/* The dense layers' host code under sanitizers: refusals, and the planning of
 * layers of every magnitude and type through the workspace-size query, which
 * launches nothing.  Device pointers are made up and never followed. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "qcnn.h"

static uint64_t state = 0x9e3779b97f4a7c15ull;

static uint64_t next(void) {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return state;
}

/* 1 .. 2^bits, every magnitude as often as the others. */
static int any_size(int bits) {
  const int b = (int)(next() % (unsigned)bits);
  return (1 << b) + (int)(next() % (1u << b));
}

#define AT(n) ((void*)((uintptr_t)(n) << 40))
#define MUST(rc, want) \
  do { \
    const int got = (int)(rc); \
    if (got != (want)) { \
      fprintf(stderr, "line %d: status %d, expected %d\n", __LINE__, got, (int)(want)); \
      exit(1); \
    } \
  } while (0)

int main(void) {
  size_t n = 0;
  int planned = 0, refused = 0;
  for (int i = 0; i < 20000; ++i) {
    const int dtype = (int)(next() % 3), act = (int)(next() % 5), N = any_size(21), Cs = any_size(20), Ct = any_size(20);
    const long long ldx = Cs + (long long)(next() % 3), ldy = Ct + (long long)(next() % 3);
    void* x = (char*)AT(1) + 4 * (next() % 4);
    int rc[6];
    rc[0] = qcnn_linear_forward(dtype, x, ldx, N, Cs, AT(2), Ct, AT(3), act, AT(4), ldy, AT(5), AT(6), ldy, NULL, &n, NULL);
    rc[1] = qcnn_linear_backward(dtype, AT(1), ldy, (char*)x + ((uintptr_t)1 << 41), ldx, N, Cs, AT(3), Ct, AT(4), act, AT(5), AT(6), AT(7), NULL, &n, NULL);
    rc[2] = qcnn_gated_forward(dtype, x, ldx, N, Cs, AT(2), Ct, AT(3), act, AT(5), AT(6), ldy, NULL, &n, NULL);
    rc[3] = qcnn_gated_backward(dtype, AT(9), ldy, x, ldx, N, Cs, AT(3), Ct, AT(4), act, AT(5), AT(6), AT(7), NULL, &n, NULL);
    rc[4] = qcnn_linear_xent_forward(dtype, x, ldx, N, Cs, AT(2), Ct, AT(3), AT(4), AT(5), AT(6), NULL, &n, NULL);
    rc[5] = qcnn_linear_xent_backward(dtype, AT(8), AT(7), x, ldx, N, Cs, AT(2), Ct, AT(3), AT(4), AT(5), AT(6), AT(9), NULL, &n, NULL);
    for (int k = 0; k < 6; ++k) {
      if (rc[k] == QCNN_OK) ++planned;
      else if (rc[k] == QCNN_ERR_UNSUPPORTED || rc[k] == QCNN_ERR_ALIAS) ++refused;
      else MUST(rc[k], QCNN_OK);
    }
  }
  if (planned < 40000) {
    fprintf(stderr, "only %d calls were planned (%d refused)\n", planned, refused);
    return 1;
  }
  /* limits, nulls, a workspace that is too small or misaligned */
  MUST(qcnn_linear_forward(0, AT(1), 8, 0, 8, AT(2), 8, NULL, 0, NULL, 0, NULL, AT(3), 8, NULL, &n, NULL), QCNN_ERR_SHAPE);
  MUST(qcnn_linear_forward(0, AT(1), 8, INT32_MAX, 8, AT(2), 8, NULL, 0, NULL, 0, NULL, AT(3), 8, NULL, &n, NULL), QCNN_ERR_UNSUPPORTED);
  MUST(qcnn_linear_forward(0, AT(1), INT64_MAX, 8, 8, AT(2), 8, NULL, 0, NULL, 0, NULL, AT(3), 8, NULL, &n, NULL), QCNN_ERR_UNSUPPORTED);
  MUST(qcnn_linear_forward(0, AT(1), 8, 8, INT32_MAX, AT(2), INT32_MAX, NULL, 0, NULL, 0, NULL, AT(3), INT32_MAX, NULL, &n, NULL), QCNN_ERR_SHAPE);
  MUST(qcnn_gated_forward(1, AT(1), 8, 8, 8, AT(2), INT32_MAX, NULL, 4, NULL, AT(3), INT32_MAX, NULL, &n, NULL), QCNN_ERR_UNSUPPORTED);
  MUST(qcnn_linear_xent_forward(1, AT(1), 8, 8, 8, AT(2), 8, NULL, NULL, AT(4), AT(5), NULL, &n, NULL), QCNN_ERR_NULL);
  MUST(qcnn_linear_xent_forward(1, AT(1), 8, 8, 8, AT(2), 8, NULL, (void*)((char*)AT(3) + 4), AT(4), AT(5), NULL, &n, NULL), QCNN_ERR_UNSUPPORTED);
  MUST(qcnn_linear_forward(1, AT(1), 1001, 99, 1001, AT(2), 50, NULL, 0, NULL, 0, NULL, AT(3), 50, NULL, &n, NULL), QCNN_OK);
  size_t small = n - 1;
  MUST(qcnn_linear_forward(1, AT(1), 1001, 99, 1001, AT(2), 50, NULL, 0, NULL, 0, NULL, AT(3), 50, AT(4), &small, NULL), QCNN_ERR_WORKSPACE);
  MUST(qcnn_linear_forward(1, AT(1), 1001, 99, 1001, AT(2), 50, NULL, 0, NULL, 0, NULL, AT(3), 50, (char*)AT(4) + 16, &n, NULL), QCNN_ERR_UNSUPPORTED);
  MUST(qcnn_linear_forward(1, AT(1), 1001, 99, 1001, AT(2), 50, NULL, 0, NULL, 0, NULL, AT(3), 50, AT(4), NULL, NULL), QCNN_ERR_NULL);
  printf("%d planned, %d refused\nok\n", planned, refused);
  return 0;
}
