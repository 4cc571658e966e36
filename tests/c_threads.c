/* Operators called from several C threads on one context at the same time, each with its own stream, width and set of inputs. Built and run
 * by tests/test_c_threads.py. Exit code 0 and a line starting with "PASS" when every call was accepted and every output is what the
 * same call wrote alone. */
#include <cuda_runtime.h>
#include <pthread.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "slidedp_ops.h"

#define CHECK_CUDA(x) do { cudaError_t e_ = (x); if (e_ != cudaSuccess) { \
  printf("FAIL cuda %s at line %d\n", cudaGetErrorString(e_), __LINE__); exit(2); } } while (0)

enum { TOKENS = 16, CALLS = 4000, THREADS = 6 };

typedef struct {
  slidedp_ctx* ctx;
  slidedp_block_norm_args args;
  slidedp_rows x, y, x_out, h, dx, dy;
  uint16_t* want;
  cudaStream_t stream;
  int status; /* of the first call that was not accepted */
} work;

static slidedp_rows rows(int64_t hidden) {
  slidedp_rows r = {NULL, hidden};
  CHECK_CUDA(cudaMalloc(&r.data, TOKENS * hidden * 2));
  CHECK_CUDA(cudaMemset(r.data, 0, TOKENS * hidden * 2));
  return r;
}
static int call(work* w) {
  const int y = w->args.has_y;
  const int rc = slidedp_block_norm(w->ctx, &w->args, &w->x, y ? &w->y : NULL, NULL, NULL, NULL, y ? &w->x_out : NULL, &w->h, w->stream);
  if (rc != SLIDEDP_OK) return rc;
  return slidedp_block_norm_backward(w->ctx, &w->args, &w->x, y ? &w->y : NULL, NULL, NULL, NULL, y ? &w->x : NULL, &w->h, &w->dx,
                                     y ? &w->dy : NULL, NULL, NULL, NULL, NULL, w->stream);
}
static void* loop(void* p) {
  work* w = p;
  for (int i = 0; i < CALLS && w->status == SLIDEDP_OK; ++i) w->status = call(w);
  return NULL;
}

int main(void) {
  static const int64_t hidden[THREADS] = {2048, 4096, 2048, 1032, 600, 3200};
  work all[THREADS];
  slidedp_ctx* ctx = NULL;
  if (slidedp_create(&ctx, 0, 0) != SLIDEDP_OK) return printf("FAIL create\n"), 3;
  for (int t = 0; t < THREADS; ++t) {
    work* w = &all[t];
    const int64_t H = hidden[t], n = TOKENS * H;
    const slidedp_block_norm_args args = {TOKENS, H, SLIDEDP_BF16, t % 3 == 2, 0, 1, 0, 0, 1.0, 1e-6};
    uint16_t* host = malloc(n * 2);
    w->ctx = ctx;
    w->args = args;
    w->status = SLIDEDP_OK;
    w->x = rows(H), w->y = rows(H), w->x_out = rows(H), w->h = rows(H), w->dx = rows(H), w->dy = rows(H);
    for (int64_t i = 0; i < n; ++i) host[i] = (uint16_t)(0x3f00 + (i * 2654435761u >> 24) % 160); /* 0.5 to 1.6 */
    CHECK_CUDA(cudaMemcpy(w->x.data, host, n * 2, cudaMemcpyHostToDevice));
    CHECK_CUDA(cudaMemcpy(w->y.data, host, n * 2, cudaMemcpyHostToDevice));
    CHECK_CUDA(cudaStreamCreateWithFlags(&w->stream, cudaStreamNonBlocking));
    CHECK_CUDA(cudaDeviceSynchronize());
    if (call(w) != SLIDEDP_OK) return printf("FAIL alone: thread %d\n", t), 3;
    CHECK_CUDA(cudaDeviceSynchronize());
    w->want = malloc(n * 4);
    CHECK_CUDA(cudaMemcpy(w->want, w->h.data, n * 2, cudaMemcpyDeviceToHost));
    CHECK_CUDA(cudaMemcpy(w->want + n, w->dx.data, n * 2, cudaMemcpyDeviceToHost));
    free(host);
  }
  pthread_t id[THREADS];
  for (int t = 0; t < THREADS; ++t) pthread_create(&id[t], NULL, loop, &all[t]);
  for (int t = 0; t < THREADS; ++t) pthread_join(id[t], NULL);
  CHECK_CUDA(cudaDeviceSynchronize());
  int bad = 0;
  for (int t = 0; t < THREADS; ++t) {
    work* w = &all[t];
    const int64_t n = TOKENS * w->args.hidden;
    uint16_t* got = malloc(n * 4);
    CHECK_CUDA(cudaMemcpy(got, w->h.data, n * 2, cudaMemcpyDeviceToHost));
    CHECK_CUDA(cudaMemcpy(got + n, w->dx.data, n * 2, cudaMemcpyDeviceToHost));
    if (w->status != SLIDEDP_OK || memcmp(got, w->want, n * 4) != 0) {
      printf("FAIL thread %d: %s, cudaError_t %d, outputs %s\n", t, slidedp_strerror(w->status), slidedp_last_cuda_error(ctx),
             memcmp(got, w->want, n * 4) ? "differ" : "agree");
      bad = 1;
    }
    free(got);
  }
  if (bad) return 4;
  slidedp_destroy(ctx);
  printf("PASS %d threads, %d calls each\n", THREADS, 2 * CALLS);
  return 0;
}
