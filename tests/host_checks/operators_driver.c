/* Host-side walk over the calls next to the step (log-probabilities of tokens, embedding rows, gradient norm) for the
 * sanitizer build: arguments that the host checks must turn into a status code, empty calls, and scratch sizes over the
 * whole range of shapes.  No GPU is needed and none of the pointers is ever dereferenced.  Exit code 0 = every status was
 * the expected one; the sanitizers abort on their own findings. */
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/sv.h"

static int failures = 0;
#define EXPECT(call, want)                                                                   \
  do {                                                                                       \
    const int got_ = (call);                                                                 \
    if (got_ != (want)) {                                                                    \
      printf("line %d: %s -> %d (%s), expected %d\n", __LINE__, #call, got_, sv_strerror(got_), (want)); \
      ++failures;                                                                            \
    }                                                                                        \
  } while (0)
#define CHECK(what)                                                                          \
  do {                                                                                       \
    if (!(what)) { printf("line %d: %s\n", __LINE__, #what); ++failures; }                   \
  } while (0)

int main(void) {
  void* p = (void*)(uintptr_t)(256 * 1024);        /* non-NULL, aligned, never dereferenced */
  void* odd = (void*)(uintptr_t)(256 * 1024 + 1);
  const size_t big = (size_t)1 << 30;
  const int Vs[] = {1, 511, 4096, 152064, 1 << 24}, Ds[] = {1, 7, 2048, 1 << 20};
  const int64_t rows[] = {0, 1, 64, 682, 683, 4096, INT_MAX};
  unsigned i, j, l;

  /* scratch sizes */
  for (i = 0; i < sizeof rows / sizeof *rows; ++i)
    for (j = 0; j < sizeof Vs / sizeof *Vs; ++j)
      for (l = 0; l <= SV_TOP_MAX; l += 8) {
        const size_t w = sv_token_logprobs_workspace_bytes(rows[i], Vs[j], l % 16 ? SV_BF16 : SV_F32, (int)l);
        CHECK(w % 256 == 0 && w < big);
      }
  CHECK(sv_token_logprobs_workspace_bytes((int64_t)INT_MAX + 1, 8, SV_F32, 0) == 0);
  CHECK(sv_token_logprobs_workspace_bytes(INT64_MIN, 8, SV_F32, 0) == 0 && sv_token_logprobs_workspace_bytes(1, INT_MAX, SV_F32, 0) == 0);
  {
    const int ns[] = {0, 1, 128, 129, 4097, 65536, SV_EMBEDDING_MAX_TOKENS};
    for (i = 0; i < sizeof ns / sizeof *ns; ++i)
      for (j = 0; j < sizeof Vs / sizeof *Vs; ++j)
        for (l = 0; l < sizeof Ds / sizeof *Ds; ++l) {
          const size_t w = sv_embedding_grad_workspace_bytes(ns[i], Vs[j], Ds[l]);
          CHECK(w >= 256 && w % 256 == 0);
          CHECK(ns[i] <= 128 || w >= (size_t)ns[i] * 16);
        }
    CHECK(sv_embedding_grad_workspace_bytes(INT_MAX, 8, 8) == 0 && sv_embedding_grad_workspace_bytes(INT_MIN, 8, 8) == 0);
    CHECK(sv_embedding_grad_workspace_bytes(8, INT_MAX, 8) == 0 && sv_embedding_grad_workspace_bytes(8, 8, INT_MAX) == 0);
  }
  {
    const int ns[] = {0, 1, 120, 121, 100000, INT_MAX - 119, INT_MAX - 1, INT_MAX};
    size_t last = 0;
    for (i = 0; i < sizeof ns / sizeof *ns; ++i) {
      const size_t w = sv_grad_norm_workspace_bytes(ns[i]);
      CHECK(w % 256 == 0 && w >= last && w > (size_t)(ns[i] / 120) * 8192);
      last = w;
    }
    CHECK(sv_grad_norm_workspace_bytes(-1) == 0 && sv_grad_norm_workspace_bytes(INT_MIN) == 0);
  }

  /* sv_token_logprobs */
  EXPECT(sv_token_logprobs(p, 8, 0, 0, p, 2, 2, 8, 7, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_DTYPE);
  EXPECT(sv_token_logprobs(p, 8, 0, 0, p, INT_MIN, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_token_logprobs(p, INT64_MIN, 0, 0, p, 2, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_token_logprobs(p, 8, p, INT_MIN, p, 2, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_token_logprobs(p, 8, 0, 0, p, 2, 2, 8, SV_F32, -1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_token_logprobs(p, 8, 0, 0, p, INT_MAX, INT_MAX, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_TOO_LARGE);
  EXPECT(sv_token_logprobs(p, INT64_MAX, 0, 0, p, 2, 2, INT_MAX, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_TOO_LARGE);
  EXPECT(sv_token_logprobs(p, 8, 0, 0, p, 2, 2, 8, SV_F32, 1.0f, INT_MAX, p, 0, 0, 0, p, p, 0, 0, 0, 0), SV_ERR_TOO_LARGE);
  EXPECT(sv_token_logprobs(0, 8, 0, 0, p, 2, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_NULL);
  EXPECT(sv_token_logprobs(0, 8, p, 1, p, 2, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_NULL);
  EXPECT(sv_token_logprobs(p, 8, 0, 0, 0, 2, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_NULL);
  EXPECT(sv_token_logprobs(p, 8, 0, 0, p, 2, 2, 8, SV_F32, 1.0f, 3, p, 0, 0, 0, p, 0, 0, 0, 0, 0), SV_ERR_NULL);
  EXPECT(sv_token_logprobs(odd, 8, 0, 0, p, 2, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_ERR_ALIGN);
  EXPECT(sv_token_logprobs(p, 8, 0, 0, p, 2, 2, 8, SV_F32, 1.0f, 0, p, 0, 0, 0, 0, 0, 0, odd, big, 0), SV_ERR_WORKSPACE);
  EXPECT(sv_token_logprobs(0, 8, 0, 0, 0, 0, 2, 8, SV_F32, 1.0f, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), SV_OK);

  /* sv_token_logprobs_grad */
  EXPECT(sv_token_logprobs_grad(p, 8, p, 2, 8, -1, 1.0f, p, 0, 0, 0, p, 8, 0, 0, 0, 0), SV_ERR_DTYPE);
  EXPECT(sv_token_logprobs_grad(p, 8, p, INT_MIN, 8, SV_BF16, 1.0f, p, 0, 0, 0, p, 8, 0, 0, 0, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_token_logprobs_grad(p, 8, p, 2, 8, SV_BF16, 1.0f, p, 0, 0, 0, p, 9, 0, 0, 0, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_token_logprobs_grad(p, INT64_MAX, p, 2, INT_MAX, SV_BF16, 1.0f, p, 0, 0, 0, p, INT64_MAX, 0, 0, 0, 0), SV_ERR_TOO_LARGE);
  EXPECT(sv_token_logprobs_grad(p, 8, p, 2, 8, SV_BF16, 1.0f, 0, 0, 0, 0, p, 8, 0, 0, 0, 0), SV_ERR_NULL);
  EXPECT(sv_token_logprobs_grad(p, 8, p, 2, 8, SV_BF16, 1.0f, odd, 0, 0, 0, p, 8, 0, 0, 0, 0), SV_ERR_ALIGN);
  EXPECT(sv_token_logprobs_grad(p, 1 << 20, p, 2, 1 << 20, SV_BF16, 1.0f, p, 0, 0, 0, p, 1 << 20, 0, p, 1, 0), SV_ERR_WORKSPACE);
  EXPECT(sv_token_logprobs_grad(0, 8, 0, 0, 8, SV_BF16, 1.0f, 0, 0, 0, 0, 0, 8, 0, 0, 0, 0), SV_OK);

  /* sv_embedding, sv_embedding_grad */
  EXPECT(sv_embedding(p, p, 2, 8, 4, 9, 1.0f, p, 0, 0), SV_ERR_DTYPE);
  EXPECT(sv_embedding(p, p, INT_MIN, 8, 4, SV_F32, 1.0f, p, 0, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_embedding(p, p, 2, INT_MAX, 4, SV_F32, 1.0f, p, 0, 0), SV_ERR_TOO_LARGE);
  EXPECT(sv_embedding(p, p, 2, 8, INT_MAX, SV_F32, 1.0f, p, 0, 0), SV_ERR_TOO_LARGE);
  EXPECT(sv_embedding(p, 0, INT_MAX, 8, 4, SV_F32, 1.0f, p, 0, 0), SV_ERR_NULL);
  EXPECT(sv_embedding(p, p, 2, 8, 4, SV_F32, 1.0f, p, odd, 0), SV_ERR_ALIGN);
  EXPECT(sv_embedding(0, 0, 0, 8, 4, SV_F32, 1.0f, 0, 0, 0), SV_OK);
  EXPECT(sv_embedding_grad(p, 5, p, 2, 8, 4, 1.0f, p, SV_F32, 0, p, big, 0), SV_ERR_DTYPE);
  EXPECT(sv_embedding_grad(p, SV_F32, p, INT_MIN, 8, 4, 1.0f, p, SV_F32, 0, p, big, 0), SV_ERR_INVALID_ARG);
  EXPECT(sv_embedding_grad(p, SV_F32, p, INT_MAX, 8, 4, 1.0f, p, SV_F32, 0, p, big, 0), SV_ERR_TOO_LARGE);
  EXPECT(sv_embedding_grad(0, SV_F32, p, 2, 8, 4, 1.0f, p, SV_F32, 0, p, big, 0), SV_ERR_NULL);
  EXPECT(sv_embedding_grad(p, SV_F32, odd, 2, 8, 4, 1.0f, p, SV_F32, 0, p, big, 0), SV_ERR_ALIGN);
  EXPECT(sv_embedding_grad(p, SV_F32, p, SV_EMBEDDING_MAX_TOKENS, 1 << 24, 1 << 20, 1.0f, p, SV_F32, 0, p, big, 0), SV_ERR_WORKSPACE);
  EXPECT(sv_embedding_grad(0, SV_F32, 0, 0, 8, 4, 1.0f, 0, SV_F32, 1, 0, 0, 0), SV_OK);

  /* sv_grad_norm, sv_clip_grad_norm */
  {
    const void* g[] = {p, p};
    void* out[] = {p, p};
    const int64_t numel[] = {4, 4}, minus[] = {4, INT64_MIN}, far[] = {(int64_t)1 << 44, INT64_MAX}, many[] = {(int64_t)1 << 44, 4};
    const int dt[] = {SV_F32, SV_BF16}, none[] = {SV_F32, 2}, other[] = {SV_BF16, SV_BF16};
    float* norm = (float*)p;
    EXPECT(sv_grad_norm(-1, g, numel, dt, norm, 0, p, big, 0), SV_ERR_INVALID_ARG);
    EXPECT(sv_grad_norm(2, 0, numel, dt, norm, 0, p, big, 0), SV_ERR_NULL);
    EXPECT(sv_grad_norm(2, g, numel, none, norm, 0, p, big, 0), SV_ERR_DTYPE);
    EXPECT(sv_grad_norm(2, g, minus, dt, norm, 0, p, big, 0), SV_ERR_INVALID_ARG);
    EXPECT(sv_grad_norm(2, g, far, dt, norm, 0, p, big, 0), SV_ERR_TOO_LARGE);
    EXPECT(sv_grad_norm(2, g, many, dt, norm, 0, p, 16, 0), SV_ERR_TOO_LARGE);
    EXPECT(sv_grad_norm(2, g, numel, dt, norm, 0, 0, 0, 0), SV_ERR_WORKSPACE);
    EXPECT(sv_clip_grad_norm(2, g, numel, dt, 0.0f, out, dt, norm, 0, p, big, 0), SV_ERR_INVALID_ARG);
    EXPECT(sv_clip_grad_norm(2, g, numel, dt, 1.0f, 0, dt, norm, 0, p, big, 0), SV_ERR_NULL);
    EXPECT(sv_clip_grad_norm(2, g, numel, dt, 1.0f, out, other, norm, 0, p, big, 0), SV_ERR_INVALID_ARG);
    EXPECT(sv_clip_grad_norm(2, g, numel, dt, 1.0f, out, dt, (float*)odd, 0, p, big, 0), SV_ERR_ALIGN);
    EXPECT(sv_clip_grad_norm(2, g, numel, dt, 1.0f, out, dt, norm, 0, p, 16, 0), SV_ERR_WORKSPACE);
  }

  if (failures) return 1;
  printf("host walk ok\n");
  return 0;
}
