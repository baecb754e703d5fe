/* Walks the host code of the model side of a step: scratch sizes over shapes up to the limits, and calls that are refused before anything is
 * enqueued.  Nothing is launched and no pointer is followed. */
#include <stdio.h>
#include <stdint.h>
#include "../../include/sv.h"

static int failures;
#define EXPECT(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); failures++; } } while (0)

int main(void) {
  char* const base = (char*)(uintptr_t)(1 << 20);
  void *p = base, *p2 = base + 4096, *odd = base + 1;
  const int sizes[] = {-1, 0, 1, 2, 7, 9, 64, 129, 1024, 2048, 65536, 1 << 20, 1 << 24, 0x7fffffff};
  const int n = sizeof(sizes) / sizeof(sizes[0]);
  const int heads[][2] = {{1, 1}, {32, 8}, {28, 4}, {1024, 1}, {1024, 1024}, {2048, 2048}, {5, 2}, {4, 0}};
  const int widths[] = {8, 64, 72, 128, 136, 256, 264};
  const int pages[][2] = {{1, 1}, {1, 65536}, {1024, 16}, {65536, 65536}, {0x7fffffff, 65536}, {0, 16}, {4, 0}, {4, 65537}};
  size_t most = 0;
  for (int b = 0; b < n; ++b)
    for (int q = 0; q < n; ++q)
      for (int h = 0; h < 8; ++h)
        for (int w = 0; w < 7; ++w)
          for (int g = 0; g < 8; ++g)
            for (int dt = 0; dt < 3; ++dt) {
              const size_t need = sv_chunk_attention_workspace_bytes(sizes[b], sizes[q], heads[h][0], heads[h][1], widths[w], dt, pages[g][0], pages[g][1]);
              EXPECT(need % 256 == 0);
              if (need > most) most = need;
            }
  EXPECT(most > 0 && most <= (1u << 28));
  for (int r = 0; r < n; ++r)
    for (int v = 0; v < n; ++v)
      for (int dt = 0; dt < 3; ++dt) EXPECT(sv_sample_workspace_bytes(sizes[r], sizes[v], dt) % 256 == 0);
  /* the last check before the launch is the workspace or an alignment: everything above it has run */
  for (int b = 0; b < n; ++b)
    for (int q = 0; q < n; ++q)
      for (int g = 0; g < 8; ++g) {
        int s = sv_chunk_attention(p, 1 << 20, NULL, 0, p, NULL, p, pages[g][0], sizes[b], sizes[q], 8, 2, 64, SV_BF16, p, p, SV_BF16, NULL, NULL, 9,
                                   pages[g][1], 1.f, 0, p2, 1 << 20, odd, NULL, NULL, 0, NULL);
        EXPECT(s != SV_OK || sizes[b] == 0);
        s = sv_chunk_attention(p, 512, p, sizes[b], p, NULL, p, pages[g][0], 4, sizes[q], 8, 2, 64, SV_BF16, p, p, SV_F8, p, p, 9, pages[g][1], 1.f, 0,
                               p2, 512, NULL, odd, NULL, 0, NULL);
        EXPECT(s != SV_OK || sizes[b] == 0);
        s = sv_cache_write(p, 1 << 20, p, 1 << 20, NULL, 0, 0, NULL, 0, NULL, 0, p, p, pages[g][0], sizes[b], sizes[q], 2, 64, SV_F32, NULL, 0, 0, 1.f, p,
                           p, SV_F32, NULL, NULL, 9, pages[g][1], odd, NULL);
        EXPECT(s != SV_OK || sizes[b] == 0);
        s = sv_cache_read(p, p, SV_F32, NULL, NULL, 9, pages[g][1], NULL, 0, p, p, pages[g][0], sizes[b], sizes[q], 2, 64, SV_F32, p, 1 << 20, p, 1 << 20,
                          odd, NULL);
        EXPECT(s != SV_OK || sizes[b] == 0);
      }
  for (int r = 0; r < n; ++r)
    for (int v = 0; v < n; ++v) {
      int s = sv_sample(p, 0x7fffffff, sizes[r], sizes[v], SV_BF16, 1.f, 5, 0.9f, 0.1f, p, odd, NULL, NULL, NULL, 0, NULL);
      EXPECT(s != SV_OK || sizes[r] == 0);
      s = sv_rope(p, 1 << 21, odd, sizes[r], 1, 64, SV_BF16, p, sizes[v], 0, 1.f, 0, p2, 1 << 21, NULL);
      EXPECT(s != SV_OK || sizes[r] == 0);
      EXPECT(sv_rope_frequencies(sizes[v], 1e4, r % 4, 2.0, 1.0, 4.0, sizes[r], odd, NULL) != SV_OK);
    }
  if (failures) return 1;
  printf("host walk ok\n");
  return 0;
}
