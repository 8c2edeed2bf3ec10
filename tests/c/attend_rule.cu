/* The form that md_attend_cache's estimate takes for launches read from stdin, and its split of their
 * rows (no GPU needed). */
#include <stdio.h>

#include "../../paper_2607_10582_gb300/csrc/md_attend.cu"

namespace md {
bool page_set(PageSet &, const int32_t *, const int32_t *, int, int, int, int, int, int, int) { return false; }
void *tile_encoder() { return nullptr; }
bool encode_tile_map(void *, CUtensorMap *, void *, size_t, int) { return false; }
}  // namespace md

int main() {
  using namespace md;
  static AttendCacheParams p;
  int e4m3, workspace;
  /* a line: eight bits or not, layers, KV heads, window, sinks, workspace or not, sequences, their tokens */
  while (scanf("%d %d %d %d %d %d %d", &e4m3, &p.L, &p.Hkv, &p.window, &p.sinks, &workspace, &p.n_seqs) == 7) {
    for (int b = 0; b < p.n_seqs; ++b)
      if (scanf("%d", &p.n_tokens[b]) != 1) return 1;
    const Form f = attend_form(p, e4m3, workspace);
    int parts = 0, partials = 0;
    for (int b = 0; b < p.n_seqs; ++b) {
      const int n = p.unit_start[b + 1] - p.unit_start[b], lh = p.L * p.Hkv;
      if (n < lh || n % lh || (n > lh && p.part_start[b] != partials)) return 2;
      parts = n / lh > parts ? n / lh : parts;
      partials += n > lh ? n : 0;
    }
    if (f.team == WARP && (f.C != 1 || parts > 1)) return 4;
    if (partials > MAX_PARTIALS || (long long)p.unit_start[p.n_seqs] * f.C >= 1LL << 31) return 3;
    printf("%d %d %d\n", f.team == WARP ? 0 : f.C, f.warps, parts);
  }
  return 0;
}
