// What the training operators launch, from the library's own rules: one question a
// line on stdin, one answer a line on stdout.
//   grouped DIRECTION EXPERTS OUT IN GATED ROWS
//   logits | dx | dw HIDDEN VOCAB TOKENS
//   vocab HIDDEN VOCAB TOKENS GRAD
#include <cinttypes>
#include <cstdio>
#include <cstring>

#include "host/train.hpp"

int main() {
  char line[256], kind[32];
  while (std::fgets(line, sizeof line, stdin)) {
    long long a[6] = {0, 0, 0, 0, 0, 0};
    std::sscanf(line, "%31s %lld %lld %lld %lld %lld %lld", kind, a, a + 1, a + 2, a + 3, a + 4, a + 5);
    if (!std::strcmp(kind, "grouped")) {
      ccl::GroupedShape s;
      s.experts = (int)a[1];
      s.out = a[2];
      s.in = a[3];
      s.gated = a[4] != 0;
      const ccl::GroupedForm f = ccl::grouped_form(s, a[5], (int)a[0]);
      std::printf("tile_m=%d tile_n=%d splits=%d tiles=%" PRId64 " workgroups=%" PRId64 " chunk=%d bytes=%" PRId64 "\n", f.tile_m,
                  f.tile_n, f.splits, f.tiles, f.workgroups, f.chunk, f.workspace_bytes);
    } else {
      ccl::VocabShape s;
      s.hidden = s.w_ld = a[0];
      s.vocab = a[1];
      if (!std::strcmp(kind, "vocab")) {
        const ccl::VocabForm f = ccl::vocab_form(s, a[2], a[3] != 0);
        std::printf("block=%" PRId64 " blocks=%" PRId64 " bytes=%" PRId64 "\n", f.block, f.blocks, f.workspace_bytes);
      } else {
        const ccl::ProductForm f = !std::strcmp(kind, "logits") ? ccl::vocab_logits_form(s, a[2])
                                   : !std::strcmp(kind, "dx")   ? ccl::vocab_dx_form(s, a[2])
                                                                : ccl::vocab_dw_form(s, a[2]);
        std::printf("tile_m=%d tile_n=%d splits=%d tiles=%" PRId64 " workgroups=%" PRId64 " chunk=%d bytes=%" PRId64 "\n", f.tile_m,
                    f.tile_n, f.splits, f.tiles, f.workgroups, f.chunk, f.splits > 1 ? (int64_t)(4 * f.splits * a[2] * a[0]) : 0);
      }
    }
  }
  return 0;
}
