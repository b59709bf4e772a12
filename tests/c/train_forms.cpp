// What the training operators launch, from the library's own rules: one question a
// line on stdin, one answer a line on stdout.
//   grouped DIRECTION EXPERTS OUT IN GATED ROWS
//   logits | dx | dw, and logits_rest | dx_rest | dw_rest HIDDEN VOCAB TOKENS (rest: of the columns, or
//     tokens of dX, behind those in whole rounds of 256x256 tiles; 0 tiles where there are none)
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
        const bool dw = kind[1] == 'w', dx = kind[1] == 'x', rest = std::strstr(kind, "rest") != nullptr;
        const int64_t large = dw ? ccl::vocab_dw_large(s, a[2]) : dx ? ccl::vocab_dx_large(s, a[2]) : ccl::vocab_logits_large(s, a[2]);
        const int64_t all = dx ? a[2] : s.vocab, columns = rest ? (large ? all - large : 0) : large ? large : all;
        if (!columns) {
          std::printf("tile_m=0 tile_n=0 splits=1 tiles=0 workgroups=8 chunk=1 bytes=0\n");
          continue;
        }
        const ccl::ProductForm f = dx   ? ccl::vocab_dx_form(s, columns, large && !rest)
                                   : dw ? ccl::vocab_dw_form(s, a[2], columns, large && !rest)
                                        : ccl::vocab_logits_form(s, a[2], columns, large && !rest);
        std::printf("tile_m=%d tile_n=%d splits=%d tiles=%" PRId64 " workgroups=%" PRId64 " chunk=%d bytes=%" PRId64 "\n", f.tile_m,
                    f.tile_n, f.splits, f.tiles, f.workgroups, f.chunk, f.splits > 1 ? (int64_t)(4 * f.splits * columns * a[0]) : 0);
      }
    }
  }
  return 0;
}
