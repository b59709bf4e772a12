// What the FFN operators launch, by the library's own rules. One question a
// line of stdin, one line of name=value pairs each:
//   ortho batch rows cols
//   moe tokens hidden ffn experts top_k fp8
//   fused M N K chiplets grid_rows page fp8 rowmajor splits grad gated dbias rows moved
#include <cstdio>
#include <cstring>
#include <string>

#include "plan.hpp"

using namespace ccl;

static void product(const char* name, const OrthoSplit& s) {
  std::printf("%s_tile=%d %s_paired=%d %s_whole=%d %s_ranges=%d ", name, s.tile, name, (int)s.paired, name, (int)s.whole, name,
              (int)s.splits);
}

int main() {
  char line[256], kind[16];
  while (std::fgets(line, sizeof line, stdin)) {
    long long v[14] = {0};
    int n = 0, used = 0;
    if (std::sscanf(line, "%15s%n", kind, &used) != 1) continue;
    for (char* at = line + used; n < 14 && std::sscanf(at, "%lld%n", &v[n], &used) == 1; at += used) ++n;
    if (!std::strcmp(kind, "ortho") && n == 3) {
      const OrthoForm f = ortho_form({v[0], v[1], v[2]});
      product("gram", f.gram);
      product("square", f.square);
      product("update", f.update);
      std::printf("pp=%d qp=%d\n", (int)f.pp, (int)f.qp);
    } else if (!std::strcmp(kind, "moe") && n == 6) {
      MoeShape s;
      s.hidden = v[1];
      s.ffn = v[2];
      s.experts = (int)v[3];
      s.top_k = (int)v[4];
      s.fp8 = v[5] != 0;
      const MoeForm f = moe_form(s, v[0]);
      std::printf("list=%d up_tiles=%d up_group=%d up_workgroups=%lld down_nt=%d down_tiles=%d down_groups=%d ranges=%d\n", (int)f.list,
                  f.up_tiles, f.up_group, (long long)f.up_workgroups, f.down_nt, f.down_tiles, f.down_groups, f.splits);
    } else if (!std::strcmp(kind, "fused") && n == 14) {
      Plan p;
      std::string why;
      const DType ab = v[6] ? DT_FP8_E4M3 : DT_BF16;
      if (make_plan(v[0], v[1], v[2], (int)v[3], (int)v[4], v[5], ab, DT_BF16, &p, &why) != Status::OK) return 2;
      const FusedForm f = fused_form(p, v[7] != 0, (int)v[8], v[9] != 0, v[10] != 0, v[11] != 0, v[12], (int)v[13]);
      const GemmForm& g = f.gemm;
      std::printf("kernel=%s tile_m=%d tile_n=%d waves=%d ranges=%d far=%d own=%d direct=%d remap=%d ragged=%d stream_b=%d\n",
                  kernel_name(g.kernel), g.tile_m, g.tile_n, g.waves, g.splits, (int)g.far, (int)f.own, (int)f.direct, (int)f.remap,
                  (int)g.ragged, (int)g.stream_b);
    } else {
      return 1;
    }
  }
  return 0;
}
