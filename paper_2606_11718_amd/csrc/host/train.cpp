#include "train.hpp"

#include <algorithm>

namespace ccl {

namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of `tiles` dealt to the 8 XCDs in runs of `chunk`.
int64_t dealt(int64_t tiles, int64_t chunk) { return 8 * chunk * up(tiles, 8 * chunk); }

}  // namespace

GroupedForm grouped_form(const GroupedShape& s, int64_t rows, int direction) {
  GroupedForm f;
  f.tile_m = f.tile_n = 128;
  f.chunk = 32;
  int64_t tiles;
  if (direction == GROUPED_WGRAD) {
    f.tiles_m = (int32_t)up(s.out, f.tile_m);
    f.tiles_n = (int32_t)up(s.in, f.tile_n);
    tiles = (int64_t)s.experts * f.tiles_m * f.tiles_n;
  } else {
    f.tiles_n = (int32_t)up(direction == GROUPED_FORWARD ? s.out : s.in, f.tile_n);
    // at most: every expert with rows has one tile that is not whole
    tiles = (rows / f.tile_m + std::min<int64_t>(s.experts, rows)) * f.tiles_n;
  }
  f.workgroups = dealt(tiles, f.chunk);
  return f;
}

namespace {

constexpr int64_t kKeptBytes = (int64_t)4 << 30;   // of exp(z - tile max) at once
constexpr int64_t kLossBlock = 16384;              // tokens at once at most

ProductForm product_form(int64_t m, int64_t n, int tile_m, int tile_n, int64_t ksteps, int splits) {
  ProductForm f;
  f.tile_m = tile_m;
  f.tile_n = tile_n;
  f.tiles_m = (int32_t)up(m, tile_m);
  f.tiles_n = (int32_t)up(n, tile_n);
  f.group = 8;
  f.chunk = 32;
  f.ksplit = (int32_t)up(ksteps, splits);
  f.splits = (int32_t)up(ksteps, f.ksplit);
  f.workgroups = dealt((int64_t)f.tiles_m * f.tiles_n * f.splits, f.chunk);
  return f;
}

}  // namespace

// 256x256 tiles where they are not mostly padding and fill the CUs.
bool large_tiles(int64_t m, int64_t n, int splits = 1) {
  return up(m, 256) * 256 <= up(m, 128) * 128 * 5 / 4 && up(m, 256) * up(n, 256) * splits >= 256;
}

ProductForm vocab_logits_form(const VocabShape& s, int64_t tokens) {
  if (large_tiles(tokens, s.vocab)) return product_form(tokens, s.vocab, 256, 256, up(s.hidden, 64), 1);
  return product_form(tokens, s.vocab, tokens <= 64 ? 64 : 128, 128, up(s.hidden, 64), 1);
}

ProductForm vocab_dx_form(const VocabShape& s, int64_t tokens) {
  if (large_tiles(tokens, s.hidden)) return product_form(tokens, s.hidden, 256, 256, up(s.vocab, 64), 1);
  const int tile_m = tokens <= 64 ? 64 : 128;
  const int64_t tiles = up(tokens, tile_m) * up(s.hidden, 128);
  const int64_t splits = tiles >= 512 ? 1 : std::min<int64_t>(std::min<int64_t>(up(512, tiles), 64), up(s.vocab, 1024));
  return product_form(tokens, s.hidden, tile_m, 128, up(s.vocab, 64), (int)splits);
}

ProductForm vocab_dw_form(const VocabShape& s, int64_t tokens) {
  if (large_tiles(s.vocab, s.hidden)) return product_form(s.vocab, s.hidden, 256, 256, up(tokens, 64), 1);
  return product_form(s.vocab, s.hidden, 128, 128, up(tokens, 64), 1);
}

VocabForm vocab_form(const VocabShape& s, int64_t tokens, bool grad) {
  VocabForm f;
  f.e_cols = (int32_t)(up(s.vocab, 64) * 64);
  f.e_ld = f.e_cols + 64;      // rows a power of two apart would share memory channels
  int64_t most = s.block ? s.block : kLossBlock;
  if (!s.block && grad) most = std::min(most, std::max<int64_t>(256, kKeptBytes / (2 * f.e_ld) / 256 * 256));
  f.blocks = std::max<int64_t>(1, up(tokens, most));
  f.block = s.block ? std::min(s.block, tokens) : std::min(tokens, up(up(tokens, f.blocks), 256) * 256);
  f.blocks = f.block ? up(tokens, f.block) : 0;
  int64_t at = 0;
  const auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up(bytes, 256) * 256;
    return here;
  };
  f.target_at = take(4 * f.block);
  f.factor_at = take(8 * f.block);
  f.stat_at = take(8 * f.block * up(s.vocab, 128));      // the narrowest tiles'
  if (grad) {
    f.e_at = take(2 * f.block * f.e_ld);
    f.rows_at = take(2 * f.block * s.hidden);
    // the last block may be cut into more ranges than the others
    int64_t part = 0;
    for (int64_t t : {f.block, tokens - (f.blocks - 1) * f.block})
      if (t > 0) {
        const ProductForm d = vocab_dx_form(s, t);
        if (d.splits > 1) part = std::max(part, 4 * d.splits * t * s.hidden);
      }
    f.part_at = take(part);
    f.sum_at = take(f.blocks > 1 ? 4 * s.vocab * s.hidden : 0);
  }
  f.workspace_bytes = at;
  return f;
}

}  // namespace ccl
