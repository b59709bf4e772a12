#include "train.hpp"

#include <algorithm>

namespace ccl {

namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// fp32 tiles of all K ranges of a product, at most: ranges are made while tiles times
// ranges fit 512 workgroups of 128 x 128, or 256 of 256 x 256.
constexpr int64_t kPartBytes = (int64_t)512 * 128 * 128 * 4, kLargePartBytes = (int64_t)256 * 256 * 256 * 4;
constexpr int kMaxRanges = 64;
int64_t part_bound(int64_t elems, int64_t most) { return std::min<int64_t>(most, 4 * kMaxRanges * elems); }

// Workgroups that stay and take `tiles` in turn, per_cu of them on a CU; one for
// every tile where there are fewer (a multiple of 8: XCDs).
int64_t resident(int64_t tiles, int per_cu) { return std::min<int64_t>(up(std::max<int64_t>(tiles, 1), 8) * 8, 256 * per_cu); }

}  // namespace

// Tiles, measured (us, 256x256 against 128x128 tiles, of which two workgroups share a
// CU): a large tile moves half as much through LDS for each product, but hides
// neither its rows' padding nor its wait for memory behind another workgroup.
//   forward  32768 rows over 128 experts of 2048 -> 1536 322 / 331, 16384 272 / 246,
//            8192 over 8 104 / 74 (fewer tiles than CUs), over one of 4096 -> 4096
//            218 / 278
//   grad     32768 over 128 of 768 -> 2048 through SwiGLU 258 / 213 (three tiles a CU,
//            uneven), 65536 372 / 369, 8192 over one of 4096 -> 4096 235 / 288
//   wgrad    32768 over 128 of 2048 -> 1536 376 / 470, 4096 172 / 230, 128 160 / 195,
//            8192 over one 223 / 288, 65536 over 4 of 256 -> 256 334 / 181 (4 tiles an
//            expert)
// All of these sides are multiples of 256, and the rule has no term for padding: a dW
// of 128 experts of 288 x 288 is taken in 256x256 tiles, which compute 512 x 512 of it
// (128x128 ones 384 x 384).
// 64x128 ones, with a third stage on its way, where few rows come to an expert (against
// 128x128): 64 rows 58 / 71 (forward as above), 1024 165 / 187, 8192 199 / 230, 12000
// 220 / 223, its grad 133 / 126.
GroupedForm grouped_form(const GroupedShape& s, int64_t rows, int direction) {
  GroupedForm f;
  const bool wgrad = direction == GROUPED_WGRAD;
  const int64_t n = direction == GROUPED_FORWARD ? s.out : s.in;
  const int64_t used = std::max<int64_t>(1, std::min<int64_t>(s.experts, rows)), mean = rows / used;
  const auto tiles = [&](int64_t tm, int64_t tn) {
    // at most: every expert with rows has one row tile that is not whole
    return wgrad ? s.experts * up(s.out, tm) * up(s.in, tn) : (rows / tm + std::min<int64_t>(s.experts, rows)) * up(n, tn);
  };
  const int64_t large = tiles(256, 256);
  if (wgrad ? large >= 256 : (mean >= 512 && large >= (direction == GROUPED_FORWARD ? 256 : 512)) ||
                                 (direction == GROUPED_FORWARD && mean >= 192 && large >= 512))
    f.tile_m = f.tile_n = 256;
  else {
    f.tile_m = wgrad || mean >= 80 ? 128 : 64;
    f.tile_n = 128;
  }
  const int per_cu = f.tile_m == 256 ? 1 : 2;
  if (wgrad) f.tiles_m = (int32_t)up(s.out, f.tile_m);
  f.tiles_n = (int32_t)up(wgrad ? s.in : n, f.tile_n);
  f.tiles = tiles(f.tile_m, f.tile_n);
  // K ranges where tiles leave half of the workgroups without one, of four steps of
  // 64 K at least; their fp32 sums are added up by a second launch.
  const int64_t steps = wgrad ? mean / 64 : up(direction == GROUPED_FORWARD ? s.in : s.out, 64);
  const int64_t fit = 256 * per_cu / std::max<int64_t>(f.tiles, 1);
  if (fit >= 2 && steps >= 8) {
    f.splits = (int32_t)std::min<int64_t>(std::min(fit, steps / 4), kMaxRanges);
    f.tiles *= f.splits;
    f.workspace_bytes = 4 * f.splits * (wgrad ? s.experts * s.out * s.in : rows * n);
  }
  // Runs of 16 tiles an XCD, against 32 and 64: 321 / 326 / 326 us (forward above). A
  // round has to be whole runs on each of the 8, or its tiles would not all be dealt.
  constexpr int kRun = 16;
  f.workgroups = resident(f.tiles, per_cu);
  if (f.workgroups > 8 * kRun) f.workgroups = up(f.workgroups, 8 * kRun) * 8 * kRun;
  f.chunk = (int32_t)std::min<int64_t>(kRun, f.workgroups / 8);
  return f;
}

int64_t grouped_workspace(const GroupedShape& s, int64_t rows, int direction) {
  const int64_t k = direction == GROUPED_WGRAD ? rows : direction == GROUPED_FORWARD ? s.in : s.out;
  if (up(k, 64) < 8 || rows == 0) return 0;
  return part_bound(direction == GROUPED_WGRAD ? s.experts * s.out * s.in : rows * (direction == GROUPED_FORWARD ? s.out : s.in),
                    kPartBytes);
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
  f.ksplit = (int32_t)up(ksteps, splits);
  f.splits = (int32_t)up(ksteps, f.ksplit);
  const int per_cu = tile_m == 256 ? 1 : 2;
  f.tiles = (int64_t)f.tiles_m * f.tiles_n * f.splits;
  f.workgroups = resident(f.tiles, per_cu);
  f.chunk = (int32_t)std::min<int64_t>(32 * per_cu, f.workgroups / 8);
  return f;
}

// 256x256 tiles where they are not mostly padding and, `ranges` of them, fill the CUs.
bool large_tiles(int64_t m, int64_t n, int64_t ranges = 1) {
  return up(m, 256) * 256 <= up(m, 128) * 128 * 5 / 4 && up(m, 256) * up(n, 256) * ranges >= 256;
}

// Of n columns (of the vocabulary, or tokens) by m, those whose 256x256 tiles are whole
// rounds of the 256 CUs, where the tiles of a last round that is not whole are a round
// or less of 128x128 ones: all otherwise. (Loss of 4096 tokens, 4096 x 4352 144 / 191 us
// in one piece, of 5461, 576 x 3216 44 / 52; with both gradients 1003 of 2048 x 50257
// 652 / 685, 1024 of 512 x 20000 131 / 140; no shape tried was slower.)
int64_t whole_rounds(int64_t n, int64_t m, int64_t k) {
  const int64_t across = up(m, 256), tiles = across * up(n, 256), whole = tiles / 256 * 256 / across * 256;
  if (tiles % 256 == 0 || whole == 0 || k < 512 || up(n - whole, 128) * up(m, 128) > 512) return n;
  return whole;
}

}  // namespace

// Few tiles wait for memory step by step: 64x128 ones while that is no more than one
// a CU (1000 tokens of 4096 x 1200 36.5 us, in tiles of 128x128 with as many stages as
// the LDS holds 41.9, with two 51.2; 135 of 4112 x 1381 36.4 / 43.3 / 58.5), and one
// 128x128 tile a CU with four stages where two would have two (250 of 4096 x 16000
// 46 / 65, 200 of 2048 x 16000 27 / 31; the kernel's choice).
ProductForm vocab_logits_form(const VocabShape& s, int64_t tokens, int64_t columns, bool large) {
  if (large) return product_form(tokens, columns, 256, 256, up(s.hidden, 64), 1);
  const bool few = tokens <= 64 || up(tokens, 64) * up(columns, 128) <= 256;
  return product_form(tokens, columns, few ? 64 : 128, 128, up(s.hidden, 64), 1);
}

int64_t vocab_logits_large(const VocabShape& s, int64_t tokens) {
  return large_tiles(tokens, s.vocab) ? whole_rounds(s.vocab, tokens, s.hidden) : 0;
}
int64_t vocab_dx_large(const VocabShape& s, int64_t tokens) {
  return large_tiles(tokens, s.hidden) ? whole_rounds(tokens, s.hidden, s.vocab) : 0;
}
int64_t vocab_dw_large(const VocabShape& s, int64_t tokens) {
  return large_tiles(s.vocab, s.hidden) ? whole_rounds(s.vocab, s.hidden, tokens) : 0;
}

// K ranges of 256x256 tiles against those of 128x128 ones, which are twice as many and
// leave half as much to add up (loss and both gradients): 1003 tokens of 2048 x 50257
// 681 / 730, 1024 of 1024 x 128000 908 / 982, 1500 of 2560 x 9000 270 / 278, but where a
// range is 1000 to 1250 columns 768 of 2048 x 8000 119 / 112, 4096 of 512 x 8000 195 / 174.
ProductForm vocab_dx_form(const VocabShape& s, int64_t tokens, bool large) {
  if (large) return product_form(tokens, s.hidden, 256, 256, up(s.vocab, 64), 1);
  const int64_t larges = up(tokens, 256) * up(s.hidden, 256);
  const int64_t ranges = std::min<int64_t>(std::min<int64_t>(256 / larges, kMaxRanges), s.vocab / 2048);
  if (larges * ranges >= 192 && large_tiles(tokens, s.hidden, 256))
    return product_form(tokens, s.hidden, 256, 256, up(s.vocab, 64), (int)ranges);
  const int tile_m = tokens <= 64 ? 64 : 128;
  const int64_t tiles = up(tokens, tile_m) * up(s.hidden, 128);
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / tiles, kMaxRanges), up(s.vocab, 1024)));
  return product_form(tokens, s.hidden, tile_m, 128, up(s.vocab, 64), (int)splits);
}

ProductForm vocab_dw_form(const VocabShape& s, int64_t tokens, int64_t columns, bool large) {
  const int tile = large ? 256 : 128;
  return product_form(columns, s.hidden, tile, tile, up(tokens, 64), 1);
}

VocabForm vocab_form(const VocabShape& s, int64_t tokens, bool grad) {
  VocabForm f;
  f.e_cols = (int32_t)(up(s.vocab, 64) * 64);
  f.e_ld = f.e_cols + 64;      // rows a power of two apart would share memory channels
  int64_t most = s.block ? s.block : kLossBlock;
  if (!s.block && grad) most = std::min(most, std::max<int64_t>(256, kKeptBytes / (2 * f.e_ld) / 256 * 256));
  f.block = std::min(tokens, most);
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
    f.part_at = take(part_bound(f.block * s.hidden, kLargePartBytes));
    f.sum_at = take(f.blocks > 1 ? 4 * s.vocab * s.hidden : 0);
  }
  f.workspace_bytes = at;
  return f;
}

}  // namespace ccl
