// Launch rules of the operators of a training step around the FFN products
// (grouped experts' products, vocabulary loss, AdamW). Plain C++, no HIP.
#pragma once

#include <cstdint>

namespace ccl {

// ---- experts' products on rows sorted by expert ----
constexpr int kGroupedMaxExperts = 512;       // eight a lane of the wave that makes a workgroup's table
enum GroupedDirection { GROUPED_FORWARD = 0, GROUPED_GRAD = 1, GROUPED_WGRAD = 2 };
struct GroupedShape {
  int64_t in = 0, out = 0;                    // K, N: an expert's weight is N x K
  int experts = 0, act = 0;
  bool gated = false;
  int64_t w_ld = 0, w_stride = 0;             // elements
};
struct GroupedForm {
  int tile_m = 0, tile_n = 0;
  int32_t tiles_m = 0, tiles_n = 0;           // tiles_m: of a weight gradient
  int32_t chunk = 1;                          // consecutive tiles of one XCD
  int32_t splits = 1;                         // K ranges of a tile
  int64_t tiles = 0;                          // at most, of all ranges
  int64_t workgroups = 0, workspace_bytes = 0;
};
GroupedForm grouped_form(const GroupedShape& s, int64_t rows, int direction);
// Workspace for that many rows or fewer (fewer may be cut into more ranges).
int64_t grouped_workspace(const GroupedShape& s, int64_t rows, int direction);

// ---- vocabulary loss ----
constexpr int64_t kVocabMaxBlock = 32768;     // the scaling pass has a grid row a token
struct VocabShape {
  int64_t hidden = 0, vocab = 0, w_ld = 0;
  int64_t block = 0;                          // tokens at once, 0: chosen
  float scale = 1.f;
};
// A product's tiles of one kind, dealt to the XCDs in a raster of `group` tile
// rows, and its K ranges.
struct ProductForm {
  int tile_m = 0, tile_n = 0;
  int32_t tiles_m = 0, tiles_n = 0, group = 1, chunk = 1;
  int32_t splits = 1, ksplit = 0;             // ksplit: steps of 64 K a range
  int64_t tiles = 0, workgroups = 0;          // tiles: of all ranges
};
struct VocabForm {
  int64_t block = 0, blocks = 0;              // tokens at once (the last block may have fewer)
  int64_t e_ld = 0;                           // elements between rows of exp(z - tile max)
  int32_t e_cols = 0;                         // of which whole 64s are used
  // bytes into the workspace
  int64_t target_at = 0, factor_at = 0, stat_at = 0, e_at = 0, rows_at = 0, part_at = 0, sum_at = 0, workspace_bytes = 0;
};
// The blocks and the workspace, which fewer tokens do not exceed; grad: with
// exp(z - tile max) kept for a block, a copy of its x, the ranges' partial dX and,
// where dW is rounded after several blocks, its fp32 sum.
VocabForm vocab_form(const VocabShape& s, int64_t tokens, bool grad);
// The products of a block of `tokens`: logits and dW, each in 256x256 tiles over the
// first vocab_..._large columns of the vocabulary (whole tiles, or all, or 0) and in
// smaller ones over the others.
int64_t vocab_logits_large(const VocabShape& s, int64_t tokens);
int64_t vocab_dw_large(const VocabShape& s, int64_t tokens);
ProductForm vocab_logits_form(const VocabShape& s, int64_t tokens, int64_t columns, bool large);
ProductForm vocab_dw_form(const VocabShape& s, int64_t tokens, int64_t columns, bool large);
// dX of the first vocab_dx_large tokens, and of the others (all, if that is 0), in two calls.
int64_t vocab_dx_large(const VocabShape& s, int64_t tokens);
ProductForm vocab_dx_form(const VocabShape& s, int64_t tokens, bool large);

// ---- AdamW ----
constexpr int kAdamwTensors[2] = {68, 54};    // of a launch (moments of 32, 8 bits): their table is a kernel argument
constexpr int kAdamwBlock = 128;              // elements of 8-bit moments that share a scale

// beta^step, the same bits on the host and the device: by squaring, in double.
#if defined(__HIPCC__)
__host__ __device__
#endif
inline double power_of(double beta, int64_t step) {
  double p = 1.0;
  for (double b = beta; step > 0; step >>= 1, b *= b)
    if (step & 1) p *= b;
  return p;
}

}  // namespace ccl
