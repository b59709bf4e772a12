// Launch rules of the operators of a training step around the FFN products
// (grouped experts' products, vocabulary loss, AdamW). Plain C++, no HIP.
#pragma once

#include <cstdint>

namespace ccl {

// ---- experts' products on rows sorted by expert ----
constexpr int kGroupedMaxExperts = 512;       // one thread each finds a workgroup's tile
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
  int64_t workgroups = 0, workspace_bytes = 0;
};
GroupedForm grouped_form(const GroupedShape& s, int64_t rows, int direction);

}  // namespace ccl
