// The library's own rule for how a product is cut (lv_cut.h), for the tests' lists of sizes.
#include "lv_cut.h"

extern "C" void cut_of(const int32_t *hold, int64_t n_tok, int32_t d_in, int32_t d_out, int32_t gated, int64_t *out) {
  const int outputs = gated ? lv::kRows / 2 : lv::kRows;
  const int64_t row_tiles = (d_out + outputs - 1) / outputs, chunks = (d_in + lv::kPiece - 1) / lv::kPiece;
  const lv::Shape s = lv::choose([&](int n) { return (int64_t)hold[n]; }, n_tok, row_tiles, chunks);
  out[0] = s.pair;
  out[1] = s.tokens;
  out[2] = s.split;
  out[3] = (s.pair ? (row_tiles + 1) / 2 : row_tiles) * ((n_tok + s.tokens - 1) / s.tokens);
  out[4] = chunks;
}
