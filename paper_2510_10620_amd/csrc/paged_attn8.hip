// Attention of one new token per sequence over a paged key-value cache in 8 bits.
#include "paged_tile8.h"

using namespace dcp;

namespace dcp {

namespace {

template <typename IO, int COLS>
void launch8(int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s) {
  if (d == 128) launch_tiles<Tile8<IO, 128>, COLS>(grid, c, a, parts, s);
  else if (d == 64) launch_tiles<Tile8<IO, 64>, COLS>(grid, c, a, parts, s);
  else launch_tiles<Tile8<IO, 32>, COLS>(grid, c, a, parts, s);
}

}  // namespace

void launch_paged_attn8(int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s) {
  if (c.io_bytes == 4) launch8<float, 16>(d, grid, c, a, parts, s);
  else if (a.group <= 8) launch8<bf16_t, 8>(d, grid, c, a, parts, s);
  else launch8<bf16_t, 16>(d, grid, c, a, parts, s);
}

}  // namespace dcp
