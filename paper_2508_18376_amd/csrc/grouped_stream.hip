// Products over groups of few rows by the kernels of grouped_streams.h: which calls they take, and their launches.
#include "grouped_streams.h"

namespace dsmoe {

// Which calls these kernels take (all times: this path against the other one, us; rows are a group's on average, the groups ragged as routing makes them, and
// the calls take three sets of inputs in turn).
//   16-bit types and 8-bit integers whose rows start on 16 bytes, against the tiles of grouped_tiles.h, which read weights through LDS: up to 12 rows
//     a group on average, 2 where 16-bit weights lie along the contraction.  y = x W on 64 experts of 2048 x 1024 at 1 / 8 / 16 rows 42 / 57 / 59
//     against 41 / 54 / 56, on 64 of 2048 x 1408 at 6 / 12 / 24 rows 57 / 59 / 65 against 72 / 72 / 75, on 8 of 4096 x 14336 at 4 / 12 / 16 rows
//     157 / 161 / 163 against 162 / 165 / 166; gradient of x on the first at 1 / 2 / 12 rows 36 / 46 / 53 against 40 / 47 / 52, on the last at 2 / 12
//     rows 181 / 198 against 169 / 186; 8 bits on the first at 1 / 4 / 12 / 16 rows 25 / 29 / 39 / 45 against 32 / 29 / 38 / 40, on the last 66 / 90 / 104 /
//     115 against 79 / 107 / 112 / 117.
//     Few pieces of long sums keep too few compute units busy, which split tiles do not: 12 rows of 14336 values, 4096 columns 70 against 36;
//     of 4096 values, 4096 columns 15.5 against 22.
//   Rows that start elsewhere, against grouped_plain.h: across, up to 16 rows a group (33 groups of 1001 x 1409 at 8 / 16 / 24 rows 31 / 33 / 40 against
//     39 / 38 / 38) or few tiles (256 rows of 1001 x 1409 in one group 12 against 20, 512 rows 23 against 20); along, 8 rows a group where the tiles
//     would not fill the card (8 groups of 2047 x 4093 56 against 89; 33 of 1001 x 1409, 264 tiles, 62 against 53).
//   fp32, against grouped_plain.h: up to 64 rows a group (48 along), or few tiles: 16 experts of 2048 x 1408 at 32 / 64 / 96 rows 66 / 100 / 129 against
//     147 / 145 / 148, along 74 / 106 / 150 against 106 / 107 / 106; 64 of 1024 x 1024 at 64 / 96 rows 133 / 191 against 149 / 151; 8 of 4096 x 4096 at
//     32 / 64 / 96 rows 196 / 284 / 387 against 300 / 290 / 294, along 240 / 346 / 477 against 290 / 287 / 288; 64 / 256 / 512 rows of 4096 x 4096 in one
//     group 52 / 97 / 180 against 277 / 284 / 286.
bool grouped_stream_sizes(const GroupedArgs& g, int type, bool b_along, bool tiles_fit) {
  if (!launch_holds(g, type, b_along, tiles_fit)) return false;
  const int64_t tiles = row_tiles_bound(g.R, g.G, g.off != nullptr, 128) * ((g.N + 127) / 128);
  if (type == kElemF32) return g.R <= (b_along ? 48 : 64) * (int64_t)g.G || tiles < 320;
  if (!tiles_fit) {
    if (b_along && type != kElemI8) return g.R <= 8 * (int64_t)g.G && tiles < 256;
    return g.R <= 16 * (int64_t)g.G || (!b_along && tiles < 64);
  }
  const bool few = g.R <= (b_along && type != kElemI8 ? 2 : 12) * (int64_t)g.G;
  const int64_t pieces = row_tiles_bound(g.R, g.G, g.off != nullptr, kStreamTile) * ((g.N + 63) / 64);
  return few && ((int64_t)g.K * elem_bytes(type) <= 16384 || (!b_along && pieces >= 128));
}
bool grouped_stream_fits(const GroupedArgs& g, int type, bool b_along) {
  const int64_t most = (int64_t)1 << 24;  // 64 rows of it are below 2^32
  return g.a_row <= most && g.b_row <= most && grouped_stream_sizes(g, type, b_along, grouped_mfma_fits(g, type, b_along));
}
hipError_t launch_grouped_stream(const GroupedArgs& g, int type, bool b_along, hipStream_t s) {
  switch (type) {
    case kElemF32: return b_along ? launch_w<kElemF32, kElemF32, false>(g, s) : launch_w<kElemF32, kElemF32, true>(g, s);
    case kElemBF16: return b_along ? launch_w<kElemBF16, kElemBF16, false>(g, s) : launch_w<kElemBF16, kElemBF16, true>(g, s);
    case kElemF16: return b_along ? launch_w<kElemF16, kElemF16, false>(g, s) : launch_w<kElemF16, kElemF16, true>(g, s);
    default:
      return g.out_type == kElemF32    ? launch_w<kElemI8, kElemF32, false>(g, s)
             : g.out_type == kElemBF16 ? launch_w<kElemI8, kElemBF16, false>(g, s)
                                       : launch_w<kElemI8, kElemF16, false>(g, s);
  }
}

}  // namespace dsmoe
