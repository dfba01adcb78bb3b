// h = f(x W1) * (x W3) over groups of rows: both products of a tile in one workgroup, so that x is read once for the two, and the products are not written
// unless a backward pass asks for them.  Tiles, streams and the plain path are those of the single products (grouped_tiles.h, grouped_streams.h,
// grouped_plain.h): a tile has half as many columns, of both weights.  Bound as those are: a step of 64 tokens on 8 experts of 4096 x 14336 326 us, 5.8 TB/s; 8192
// rows there, with both sums written, 1745 us, 1102 TFLOP/s; 65536 rows on 64 experts of 2048 x 1024 592 us, 929 TFLOP/s and 3.9 TB/s at once.
#include "gated.h"
#include "grouped_plain.h"
#include "grouped_streams.h"
#include "grouped_tiles.h"

namespace dsmoe {

namespace {

bool tiles_fit(const GroupedArgs& g, int type) {
  if (type == kElemF32 || g.N % 8 != 0 || g.K % 8 != 0) return false;
  return rows_fit(g.a, g.a_row, g.K * 2ll) && rows_fit(g.b, g.b_row, g.N * 2ll) && rows_fit(g.b2, g.b_row, g.N * 2ll) && (g.b_group & 15) == 0 &&
         rows_fit(g.c, g.c_row, g.N * 2ll) && ((uintptr_t)g.sums & 15) == 0;
}

// As for the single product (grouped_stream.hip), but that the weights are two.  Streams against tiles, rows on 16 bytes, as many rows in each group: 1 / 12 / 32
// rows on 64 experts of 2048 x 1024 100 / 102 / 109 us against 106 / 106 / 108, on 8 of 4096 x 14336 307 / 314 / 341 against 344 / 344 / 348, on 64 of
// 2048 x 1408 107 / 109 / 122 against 127 / 129 / 132; 1 / 32 rows of 2048 x 1024 in one group 11 / 18 against 23 / 23.
bool stream_sizes(const GroupedArgs& g, int type, bool fit) {
  if (!launch_holds(g, type, false, fit)) return false;
  const int64_t tiles = row_tiles_bound(g.R, g.G, g.off != nullptr, 128) * ((g.N + 63) / 64);
  if (type == kElemF32) return g.R <= 64 * (int64_t)g.G || tiles < 320;
  if (!fit) return g.R <= 16 * (int64_t)g.G || tiles < 64;
  const int64_t pieces = row_tiles_bound(g.R, g.G, g.off != nullptr, kStreamTile) * ((g.N + 63) / 64);
  return g.R <= 24 * (int64_t)g.G && ((int64_t)g.K * 2 <= 16384 || pieces >= 128);
}

template <int TY>
hipError_t launch_one(const GroupedArgs& g, hipStream_t s) {
  const int64_t most = (int64_t)1 << 24;
  const bool fit = tiles_fit(g, TY);
  if (g.a_row <= most && g.b_row <= most && stream_sizes(g, TY, fit)) return launch_w<TY, TY, true, kGatedPair>(g, s);
  if constexpr (TY != kElemF32) {
    if (fit) return launch_rows<TY, TY, true, kGatedPair>(g, s);
  }
  return launch<TY, true, false, kGatedPair>(g, row_tiles_bound(g.R, g.G, g.off != nullptr, kPT) * ((g.N + kPT / 2 - 1) / (kPT / 2)), s);
}

}  // namespace

size_t gated_pair_bytes(const GroupedArgs& g, int type) {
  if (type == kElemF32 || g.R == 0 || stream_sizes(g, type, true)) return 0;
  const int BM = tile_rows(g, type, kGatedPair);
  return (size_t)(rows_room(g, type, BM, kGatedPair).parts * (kPartialBytes / kGT * BM));
}

hipError_t launch_gated_pair(const GroupedArgs& g, int type, hipStream_t s) {
  return type == kElemF32 ? launch_one<kElemF32>(g, s) : type == kElemBF16 ? launch_one<kElemBF16>(g, s) : launch_one<kElemF16>(g, s);
}

}  // namespace dsmoe
