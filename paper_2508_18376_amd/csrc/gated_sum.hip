// dx = da W1^T + db W3^T over groups of rows: one contraction, first along the columns of the one weight, then along the other's (tiles, streams and the plain
// path of grouped_tiles.h, grouped_streams.h and grouped_plain.h), so that the sum stays in registers and dx is rounded once.
// Bound by the matrix cores: 8192 rows on 8 experts of 4096 x 14336 1602 us with the launch that joins parts, 1201 TFLOP/s; 65536 rows on 64 of 2048 x 1024 508 us,
// 1083 TFLOP/s.
#include "gated.h"
#include "grouped_plain.h"
#include "grouped_streams.h"
#include "grouped_tiles.h"

namespace dsmoe {

namespace {

bool tiles_fit(const GroupedArgs& g, int type) {
  if (type == kElemF32 || g.N % 8 != 0 || g.K % 8 != 0) return false;
  return rows_fit(g.a, g.a_row, g.K * 2ll) && rows_fit(g.a2, g.a_row, g.K * 2ll) && rows_fit(g.b, g.b_row, g.K * 2ll) && rows_fit(g.b2, g.b_row, g.K * 2ll) &&
         (g.b_group & 15) == 0 && rows_fit(g.c, g.c_row, g.N * 2ll);
}

// Streams against tiles, the whole backward pass, as many rows in each group: 1 / 12 / 24 rows on 64 experts of 2048 x 1024 275 / 280 / 285 us against 282 / 288 /
// 289, on 8 of 4096 x 14336 777 / 824 / 867 against 818 / 831 / 831, on 8 of 14336 x 4096 726 / 778 / 821 against 814 / 837 / 848; long sums in few
// pieces keep too few compute units busy: 1 / 12 rows of 4096 x 14336 in one group 193 / 209 against 163 / 164.
bool stream_sizes(const GroupedArgs& g, int type, bool fit) {
  if (!launch_holds(g, type, true, fit)) return false;
  const int64_t tiles = row_tiles_bound(g.R, g.G, g.off != nullptr, 128) * ((g.N + 127) / 128);
  if (type == kElemF32) return g.R <= 48 * (int64_t)g.G || tiles < 320;
  if (!fit) return g.R <= 8 * (int64_t)g.G && tiles < 256;
  const int64_t pieces = row_tiles_bound(g.R, g.G, g.off != nullptr, kStreamTile) * ((g.N + 63) / 64);
  return g.R <= 12 * (int64_t)g.G && ((int64_t)g.K * 2 <= 16384 || pieces >= 256);
}

template <int TY>
hipError_t launch_one(const GroupedArgs& g, hipStream_t s) {
  const int64_t most = (int64_t)1 << 24;
  const bool fit = tiles_fit(g, TY);
  if (g.a_row <= most && g.b_row <= most && stream_sizes(g, TY, fit)) return launch_w<TY, TY, false, kSumOfTwo>(g, s);
  if constexpr (TY != kElemF32) {
    if (fit) return launch_rows<TY, TY, false, kSumOfTwo>(g, s);
  }
  return launch<TY, false, false, kSumOfTwo>(g, row_tiles_bound(g.R, g.G, g.off != nullptr, kPT) * ((g.N + kPT - 1) / kPT), s);
}

}  // namespace

size_t sum_of_two_bytes(const GroupedArgs& g, int type) {
  if (type == kElemF32 || g.R == 0 || stream_sizes(g, type, true)) return 0;
  const int BM = tile_rows(g, type, kSumOfTwo);
  return (size_t)(rows_room(g, type, BM, kSumOfTwo).parts * (kPartialBytes / kGT * BM));
}

hipError_t launch_sum_of_two(const GroupedArgs& g, int type, hipStream_t s) {
  return type == kElemF32 ? launch_one<kElemF32>(g, s) : type == kElemBF16 ? launch_one<kElemBF16>(g, s) : launch_one<kElemF16>(g, s);
}

}  // namespace dsmoe
