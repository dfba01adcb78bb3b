// Products with weights in 4 bits: which calls go where.
#include "int4_matmul.h"

namespace dsmoe {

namespace {

// The tiles of few rows against those of many (us; as many rows in each group): 96 / 192 / 256 rows a group on 8 groups of 4096 x 14336 172 / 264 / 327
// against 199 / 265 / 298, on 64 of 2048 x 1408 75 / 117 / 137 against 90 / 123 / 128; where the latter are too few for the card, up to more: 256 /
// 512 / 1024 rows of 4096 x 14336 in one group 60 / 93 / 178 against 92 / 96 / 130, of 1024 x 2048 17 / 19 / 24 against 25 / 25 / 26.
bool short_sizes(const Int4Args& a) {
  return a.type != kElemF32 && (a.R <= 192 * (int64_t)a.G || row_tiles_bound(a.R, a.G, a.off != nullptr, 256) * ((a.N + 255) / 256) <= 112);
}

// The streams against the tiles of few rows: pieces of a single round with a few steps for each wavefront.  1 / 16 rows of 4096 x 14336 13 / 15 us against
// 16 / 20, of 14336 x 4096 33 / 42 against 19 / 22; 8 rows on 8 groups of 2048 x 1408 10.6 against 13.1; 1 / 16 rows on 2 groups of 4096 x 14336, 448
// pieces, 26 / 31 against 23 / 28.
bool stream_sizes(const Int4Args& a) {
  return a.type != kElemF32 && a.R <= 16 * (int64_t)a.G && a.K <= 4096 && row_tiles_bound(a.R, a.G, a.off != nullptr, 16) * ((a.N + 63) / 64) <= 256;
}

}  // namespace

size_t int4_workspace_bytes(const Int4Args& a) { return a.type == kElemF32 || a.R == 0 || stream_sizes(a) ? 0 : short_sizes(a) ? int4_short_bytes(a) : int4_tiles_bytes(a); }

hipError_t launch_int4_matmul(const Int4Args& a, hipStream_t s) {
  if (stream_sizes(a) && int4_stream_fits(a)) return launch_int4_stream(a, s);
  if (short_sizes(a) && int4_short_fits(a)) return launch_int4_short(a, s);
  if (!short_sizes(a) && int4_tiles_fit(a)) return launch_int4_tiles(a, s);
  return int4_stream_fits(a) ? launch_int4_stream(a, s) : launch_int4_plain(a, s);
}

}  // namespace dsmoe
