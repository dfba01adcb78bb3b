// Products with weights in 4 bits: which calls go where.
#include "int4_matmul.h"

namespace dsmoe {

namespace {

// few rows a group
bool short_sizes(const Int4Args& a) { return a.type != kElemF32 && a.R <= 64 * (int64_t)a.G; }

}  // namespace

size_t int4_workspace_bytes(const Int4Args& a) { return a.type == kElemF32 || a.R == 0 ? 0 : short_sizes(a) ? int4_short_bytes(a) : int4_tiles_bytes(a); }

hipError_t launch_int4_matmul(const Int4Args& a, hipStream_t s) {
  if (short_sizes(a) && int4_short_fits(a)) return launch_int4_short(a, s);
  if (!short_sizes(a) && int4_tiles_fit(a)) return launch_int4_tiles(a, s);
  return int4_stream_fits(a) ? launch_int4_stream(a, s) : launch_int4_plain(a, s);
}

}  // namespace dsmoe
