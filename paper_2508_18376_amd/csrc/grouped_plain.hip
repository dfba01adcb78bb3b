// Products over groups of rows by the kernel of grouped_plain.h: launches.
#include "grouped_plain.h"

namespace dsmoe {

hipError_t launch_grouped_plain(const GroupedArgs& g, int type, bool b_along, hipStream_t s) {
  const int64_t blocks = row_tiles_bound(g.R, g.G, g.off != nullptr, kPT) * ((g.N + kPT - 1) / kPT);
  switch (type) {
    case kElemF32: return b_along ? launch<kElemF32, false, false>(g, blocks, s) : launch<kElemF32, true, false>(g, blocks, s);
    case kElemBF16: return b_along ? launch<kElemBF16, false, false>(g, blocks, s) : launch<kElemBF16, true, false>(g, blocks, s);
    case kElemF16: return b_along ? launch<kElemF16, false, false>(g, blocks, s) : launch<kElemF16, true, false>(g, blocks, s);
    default: return launch<kElemI8, false, false>(g, blocks, s);
  }
}

namespace {

// pair: one or both gradients of a gated pair
hipError_t launch_dw(const GroupedArgs& g, int type, bool pair, hipStream_t s) {
  const int64_t each = (int64_t)g.G * ((g.M + kPT - 1) / kPT) * ((g.N + kPT - 1) / kPT), blocks = g.c2 != nullptr ? 2 * each : each;
  if (g.c2 != nullptr && blocks * 256 >= (int64_t)1 << 32) {  // (a launch of 2^32 threads is silently cut short; of one product's tiles there are less)
    GroupedArgs one = g, two = g;
    one.c2 = two.c2 = nullptr;
    two.b = g.b2;
    two.c = g.c2;
    const hipError_t e = launch_dw(one, type, pair, s);
    return e != hipSuccess ? e : launch_dw(two, type, pair, s);
  }
  switch (type) {
    case kElemF32: return pair ? launch<kElemF32, true, true, kGatedPair>(g, blocks, s) : launch<kElemF32, true, true>(g, blocks, s);
    case kElemBF16: return launch<kElemBF16, true, true>(g, blocks, s);
    default: return launch<kElemF16, true, true>(g, blocks, s);
  }
}

}  // namespace

hipError_t launch_grouped_dw_plain(const GroupedArgs& g, int type, hipStream_t s) { return launch_dw(g, type, g.c2 != nullptr, s); }

}  // namespace dsmoe
