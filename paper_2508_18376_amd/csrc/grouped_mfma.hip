// Products over groups of rows on the tiles of grouped_tiles.h: which calls they take, and their launches.
#include "grouped_tiles.h"

namespace dsmoe {

bool grouped_mfma_fits(const GroupedArgs& g, int type, bool b_along) {
  if (type == kElemF32 || g.N % 8 != 0 || (type != kElemI8 && g.K % 8 != 0)) return false;
  const int64_t e = elem_bytes(type), oe = type == kElemI8 ? elem_bytes(g.out_type) : e;
  return rows_fit(g.a, g.a_row, g.K * e) && rows_fit(g.b, g.b_row, (b_along ? g.K : g.N) * e) && (g.b_group & 15) == 0 && rows_fit(g.c, g.c_row, g.N * oe);
}
hipError_t launch_grouped_mfma(const GroupedArgs& g, int type, bool b_along, hipStream_t s) {
  if (type == kElemI8)
    return g.out_type == kElemF32    ? launch_rows<kElemI8, kElemF32, false>(g, s)
           : g.out_type == kElemBF16 ? launch_rows<kElemI8, kElemBF16, false>(g, s)
                                     : launch_rows<kElemI8, kElemF16, false>(g, s);
  if (type == kElemBF16) return b_along ? launch_rows<kElemBF16, kElemBF16, false>(g, s) : launch_rows<kElemBF16, kElemBF16, true>(g, s);
  return b_along ? launch_rows<kElemF16, kElemF16, false>(g, s) : launch_rows<kElemF16, kElemF16, true>(g, s);
}

size_t grouped_split_bytes(const GroupedArgs& g, int type) {
  const int BM = tile_rows(g, type);
  return (size_t)(rows_room(g, type, BM).parts * (kPartialBytes / kGT * BM));
}
size_t grouped_dw_split_bytes(const GroupedArgs& g) {
  const Split s = split_of(dw_tiles(g), dw_stages(g), kGT, split_room(dw_tiles(g), dw_stages(g), kGT));
  return (size_t)((s.cols ? 0 : dw_tiles(g) - s.whole) * s.parts * kPartialBytes);
}

bool grouped_dw_mfma_fits(const GroupedArgs& g, int type) {
  if (type == kElemF32 || g.M % 8 != 0 || g.N % 8 != 0) return false;
  return rows_fit(g.a, g.a_row, g.M * 2ll) && rows_fit(g.b, g.b_row, g.N * 2ll) && rows_fit(g.c, g.c_row, g.N * 2ll) && (g.c_group & 15) == 0;
}
hipError_t launch_grouped_dw_mfma(const GroupedArgs& g, int type, hipStream_t s) {
  return type == kElemBF16 ? launch_dw<kElemBF16>(g, s) : launch_dw<kElemF16>(g, s);
}

}  // namespace dsmoe
