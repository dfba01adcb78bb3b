// Products with weights in 4 bits: which calls go where.
#include "int4_matmul.h"

namespace dsmoe {

hipError_t launch_int4_matmul(const Int4Args& a, hipStream_t s) {
  return int4_stream_fits(a) ? launch_int4_stream(a, s) : launch_int4_plain(a, s);
}

}  // namespace dsmoe
