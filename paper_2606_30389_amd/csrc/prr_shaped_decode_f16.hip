// Attention of single tokens with shaped scores, float16.
#include "prr_decode_impl.h"

namespace prr {

template <>
const void* shaped_decode_fn<false>(const DecodeLaunch& a, bool join) {
  if (join) return (const void*)merge_parts_kernel<false, kShapeSpan>;
  switch (a.shape) {
    case kShapeSpan: return decode_fn<false, kShapeSpan>(a.e4m3);
    case kShapeSpan | kShapeCap: return decode_fn<false, kShapeSpan | kShapeCap>(a.e4m3);
    case kShapeSpan | kShapeSlopes: return decode_fn<false, kShapeSpan | kShapeSlopes>(a.e4m3);
    default: return decode_fn<false, kShapeSpan | kShapeCap | kShapeSlopes>(a.e4m3);
  }
}

}  // namespace prr
