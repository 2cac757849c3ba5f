// Attention of single tokens with shaped scores, bfloat16.
#include "prr_decode_impl.h"

namespace prr {

template <>
const void* shaped_decode_fn<true>(const DecodeLaunch& a, bool join) {
  if (join) return (const void*)merge_parts_kernel<true, kShapeSpan>;
  switch (a.shape) {
    case kShapeSpan: return decode_fn<true, kShapeSpan>(a.e4m3);
    case kShapeSpan | kShapeCap: return decode_fn<true, kShapeSpan | kShapeCap>(a.e4m3);
    case kShapeSpan | kShapeSlopes: return decode_fn<true, kShapeSpan | kShapeSlopes>(a.e4m3);
    default: return decode_fn<true, kShapeSpan | kShapeCap | kShapeSlopes>(a.e4m3);
  }
}

}  // namespace prr
