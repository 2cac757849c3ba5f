// Prompt attention with shaped scores, float16.
#include "prr_prompt_impl.h"

namespace prr {

template <>
const void* shaped_prompt_fn<false>(const PromptLaunch& a) {
  const bool paged = a.b.page_table != nullptr;
  switch (a.shape) {
    case kShapeSpan: return prompt_fn<false, kShapeSpan>(paged, a.waves);
    case kShapeSpan | kShapeCap: return prompt_fn<false, kShapeSpan | kShapeCap>(paged, a.waves);
    case kShapeSpan | kShapeSlopes: return prompt_fn<false, kShapeSpan | kShapeSlopes>(paged, a.waves);
    default: return prompt_fn<false, kShapeSpan | kShapeCap | kShapeSlopes>(paged, a.waves);
  }
}

}  // namespace prr
