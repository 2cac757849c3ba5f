// Prompt attention with shaped scores, bfloat16.
#include "prr_prompt_impl.h"

namespace prr {

template <>
const void* shaped_prompt_fn<true>(const PromptLaunch& a) {
  const bool paged = a.b.page_table != nullptr;
  switch (a.shape) {
    case kShapeSpan: return prompt_fn<true, kShapeSpan>(paged, a.waves);
    case kShapeSpan | kShapeCap: return prompt_fn<true, kShapeSpan | kShapeCap>(paged, a.waves);
    case kShapeSpan | kShapeSlopes: return prompt_fn<true, kShapeSpan | kShapeSlopes>(paged, a.waves);
    default: return prompt_fn<true, kShapeSpan | kShapeCap | kShapeSlopes>(paged, a.waves);
  }
}

}  // namespace prr
