// prr_shape.h's spans on the CPU, behind a C entry.
#include <stdint.h>

#include <algorithm>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;

#include "prr_shape.h"

extern "C" void span_host(int window, const int32_t* prefix, const int32_t* first, int pos, int row, int s, int kv, int32_t* out) {
  prr::ShapeArgs a{};
  a.window = window;
  a.prefix = prefix;
  a.first = first;
  const prr::Span r = prr::span_of(a, pos, row, s, kv);
  out[0] = r.lo;
  out[1] = r.hi;
}
