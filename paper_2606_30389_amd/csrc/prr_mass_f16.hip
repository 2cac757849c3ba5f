// The weight that cached tokens receive, float16 queries.
#include "prr_mass_impl.h"

namespace prr {

template <>
const void* mass_kernel_of<false>(const MassLaunch& a) {
  return mass_fn_of<false>(a);
}

}  // namespace prr
