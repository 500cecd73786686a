// New keys and values into the cache's pages, turned by positions on several
// axes (a unit of its own, as append_impl.h makes 16 kernels of each form).
#include "append_impl.h"

namespace epikv {

hipError_t launch_append_axes(const AppendAxesArgs& a, bool q4, hipStream_t s) {
  return q4 ? launch_append_fmt<true>(a, s) : launch_append_fmt<false>(a, s);
}

}  // namespace epikv
