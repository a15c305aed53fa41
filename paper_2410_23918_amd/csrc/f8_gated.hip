// The products in 8-bit floating point whose rows are gates and values (kernels: f8_product.h).
#include "f8_product.h"

namespace bitstack {

hipError_t launch_f8_gated(const F8Params& p, const F8Plan& plan, hipStream_t st) { return launch_f8_kernel<kEpiGated>(p, plan, st); }

}  // namespace bitstack
