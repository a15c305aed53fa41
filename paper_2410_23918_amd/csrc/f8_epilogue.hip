// The products in 8-bit floating point with a bias, an activation and a residual after them (kernels: f8_product.h).
#include "f8_product.h"

namespace bitstack {

hipError_t launch_f8_epilogue(const F8Params& p, const F8Plan& plan, hipStream_t st) { return launch_f8_kernel<kEpiPlain>(p, plan, st); }

}  // namespace bitstack
