// Products of the dense operators, bf16 operands.
#include "dense_kernel.h"

namespace geot {

GEOT_DENSE_LAUNCHER(launch_dense_bf16) { return launch_float<ELEM_BF16>(epi, mode, tile, direct, a, blocks, st); }

}  // namespace geot
