// Products of the dense operators, f16 operands.
#include "dense_kernel.h"

namespace geot {

GEOT_DENSE_LAUNCHER(launch_dense_f16) { return launch_float<ELEM_F16>(epi, mode, tile, direct, a, blocks, st); }

}  // namespace geot
