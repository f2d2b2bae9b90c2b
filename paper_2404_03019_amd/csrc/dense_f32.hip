// Products of the dense operators, f32 operands.
#include "dense_kernel.h"

namespace geot {

GEOT_DENSE_LAUNCHER(launch_dense_f32) { return launch_float<ELEM_F32>(epi, mode, tile, direct, a, blocks, st); }

}  // namespace geot
