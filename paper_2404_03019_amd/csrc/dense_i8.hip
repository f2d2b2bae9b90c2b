// Products of the dense operators, 8-bit operands with 32-bit sums.
#include "dense_kernel.h"
#include "dense_small.h"

namespace geot {

GEOT_DENSE_LAUNCHER(launch_dense_i8) {
    if (mode != DENSE_NT) return hipErrorInvalidValue;
    if (tile == DENSE_TILE_SMALL)
        return epi == DENSE_I8 ? launch_small<ELEM_I8, DENSE_I8, false>(a, fm, fn, blocks, st) : hipErrorInvalidValue;
    if (epi == DENSE_I8) return launch_tile<ELEM_I8, DENSE_I8, false, DENSE_NT>(tile, direct, a, blocks, st);
    if (epi == DENSE_PART) return launch_tile<ELEM_I8, DENSE_PART, false, DENSE_NT>(tile, direct, a, blocks, st);
    return hipErrorInvalidValue;
}

}  // namespace geot
