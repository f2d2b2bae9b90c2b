// Products of the dense operators, f32 operands.
#include "dense_kernel.h"
#include "dense_narrow.h"
#include "dense_small.h"

namespace geot {

GEOT_DENSE_LAUNCHER(launch_dense_f32) {
    if (tile == DENSE_TILE_SMALL) {
        if (epi == DENSE_GATED) return launch_small<ELEM_F32, DENSE_GATED, true>(a, fm, fn, blocks, st);
        if (epi == DENSE_GATED_BWD) return launch_small<ELEM_F32, DENSE_GATED_BWD, true>(a, fm, fn, blocks, st);
        return hipErrorInvalidValue;
    }
    if (tile == DENSE_TILE_NARROW) {   // fm: 64-byte pieces, fn: waves over the columns
        if (epi == DENSE_GATED) return launch_narrow<ELEM_F32, DENSE_GATED>(a, fm, fn, (int)a.tiles_n, blocks, st);
        if (epi == DENSE_GATED_BWD) return launch_narrow<ELEM_F32, DENSE_GATED_BWD>(a, fm, fn, (int)a.tiles_n, blocks, st);
        return hipErrorInvalidValue;
    }
    return launch_float<ELEM_F32>(epi, mode, tile, direct, a, blocks, st);
}

}  // namespace geot
