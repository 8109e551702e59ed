// The instances of attention_rows.h for drafted trees.
#include "attention_rows.h"
#include "nnjit.h"

namespace nnjit {

hipError_t launch_tree_rows(const AttentionParams &p, int dtype, bool vec, int waves, int grid, hipStream_t stream)
{
    return dtype == NNJIT_F16 ? launch_typed<_Float16, true>(p, vec, waves, grid, stream) : launch_typed<float, true>(p, vec, waves, grid, stream);
}

}  // namespace nnjit
