// The fp32 instances of attention_tiles.h (a file each: they take the longest to compile).
#include "attention_tiles.h"

namespace nnjit {

hipError_t launch_attention_tiles_f32(const AttentionParams &p, int tile_rows, bool vec, int grid, hipStream_t stream)
{
    return launch_tiles<float>(p, tile_rows, vec, grid, stream);
}

}  // namespace nnjit
