// The fp16 instances of attention_tiles.h (a file each: they take the longest to compile).
#include "attention_tiles.h"

namespace nnjit {

hipError_t launch_attention_tiles_f16(const AttentionParams &p, int tile_rows, bool vec, int grid, hipStream_t stream)
{
    return launch_tiles<_Float16>(p, tile_rows, vec, grid, stream);
}

}  // namespace nnjit
