// The fp16 instances of attention_tiles.h (a file a type: they take the longest to compile).
#include "attention_tiles.h"

namespace nnjit {

hipError_t launch_attention_tiles_f16(const AttentionParams &p, int tile_rows, bool vec, int grid, hipStream_t stream)
{
    if (!vec) {
        return p.dim <= 128 ? launch_shape<_Float16, 128, ANY, 2>(p, tile_rows, grid, stream)
                            : launch_shape<_Float16, 256, ANY, 1>(p, tile_rows, grid, stream);
    }
    if (p.dim <= 64) return launch_chunks<_Float16, 64, 2>(p, tile_rows, grid, stream);
    if (p.dim <= 96) return launch_chunks<_Float16, 96, 2>(p, tile_rows, grid, stream);
    if (p.dim <= 128) return launch_chunks<_Float16, 128, 2>(p, tile_rows, grid, stream);
    return launch_chunks<_Float16, 256, 1>(p, tile_rows, grid, stream);
}

}  // namespace nnjit
