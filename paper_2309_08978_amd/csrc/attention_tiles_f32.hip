// The fp32 instances of attention_tiles.h.
#include "attention_tiles.h"

namespace nnjit {

// Up to 128 dims on the bf16 matrix cores; above, a row's parts do not fit the
// registers, and the fp32 matrix cores take it.
hipError_t launch_attention_tiles_f32(const AttentionParams &p, int tile_rows, bool vec, int grid, hipStream_t stream)
{
    if (!vec) {
        return p.dim <= 128 ? launch_shape<float, 128, SPLIT_ANY, 1>(p, tile_rows, grid, stream)
                            : launch_shape<float, 256, ANY, 1>(p, tile_rows, grid, stream);
    }
    if (p.dim <= 64) return launch_shape<float, 64, SPLIT, 1>(p, tile_rows, grid, stream);
    if (p.dim <= 96) return launch_shape<float, 96, SPLIT, 1>(p, tile_rows, grid, stream);
    if (p.dim <= 128) return launch_shape<float, 128, SPLIT, 1>(p, tile_rows, grid, stream);
    return launch_chunks<float, 256, 1>(p, tile_rows, grid, stream);
}

}  // namespace nnjit
