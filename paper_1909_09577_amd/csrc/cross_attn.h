// What the files of cross attention share on the host.
#pragma once

#include "attn_tiles.h"

#include <math.h>

namespace nm {

struct AttnPlan {
    int col_tiles, splits, tiles_per_split;
    size_t part_bytes, ml_bytes;  // of workspace
};
// columns: tokens of a workgroup; tile: positions of a tile; waves: tiles that a workgroup takes at a time
AttnPlan attn_plan(int columns, int tile, int waves, int B, int H, int Hkv, int D, int U, int T);
AttnPlan attn_fwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T);
hipError_t launch_attn_fwd(bool bf16, const AttnArgs &a, hipStream_t s);

// plan of the kernel of dq; its workspace: the sums over channels of o * dout, then parts of dq
AttnPlan attn_bwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T);
hipError_t launch_attn_bwd(bool bf16, const AttnArgs &a, hipStream_t s);

}  // namespace nm
