// What the files of cross attention share on the host.
#pragma once

#include "attn_tiles.h"

#include <math.h>

namespace nm {

constexpr int kMaxSplits = 64;

struct AttnPlan {
    int col_tiles, splits, tiles_per_split;   // of the forward pass or of dq
    int pos_tiles, parts, units_per_part;     // of dk and dv
    size_t part_bytes, ml_bytes, kv_part_bytes;  // of workspace
};
// Rounds of a workgroup, of `rounds`, where `groups` workgroups may each be shared among several: as many as are fastest by an
// estimate of round_us a round, and of writing and reading join_bytes for every share.
int attn_share(long long groups, int rounds, double round_us, double join_bytes);
// columns: tokens of a workgroup; tile: positions of a tile; waves: tiles that a workgroup takes at a time
AttnPlan attn_plan(int columns, int tile, int waves, int B, int H, int Hkv, int D, int U, int T);
AttnPlan attn_fwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T);
hipError_t launch_attn_fwd(bool bf16, const AttnArgs &a, hipStream_t s);

AttnPlan attn_bwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T);
hipError_t launch_attn_bwd(bool bf16, const AttnArgs &a, hipStream_t s);

}  // namespace nm
