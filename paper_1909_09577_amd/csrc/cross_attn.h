// What the files of cross attention share on the host.
#pragma once

#include "attn_tiles.h"

#include <initializer_list>
#include <math.h>

namespace nm {

constexpr int kMaxSplits = 64;

// Bytes of LDS of a workgroup whose phases want these
constexpr int most(std::initializer_list<int> phases)
{
    int bytes = 0;
    for (const int b : phases) bytes = b > bytes ? b : bytes;
    return bytes;
}

struct AttnPlan {
    int col_tiles, head_tiles, head_waves_log, splits;   // of the forward pass or of dq
    int pos_tiles, parts, units_per_part;     // of dk and dv
    bool dq_first;                            // workgroups of dq take longer
    size_t part_bytes, ml_bytes, kv_part_bytes;  // of workspace
};
struct AttnForm {
    int columns, tile, waves;  // of a workgroup: tokens, positions of a tile, tiles that it takes at a time
    int per_cu;                // workgroups that run on a CU at a time
    int work;                  // of a position, in those of bfloat16: float matrix instructions make an eighth as many products a cycle
};
constexpr int attn_work(bool bf16) { return bf16 ? 1 : 4; }  // (the rest of a round is no slower)
// Rounds of a workgroup, of `rounds`, where `groups` workgroups may each be shared among several: as many as are fastest by an
// estimate of round_us a round, and of writing and reading join_bytes for every share.
int attn_share(long long groups, int rounds, double round_us, double join_bytes, int per_cu);
AttnPlan attn_plan(const AttnForm &f, int B, int H, int Hkv, int D, int U, int T);
AttnPlan attn_fwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T);
hipError_t launch_attn_fwd(bool bf16, const AttnArgs &a, hipStream_t s);

AttnPlan attn_bwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T);
hipError_t launch_attn_bwd(bool bf16, const AttnArgs &a, hipStream_t s);

}  // namespace nm
