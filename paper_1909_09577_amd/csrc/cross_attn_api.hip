// Entry points of cross attention (include/nm_attention.h): checks of arguments, plans, workspace.
#include "../../include/nm_attention.h"
#include "../../include/nm_conv1d.h"
#include "cross_attn.h"

namespace nm {

// of the estimates below, in microseconds: a round of 64 positions at 64 channels, what comes before and after the rounds, a second launch
constexpr double kRoundUs = 1.2, kStartUs = 3.0, kJoinUs = 4.0;

int attn_share(long long groups, int rounds, double round_us, double join_bytes, int per_cu)
{
    const long long slots = 256LL * per_cu;
    double best = 0;
    int per = rounds;
    for (int n = 1; n <= rounds && n <= kMaxSplits; ++n) {
        const int each = (rounds + n - 1) / n;
        if ((rounds + each - 1) / each != n) continue;
        const double us = (double)((groups * n + slots - 1) / slots) * (kStartUs + each * round_us) + (n > 1 ? kJoinUs + n * join_bytes / 4.0e6 : 0.0);
        if (n == 1 || us < best) {
            best = us;
            per = each;
        }
    }
    return per;
}

AttnPlan attn_plan(const AttnForm &f, int B, int H, int Hkv, int D, int U, int T)
{
    AttnPlan p = {};
    const int columns = f.columns;
    // Tiles of one head have their tokens side by side in memory, which are then read in 16-byte groups; where they would be less than
    // two thirds full, tiles run over the heads.
    // A workgroup's wavefronts take the same tokens of as many heads as there are (a power of two that divides them): fewer tiles are
    // half empty, and windows of neighbouring tokens overlap more than those of distant ones (windows of a quarter of 3001 frames, 333
    // tokens, 4 heads on one: dq 42 -> 34 us).
    const int G = H / Hkv;
    int log = 0;
    while (32 << (log + 1) <= columns && G % (2 << log) == 0) ++log;
    const int head_columns = columns >> log, head_tiles = (U + head_columns - 1) / head_columns;
    p.head_tiles = G == 1 || 3LL * U >= 2LL * head_tiles * head_columns ? head_tiles : 0;
    p.head_waves_log = p.head_tiles ? log : 0;
    p.col_tiles = p.head_tiles ? (G >> log) * head_tiles : (int)(((long long)G * U + columns - 1) / columns);
    const int tiles = (T + f.tile - 1) / f.tile, rounds = (tiles + f.waves - 1) / f.waves;
    const int per = attn_share((long long)B * Hkv * p.col_tiles, rounds, kRoundUs * f.work * D / 64 * f.tile / 64, 2.0 * 4 * B * H * U * D, f.per_cu);
    p.splits = (rounds + per - 1) / per;
    const size_t rows = (size_t)B * H * U;
    p.part_bytes = p.splits > 1 ? align_up((size_t)p.splits * rows * D * sizeof(float), 256) : 0;
    p.ml_bytes = p.splits > 1 ? align_up((size_t)p.splits * rows * 2 * sizeof(float), 256) : 0;
    return p;
}

namespace {

constexpr int kMaxD = 128;

int check(int B, int H, int Hkv, int D, int U, int T, int dtype)
{
    if (B <= 0 || H <= 0 || Hkv <= 0 || D <= 0 || U <= 0 || T <= 0 || H % Hkv || (dtype != NM_BF16 && dtype != NM_F32)) return NM_ERR_BAD_ARG;
    const long long most = (1LL << 31) - 1;
    const int element = dtype == NM_BF16 ? 2 : 4;
    if ((long long)D * element > ((1LL << 32) - 1) / U || (long long)D * element > ((1LL << 32) - 1) / T) return NM_ERR_UNSUPPORTED;  // a head's rows
    if (D > kMaxD || (long long)H * D > most / U || (long long)Hkv * D > most / T || (long long)B * H > (1 << 24)) return NM_ERR_UNSUPPORTED;
    if ((long long)B * H * U > most / 2) return NM_ERR_UNSUPPORTED;
    // The grids, with as many column tiles, position tiles and parts as there can be: below 2^32 work items.  (Workgroups of 512 take
    // 256 tokens, or few tokens and then those of all heads that share keys and values; those of 256 take 128 tokens or positions, or one
    // head's if it has fewer.)
    if ((long long)B * Hkv >= 1LL << 23 || (long long)B * H * ((U + 31) / 32) >= 1LL << 24 || (long long)B * Hkv * ((T + 31) / 32) >= 1LL << 24 ||
        (long long)B * H * D > ((1LL << 31) * 256 - 1) / U)
        return NM_ERR_UNSUPPORTED;
    return NM_OK;
}

struct Span {
    const void *p;
    size_t bytes;
};
Span span(const void *p, long long stride, int B, long long item, int dtype)
{
    return {p, (size_t)((B - 1) * stride + item) * (dtype == NM_BF16 ? 2 : 4)};
}
bool strides_ok(long long s, long long item) { return s >= item && s < 1LL << 40; }
bool overlap(const Span &a, const Span &b)
{
    if (!a.p || !b.p) return false;
    const char *pa = (const char *)a.p, *pb = (const char *)b.p;
    return pa < pb + b.bytes && pb < pa + a.bytes;
}
// Items of two tensors that lie between each other's (the halves of one projection's output) overlap as spans but not as tensors.
bool overlap_items(const Span &a, long long as, const Span &b, long long bs, long long item_a, long long item_b, int B, int dtype)
{
    if (!overlap(a, b)) return false;
    if (B == 1 || as != bs) return true;
    const long long e = dtype == NM_BF16 ? 2 : 4, stride = as * e;
    long long d = ((const char *)b.p - (const char *)a.p) % stride;  // of b's items behind a's
    if (d < 0) d += stride;
    return d < item_a * e || d + item_b * e > stride;
}
int workspace_status(const void *ws, size_t have, size_t need)
{
    return need && (!ws || have < need || (uintptr_t)ws % 256) ? NM_ERR_WORKSPACE : NM_OK;
}
int dev(hipError_t e) { return e == hipSuccess ? NM_OK : NM_ERR_DEVICE; }

bool fill_scale(AttnArgs &a, float scale)
{
    if (!(scale - scale == 0.f)) return false;
    a.scale = scale;
    const float c = (scale < 0.f ? -scale : scale) * 1.4426950408889634f;
    a.c = c < 1e-37f ? 1e-37f : c;  // (not zero: masked scores are -infinity times this)
    a.flip = scale < 0.f ? 0x80000000u : 0u;
    return true;
}

}  // namespace
}  // namespace nm

using namespace nm;

extern "C" {

size_t nm_cross_attn_workspace_bytes(int op, int B, int heads, int kv_heads, int D, int U, int T, int dtype)
{
    if (check(B, heads, kv_heads, D, U, T, dtype) != NM_OK) return 0;
    if (op == NM_OP_ATTN_FWD) {
        const AttnPlan p = attn_fwd_plan(dtype == NM_BF16, B, heads, kv_heads, D, U, T);
        return p.part_bytes + p.ml_bytes;
    }
    if (op == NM_OP_ATTN_BWD) {
        const AttnPlan p = attn_bwd_plan(dtype == NM_BF16, B, heads, kv_heads, D, U, T);
        return align_up(align_up((size_t)B * heads * U * sizeof(float), 256) + p.part_bytes + p.kv_part_bytes, 256);
    }
    return 0;
}

int nm_cross_attn_fwd(int B, int heads, int kv_heads, int D, int U, int T, const void *q, long long q_stride,
                      const void *k, long long k_stride, const void *v, long long v_stride, const int *lengths,
                      const int *q_lengths, const int *windows, float scale, void *o, long long o_stride, float *lse,
                      int dtype, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check(B, heads, kv_heads, D, U, T, dtype);
    if (st != NM_OK) return st;
    AttnArgs a = {};
    if (!q || !k || !v || !o || !fill_scale(a, scale)) return NM_ERR_BAD_ARG;
    const long long qi = (long long)heads * D * U, ki = (long long)kv_heads * D * T;
    if (!strides_ok(q_stride, qi) || !strides_ok(o_stride, qi) || !strides_ok(k_stride, ki) || !strides_ok(v_stride, ki)) return NM_ERR_BAD_ARG;
    const Span so = span(o, o_stride, B, qi, dtype), sl = {lse, (size_t)B * heads * U * sizeof(float)};
    const Span in[3] = {span(q, q_stride, B, qi, dtype), span(k, k_stride, B, ki, dtype), span(v, v_stride, B, ki, dtype)};
    const long long stride[3] = {q_stride, k_stride, v_stride}, item[3] = {qi, ki, ki};
    for (int i = 0; i < 3; ++i)
        if (overlap_items(so, o_stride, in[i], stride[i], qi, item[i], B, dtype) || overlap(sl, in[i])) return NM_ERR_BAD_ARG;
    if (overlap(so, sl)) return NM_ERR_BAD_ARG;
    const AttnPlan p = attn_fwd_plan(dtype == NM_BF16, B, heads, kv_heads, D, U, T);
    const int ws = workspace_status(workspace, workspace_bytes, p.part_bytes + p.ml_bytes);
    if (ws != NM_OK) return ws;
    a.B = B; a.H = heads; a.Hkv = kv_heads; a.G = heads / kv_heads; a.D = D; a.U = U; a.T = T;
    a.q = q; a.k = k; a.v = v; a.qs = q_stride; a.ks = k_stride; a.vs = v_stride;
    a.len = lengths; a.q_len = q_lengths; a.windows = windows;
    a.out = o; a.os = o_stride; a.lse = lse;
    a.part = (float *)workspace;
    a.part_ml = (float *)((char *)workspace + p.part_bytes);
    a.col_tiles = p.col_tiles; a.head_tiles = p.head_tiles; a.head_waves_log = p.head_waves_log; a.splits = p.splits;
    return dev(launch_attn_fwd(dtype == NM_BF16, a, (hipStream_t)hip_stream));
}

int nm_cross_attn_bwd(int B, int heads, int kv_heads, int D, int U, int T, const void *dout, long long dout_stride,
                      const void *q, long long q_stride, const void *k, long long k_stride, const void *v,
                      long long v_stride, const void *o, long long o_stride, const float *lse, const int *lengths,
                      const int *q_lengths, const int *windows, float scale, void *dq, long long dq_stride, void *dk,
                      long long dk_stride, void *dv, long long dv_stride, int dtype, void *workspace,
                      size_t workspace_bytes, void *hip_stream)
{
    const int st = check(B, heads, kv_heads, D, U, T, dtype);
    if (st != NM_OK) return st;
    AttnArgs a = {};
    if (!dout || !q || !k || !v || !o || !lse || !dq || !dk || !dv || !fill_scale(a, scale)) return NM_ERR_BAD_ARG;
    const long long qi = (long long)heads * D * U, ki = (long long)kv_heads * D * T;
    const void *ptr[8] = {dout, q, o, k, v, dq, dk, dv};
    const long long stride[8] = {dout_stride, q_stride, o_stride, k_stride, v_stride, dq_stride, dk_stride, dv_stride};
    const long long item[8] = {qi, qi, qi, ki, ki, qi, ki, ki};
    for (int i = 0; i < 8; ++i)
        if (!strides_ok(stride[i], item[i])) return NM_ERR_BAD_ARG;
    const Span sl = {lse, (size_t)B * heads * U * sizeof(float)};
    for (int i = 5; i < 8; ++i) {  // an output
        const Span out = span(ptr[i], stride[i], B, item[i], dtype);
        if (overlap(out, sl)) return NM_ERR_BAD_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap_items(out, stride[i], span(ptr[j], stride[j], B, item[j], dtype), stride[j], item[i], item[j], B, dtype)) return NM_ERR_BAD_ARG;
    }
    const AttnPlan p = attn_bwd_plan(dtype == NM_BF16, B, heads, kv_heads, D, U, T);
    const size_t delta_bytes = align_up((size_t)B * heads * U * sizeof(float), 256);
    const int ws = workspace_status(workspace, workspace_bytes, delta_bytes + p.part_bytes + p.kv_part_bytes);
    if (ws != NM_OK) return ws;
    a.B = B; a.H = heads; a.Hkv = kv_heads; a.G = heads / kv_heads; a.D = D; a.U = U; a.T = T;
    a.q = q; a.k = k; a.v = v; a.o = o; a.dout = dout;
    a.qs = q_stride; a.ks = k_stride; a.vs = v_stride; a.os = o_stride; a.dos = dout_stride;
    a.len = lengths; a.q_len = q_lengths; a.windows = windows;
    a.dq = dq; a.dk = dk; a.dv = dv; a.dqs = dq_stride; a.dks = dk_stride; a.dvs = dv_stride;
    a.lse = const_cast<float *>(lse);
    a.delta = (float *)workspace;
    a.part = (float *)((char *)workspace + delta_bytes);
    a.kv_part = (float *)((char *)workspace + delta_bytes + p.part_bytes);
    a.pos_tiles = p.pos_tiles; a.parts = p.parts; a.units_per_part = p.units_per_part; a.dq_first = p.dq_first;
    a.col_tiles = p.col_tiles; a.head_tiles = p.head_tiles; a.head_waves_log = p.head_waves_log; a.splits = p.splits;
    return dev(launch_attn_bwd(dtype == NM_BF16, a, (hipStream_t)hip_stream));
}

}  // extern "C"
