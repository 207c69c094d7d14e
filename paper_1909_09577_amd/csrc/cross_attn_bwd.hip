// Cross attention, backward (definition: include/nm_attention.h).
//
// A small kernel makes delta, the sums over channels of o * dout.  Then one launch makes all three gradients: workgroups of dq own tokens
// and go over the positions, in the two forms of the forward pass; workgroups of dk and dv own positions and go over the tokens of all
// heads that share them.  Scores and probabilities are made again in both from the saved log-sum-exp: two of seven products,
// against writing and reading them.  In each the result of the first products (scores and dp) is the second operand of the next ones,
// in the registers it was made in (attn_tiles.h).  Where either has too few workgroups, several share one's positions or tokens,
// and their sums are joined by another kernel, in order.
//
// Measured in bfloat16: 32 x 150 tokens, up to 800 frames, 16 heads of 64: delta 7 us, gradients 116 (215 MB that have to move: 1.8 TB/s);
// 4 x 333 tokens with windows of a quarter of 3001 frames, 8 heads of 128 over 2: 5, 71 and 19 for the join.  In launches of their own, with
// delta made by dq, they took 57 + 76 us and 37 + 55 + 8 + 12: neither fills the chip to its end.  The former's dk and dv alone kept the matrix
// pipes busy in 14 % of the cycles and the vector units in 33 %, with 1.4 of two possible wavefronts a SIMD on average: a
// workgroup has two or three tiles of tokens between its first loads and its stores.  Three wavefronts a SIMD sent 44 registers to
// scratch memory (76 -> 95 us); loads two tiles ahead changed nothing.  Heads of 65 to 96 channels in bfloat16 keep 8 bytes a lane in scratch memory.
#include "cross_attn.h"

namespace nm {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Probability from a score and the log-sum-exp, both in halves of powers of two: the square of its root.  The exponential of the
// hardware makes zeros of results below 2^-126, which scores and gradients of hundreds lift to values that a sum may consist of.
__device__ __forceinline__ float probability(float score, float half_c, float half_lse)
{
    const float root = __builtin_amdgcn_exp2f(__builtin_fmaf(score, half_c, -half_lse));
    return root * root;
}

// ---- dk and dv: a wavefront owns 32 positions, the columns of its products; tokens are rows ------------------------------
constexpr int kReach = 256;  // tiles of tokens

template <int TT>
struct TokenRows {  // of a tile of tokens
    float lse[TT], delta[TT];  // log-sum-exp in halves of powers of two, infinite where a token is not there
    int lo[TT], hi[TT];
};

// Of the widest heads, keys and values of a wavefront's positions and both sums do not fit the registers of two wavefronts a SIMD: the
// values stay in LDS (60 registers went to scratch memory otherwise).
constexpr bool values_in_lds(bool bf16, int DP) { return bf16 && DP > 96; }

template <typename S, int DP, int NB, int NW>
__device__ __forceinline__ void attn_dkv(const AttnArgs &a, const int id)
{
    typedef Mma<S> M;
    constexpr int TT = NB * 32, NT = NW * 64, KS = DP / M::kSteps;
    typedef Tile<S, DP, NB, NT> T;
    typedef TokenRows<TT> Rows;
    constexpr int kBuf = 2 * T::kBytes + (int)((sizeof(Rows) + 15) / 16 * 16);
    constexpr bool kValuesInLds = values_in_lds(sizeof(S) == 2, DP);
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int bh = id % (a.B * a.Hkv), rest = id / (a.B * a.Hkv);
    const int tile = rest % a.pos_tiles, part = rest / a.pos_tiles;
    const int b = bh / a.Hkv, kvh = bh - b * a.Hkv;
    const int len = a.len ? clipped(a.len[b], a.T) : a.T, q_len = a.q_len ? clipped(a.q_len[b], a.U) : a.U;
    const int w0 = (tile * NW + wave) * 32, t = w0 + (lane & 31);
    const float c = (a.flip ? -0.5f : 0.5f) * a.c;
    const int t_first = tile * NW * 32, t_last = t_first + NW * 32;
    typename M::Frag kf[KS], vf[kValuesInLds ? 1 : KS];
    unsigned char *values = smem + 2 * kBuf;
    OwnColumns<S, DP, NW> k_own, v_own;
    if (t_first < len) {  // (uniform)
        k_own.load((const S *)a.k + (size_t)b * a.ks + (size_t)kvh * a.D * a.T, a.D, a.T, t_first);
        v_own.load((const S *)a.v + (size_t)b * a.vs + (size_t)kvh * a.D * a.T, a.D, a.T, t_first);
    }
    f32x16_t dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[d][r] = dv[d][r] = 0.f;
    // Frames that some token of a tile looks at, so that tiles which look elsewhere are left out, and frames that all of them look at,
    // which need no masks (of as many tiles as there is room for; those behind are taken, with masks).
    __shared__ int reach[4][kReach];
    const int tiles = (q_len + TT - 1) / TT;
    if (a.windows) {
        for (int u0 = wave * 64; u0 < min(tiles * TT, kReach * TT); u0 += NT) {
            const int u = u0 + lane;
            int lo = a.T, hi = 0, all_lo = 0, all_hi = a.T;
            if (u < q_len) {
                frames_of(a, b, u, len, all_lo, all_hi);
                if (all_lo < all_hi) {
                    lo = all_lo;
                    hi = all_hi;
                }
            }
#pragma unroll
            for (int d = 1; d < TT; d <<= 1) {
                lo = min(lo, __shfl_xor(lo, d));
                hi = max(hi, __shfl_xor(hi, d));
                all_lo = max(all_lo, __shfl_xor(all_lo, d));
                all_hi = min(all_hi, __shfl_xor(all_hi, d));
            }
            if (lane % TT == 0 && u / TT < kReach) {
                reach[0][u / TT] = lo;
                reach[1][u / TT] = hi;
                reach[2][u / TT] = all_lo;
                reach[3][u / TT] = all_hi;
            }
        }
        __syncthreads();
    }
    // units: tiles of the heads, one head after the other; this workgroup's are those of its part
    const int units = t_first < len ? tiles * a.G : 0, unit_end = min(units, (part + 1) * a.units_per_part);
    auto next_from = [&](int i) {  // (uniform) the first unit from i on that has something to look at
        if (a.windows) {
            for (; i < unit_end; ++i) {
                const int at = i % tiles;
                if (at >= kReach || (reach[0][at] < t_last && reach[1][at] > t_first)) break;
            }
        }
        return __builtin_amdgcn_readfirstlane(i);
    };
    T qt, gt;
    typename T::Places at;
    at.set(a.D, a.U, threadIdx.x);
    float row_lse = 0.f, row_delta = 0.f;
    int row_lo = 0, row_hi = 0;
    auto load = [&](int i) {
        const int g = i / tiles, u0 = (i - g * tiles) * TT, head = kvh * a.G + g;
        qt.load((const S *)a.q + (size_t)b * a.qs + (size_t)head * a.D * a.U, at, a.U, u0, threadIdx.x);
        gt.load((const S *)a.dout + (size_t)b * a.dos + (size_t)head * a.D * a.U, at, a.U, u0, threadIdx.x);
        if (threadIdx.x < TT) {
            const int u = u0 + threadIdx.x, uc = min(u, a.U - 1);
            const size_t row = ((size_t)b * a.H + head) * a.U + uc;
            row_lse = a.lse[row];
            row_delta = a.delta[row];
            frames_of(a, b, uc, len, row_lo, row_hi);
            if (u >= q_len) row_lo = row_hi = 0;
        }
    };
    int i = next_from(part * a.units_per_part), turn = 0;
    if (i < unit_end) load(i);
    if (t_first < len) {
        if constexpr (kValuesInLds) {
            v_own.own.write(values, a.D, a.T, len, t_first, threadIdx.x);  // (read behind the barrier of the first unit)
            k_own.take(smem, a.D, a.T, len, t_first, wave, lane, kf);
        } else {
            v_own.own.write(smem + OwnColumns<S, DP, NW>::Own::kBytes, a.D, a.T, len, t_first, threadIdx.x);
            k_own.take(smem, a.D, a.T, len, t_first, wave, lane, kf, vf);
        }
    }
    values += wave * OwnColumns<S, DP, NW>::Own::kBlock;
    int off[2], own_off[2];
    M::template across_offsets<true>(lane, off);
    M::template across_offsets<false>(lane, own_off);
    for (int after; i < unit_end; i = after, turn ^= 1) {
        unsigned char *buf = smem + turn * kBuf;
        Rows &rows = *reinterpret_cast<Rows *>(buf + 2 * T::kBytes);
        const int u0 = (i % tiles) * TT;
        qt.write(buf, a.D, a.U, q_len, u0, threadIdx.x);
        gt.write(buf + T::kBytes, a.D, a.U, q_len, u0, threadIdx.x);
        if (threadIdx.x < TT) {
            const bool some = row_lo < row_hi;
            rows.lse[threadIdx.x] = some && row_lse != -INFINITY ? row_lse * (0.5f * kLog2e) : INFINITY;
            rows.delta[threadIdx.x] = some ? row_delta : 0.f;
            rows.lo[threadIdx.x] = row_lo;
            rows.hi[threadIdx.x] = row_hi;
        }
        __syncthreads();
        after = next_from(i + 1);
        if (after < unit_end) load(after);
        if (w0 >= len) continue;
        const int at_tile = u0 / TT;
        bool masked = a.windows;
        if (a.windows && at_tile < kReach) {
            if (reach[0][at_tile] >= w0 + 32 || reach[1][at_tile] <= w0) continue;
            masked = reach[2][at_tile] > w0 || reach[3][at_tile] < w0 + 32;
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const unsigned char *qb = buf + n * T::kBlock, *gb = qb + T::kBytes;
            f32x16_t s, dp;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                s = M::mul(M::across(qb, off, st), kf[st], s);
                if constexpr (kValuesInLds)
                    dp = M::mul(M::across(gb, off, st), M::across(values, own_off, st), dp);
                else
                    dp = M::mul(M::across(gb, off, st), vf[st], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int u = 32 * n + M::position(r, half);
                const float p = probability(s[r], c, rows.lse[u]);  // (columns beyond the sequence are not stored)
                s[r] = p;
                dp[r] = p * (dp[r] - rows.delta[u]);
            }
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int u = 32 * n + M::position(r, half);
                    const bool ok = t >= rows.lo[u] && t < rows.hi[u];
                    s[r] = ok ? s[r] : 0.f;
                    dp[r] = ok ? dp[r] : 0.f;
                }
            }
            const typename M::Probs pp = M::probs(s);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) dv[d] = M::mul(M::along(gb, d * 32, lane), pp, dv[d]);
            __builtin_amdgcn_sched_barrier(0);
            M::add_in_two_terms(dk, qb, lane, dp);
        }
    }
    __syncthreads();  // (the tiles give way to the results)
    if (w0 >= a.T) return;
    const size_t item = (size_t)kvh * a.D * a.T;
    if (a.parts > 1) {
        unsigned char *block = smem + wave * DP * 128;
        const size_t all = (size_t)a.B * a.Hkv * a.D * a.T, to = ((size_t)part * 2 * a.B + b) * a.Hkv * a.D * a.T + item;
        store_block<float, DP>(block, dk, 1.f, a.kv_part + to, a.D, a.T, w0, len, lane);
        wave_fence();
        store_block<float, DP>(block, dv, 1.f, a.kv_part + all + to, a.D, a.T, w0, len, lane);
        return;
    }
    unsigned char *block = smem + wave * 2 * DP * M::kRow;
    store_block<S, DP>(block, dk, a.scale, (S *)a.dk + (size_t)b * a.dks + item, a.D, a.T, w0, len, lane);
    store_block<S, DP>(block + DP * M::kRow, dv, 1.f, (S *)a.dv + (size_t)b * a.dvs + item, a.D, a.T, w0, len, lane);
}

// Adds the parts of dk and dv, in order.
template <typename S>
__device__ __forceinline__ void attn_dkv_join(const AttnArgs &a, unsigned id)
{
    const size_t item = (size_t)a.Hkv * a.D * a.T, all = item * a.B;
    const size_t e = (size_t)id * 256 + threadIdx.x;
    if (e >= all) return;
    float k = 0.f, v = 0.f;
#pragma unroll 4
    for (int p = 0; p < a.parts; ++p) {
        k += a.kv_part[2 * p * all + e];
        v += a.kv_part[(2 * p + 1) * all + e];
    }
    const size_t b = e / item;
    store_from_f32((S *)a.dk, b * a.dks + (e - b * item), k * a.scale);
    store_from_f32((S *)a.dv, b * a.dvs + (e - b * item), v);
}

// ---- dq: a wavefront's columns are tokens, rows are positions; shared and apart as in the forward pass ---------------------
template <typename S, int DP, int NB, int NW, bool SHARED>
__device__ __forceinline__ void attn_dq(const AttnArgs &a, const int id)
{
    typedef Mma<S> M;
    constexpr int TT = NB * 32, NT = SHARED ? NW * 64 : 64, KS = DP / M::kSteps;
    typedef Tile<S, DP, NB, NT> T;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int bh = id % (a.B * a.Hkv), rest = id / (a.B * a.Hkv);
    const int ct = rest % a.col_tiles, split = rest / a.col_tiles;
    const int b = bh / a.Hkv, kvh = bh - b * a.Hkv;
    const int len = a.len ? clipped(a.len[b], a.T) : a.T, q_len = a.q_len ? clipped(a.q_len[b], a.U) : a.U;
    const S *krows = (const S *)a.k + (size_t)b * a.ks + (size_t)kvh * a.D * a.T;
    const S *vrows = (const S *)a.v + (size_t)b * a.vs + (size_t)kvh * a.D * a.T;

    // this lane's column
    const int block = SHARED ? wave : 0;
    int g, u;
    bool exists;
    if (a.head_tiles) {
        const int gt = ct / a.head_tiles, log = a.head_waves_log;
        g = (gt << log) + (block & ((1 << log) - 1));
        u = ((ct - gt * a.head_tiles) * ((SHARED ? NW : 1) >> log) + (block >> log)) * 32 + (lane & 31);
        exists = u < a.U;
    } else {
        const int m = (ct * (SHARED ? NW : 1) + block) * 32 + (lane & 31);
        exists = m < a.G * a.U;
        g = exists ? m / a.U : 0;
        u = m - g * a.U;
    }
    if (!exists) u = 0;
    const int head = kvh * a.G + g;
    const bool there = exists && u < q_len;
    const float half_c = 0.5f * a.c;
    int lo = 0, hi = 0x7fffffff, first = a.T, last = 0;
    float lse = INFINITY, delta = 0.f;  // a token that is not there, or without frames: every probability is zero
    if (there) {
        frames_of(a, b, u, len, lo, hi);
        first = lo;
        last = hi;
        if (lo < hi) {
            const size_t row = ((size_t)b * a.H + head) * a.U + u;
            lse = a.lse[row] * (0.5f * kLog2e);
            delta = a.delta[row];
            if (lse == -INFINITY) lse = INFINITY;
        }
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        first = min(first, __shfl_xor(first, d));
        last = max(last, __shfl_xor(last, d));
    }
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    const int wave_first = first, wave_last = last;
    if constexpr (SHARED) {  // of the workgroup
        int *range = reinterpret_cast<int *>(smem);
        if (lane == 0) {
            range[wave] = first;
            range[NW + wave] = last;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            first = min(first, range[w]);
            last = max(last, range[NW + w]);
        }
        __syncthreads();
    }
    // this workgroup's share of the tiles between them
    const int t_first = first / TT, t_last = (last + TT - 1) / TT, t_share = (t_last - t_first + a.splits - 1) / a.splits;
    const int t_begin = t_first + split * t_share, t_end = min(t_last, t_begin + t_share);

    // the first tiles and the tokens are loaded together
    T kt, vt;
    typename T::Places at;
    const int loader = SHARED ? threadIdx.x : lane, t_mine = SHARED ? t_begin : t_begin + wave;
    at.set(a.D, a.T, loader);
    if (t_mine < t_end) {
        kt.load(krows, at, a.T, t_mine * TT, loader);
        vt.load(vrows, at, a.T, t_mine * TT, loader);
    }
    typename M::Frag q[KS], go[KS];
    {
        const size_t item = (size_t)head * a.D * a.U;
        const S *qr = (const S *)a.q + (size_t)b * a.qs + item, *gr = (const S *)a.dout + (size_t)b * a.dos + item;
        bool taken = false;
        if constexpr (SHARED) {
            if (a.head_tiles && a.head_waves_log == 0) {  // (uniform)
                const int u0 = (ct - g * a.head_tiles) * NW * 32;
                OwnColumns<S, DP, NW> q_own, g_own;
                g_own.load(gr, a.D, a.U, u0);
                q_own.load(qr, a.D, a.U, u0);
                g_own.take(smem, a.D, a.U, q_len, u0, wave, lane, go);
                q_own.take(smem, a.D, a.U, q_len, u0, wave, lane, q);
                taken = true;
            } else if (a.head_tiles) {
                const int u0 = __builtin_amdgcn_readfirstlane(exists ? u : a.U);
                unsigned char *own = smem + wave * DP * M::kRow;
                WaveColumns<S, DP> q_own, g_own;
                g_own.load(gr, a.D, a.U, u0, lane);
                q_own.load(qr, a.D, a.U, u0, lane);
                g_own.take(own, a.D, a.U, q_len, u0, lane, go);
                q_own.take(own, a.D, a.U, q_len, u0, lane, q);
                __syncthreads();
                taken = true;
            }
        }
        if (!taken) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                q[s] = M::column(qr + u, s, half, a.D, a.U, there);
                go[s] = M::column(gr + u, s, half, a.D, a.U, there);
            }
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = M::flipped(q[s], a.flip);
    }
    f32x16_t acc[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
    int off[2];
    M::template across_offsets<true>(lane, off);

    auto compute = [&](const unsigned char *ktile, const unsigned char *vtile, int t0) {
        const bool whole = __all(lo <= t0 && t0 + TT <= hi);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const unsigned char *kb = ktile + n * T::kBlock, *vb = vtile + n * T::kBlock;
            f32x16_t s, dp;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                s = M::mul(M::across(kb, off, st), q[st], s);
                dp = M::mul(M::across(vb, off, st), go[st], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = probability(s[r], half_c, lse);
                dp[r] = p * (dp[r] - delta);
            }
            if (!whole) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = t0 + 32 * n + M::position(r, half);
                    dp[r] = t >= lo && t < hi ? dp[r] : 0.f;
                }
            }
            M::add_in_two_terms(acc, kb, lane, dp);
        }
    };
    if constexpr (SHARED) {
        for (int t = t_begin, turn = 0; t < t_end; ++t, turn ^= 1) {
            unsigned char *buf = smem + turn * 2 * T::kBytes;
            kt.write(buf, a.D, a.T, len, t * TT, threadIdx.x);
            vt.write(buf + T::kBytes, a.D, a.T, len, t * TT, threadIdx.x);
            __syncthreads();  // (the other buffer is written next: all are through with it before they pass here again)
            if (t + 1 < t_end) {
                kt.load(krows, at, a.T, (t + 1) * TT, threadIdx.x);
                vt.load(vrows, at, a.T, (t + 1) * TT, threadIdx.x);
            }
            if (t * TT < wave_last && (t + 1) * TT > wave_first) compute(buf, buf + T::kBytes, t * TT);
        }
    } else {
        unsigned char *buf = smem + wave * 2 * T::kBytes;
        for (int t = t_mine; t < t_end; t += NW) {
            wave_fence();
            kt.write(buf, a.D, a.T, len, t * TT, lane);
            vt.write(buf + T::kBytes, a.D, a.T, len, t * TT, lane);
            wave_fence();
            if (t + NW < t_end) {
                kt.load(krows, at, a.T, (t + NW) * TT, lane);
                vt.load(vrows, at, a.T, (t + NW) * TT, lane);
            }
            compute(buf, buf + T::kBytes, t * TT);
        }
    }
    auto put = [&](int d, int r, float v) {
        const int ch = d * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
        if (!exists || ch >= a.D) return;
        if (!there) v = 0.f;
        if (a.splits > 1)
            a.part[(((size_t)split * a.B + b) * a.H + head) * a.D * a.U + (size_t)ch * a.U + u] = v;
        else
            store_from_f32((S *)a.dq, (size_t)b * a.dqs + ((size_t)head * a.D + ch) * a.U + u, v * a.scale);
    };
    if constexpr (SHARED) {
        const int u0 = __builtin_amdgcn_readfirstlane(u), g0 = __builtin_amdgcn_readfirstlane(g);  // of column 0
        __syncthreads();  // (the tiles give way to the results)
        if (!__any(exists)) return;
        if (a.head_tiles || g0 == a.G - 1 || u0 + 32 <= a.U) {  // (uniform) tokens of one head
            unsigned char *block = smem + wave * DP * (a.splits > 1 ? 128 : M::kRow);
            const size_t item = (size_t)(kvh * a.G + g0) * a.D * a.U;
            if (a.splits > 1)
                store_block<float, DP>(block, acc, 1.f, a.part + ((size_t)split * a.B + b) * a.H * a.D * a.U + item, a.D, a.U, u0, q_len, lane);
            else
                store_block<S, DP>(block, acc, a.scale, (S *)a.dq + (size_t)b * a.dqs + item, a.D, a.U, u0, q_len, lane);
            return;
        }
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) put(d, r, acc[d][r]);
    } else {
        constexpr int PAIRS = DP / 32 * 16;
        float *prod = reinterpret_cast<float *>(smem);  // [NW][PAIRS][64]
        __syncthreads();
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) prod[(wave * PAIRS + d * 16 + r) * 64 + lane] = acc[d][r];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < PAIRS / NW; ++n) {
            const int pair = n * NW + wave;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) v += prod[(w * PAIRS + pair) * 64 + lane];
            put(pair / 16, pair % 16, v);
        }
    }
}

// Adds the parts of dq of `splits` workgroups, in order.
template <typename S>
__device__ __forceinline__ void attn_dq_join(const AttnArgs &a, unsigned id)
{
    const size_t item = (size_t)a.H * a.D * a.U, all = item * a.B;
    const size_t e = (size_t)id * 256 + threadIdx.x;
    if (e >= all) return;
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) v += a.part[s * all + e];
    const size_t b = e / item;
    store_from_f32((S *)a.dq, b * a.dqs + (e - b * item), v * a.scale);
}

// Both joins in one launch, as far as there are parts.
template <typename S>
__global__ __launch_bounds__(256) void attn_bwd_join_kernel(AttnArgs a, unsigned dq_groups)
{
    if (blockIdx.x < dq_groups)
        attn_dq_join<S>(a, blockIdx.x);
    else
        attn_dkv_join<S>(a, blockIdx.x - dq_groups);
}

// ---- delta: the sums over channels of o * dout of every token, 64 tokens of a head and four shares of the channels a workgroup ------
template <typename S>
__global__ __launch_bounds__(256) void attn_delta_kernel(AttnArgs a)
{
    __shared__ float parts[4][64];
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6;
    const int tiles = (a.U + 63) / 64, bh = blockIdx.x / tiles, u = (blockIdx.x - bh * tiles) * 64 + lane;
    const int b = bh / a.H, h = bh - b * a.H;
    const int q_len = a.q_len ? clipped(a.q_len[b], a.U) : a.U;
    float v = 0.f;
    if (u < q_len) {
        const S *o = (const S *)a.o + (size_t)b * a.os + (size_t)h * a.D * a.U + u, *g = (const S *)a.dout + (size_t)b * a.dos + (size_t)h * a.D * a.U + u;
#pragma unroll 8
        for (int d = share; d < a.D; d += 4) v += load_as_f32(o, (size_t)d * a.U) * load_as_f32(g, (size_t)d * a.U);
    }
    parts[share][lane] = v;
    __syncthreads();
    if (share == 0 && u < a.U) a.delta[(size_t)bh * a.U + u] = (parts[0][lane] + parts[1][lane]) + (parts[2][lane] + parts[3][lane]);
}

// All three gradients in one launch: few workgroups of either leave the chip half empty.  Those that take longer come first.
template <typename S, int DP, int NBQ, int NBKV, int NW, bool SHARED>
__global__ __launch_bounds__(NW * 64, sizeof(S) * DP <= (SHARED ? 256 : 192) ? 2 : 1) void attn_bwd_kernel(AttnArgs a, int dq_groups, int dkv_groups)
{
    const int id = a.dq_first ? (int)blockIdx.x - dq_groups : (int)blockIdx.x;
    if (id >= 0 && id < dkv_groups)
        attn_dkv<S, DP, NBKV, NW>(a, id);
    else
        attn_dq<S, DP, NBQ, NW, SHARED>(a, a.dq_first ? (int)blockIdx.x : (int)blockIdx.x - dkv_groups);
}

// ---- sizes ------------------------------------------------------------------------------------------------------
constexpr int kWaves = 4;
constexpr int token_blocks(bool bf16, int DP) { return bf16 && DP <= 96 ? 2 : 1; }  // of a tile of the kernel of dk and dv

template <typename S, int DP>
constexpr int dkv_lds()
{
    constexpr int NB = token_blocks(sizeof(S) == 2, DP);
    constexpr int own = OwnColumns<S, DP, kWaves>::Own::kBytes;
    constexpr int tiles = 2 * (2 * Tile<S, DP, NB, kWaves * 64>::kBytes + (int)((sizeof(TokenRows<NB * 32>) + 15) / 16 * 16));
    constexpr int out = kWaves * DP * (sizeof(S) == 2 ? 128 : 256);
    if (values_in_lds(sizeof(S) == 2, DP)) {  // the values lie behind the tiles, whose place the keys take before
        static_assert(!values_in_lds(sizeof(S) == 2, DP) || own <= tiles, "keys in front of the values");
        return most({tiles + own, out});
    }
    return most({tiles, 2 * own, out});
}

constexpr bool two_blocks(bool bf16, int DP, bool shared) { return bf16 && (shared || DP <= 64); }
// (float tiles of wide heads, one per wavefront, do not fit the registers)
bool is_shared(bool bf16, int DP, long long columns) { return columns > 32 || (!bf16 && DP > 64); }
AttnForm form_of(bool bf16, int DP, long long columns)
{
    const bool shared = is_shared(bf16, DP, columns);
    return {shared ? 128 : 32, two_blocks(bf16, DP, shared) ? 64 : 32, shared ? 1 : kWaves, bf16 || DP <= 64 ? 2 : 1, attn_work(bf16)};
}
template <typename S, int DP, bool SHARED>
hipError_t run(const AttnArgs &a, hipStream_t s)
{
    static LdsOptIn opt;
    constexpr int NB = two_blocks(sizeof(S) == 2, DP, SHARED) ? 2 : 1, NT = SHARED ? kWaves * 64 : 64;
    constexpr int tiles = (SHARED ? 4 : kWaves * 2) * Tile<S, DP, NB, NT>::kBytes, join = SHARED ? kWaves * DP * 128 : kWaves * DP / 32 * 16 * 64 * 4;
    constexpr int own = SHARED ? most({OwnColumns<S, DP, kWaves>::Own::kBytes, kWaves * WaveColumns<S, DP>::Own::kBytes}) : 0;  // of dq's tokens
    constexpr int bytes = most({tiles, join, own, dkv_lds<S, DP>()});
    static_assert(bytes + 4 * kReach * 4 <= 160 * 1024, "LDS of a CU");
    auto *fn = attn_bwd_kernel<S, DP, NB, token_blocks(sizeof(S) == 2, DP), kWaves, SHARED>;
    const hipError_t e = ensure_dynamic_lds(opt, (const void *)fn, bytes);
    if (e != hipSuccess) return e;
    attn_delta_kernel<S><<<dim3((unsigned)(a.B * a.H) * ((a.U + 63) / 64)), dim3(256), 0, s>>>(a);
    const int dkv_groups = a.B * a.Hkv * a.pos_tiles * a.parts, dq_groups = a.B * a.Hkv * a.col_tiles * a.splits;
    fn<<<dim3((unsigned)dkv_groups + dq_groups), dim3(kWaves * 64), bytes, s>>>(a, dq_groups, dkv_groups);
    return hipGetLastError();
}
template <typename S, int DP>
hipError_t run_both(const AttnArgs &a, hipStream_t s)
{
    if constexpr (sizeof(S) == 2 || DP <= 64) {
        if (!is_shared(sizeof(S) == 2, DP, (long long)a.G * a.U)) return run<S, DP, false>(a, s);
    }
    return run<S, DP, true>(a, s);
}
template <typename S>
hipError_t run_any(const AttnArgs &a, hipStream_t s)
{
    hipError_t e;
    if (a.D <= 32) e = run_both<S, 32>(a, s);
    else if (a.D <= 64) e = run_both<S, 64>(a, s);
    else if (a.D <= 96) e = run_both<S, 96>(a, s);
    else e = run_both<S, 128>(a, s);
    if (e != hipSuccess) return e;
    const unsigned dq_groups = a.splits > 1 ? (unsigned)(((size_t)a.B * a.H * a.U * a.D + 255) / 256) : 0;
    const unsigned dkv_groups = a.parts > 1 ? (unsigned)(((size_t)a.B * a.Hkv * a.T * a.D + 255) / 256) : 0;
    if (dq_groups + dkv_groups) attn_bwd_join_kernel<S><<<dim3(dq_groups + dkv_groups), dim3(256), 0, s>>>(a, dq_groups);
    return hipGetLastError();
}

}  // namespace

// a unit of the kernel of dk and dv, in microseconds at 64 tokens and channels
constexpr double kUnitUs = 2.0, kDqRoundUs = 1.5;  // (and a tile of dq)

AttnPlan attn_bwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T)
{
    const int DP = (D + 31) / 32 * 32;
    const long long columns = (long long)(H / Hkv) * U;
    AttnPlan p = attn_plan(form_of(bf16, DP, columns), B, H, Hkv, D, U, T);
    // dk and dv: units of a tile of tokens of a head
    const int per = kWaves * 32, tokens = 32 * token_blocks(bf16, DP), units = (U + tokens - 1) / tokens * (H / Hkv);
    p.pos_tiles = (T + per - 1) / per;
    p.units_per_part = attn_share((long long)B * Hkv * p.pos_tiles, units, kUnitUs * attn_work(bf16) * DP / 64 * tokens / 64, 2.0 * 2 * 4 * B * Hkv * T * D,
                                  bf16 || DP <= 64 ? 2 : 1);
    p.parts = (units + p.units_per_part - 1) / p.units_per_part;
    const AttnForm f = form_of(bf16, DP, columns);
    const int rounds = ((T + f.tile - 1) / f.tile + f.waves * p.splits - 1) / (f.waves * p.splits);
    p.dq_first = rounds * kDqRoundUs * f.tile > p.units_per_part * kUnitUs * tokens;  // (both at 64 positions or tokens, of as many channels)
    p.kv_part_bytes = p.parts > 1 ? (size_t)p.parts * 2 * B * Hkv * D * T * sizeof(float) : 0;
    return p;
}

hipError_t launch_attn_bwd(bool bf16, const AttnArgs &a, hipStream_t s) { return bf16 ? run_any<bf16_t>(a, s) : run_any<float>(a, s); }

}  // namespace nm
