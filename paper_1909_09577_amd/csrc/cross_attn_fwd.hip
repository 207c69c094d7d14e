// Cross attention, forward (definition: include/nm_attention.h).
//
// One pass over the keys and values with a running maximum and sum per token: the scores of a tile of positions are made with
// the positions as rows and the tokens as columns, so that a lane holds scores of one token and a softmax needs one exchange
// between the two lanes that share it; the probabilities stay in the registers they were made in (attn_tiles.h).  The tokens of
// the heads that share keys and values are columns side by side, so that those are read once for all of them.
//
// Two divisions of the work, by the number of columns:
//   shared   many columns: the wavefronts of a workgroup have columns of their own and share every tile, in two buffers;
//   apart    few columns (single tokens, beams): every wavefront has all columns and tiles of its own; the wavefronts' sums are
//            joined through LDS at the end.  This form reads keys and values at the rate of memory, and nothing in it waits
//            for another wavefront.
// Calls with too few workgroups for the chip share a token's positions among several, whose sums are joined by a second kernel.
//
// Measured in bfloat16: 32 x 150 tokens, up to 800 frames, 16 heads of 64: 35 us (96 MB that have to move: 2.7 TB/s; the longest
// utterance's 13 tiles one after the other); 4 x 700 tokens, 7501 frames, 8 heads of 128: 127 us and 17 for the join (0.68 PFLOP/s in the
// first).  Nothing is busy all the time there: matrix pipes 30 % of the cycles, vector units 28 % and as much again for
// exponentials, LDS 26 %; a wavefront's products, exponentials and reads of LDS follow one another, and the registers hold two wavefronts
// a SIMD.  Scores of the next block written beside the exponentials of this one (5 % slower), loads two tiles ahead and a higher priority
// for wavefronts in their matrix instructions (no change) did not help.
#include "cross_attn.h"

namespace nm {
namespace {

constexpr float kLag = 8.f;

// Wavefronts of a SIMD that the registers are made to last for: two, and four where a workgroup's eight wavefronts have narrow heads
// (a tile's groups are then few for each of them).
template <typename S, int DP, int NW, bool SHARED>
constexpr int kSimdWaves = sizeof(S) * DP > 256 ? NW / 4 : (NW == 8 && SHARED && sizeof(S) * DP <= 128 ? 4 : 2);

template <typename S, int DP, int NB, int NW, bool SHARED>
__global__ __launch_bounds__(NW * 64, (kSimdWaves<S, DP, NW, SHARED>)) void attn_fwd_kernel(AttnArgs a)
{
    typedef Mma<S> M;
    constexpr int TT = NB * 32, NT = SHARED ? NW * 64 : 64, KS = DP / M::kSteps;
    typedef Tile<S, DP, NB, NT> T;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int bh = blockIdx.x % (a.B * a.Hkv), rest = blockIdx.x / (a.B * a.Hkv);
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
    int lo = 0, hi = 0x7fffffff;  // a column that is not there is masked nowhere: it must not slow the others down
    int first = a.T, last = 0;    // frames that some column may look at
    if (there) {
        frames_of(a, b, u, len, lo, hi);
        first = lo;
        last = hi;
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
    typename M::Frag q[KS];
    {
        const S *rows = (const S *)a.q + (size_t)b * a.qs + (size_t)head * a.D * a.U;
        bool taken = false;
        if constexpr (SHARED) {
            if (a.head_tiles && a.head_waves_log == 0) {  // (uniform)
                const int u0 = (ct - g * a.head_tiles) * NW * 32;
                OwnColumns<S, DP, NW> own;
                own.load(rows, a.D, a.U, u0);
                own.take(smem, a.D, a.U, q_len, u0, wave, lane, q);
                taken = true;
            } else if (a.head_tiles) {
                const int u0 = __builtin_amdgcn_readfirstlane(exists ? u : a.U);
                WaveColumns<S, DP> own;
                own.load(rows, a.D, a.U, u0, lane);
                own.take(smem + wave * DP * M::kRow, a.D, a.U, q_len, u0, lane, q);
                __syncthreads();
                taken = true;
            }
        }
        if (!taken) {
#pragma unroll
            for (int s = 0; s < KS; ++s) q[s] = M::column(rows + u, s, half, a.D, a.U, there);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = M::flipped(q[s], a.flip);
    }

    float mx = -INFINITY, sum = 0.f;  // in powers of two, and of this lane's positions
    f32x16_t acc[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
    int koff[2];
    M::template across_offsets<true>(lane, koff);

    auto compute = [&](const unsigned char *kt, const unsigned char *vt, int t0) {
        f32x16_t s[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[n][r] = 0.f;
#pragma unroll
        for (int st = 0; st < KS; ++st)
#pragma unroll
            for (int n = 0; n < NB; ++n) s[n] = M::mul(M::across(kt + n * T::kBlock, koff, st), q[st], s[n]);
        if (!__all(lo <= t0 && t0 + TT <= hi)) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = t0 + 32 * n + M::position(r, half);
                    s[n][r] = t >= lo && t < hi ? s[n][r] : -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
        top = half_max(top) * a.c;
        // The base that sums are taken to follows the maximum only where that has grown by kLag powers of two: probabilities up to
        // 2^kLag do no harm, and multiplying what has been added so far is a third of the work otherwise.
        if (__any(top > mx + kLag)) {
            top = fmaxf(top, mx);
            const float shrink = __builtin_amdgcn_exp2f(mx - (top == -INFINITY ? 0.f : top));
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= shrink;
            mx = top;
        }
        const float base = mx == -INFINITY ? 0.f : mx;  // (nothing allowed so far: every probability is zero)
        typename M::Probs p[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            float part = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], a.c, -base));
                part += s[n][r];
            }
            sum += part;
            p[n] = M::probs(s[n]);
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) acc[d] = M::mul(M::along(vt + n * T::kBlock, d * 32, lane), p[n], acc[d]);
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

    // one value per (column, channel) and its place; sum_all: of the column
    auto put = [&](int d, int r, float v, float sum_all) {
        const int ch = d * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
        if (!exists || ch >= a.D) return;
        if (a.splits > 1) {
            a.part[(((size_t)split * a.B + b) * a.H + head) * a.D * a.U + (size_t)ch * a.U + u] = there ? v : 0.f;
        } else {
            const float inv = sum_all == 0.f ? 0.f : 1.f / sum_all;
            store_from_f32((S *)a.out, (size_t)b * a.os + ((size_t)head * a.D + ch) * a.U + u, there ? v * inv : 0.f);
        }
    };
    auto put_sums = [&](float mx_all, float sum_all) {
        if (!exists || half) return;
        const size_t row = ((size_t)b * a.H + head) * a.U + u;
        if (a.splits > 1) {
            float *ml = a.part_ml + ((size_t)split * a.B * a.H * a.U + row) * 2;
            ml[0] = there ? mx_all : -INFINITY;
            ml[1] = there ? sum_all : 0.f;
        } else if (a.lse) {
            a.lse[row] = there && sum_all != 0.f ? (mx_all + __builtin_amdgcn_logf(sum_all)) * 0.69314718055994531f : -INFINITY;
        }
    };
    if constexpr (SHARED) {
        __syncthreads();  // (the tiles give way to the results)
        const float total = half_sum(sum);
        put_sums(mx, total);
        const int u0 = __builtin_amdgcn_readfirstlane(u), g0 = __builtin_amdgcn_readfirstlane(g);  // of column 0
        if (!__any(exists)) return;
        if (a.head_tiles || g0 == a.G - 1 || u0 + 32 <= a.U) {  // (uniform) tokens of one head
            unsigned char *block = smem + wave * DP * (a.splits > 1 ? 128 : M::kRow);
            const size_t item = (size_t)(kvh * a.G + g0) * a.D * a.U;
            if (a.splits > 1)
                store_block<float, DP>(block, acc, 1.f, a.part + ((size_t)split * a.B + b) * a.H * a.D * a.U + item, a.D, a.U, u0, q_len, lane);
            else
                store_block<S, DP>(block, acc, total == 0.f ? 0.f : 1.f / total, (S *)a.out + (size_t)b * a.os + item, a.D, a.U, u0, q_len, lane);
            return;
        }
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) put(d, r, acc[d][r], total);
    } else {
        // joined through LDS: every wavefront's maxima and sums, and its products
        constexpr int PAIRS = DP / 32 * 16;
        float *sums = reinterpret_cast<float *>(smem);  // [NW][2][64]
        float *prod = sums + NW * 128;                  // [NW][PAIRS][64]
        __syncthreads();
        sums[wave * 128 + lane] = mx;
        sums[wave * 128 + 64 + lane] = half_sum(sum);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) prod[(wave * PAIRS + d * 16 + r) * 64 + lane] = acc[d][r];
        __syncthreads();
        float top = -INFINITY, total = 0.f, weight[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, sums[w * 128 + lane]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            weight[w] = __builtin_amdgcn_exp2f(sums[w * 128 + lane] - (top == -INFINITY ? 0.f : top));
            total += weight[w] * sums[w * 128 + 64 + lane];
        }
        if (wave == 0) put_sums(top, total);
#pragma unroll
        for (int n = 0; n < PAIRS / NW; ++n) {
            const int pair = n * NW + wave;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) v += weight[w] * prod[(w * PAIRS + pair) * 64 + lane];
            put(pair / 16, pair % 16, v, total);
        }
    }
}

// Joins the sums of `splits` workgroups, in order: a workgroup takes 64 tokens of a head, whose weights lie in LDS, and 32 channels.  The
// wavefronts fetch the maxima and sums of different splits (one after the other, 22 splits took 17 us).
template <typename S>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    __shared__ float top_of[kMaxSplits][64], sum_of[kMaxSplits][64];
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6;
    const int tiles = (a.U + 63) / 64, bh = blockIdx.x / tiles, u = (blockIdx.x - bh * tiles) * 64 + lane;
    const int b = bh / a.H, h = bh - b * a.H;
    const size_t rows = (size_t)a.B * a.H * a.U, all = rows * a.D, row = (size_t)bh * a.U + min(u, a.U - 1);
#pragma unroll 4
    for (int s = share; s < a.splits; s += 4) {
        const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + (s * rows + row) * 2);
        top_of[s][lane] = ml.x;
        sum_of[s][lane] = ml.y;
    }
    __syncthreads();
    float top = -INFINITY, total = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, top_of[s][lane]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) total += __builtin_amdgcn_exp2f(top_of[s][lane] - base) * sum_of[s][lane];
    if (u >= a.U) return;
    if (a.lse && share == 0 && blockIdx.y == 0) a.lse[row] = total != 0.f ? (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f : -INFINITY;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int d0 = blockIdx.y * 32 + share;
    const float *part = a.part + (size_t)bh * a.D * a.U + u;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    for (int s = 0; s < a.splits; ++s) {  // (eight channels' loads at a time)
        const float w = __builtin_amdgcn_exp2f(top_of[s][lane] - base) * inv;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += w * part[s * all + (size_t)min(d0 + 4 * i, a.D - 1) * a.U];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (d0 + 4 * i < a.D) store_from_f32((S *)a.out, (size_t)b * a.os + ((size_t)h * a.D + d0 + 4 * i) * a.U + u, v[i]);
}

// ---- which form, and its sizes --------------------------------------------------------------------------------
template <typename S, int DP, int NB, int NW, bool SHARED>
constexpr int lds_bytes()
{
    if constexpr (SHARED) {  // two tiles of keys and of values in turn; before them the workgroup's tokens, after them its results as float blocks
        return most({4 * Tile<S, DP, NB, NW * 64>::kBytes, OwnColumns<S, DP, NW>::Own::kBytes, NW * WaveColumns<S, DP>::Own::kBytes, NW * DP * 128});
    }
    return most({NW * 2 * Tile<S, DP, NB, 64>::kBytes, NW * 128 * 4 + NW * (DP / 32 * 16) * 64 * 4});
}

template <typename S, int DP, int NB, int NW, bool SHARED>
hipError_t run(AttnArgs a, hipStream_t s)
{
    static LdsOptIn opt;
    constexpr int bytes = lds_bytes<S, DP, NB, NW, SHARED>();
    static_assert(bytes <= 160 * 1024, "LDS of a CU");
    auto *fn = attn_fwd_kernel<S, DP, NB, NW, SHARED>;
    const hipError_t e = ensure_dynamic_lds(opt, (const void *)fn, bytes);
    if (e != hipSuccess) return e;
    fn<<<dim3((unsigned)(a.B * a.Hkv) * a.col_tiles * a.splits), dim3(NW * 64), bytes, s>>>(a);
    return hipGetLastError();
}

constexpr int kApartColumns = 32, kApartWaves = 8;  // (one token, 600 frames: 4 wavefronts 12.5 us, 8 11.1, 16 with half tiles 13.9)
// Few columns go apart (but float tiles of wide heads, one per wavefront, do not fit the registers).  Of the others, 256 share keys and
// values where there are that many: they are then read and written to LDS half as often.
AttnForm form_of(bool bf16, int DP, int U, int G)
{
    if ((long long)U * G <= kApartColumns && (bf16 || DP <= 64)) return {32, bf16 && DP <= 64 ? 64 : 32, kApartWaves, 1, attn_work(bf16)};
    if (bf16 && U > 128) return {256, 64, 1, DP <= 64 ? 2 : 1, 1};
    return {128, bf16 ? 64 : 32, 1, bf16 || DP <= 64 ? 2 : 1, attn_work(bf16)};
}

template <typename S, int DP>
hipError_t run_form(const AttnArgs &a, hipStream_t s)
{
    constexpr bool bf16 = sizeof(S) == 2;
    const AttnForm f = form_of(bf16, DP, a.U, a.G);
    if constexpr (bf16 || DP <= 64) {
        if (f.columns == 32) return run<S, DP, bf16 && DP <= 64 ? 2 : 1, kApartWaves, false>(a, s);
    }
    if constexpr (bf16) {
        if (f.columns == 256) return run<S, DP, 2, 8, true>(a, s);
    }
    return run<S, DP, bf16 ? 2 : 1, 4, true>(a, s);
}
template <typename S>
hipError_t run_any(const AttnArgs &a, hipStream_t s)
{
    hipError_t e;
    if (a.D <= 32) e = run_form<S, 32>(a, s);
    else if (a.D <= 64) e = run_form<S, 64>(a, s);
    else if (a.D <= 96) e = run_form<S, 96>(a, s);
    else e = run_form<S, 128>(a, s);
    if (e != hipSuccess || a.splits == 1) return e;
    attn_join_kernel<S><<<dim3((unsigned)(a.B * a.H) * ((a.U + 63) / 64), (a.D + 31) / 32), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

AttnPlan attn_fwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T)
{
    return attn_plan(form_of(bf16, (D + 31) / 32 * 32, U, H / Hkv), B, H, Hkv, D, U, T);
}

hipError_t launch_attn_fwd(bool bf16, const AttnArgs &a, hipStream_t s) { return bf16 ? run_any<bf16_t>(a, s) : run_any<float>(a, s); }

}  // namespace nm
