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
#include "cross_attn.h"

namespace nm {
namespace {

template <typename S, int DP, int NU, int NB, int NW, bool SHARED>
__global__ __launch_bounds__(NW * 64, sizeof(S) * DP <= 256 ? 2 : 1) void attn_fwd_kernel(AttnArgs a)
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

    // columns of this lane
    int head[NU], u[NU], lo[NU], hi[NU];
    bool exists[NU], there[NU];
    typename M::Frag q[NU][KS];
    int first = a.T, last = 0;  // frames that some column may look at
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const int m = (SHARED ? (ct * NW + wave) * NU + i : ct * NU + i) * 32 + (lane & 31);
        exists[i] = m < a.G * a.U;
        const int g = exists[i] ? m / a.U : 0;
        u[i] = exists[i] ? m - g * a.U : 0;
        head[i] = kvh * a.G + g;
        there[i] = exists[i] && u[i] < q_len;
        lo[i] = 0;
        hi[i] = 0x7fffffff;  // a column that is not there is masked nowhere: it must not slow the others down
        if (there[i]) {
            frames_of(a, b, u[i], len, lo[i], hi[i]);
            first = min(first, lo[i]);
            last = max(last, hi[i]);
        }
        const S *col = (const S *)a.q + (size_t)b * a.qs + (size_t)head[i] * a.D * a.U + u[i];
#pragma unroll
        for (int s = 0; s < KS; ++s) q[i][s] = M::column(col, s, half, a.D, a.U, there[i], a.flip);
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        first = min(first, __shfl_xor(first, d));
        last = max(last, __shfl_xor(last, d));
    }
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    const bool active = last > first;
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
    int t_begin = max(first / TT, split * a.tiles_per_split), t_end = min((last + TT - 1) / TT, (split + 1) * a.tiles_per_split);

    float mx[NU], sum[NU];  // in powers of two, and of this lane's positions
    f32x16_t acc[NU][DP / 32];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        mx[i] = -INFINITY;
        sum[i] = 0.f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][d][r] = 0.f;
    }
    int koff[2];
    M::template across_offsets<true>(lane, koff);

    auto compute = [&](const unsigned char *kt, const unsigned char *vt, int t0) {
        f32x16_t s[NU][NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int i = 0; i < NU; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[i][n][r] = 0.f;
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                const typename M::Frag f = M::across(kt + n * T::kBlock, koff, st);
#pragma unroll
                for (int i = 0; i < NU; ++i) s[i][n] = M::mul(f, q[i][st], s[i][n]);
            }
        }
        typename M::Probs p[NU][NB];
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            if (!__all(lo[i] <= t0 && t0 + TT <= hi[i])) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int t = t0 + 32 * n + M::position(r, half);
                        s[i][n][r] = t >= lo[i] && t < hi[i] ? s[i][n][r] : -INFINITY;
                    }
            }
            float top = s[i][0][0];
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][n][r]);
            top = fmaxf(mx[i], half_max(top) * a.c);
            const float base = top == -INFINITY ? 0.f : top;  // (nothing allowed so far: every probability is zero)
            if (!__all(top == mx[i])) {
                const float shrink = __builtin_amdgcn_exp2f(mx[i] - base);
                sum[i] *= shrink;
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][d][r] *= shrink;
                mx[i] = top;
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[i][n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][n][r], a.c, -base));
                    sum[i] += s[i][n][r];
                }
                p[i][n] = M::probs(s[i][n]);
            }
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                const typename M::Along f = M::along(vt + n * T::kBlock, d * 32, lane);
#pragma unroll
                for (int i = 0; i < NU; ++i) acc[i][d] = M::mul(f, p[i][n], acc[i][d]);
            }
    };

    T kt, vt;
    if constexpr (SHARED) {
        if (t_begin < t_end) {
            kt.load(krows, a.D, a.T, t_begin * TT, threadIdx.x);
            vt.load(vrows, a.D, a.T, t_begin * TT, threadIdx.x);
        }
        for (int t = t_begin, turn = 0; t < t_end; ++t, turn ^= 1) {
            unsigned char *buf = smem + turn * 2 * T::kBytes;
            kt.write(buf, a.D, a.T, len, t * TT, threadIdx.x);
            vt.write(buf + T::kBytes, a.D, a.T, len, t * TT, threadIdx.x);
            __syncthreads();  // (the other buffer is written next: all are through with it before they pass here again)
            if (t + 1 < t_end) {
                kt.load(krows, a.D, a.T, (t + 1) * TT, threadIdx.x);
                vt.load(vrows, a.D, a.T, (t + 1) * TT, threadIdx.x);
            }
            if (active) compute(buf, buf + T::kBytes, t * TT);
        }
    } else {
        unsigned char *buf = smem + wave * 2 * T::kBytes;
        int t = t_begin + wave;
        if (t < t_end) {
            kt.load(krows, a.D, a.T, t * TT, lane);
            vt.load(vrows, a.D, a.T, t * TT, lane);
        }
        for (; t < t_end; t += NW) {
            wave_fence();
            kt.write(buf, a.D, a.T, len, t * TT, lane);
            vt.write(buf + T::kBytes, a.D, a.T, len, t * TT, lane);
            wave_fence();
            if (t + NW < t_end) {
                kt.load(krows, a.D, a.T, (t + NW) * TT, lane);
                vt.load(vrows, a.D, a.T, (t + NW) * TT, lane);
            }
            compute(buf, buf + T::kBytes, t * TT);
        }
    }

    // one value per (column, channel) and its place
    auto put = [&](int i, int d, int r, float v, float mx_all, float sum_all) {
        const int ch = d * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
        if (!exists[i] || ch >= a.D) return;
        if (a.splits > 1) {
            a.part[(((size_t)split * a.B + b) * a.H + head[i]) * a.D * a.U + (size_t)ch * a.U + u[i]] = v;
        } else {
            const float inv = sum_all == 0.f ? 0.f : 1.f / sum_all;
            store_from_f32((S *)a.out, (size_t)b * a.os + ((size_t)head[i] * a.D + ch) * a.U + u[i], there[i] ? v * inv : 0.f);
        }
    };
    auto put_sums = [&](int i, float mx_all, float sum_all) {
        if (!exists[i] || half) return;
        const size_t row = ((size_t)b * a.H + head[i]) * a.U + u[i];
        if (a.splits > 1) {
            float *ml = a.part_ml + ((size_t)split * a.B * a.H * a.U + row) * 2;
            ml[0] = there[i] ? mx_all : -INFINITY;
            ml[1] = there[i] ? sum_all : 0.f;
        } else if (a.lse) {
            a.lse[row] = there[i] && sum_all != 0.f ? (mx_all + __builtin_amdgcn_logf(sum_all)) * 0.69314718055994531f : -INFINITY;
        }
    };
    if constexpr (SHARED) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const float total = half_sum(sum[i]);
            put_sums(i, mx[i], total);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) put(i, d, r, acc[i][d][r], mx[i], total);
        }
    } else {
        // joined through LDS: every wavefront's maxima and sums, then its products, one column block after the other
        constexpr int PAIRS = DP / 32 * 16;
        float *sums = reinterpret_cast<float *>(smem);            // [NW][2][64]
        float *prod = sums + NW * 128;                            // [NW][PAIRS][64]
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            __syncthreads();
            sums[wave * 128 + lane] = mx[i];
            sums[wave * 128 + 64 + lane] = half_sum(sum[i]);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) prod[(wave * PAIRS + d * 16 + r) * 64 + lane] = acc[i][d][r];
            __syncthreads();
            float top = -INFINITY, total = 0.f, weight[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) top = fmaxf(top, sums[w * 128 + lane]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                weight[w] = __builtin_amdgcn_exp2f(sums[w * 128 + lane] - (top == -INFINITY ? 0.f : top));
                total += weight[w] * sums[w * 128 + 64 + lane];
            }
            if (wave == 0) put_sums(i, top, total);
#pragma unroll
            for (int n = 0; n < PAIRS / NW; ++n) {
                const int pair = n * NW + wave;
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) v += weight[w] * prod[(w * PAIRS + pair) * 64 + lane];
                put(i, pair / 16, pair % 16, v, top, total);
            }
        }
    }
}

// Joins the sums of `splits` workgroups, in order.
template <typename S>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    const size_t rows = (size_t)a.B * a.H * a.U, all = rows * a.D;
    const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= all) return;
    const int u = (int)(e % a.U);
    const size_t hd = e / a.U, bh = hd / a.D;
    const int d = (int)(hd - bh * a.D), b = (int)(bh / a.H), h = (int)(bh - (size_t)b * a.H);
    const size_t row = bh * a.U + u;
    float top = -INFINITY, total = 0.f, v = 0.f;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_ml[(s * rows + row) * 2]);
    const float base = top == -INFINITY ? 0.f : top;
    for (int s = 0; s < a.splits; ++s) {
        const float w = __builtin_amdgcn_exp2f(a.part_ml[(s * rows + row) * 2] - base);
        total += w * a.part_ml[(s * rows + row) * 2 + 1];
        v += w * a.part[s * all + e];
    }
    store_from_f32((S *)a.out, (size_t)b * a.os + ((size_t)h * a.D + d) * a.U + u, total == 0.f ? 0.f : v / total);
    if (a.lse && d == 0) a.lse[row] = total != 0.f ? (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f : -INFINITY;
}

// ---- which form, and its sizes --------------------------------------------------------------------------------
template <typename S, int DP, int NU, int NB, int NW, bool SHARED>
constexpr int lds_bytes()
{
    if constexpr (SHARED) return 4 * Tile<S, DP, NB, NW * 64>::kBytes;
    constexpr int tiles = NW * 2 * Tile<S, DP, NB, 64>::kBytes, join = NW * 128 * 4 + NW * (DP / 32 * 16) * 64 * 4;
    return tiles > join ? tiles : join;
}

struct Form {
    int columns, tile, waves;  // of a workgroup: tokens, positions of a tile, wavefronts with tiles of their own
};
template <typename S, int DP, int NU, int NB, int NW, bool SHARED>
hipError_t run(AttnArgs a, hipStream_t s)
{
    static LdsOptIn opt;
    constexpr int bytes = lds_bytes<S, DP, NU, NB, NW, SHARED>();
    static_assert(bytes <= 160 * 1024, "LDS of a CU");
    auto *fn = attn_fwd_kernel<S, DP, NU, NB, NW, SHARED>;
    const hipError_t e = ensure_dynamic_lds(opt, (const void *)fn, bytes);
    if (e != hipSuccess) return e;
    fn<<<dim3((unsigned)(a.B * a.Hkv) * a.col_tiles * a.splits), dim3(NW * 64), bytes, s>>>(a);
    return hipGetLastError();
}

constexpr int kApartColumns = 32;
Form form_of(bool bf16, int DP, long long columns)
{
    // (float tiles of wide heads, one per wavefront, do not fit the registers)
    if (columns <= kApartColumns && (bf16 || DP <= 64)) return {32, bf16 && DP <= 64 ? 64 : 32, 4};
    if (!bf16) return {128, 32, 1};
    return columns <= 128 || DP > 64 ? Form{128, 64, 1} : Form{256, 64, 1};
}

template <typename S, int DP>
hipError_t run_form(const AttnArgs &a, hipStream_t s)
{
    constexpr bool bf16 = sizeof(S) == 2;
    const Form f = form_of(bf16, DP, (long long)a.G * a.U);
    if constexpr (bf16 || DP <= 64) {
        if (f.columns == 32) return run<S, DP, 1, bf16 && DP <= 64 ? 2 : 1, 4, false>(a, s);
    }
    if constexpr (bf16 && DP <= 64) {
        if (f.columns == 256) return run<S, DP, 2, 2, 4, true>(a, s);
    }
    return run<S, DP, 1, bf16 ? 2 : 1, 4, true>(a, s);
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
    attn_join_kernel<S><<<dim3((unsigned)(((size_t)a.B * a.H * a.U * a.D + 255) / 256)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

AttnPlan attn_fwd_plan(bool bf16, int B, int H, int Hkv, int D, int U, int T)
{
    const int DP = (D + 31) / 32 * 32;
    const long long columns = (long long)(H / Hkv) * U;
    const Form f = form_of(bf16, DP, columns);
    return attn_plan(f.columns, f.tile, f.waves, B, H, Hkv, D, U, T);
}

hipError_t launch_attn_fwd(bool bf16, const AttnArgs &a, hipStream_t s) { return bf16 ? run_any<bf16_t>(a, s) : run_any<float>(a, s); }

}  // namespace nm
