// Norms of queries and keys for each head and their rotation by position (definition: include/nm_head_norm.h).
//
// Work goes by units of two channels: the pairs that turn together, then the channels that do not turn, two by two.  Two divisions:
//   tiles  one to four wavefronts own 32 tokens of a head, a lane eight neighbouring tokens of a unit, so that the sums over a head's
//          channels are eight values of a lane, a few exchanges and LDS, and every tensor is read and written once.  A lane makes the angles of
//          its unit and tokens once for all heads that the workgroup takes.  The last tile of a row begins as many tokens before its end; what
//          two tiles share is made twice, alike.  Tiles that share 128-byte lines of memory run on the same XCD: with 64 tokens a tile has
//          lines of its own, but half as many workgroups (backward of 4 x 1333 tokens, 10 heads of 128: 21 us instead of 17).
//   single a wavefront owns one token of a head, a lane a unit: rows of fewer than eight tokens, and everything that goes into the cache.
//          (32 items, 20 heads of 64, forward and backward with its join: 8 tokens each 5.1 and 14 us, as tiles 5.6 and 10; 16 tokens 8.2 and
//          18 against 5.7 and 10.)
// Forward of 32 x 150 tokens, 20 heads of 64: 11 us, backward of 4 x 1333, 10 heads of 128: 17 + 4; their bytes would take 4 and 8.  Vector units are
// busy a quarter of the time and memory at a third to half of its rate: a launch of few short workgroups, whose loads, sums and stores
// follow one another.  Single tokens of 32 items into the cache: 3.9 us, the launch and one chain of loads.
// An angle is position * freqs[i] as a part of a turn in double, of which only the fraction goes on in float: 500000 tokens into a
// recording a float product would leave the angle to 1/30.
#include "../../include/nm_head_norm.h"
#include "token_ops.h"

namespace nm {
namespace {

constexpr int kMostTiles = 1024;   // that workgroups of the backward pass have side by side: rows of partial sums
constexpr int kMaxD = 128;
constexpr int kGroups = 4;         // of eight tokens, that a tile has

struct Heads {
    int B, H, Hkv, D, U;
    const void *x, *dout;
    long long xs, ds, os;
    const float *qw, *kw;
    float eps;
    const double *freqs;
    int rot;
    const int *positions, *len;
    void *out;     // out, dx or the returned queries
    bool norm, pairs;
    int u_tiles, heads_each, q_chunks;  // heads of a workgroup; the first chunks are of queries
    float *part;   // [chunks][workgroups][D]
    // of the cache
    int pages, log_page, max_pages;
    const int *page_table, *q_len;
    void *k_cache, *v_cache;
};

__device__ __forceinline__ void channels_of(const Heads &a, int unit, int &c0, int &c1)
{
    const int half = a.rot >> 1;
    const bool apart = !a.pairs && unit < half;
    c0 = apart ? unit : 2 * unit;
    c1 = apart ? unit + half : 2 * unit + 1;
}

// Cosine and sine of a position's angle; per_turn: turns from one position to the next.  The fraction of a turn is made in double and goes on as
// the nearest quarter and what is left of it, at most an eighth: there the series of both functions end after x^9 and x^8 within half a unit of float.
__device__ __forceinline__ float2 turn(int position, double per_turn)
{
    const double t = (double)position * per_turn;
    const float f = (float)(t - rint(t)), quarter = rintf(4.f * f);
    const float x = __builtin_fmaf(quarter, -0.25f, f) * 6.28318530717958648f, z = x * x;
    const float s = __builtin_fmaf(x * z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
    const float c = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const uint32_t n = (uint32_t)(int)quarter;
    const float co = n & 1 ? s : c, si = n & 1 ? c : s;
    return {__uint_as_float(__float_as_uint(co) ^ ((n + 1) & 2) << 30), __uint_as_float(__float_as_uint(si) ^ (n & 2) << 30)};
}
constexpr double kPerRadian = 0.15915494309189533577;  // turns

// Eight tokens of a channel as they lie in memory
template <typename S>
struct Eight;
template <>
struct Eight<bf16_t> {
    u32x4_t r;
    __device__ __forceinline__ void load(const bf16_t *head, uint32_t at) { __builtin_memcpy(&r, reinterpret_cast<const char *>(head) + at, 16); }
    __device__ __forceinline__ float at(int e) const { return __uint_as_float(e & 1 ? r[e >> 1] & 0xffff0000u : r[e >> 1] << 16); }
};
template <>
struct Eight<float> {
    float r[8];
    __device__ __forceinline__ void load(const float *head, uint32_t at) { __builtin_memcpy(r, reinterpret_cast<const char *>(head) + at, 32); }
    __device__ __forceinline__ float at(int e) const { return r[e]; }
};

// PER wavefronts take a head, 64 / GROUPS units each and GROUPS groups of eight tokens: with all channels of a head in one wavefront, a lane's
// registers would be too many for more than one or two wavefronts a SIMD.
template <int GROUPS, int PER>
struct TileForm {
    static constexpr int kTile = 8 * GROUPS, kUnits = 64 / GROUPS;                                           // tokens; units of a wavefront
    static constexpr int kHeads = PER < 4 ? 4 / PER : 1, kWaves = kHeads * PER, kThreads = kWaves * 64;  // heads side by side
};

template <typename S, int GROUPS, int PER, bool BACK>
__global__ __launch_bounds__((TileForm<GROUPS, PER>::kThreads), sizeof(S) == 2 ? 4 : 2) void heads_tile_kernel(Heads a)
{
    typedef TileForm<GROUPS, PER> F;
    typedef Eight<S> E;
    constexpr int kTile = F::kTile;
    __shared__ float sums[2][F::kWaves][kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane % GROUPS;
    const int slot = wave / PER, unit = wave % PER * F::kUnits + lane / GROUPS, units = a.D >> 1, half = a.rot >> 1;
    const bool is = unit < units, keys = blockIdx.y >= a.q_chunks;
    const int h_begin = keys ? a.H + (blockIdx.y - a.q_chunks) * a.heads_each : blockIdx.y * a.heads_each;
    const int h_end = min(h_begin + a.heads_each, keys ? a.H + a.Hkv : a.H);
    int i0, i1;
    channels_of(a, min(unit, units - 1), i0, i1);
    const float *weight = a.norm ? (keys ? a.kw : a.qw) : nullptr;
    const float w0 = weight ? weight[i0] : 1.f, w1 = weight ? weight[i1] : 1.f, per_d = 1.f / (float)a.D;
    const uint32_t c0 = (uint32_t)i0 * (uint32_t)a.U * (uint32_t)sizeof(S), c1 = (uint32_t)i1 * (uint32_t)a.U * (uint32_t)sizeof(S);  // bytes in a head
    float dw0 = 0.f, dw1 = 0.f;
    // sums over a head's channels, for the lane's eight tokens, in order
    auto over_head = [&](float (&v)[8], int buffer) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sum_of_every<GROUPS>(v[e]);
        if constexpr (PER > 1) {
            if (lane < GROUPS) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[buffer][wave][8 * lane + e] = v[e];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = sums[buffer][slot * PER][8 * g + e];
#pragma unroll
                for (int w = 1; w < PER; ++w) v[e] += sums[buffer][slot * PER + w][8 * g + e];
            }
        }
    };
    // neighbouring workgroups go to different XCDs: neighbouring tiles, which share lines of memory, are eight apart
    const int tiles = a.B * a.u_tiles, each = (tiles + 7) / 8;
    for (int i = blockIdx.x; i < each * 8; i += gridDim.x) {
        const int tile = i % 8 * each + i / 8;
        if (tile >= tiles) continue;  // (uniform)
        const int b = tile / a.u_tiles, u0 = (tile - b * a.u_tiles) * kTile, ub = max(0, min(u0, a.U - kTile));
        const int len = length_in(a.len, b, a.U);
        const bool active = is && ub + 8 * g < a.U, some = ub < len;                // (rows shorter than a tile)
        const int t = min(ub + 8 * g, a.U - 8), first = a.U < kTile ? 8 * g : u0;  // tokens before `first` are another lane's too
        const uint32_t at0 = c0 + (uint32_t)t * (uint32_t)sizeof(S), at1 = c1 + (uint32_t)t * (uint32_t)sizeof(S);
        const size_t head = (size_t)a.D * a.U;
        E x0, x1, d0, d1;
        auto load = [&](int h) {
            const int from = min(h, h_end - 1);
            if (!BACK || a.norm) {
                const S *x = (const S *)a.x + (size_t)b * a.xs + from * head;
                x0.load(x, at0);
                x1.load(x, at1);
            }
            if constexpr (BACK) {
                const S *d = (const S *)a.dout + (size_t)b * a.ds + from * head;
                d0.load(d, at0);
                d1.load(d, at1);
            }
        };
        if (some) load(h_begin + slot);  // (on its way while the angles are made)
        float2 cs[8];  // of the lane's tokens, for its unit of every head
        if (a.rot && some) {
            const double per_turn = unit < half ? a.freqs[unit] * kPerRadian : 0.0;
            const int *positions = a.positions ? a.positions + (size_t)b * a.U + t : nullptr;
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = turn(positions ? positions[e] : t + e, per_turn);
        }
        for (int hh = h_begin, turn_of = 0; hh < h_end; hh += F::kHeads, turn_of ^= 1) {
            const int h = hh + slot;
            const bool stores = active && h < h_end;
            char *out = reinterpret_cast<char *>((S *)a.out + (size_t)b * a.os + min(h, h_end - 1) * head);
            float y0[8], y1[8];
            if (!some) {  // (uniform)
#pragma unroll
                for (int e = 0; e < 8; ++e) y0[e] = y1[e] = 0.f;
            } else {
                float r[8], v0[8], v1[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v0[e] = (!BACK || a.norm) ? x0.at(e) : 0.f;
                    v1[e] = (!BACK || a.norm) ? x1.at(e) : 0.f;
                    y0[e] = BACK ? d0.at(e) : 0.f;
                    y1[e] = BACK ? d1.at(e) : 0.f;
                }
                if (hh + F::kHeads < h_end) load(h + F::kHeads);
                if (a.norm) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[e] = is ? v0[e] * v0[e] + v1[e] * v1[e] : 0.f;
                    over_head(r, BACK ? 0 : turn_of);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        r[e] = rsqrtf(r[e] * per_d + a.eps);
                        v0[e] *= r[e];
                        v1[e] *= r[e];
                    }
                }
                if constexpr (!BACK) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float n0 = v0[e] * w0, n1 = v1[e] * w1;
                        y0[e] = a.rot ? n0 * cs[e].x - n1 * cs[e].y : n0;
                        y1[e] = a.rot ? n1 * cs[e].x + n0 * cs[e].y : n1;
                    }
                } else {
                    if (a.rot) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float v = y0[e];
                            y0[e] = v * cs[e].x + y1[e] * cs[e].y;
                            y1[e] = y1[e] * cs[e].x - v * cs[e].y;
                        }
                    }
                    if (a.norm) {
                        float m[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float p0 = y0[e] * v0[e], p1 = y1[e] * v1[e];
                            const bool mine = stores && t + e >= first && t + e < len;
                            dw0 += mine ? p0 : 0.f;
                            dw1 += mine ? p1 : 0.f;
                            m[e] = is ? w0 * p0 + w1 * p1 : 0.f;
                        }
                        over_head(m, 1);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float mean = m[e] * per_d;
                            y0[e] = r[e] * (w0 * y0[e] - v0[e] * mean);
                            y1[e] = r[e] * (w1 * y1[e] - v1[e] * mean);
                        }
                    }
                }
                if (t + 8 > len) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        y0[e] = t + e < len ? y0[e] : 0.f;
                        y1[e] = t + e < len ? y1[e] : 0.f;
                    }
                }
            }
            if (stores) {
                store8(reinterpret_cast<S *>(out + at0), 8, y0);
                store8(reinterpret_cast<S *>(out + at1), 8, y1);
            }
        }
    }
    if constexpr (BACK) {
        if (!a.part) return;  // (uniform)
        __shared__ float all[F::kHeads][kMaxD];
#pragma unroll
        for (int d = 1; d < GROUPS; d <<= 1) {
            dw0 += __shfl_xor(dw0, d);
            dw1 += __shfl_xor(dw1, d);
        }
        if (g == 0 && is) {
            all[slot][i0] = dw0;
            all[slot][i1] = dw1;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += F::kThreads) {
            float s = all[0][c];
#pragma unroll
            for (int i = 1; i < F::kHeads; ++i) s += all[i][c];
            a.part[((size_t)blockIdx.y * gridDim.x + blockIdx.x) * a.D + c] = s;
        }
    }
}

// A token of a head for each wavefront.  CACHE: keys go to their page, values too, queries to `out`.
template <typename S, bool BACK, bool CACHE>
__global__ __launch_bounds__(256) void heads_single_kernel(Heads a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int all = a.H + (CACHE ? 2 : 1) * a.Hkv, tokens = a.B * a.U;
    const int units = a.D >> 1, half = a.rot >> 1;
    int c0, c1;
    channels_of(a, min(lane, units - 1), c0, c1);
    const bool mine = lane < units;
    // the backward pass: a workgroup takes every gridDim.x-th token of its chunk of heads and leaves their sums
    const int chunk = BACK ? blockIdx.y : 0;
    const bool keys_chunk = BACK && chunk >= a.q_chunks;
    const int h_first = !BACK ? 0 : keys_chunk ? a.H + (chunk - a.q_chunks) * a.heads_each : chunk * a.heads_each;
    const int h_count = !BACK ? all : min(a.heads_each, (keys_chunk ? a.H + a.Hkv : a.H) - h_first);
    const int count = tokens * h_count, stride = gridDim.x * 4;  // (below 2^25 and, of the grid, 2^26)
    float dw0 = 0.f, dw1 = 0.f;
    for (int i = blockIdx.x * 4 + wave; i < count; i += stride) {
        const int bh = i / a.U, u = i - bh * a.U, b = bh / h_count, h = h_first + bh - b * h_count;
        const S *x = (const S *)a.x + (size_t)b * a.xs + (size_t)h * a.D * a.U + u;
        int len, position = u;
        if constexpr (CACHE) {
            len = length_in(a.q_len, b, a.U);
            position = max(a.len[b], 0) - len + u;
        } else {
            len = length_in(a.len, b, a.U);
            if (a.positions) position = a.positions[(size_t)b * a.U + u];
        }
        const bool there = u < len, key = h >= a.H, value = CACHE && h >= a.H + a.Hkv;
        S *out = (S *)a.out + (size_t)b * a.os + (size_t)h * a.D * a.U + u;
        size_t row = 0;
        if (CACHE && key) {
            const int page_at = position >> a.log_page;
            if (!there || position < 0 || page_at >= a.max_pages) continue;
            const int page = a.page_table[(size_t)b * a.max_pages + page_at];
            if (page < 0 || page >= a.pages) continue;
            const int kvh = h - a.H - (value ? a.Hkv : 0), size = 1 << a.log_page, at = position & (size - 1);
            row = ((size_t)page * a.Hkv + kvh) * size * a.D + (value ? (size_t)at : (size_t)at * a.D);
            if (value) {
                S *v = (S *)a.v_cache + row;
                for (int d = lane; d < a.D; d += 64) v[(size_t)d << a.log_page] = x[(size_t)d * a.U];
                continue;
            }
        }
        float y0 = 0.f, y1 = 0.f;
        if (there) {  // (uniform)
            float2 cs = {1.f, 0.f};
            if (lane < half) cs = turn(position, a.freqs[lane] * kPerRadian);
            const float *weight = a.norm ? (key ? a.kw : a.qw) : nullptr;
            const float w0 = weight ? weight[c0] : 1.f, w1 = weight ? weight[c1] : 1.f;
            float x0 = 0.f, x1 = 0.f, r = 1.f;
            if (mine && (!BACK || a.norm)) {
                x0 = load_as_f32(x, (size_t)c0 * a.U);
                x1 = load_as_f32(x, (size_t)c1 * a.U);
            }
            if (a.norm) {
                float s = x0 * x0 + x1 * x1;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
                r = rsqrtf(s / (float)a.D + a.eps);
                x0 *= r;
                x1 *= r;
            }
            if constexpr (!BACK) {
                const float n0 = a.norm ? x0 * w0 : x0, n1 = a.norm ? x1 * w1 : x1;
                y0 = n0 * cs.x - n1 * cs.y;
                y1 = n1 * cs.x + n0 * cs.y;
                if (lane >= half) {
                    y0 = n0;
                    y1 = n1;
                }
            } else if (mine) {
                const S *d = (const S *)a.dout + (size_t)b * a.ds + (size_t)h * a.D * a.U + u;
                const float g0 = load_as_f32(d, (size_t)c0 * a.U), g1 = load_as_f32(d, (size_t)c1 * a.U);
                y0 = lane < half ? g0 * cs.x + g1 * cs.y : g0;
                y1 = lane < half ? g1 * cs.x - g0 * cs.y : g1;
            }
            if (BACK && a.norm) {
                const float p0 = y0 * x0, p1 = y1 * x1;
                dw0 += p0;
                dw1 += p1;
                float m = w0 * p0 + w1 * p1;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) m += __shfl_xor(m, d);
                m /= (float)a.D;
                y0 = r * (w0 * y0 - x0 * m);
                y1 = r * (w1 * y1 - x1 * m);
            }
        }
        if (!mine) continue;
        if (CACHE && key) {
            store_from_f32((S *)a.k_cache + row, c0, y0);
            store_from_f32((S *)a.k_cache + row, c1, y1);
        } else {
            store_from_f32(out, (size_t)c0 * a.U, y0);
            store_from_f32(out, (size_t)c1 * a.U, y1);
        }
    }
    if constexpr (BACK) {
        if (!a.part) return;
        __shared__ float sums[4][kMaxD];
        if (mine) {
            sums[wave][c0] = dw0;
            sums[wave][c1] = dw1;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += 256)
            a.part[((size_t)chunk * gridDim.x + blockIdx.x) * a.D + c] = sums[0][c] + sums[1][c] + sums[2][c] + sums[3][c];
    }
}

// Sums of the workgroups' rows in order: 32 channels of the queries' or the keys' weight, eight rows at a time
__global__ __launch_bounds__(256) void heads_join_kernel(const float *part, int D, int q_rows, int k_rows, float *dq, float *dk)
{
    __shared__ float sums[8][32];
    const int c = threadIdx.x & 31, lane = threadIdx.x >> 5, tiles = (D + 31) / 32, tile = blockIdx.x % tiles, keys = blockIdx.x / tiles;
    float *out = keys ? dk : dq;
    if (!out) return;
    const int rows = keys ? k_rows : q_rows, ch = min(tile * 32 + c, D - 1);
    const float *p = part + (keys ? (size_t)q_rows * D : 0) + ch;
    float s = 0.f;
#pragma unroll 8
    for (int r = lane; r < rows; r += 8) s += p[(size_t)r * D];
    sums[lane][c] = s;
    __syncthreads();
    if (lane || tile * 32 + c >= D) return;
    for (int i = 1; i < 8; ++i) s += sums[i][c];
    out[ch] = s;
}

// How the heads and tokens are shared among workgroups
struct Plan {
    bool tiles;
    int u_tiles, heads_each, q_chunks, k_chunks, side;  // side: workgroups along the tokens
};
Plan plan_of(int B, int H, int Hkv, int D, int U, bool back)
{
    Plan p = {};
    p.tiles = U >= 8;
    p.u_tiles = (U + 8 * kGroups - 1) / (8 * kGroups);
    // forward and backward with its join, of 32 x 150 tokens (10 heads of 96) and 4 x 1333 (10 of 128): with four heads a workgroup 11.2 and 20, 12 and 22 us, with
    // two 9.7 and 19, 11 and 23 (20 heads of 64: 11.0 and 21, 11.4 and 25), with eight 13 and 23, 14 and 26
    p.heads_each = 4;
    const long long work = p.tiles ? (long long)B * p.u_tiles : ((long long)B * U + 3) / 4;
    const long long side = p.tiles ? (work + 7) / 8 * 8 : work;
    p.side = (int)(back && side > kMostTiles ? kMostTiles : side);
    p.q_chunks = (H + p.heads_each - 1) / p.heads_each;
    p.k_chunks = (Hkv + p.heads_each - 1) / p.heads_each;
    return p;
}

template <typename S, int GROUPS, int PER, bool BACK>
hipError_t run_tile(const Heads &a, const Plan &p, hipStream_t s)
{
    heads_tile_kernel<S, GROUPS, PER, BACK><<<dim3(p.side, p.q_chunks + p.k_chunks), dim3(TileForm<GROUPS, PER>::kThreads), 0, s>>>(a);
    return hipGetLastError();
}
template <typename S, bool BACK>
hipError_t run(Heads a, hipStream_t s)
{
    const Plan p = plan_of(a.B, a.H, a.Hkv, a.D, a.U, BACK);
    a.u_tiles = p.u_tiles;
    a.heads_each = p.heads_each;
    a.q_chunks = p.q_chunks;
    if (!p.tiles) {
        const long long waves = (long long)a.B * a.U * (a.H + a.Hkv);
        const dim3 grid = BACK ? dim3(p.side, p.q_chunks + p.k_chunks) : dim3((unsigned)((waves + 3) / 4));
        heads_single_kernel<S, BACK, false><<<grid, dim3(256), 0, s>>>(a);
        return hipGetLastError();
    }
    constexpr int kUnits = 64 / kGroups;
    switch ((a.D / 2 + kUnits - 1) / kUnits) {
    case 1: return run_tile<S, kGroups, 1, BACK>(a, p, s);
    case 2: return run_tile<S, kGroups, 2, BACK>(a, p, s);
    case 3: return run_tile<S, kGroups, 3, BACK>(a, p, s);
    default: return run_tile<S, kGroups, 4, BACK>(a, p, s);
    }
}

int check(int B, int H, int Hkv, int D, int U, const void *q_weight, const void *k_weight, float eps, const void *freqs, int rot, unsigned flags, int dtype)
{
    if (B <= 0 || H <= 0 || Hkv < 0 || D <= 0 || U <= 0 || rot < 0 || rot > D || rot % 2 || (rot != 0) != (freqs != nullptr) || !known_dtype(dtype) ||
        (flags & ~3u) || !(eps >= 0.f) || !finite_float(eps) || (!(flags & NM_HEADS_NORM) && (q_weight || k_weight)) || (!Hkv && k_weight))
        return NM_ERR_BAD_ARG;
    if (D % 2 || D > kMaxD) return NM_ERR_UNSUPPORTED;
    const long long most = (1LL << 31) - 1, heads = (long long)H + 2LL * Hkv;
    if (heads > most / D || heads * D > most / U || (long long)D * (long long)element(dtype) > ((1LL << 32) - 1) / U) return NM_ERR_UNSUPPORTED;  // (a head's rows: below 4 GiB)
    // the grids: below 2^32 work items, of 64 for a token of a head or 256 for a tile of four heads; no more than 2^16 chunks of heads
    if ((long long)B * U > most / 2 || heads > 1 << 16 || (U < 8 ? (long long)B * U * heads >= 1LL << 25 : (long long)B * ((U + 31) / 32) * (heads / 4 + 2) >= 1LL << 23))
        return NM_ERR_UNSUPPORTED;
    return NM_OK;
}
Heads common(int B, int H, int Hkv, int D, int U, const void *x, long long x_stride, const float *qw, const float *kw, float eps, const double *freqs,
             int rot, unsigned flags)
{
    Heads a = {};
    a.B = B; a.H = H; a.Hkv = Hkv; a.D = D; a.U = U;
    a.x = x; a.xs = x_stride;
    a.qw = qw; a.kw = kw; a.eps = eps;
    a.freqs = freqs; a.rot = rot;
    a.norm = flags & NM_HEADS_NORM;
    a.pairs = flags & NM_HEADS_PAIRS;
    return a;
}

}  // namespace
}  // namespace nm

using namespace nm;

extern "C" {

int nm_head_norm_fwd(int B, int heads, int kv_heads, int D, int U, const void *x, long long x_stride, const float *q_weight,
                     const float *k_weight, float eps, const double *freqs, int rot, const int *positions, const int *lengths, void *out,
                     long long out_stride, unsigned flags, int dtype, void *hip_stream)
{
    const int st = check(B, heads, kv_heads, D, U, q_weight, k_weight, eps, freqs, rot, flags, dtype);
    if (st != NM_OK) return st;
    const long long item = (long long)(heads + kv_heads) * D * U;
    if (!x || !out || !stride_ok(x_stride, item) || !stride_ok(out_stride, item)) return NM_ERR_BAD_ARG;
    const int size = (int)element(dtype);
    const Items to = {out, out_stride, item, B, size};
    const Region in[5] = {{q_weight, (size_t)D * 4}, {k_weight, (size_t)D * 4}, {freqs, (size_t)rot * 4}, {positions, (size_t)B * U * 4}, {lengths, (size_t)B * 4}};
    if (meet(to, Items{x, x_stride, item, B, size}) || meets(to.region(), in)) return NM_ERR_BAD_ARG;
    Heads a = common(B, heads, kv_heads, D, U, x, x_stride, q_weight, k_weight, eps, freqs, rot, flags);
    a.positions = positions; a.len = lengths;
    a.out = out; a.os = out_stride;
    hipStream_t s = (hipStream_t)hip_stream;
    return status_of(dtype == NM_BF16 ? run<bf16_t, false>(a, s) : run<float, false>(a, s));
}

size_t nm_head_norm_bwd_workspace_bytes(int B, int heads, int kv_heads, int D, int U, int dtype)
{
    if (check(B, heads, kv_heads, D, U, nullptr, nullptr, 0.f, nullptr, 0, NM_HEADS_NORM, dtype) != NM_OK) return 0;
    const Plan p = plan_of(B, heads, kv_heads, D, U, true);
    return align_up((size_t)p.side * (p.q_chunks + p.k_chunks) * D * 4, 256);
}

int nm_head_norm_bwd(int B, int heads, int kv_heads, int D, int U, const void *dout, long long dout_stride, const void *x,
                     long long x_stride, const float *q_weight, const float *k_weight, float eps, const double *freqs, int rot,
                     const int *positions, const int *lengths, void *dx, long long dx_stride, float *dq_weight, float *dk_weight,
                     unsigned flags, int dtype, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check(B, heads, kv_heads, D, U, q_weight, k_weight, eps, freqs, rot, flags, dtype);
    if (st != NM_OK) return st;
    const long long item = (long long)(heads + kv_heads) * D * U;
    if (!dout || !x || !dx || !stride_ok(x_stride, item) || !stride_ok(dout_stride, item) || !stride_ok(dx_stride, item) || (dq_weight && !q_weight) ||
        (dk_weight && !k_weight))
        return NM_ERR_BAD_ARG;
    const int size = (int)element(dtype);
    const size_t vec = (size_t)D * 4;
    const Items to = {dx, dx_stride, item, B, size}, from[2] = {{dout, dout_stride, item, B, size}, {x, x_stride, item, B, size}};
    const Region in[7] = {{q_weight, vec}, {k_weight, vec}, {freqs, (size_t)rot * 4}, {positions, (size_t)B * U * 4}, {lengths, (size_t)B * 4},
                          from[0].region(), from[1].region()};
    const Region small[5] = {in[0], in[1], in[2], in[3], in[4]}, wq = {dq_weight, vec}, wk = {dk_weight, vec};
    if (meet(to, from[0]) || meet(to, from[1]) || meets(to.region(), small) || meets(wq, in) || meets(wk, in) || meet(wq, wk) || meet(wq, to.region()) ||
        meet(wk, to.region()))
        return NM_ERR_BAD_ARG;
    const bool sums = dq_weight || dk_weight;
    if (sums && workspace_missing(workspace, workspace_bytes, nm_head_norm_bwd_workspace_bytes(B, heads, kv_heads, D, U, dtype))) return NM_ERR_WORKSPACE;
    Heads a = common(B, heads, kv_heads, D, U, x, x_stride, q_weight, k_weight, eps, freqs, rot, flags);
    a.dout = dout; a.ds = dout_stride;
    a.positions = positions; a.len = lengths;
    a.out = dx; a.os = dx_stride;
    a.part = sums ? (float *)workspace : nullptr;
    hipStream_t s = (hipStream_t)hip_stream;
    hipError_t e = dtype == NM_BF16 ? run<bf16_t, true>(a, s) : run<float, true>(a, s);
    if (e != hipSuccess || !sums) return status_of(e);
    const Plan p = plan_of(B, heads, kv_heads, D, U, true);
    heads_join_kernel<<<dim3(2 * ((D + 31) / 32)), dim3(256), 0, s>>>(a.part, D, p.side * p.q_chunks, p.side * p.k_chunks, dq_weight, dk_weight);
    return status_of(hipGetLastError());
}

int nm_head_norm_cache(int B, int heads, int kv_heads, int D, int U, const void *x, long long x_stride, const float *q_weight,
                       const float *k_weight, float eps, const double *freqs, int rot, int pages, int page_size, const int *page_table,
                       int max_pages, const int *lengths, const int *q_lengths, void *k_cache, void *v_cache, void *q_out,
                       long long q_stride, unsigned flags, int dtype, void *hip_stream)
{
    const int st = check(B, heads, kv_heads, D, U, q_weight, k_weight, eps, freqs, rot, flags, dtype);
    if (st != NM_OK) return st;
    const long long item = (long long)(heads + 2 * kv_heads) * D * U, q_item = (long long)heads * D * U, most = (1LL << 31) - 1;
    if (kv_heads <= 0 || pages <= 0 || max_pages <= 0 || !x || !page_table || !lengths || !k_cache || !v_cache || !q_out || !stride_ok(x_stride, item) ||
        !stride_ok(q_stride, q_item))
        return NM_ERR_BAD_ARG;
    int log_page = 4;
    while (log_page < 8 && 1 << log_page != page_size) ++log_page;
    if (1 << log_page != page_size) return NM_ERR_UNSUPPORTED;
    if ((long long)B * max_pages > most || (long long)B * U * (heads + 2LL * kv_heads) >= 1LL << 25 || (long long)pages * kv_heads > (1LL << 40) / (page_size * D)) return NM_ERR_UNSUPPORTED;
    const int size = (int)element(dtype);
    const size_t cache = (size_t)pages * kv_heads * page_size * D * size;
    const Region q = Items{q_out, q_stride, q_item, B, size}.region(), from = Items{x, x_stride, item, B, size}.region(), k = {k_cache, cache}, v = {v_cache, cache};
    const Region in[6] = {{q_weight, (size_t)D * 4}, {k_weight, (size_t)D * 4}, {freqs, (size_t)rot * 4}, {page_table, (size_t)B * max_pages * 4},
                          {lengths, (size_t)B * 4}, {q_lengths, (size_t)B * 4}};
    if (meets(q, in) || meets(k, in) || meets(v, in) || meet(q, k) || meet(q, v) || meet(k, v) || meet(k, from) || meet(v, from) ||
        meet(Items{q_out, q_stride, q_item, B, size}, Items{x, x_stride, item, B, size}))
        return NM_ERR_BAD_ARG;
    Heads a = common(B, heads, kv_heads, D, U, x, x_stride, q_weight, k_weight, eps, freqs, rot, flags);
    a.len = lengths; a.q_len = q_lengths;
    a.out = q_out; a.os = q_stride;
    a.pages = pages; a.log_page = log_page; a.max_pages = max_pages; a.page_table = page_table;
    a.k_cache = k_cache; a.v_cache = v_cache;
    const long long waves = (long long)B * U * (heads + 2 * kv_heads);
    const dim3 grid((unsigned)((waves + 3) / 4));
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == NM_BF16) heads_single_kernel<bf16_t, false, true><<<grid, dim3(256), 0, s>>>(a);
    else heads_single_kernel<float, false, true><<<grid, dim3(256), 0, s>>>(a);
    return status_of(hipGetLastError());
}

}  // extern "C"
