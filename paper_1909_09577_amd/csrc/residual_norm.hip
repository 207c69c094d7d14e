// The norms around a block with its gate and residual scale, forward and backward (definition: include/nm_norm.h).
//
// A norm runs over the channels of a position, and positions lie side by side in memory: a workgroup owns a tile of
// positions of one item with all their channels, so that the sums stay inside it and every tensor is read once and written
// once.  A thread holds groups of 16 bytes of neighbouring positions (eight bfloat16, four float) of every CL-th channel in
// registers, as they were read; sums over channels go over the lanes of a wavefront that hold the same positions and then
// over the wavefronts through LDS, always in the same order.
//
// Rows of any length: the last group of a row is read from where the row's last whole group begins, so that some of its
// positions are there twice, in one workgroup or in two neighbouring ones.  Both copies are made in full from the same inputs and
// stored over each other; sums over time leave one out.
// Rows shorter than a group go to kernels that work by elements.
//
// Bound by memory, and by the phases of a workgroup that loads, sums, stores: forward, 32 x 1024 x 800, bfloat16: 58 us when inputs come
// from the Infinity Cache, 74 from memory (2.8 TB/s); backward, 16 x 768 x up to 777 with a gate per element: 60 and 4 for the sums over
// time (78 from memory, 1.7 TB/s): 300 tiles that are not padding on 256 CUs, one a CU.  Backward with 1024 threads a tile: 69 us (scratch
// memory); without the selections between summands in whole tiles: no change.  In bfloat16 some backward instances keep a few registers
// in scratch memory: 28 to 72 bytes a lane at 129 to 192 and 257 to 384 channels, 20 to 124 at 769 to 896 with LayerNorm and 897 to 1024.
// 16 x 800 positions without a gate, from the Infinity Cache: 384 channels 31 us, 768 (no scratch) 57, 1024 76, with LayerNorm 98.
#include "../../include/nm_norm.h"
#include "../../include/nm_conv1d.h"
#include "nm_common.h"

#include <math.h>

namespace nm {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxChannels = 8192;

struct NormFwd {
    int B, C, T;
    const void *x, *f, *gate;
    int gate_kind;
    const float *rscale, *post_w, *post_b, *next_w, *next_b;
    float eps;
    const int *len;
    void *y, *n;
    bool post, next, layer;
};

struct NormBwd {
    int B, C, T;
    const void *dy, *dn, *y, *f, *gate;
    int gate_kind;
    const float *rscale, *post_w, *post_b, *next_w;
    float eps;
    const int *len;
    void *dx, *df, *dgate;
    float *part;   // [kSums][B*splits][C]: sums over time of a workgroup's positions
    int splits;    // workgroups of an item
    bool post, next, layer;
    unsigned sums;  // which of the sums below are wanted
};
enum { kDnw, kDnb, kDrs, kDpw, kDpb, kDgate, kSums };

template <typename S>
struct Group;  // 16 bytes
template <>
struct Group<bf16_t> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void unpack(u32x4_t r, float (&v)[8])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(r[j] << 16);
            v[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4_t pack(const float (&v)[8])
    {
        return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
};
template <>
struct Group<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void unpack(u32x4_t r, float (&v)[4])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(r[j]);
    }
    static __device__ __forceinline__ u32x4_t pack(const float (&v)[4])
    {
        return u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};

// (at: byte offset in the item, in 32 bits beside a base that all lanes share, so that an address takes one register)
template <typename S>
__device__ __forceinline__ u32x4_t load_group(const S *item, uint32_t at)
{
    u32x4_t r;
    __builtin_memcpy(&r, reinterpret_cast<const char *>(item) + at, 16);
    return r;
}
template <typename S>
__device__ __forceinline__ void store_group(S *item, uint32_t at, u32x4_t r)
{
    __builtin_memcpy(reinterpret_cast<char *>(item) + at, &r, 16);
}
// zeros from position n of the group on
template <typename S>
__device__ __forceinline__ u32x4_t first_positions(u32x4_t r, int n)
{
    if constexpr (sizeof(S) == 2) return first_of8(r, n);
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = j < n ? r[j] : 0u;
    return r;
}

// The same register contents, but values the compiler takes for new ones: what was unpacked from them before is unpacked again
// instead of being kept, which takes twice the registers that the packed groups do (without it the backward kernel spills).
__device__ __forceinline__ void unpack_again(u32x4_t &r) { asm volatile("" : "+v"(r)); }

__device__ __forceinline__ int length_of(const int *len, int b, int T)
{
    if (!len) return T;
    const int n = len[b];
    return n < 0 ? 0 : (n > T ? T : n);
}

// Neighbouring tiles share lines of memory: they go to workgroups of one XCD (every eighth), one after the other.  The grid is a
// multiple of eight; numbers beyond the work return.
__device__ __forceinline__ int neighbours_together() { return (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3); }
inline dim3 eights(size_t n) { return dim3((unsigned)((n + 7) / 8 * 8)); }

// Sums N quantities of each of the V positions over all lanes that hold the same positions (lane % TG): over a wavefront by
// exchanges, over the wavefronts by one thread for every sum, which all threads then read.  (The first barrier keeps a call's
// writes of `total` behind the last call's reads of it, the second one its writes of `part`.)
template <int TG, int V, int NQ>
struct ColumnSums {
    float part[NQ][kWaves][TG * V];
    __attribute__((aligned(16))) float total[NQ][TG * V];
};
template <int TG, int V, int NQ>
__device__ __forceinline__ void sum_columns(ColumnSums<TG, V, NQ> &lds, float (&v)[NQ][V])
{
    static_assert(NQ * TG * V <= kThreads, "a thread for every sum");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tg = lane % TG;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float t = v[q][j];
#pragma unroll
            for (int d = TG; d < 64; d <<= 1) t += __shfl_xor(t, d);
            if (lane < TG) lds.part[q][wave][tg * V + j] = t;
        }
    __syncthreads();
    if (threadIdx.x < NQ * TG * V) {
        const int q = threadIdx.x / (TG * V), at = threadIdx.x % (TG * V);
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) t += lds.part[q][w][at];
        lds.total[q][at] = t;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int j = 0; j < V; ++j) v[q][j] = lds.total[q][tg * V + j];
}

// ---- forward ----------------------------------------------------------------------------------------------------
// TG lanes side by side along a row, NR rows of every kThreads/TG-th channel per thread (NR * kThreads/TG >= C).
template <typename S, int TG, int NR, bool LAYER>
__global__ __launch_bounds__(kThreads) void residual_norm_fwd_kernel(NormFwd p)
{
    constexpr int V = Group<S>::V, CL = kThreads / TG, TW = TG * V;
    __shared__ ColumnSums<TG, V, 1> lds;
    const int tg = threadIdx.x % TG, cl = threadIdx.x / TG;
    const int tiles = (p.T + TW - 1) / TW;
    const int at_tile = neighbours_together();
    if (at_tile >= p.B * tiles) return;
    const int b = at_tile / tiles, tile = at_tile - b * tiles;
    const int t_own = tile * TW + tg * V;  // the group's place; it is read at t0
    const int t0 = min(t_own, p.T - V);
    const bool store = t_own < p.T;
    const int len = length_of(p.len, b, p.T);
    const float per_c = 1.f / (float)p.C;
    const size_t item = (size_t)b * p.C * p.T;
    const S *x = (const S *)p.x + item, *f = p.f ? (const S *)p.f + item : nullptr;
    S *y = (S *)p.y + item, *n = (S *)p.n + item;
    auto at = [&](int i) { return (uint32_t)(min(cl + i * CL, p.C - 1) * p.T + t0) * (uint32_t)sizeof(S); };
    // (uniform) some position that the tile stores is no padding: a last tile of less than a group stores positions of the one before
    const bool any = min(tile * TW, p.T - V) < len;

    u32x4_t xr[NR], fr[NR];
    if (any) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            if (i * CL >= p.C) break;
            if (f) fr[i] = load_group<S>(f, at(i));
            xr[i] = load_group<S>(x, at(i));
        }
    }
    float mean[V], rstd[V];
    // mean (zero without LAYER) and 1/deviation of the rows r
    auto statistics = [&](const u32x4_t (&r)[NR]) {
        float s[1][V];
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) mean[j] = 0.f;
        if constexpr (LAYER) {
#pragma unroll
            for (int j = 0; j < V; ++j) s[0][j] = 0.f;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if (cl + i * CL >= p.C) break;
                Group<S>::unpack(r[i], v);
#pragma unroll
                for (int j = 0; j < V; ++j) s[0][j] += v[j];
            }
            sum_columns(lds, s);
#pragma unroll
            for (int j = 0; j < V; ++j) mean[j] = s[0][j] * per_c;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) s[0][j] = 0.f;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            if (cl + i * CL >= p.C) break;
            Group<S>::unpack(r[i], v);
#pragma unroll
            for (int j = 0; j < V; ++j) s[0][j] += (v[j] - mean[j]) * (v[j] - mean[j]);
        }
        sum_columns(lds, s);
#pragma unroll
        for (int j = 0; j < V; ++j) rstd[j] = 1.f / sqrtf(s[0][j] * per_c + p.eps);
    };
    if (f) {
        if (any && p.post) statistics(fr);
        const float *gate_item = p.gate_kind == NM_GATE_ITEM ? (const float *)p.gate + (size_t)b * p.C : nullptr;
        const S *gate = p.gate_kind == NM_GATE_ELEMENT ? (const S *)p.gate + item : nullptr;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int c = cl + i * CL;
            if (c >= p.C) break;
            u32x4_t out = {0u, 0u, 0u, 0u};
            if (any) {
                float xv[V], hv[V], gv[V];
                Group<S>::unpack(xr[i], xv);
                Group<S>::unpack(fr[i], hv);
                if (p.post) {
                    const float w = p.post_w ? p.post_w[c] : 1.f, bias = p.post_b ? p.post_b[c] : 0.f;
#pragma unroll
                    for (int j = 0; j < V; ++j) hv[j] = (hv[j] - mean[j]) * rstd[j] * w + bias;
                }
                const float rs = (p.rscale ? p.rscale[c] : 1.f) * (gate_item ? gate_item[c] : 1.f);
                if (gate) {
                    Group<S>::unpack(load_group<S>(gate, at(i)), gv);
#pragma unroll
                    for (int j = 0; j < V; ++j) hv[j] *= gv[j];
                }
#pragma unroll
                for (int j = 0; j < V; ++j) xv[j] += rs * hv[j];
                out = Group<S>::pack(xv);
            }
            xr[i] = out;
            if (store) store_group<S>(y, at(i), first_positions<S>(out, len - t0));
        }
    }
    if (p.next) {
        if (any) statistics(xr);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int c = cl + i * CL;
            if (c >= p.C) break;
            u32x4_t out = {0u, 0u, 0u, 0u};
            if (any) {
                const float w = p.next_w ? p.next_w[c] : 1.f, bias = p.next_b ? p.next_b[c] : 0.f;
                float v[V];
                Group<S>::unpack(xr[i], v);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = (v[j] - mean[j]) * rstd[j] * w + bias;
                out = first_positions<S>(Group<S>::pack(v), len - t0);
            }
            if (store) store_group<S>(n, at(i), out);
        }
    }
}

// Any number of channels, rows of any length: `positions` (a power of two up to 64) threads side by side along a row, the others
// share the channels, and the tensors are read again for every sum.  A wavefront's threads of one position add by exchanges, the
// wavefronts through LDS.  Made for few positions (a decoding step), not for wide rows of many: 16 x 2048 x 800 in bfloat16 takes 598 us
// forward and 1590 backward, 1024 channels in registers 26 and 76.
constexpr int kPlainThreads = 512, kPlainWaves = kPlainThreads / 64;
struct PlainSums {
    float of[kPlainWaves][64];
};
__device__ __forceinline__ float plain_total(PlainSums &lds, int positions, float v)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = positions; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    lds.of[wave][lane] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kPlainWaves; ++w) v += lds.of[w][lane];
    return v;
}

template <typename S>
__global__ __launch_bounds__(kPlainThreads) void residual_norm_fwd_plain_kernel(NormFwd p, int positions)
{
    __shared__ PlainSums lds;
    const int part = threadIdx.x / positions, parts = kPlainThreads / positions;
    const int tiles = (p.T + positions - 1) / positions;
    const int b = blockIdx.x / tiles, t = (blockIdx.x - b * tiles) * positions + threadIdx.x % positions, tc = min(t, p.T - 1);
    const bool valid = t < length_of(p.len, b, p.T);
    const S *x = (const S *)p.x, *f = (const S *)p.f;
    S *y = (S *)p.y, *n = (S *)p.n;
    auto at = [&](int c) { return ((size_t)b * p.C + c) * p.T + tc; };
    auto total = [&](float v) { return plain_total(lds, positions, v); };
    auto statistics = [&](auto value, float &mean, float &rstd) {
        mean = 0.f;
        float s = 0.f;
        if (p.layer) {
            for (int c = part; c < p.C; c += parts) s += value(c);
            mean = total(s) / (float)p.C;
        }
        s = 0.f;
        for (int c = part; c < p.C; c += parts) s += (value(c) - mean) * (value(c) - mean);
        rstd = 1.f / sqrtf(total(s) / (float)p.C + p.eps);
    };
    float fm = 0.f, fr = 1.f, ym, yr;
    if (f && p.post) statistics([&](int c) { return load_as_f32(f, at(c)); }, fm, fr);
    auto out = [&](int c) {  // y
        float v = load_as_f32(x, at(c));
        if (!f) return v;
        float h = load_as_f32(f, at(c));
        if (p.post) h = (h - fm) * fr * (p.post_w ? p.post_w[c] : 1.f) + (p.post_b ? p.post_b[c] : 0.f);
        float r = p.rscale ? p.rscale[c] : 1.f;
        if (p.gate_kind == NM_GATE_ITEM) r *= ((const float *)p.gate)[(size_t)b * p.C + c];
        if (p.gate_kind == NM_GATE_ELEMENT) h *= load_as_f32((const S *)p.gate, at(c));
        return round_to_storage(v + r * h, y);
    };
    if (p.next) statistics(out, ym, yr);
    for (int c = part; c < p.C; c += parts) {
        const float v = out(c);
        if (t < p.T) {
            if (f) store_from_f32(y, at(c), valid ? v : 0.f);
            if (p.next) store_from_f32(n, at(c), valid ? (v - ym) * yr * (p.next_w ? p.next_w[c] : 1.f) + (p.next_b ? p.next_b[c] : 0.f) : 0.f);
        }
    }
}

// ---- backward ----------------------------------------------------------------------------------------------------
// A workgroup owns every splits-th tile of an item and adds its sums over time in registers: the TG lanes of a row add
// theirs and each keeps every TG-th sum, so that the six sums of a row take 6/TG registers.
template <int TG>
__device__ __forceinline__ float row_sum(float v)
{
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xf, 0xf, true));              // lanes 1 0 3 2
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xf, 0xf, true));                                // 2 3 0 1
    if constexpr (TG > 4) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xf, 0xf, true)); // 7 6 5 4 3 2 1 0
    return v;
}

template <typename S, int TG, int NR, bool LAYER>
struct NormBwdLds {
    ColumnSums<TG, Group<S>::V, LAYER ? 4 : 3> sums;
    float vectors[5][NR * kThreads / TG];
    u32x4_t f[NR * kThreads];  // behind it as much for an element gate
};

// Few channels have many positions in a tile (TG), so that a thread has groups enough for the work around them.
// The per-channel vectors lie in LDS, ones and zeros for those that are not given, so that nothing branches between the rows.
// The groups of f and of an element gate wait in LDS, each thread's its own, until g is made: five tensors' groups and all that is
// made of them do not fit the registers.  NR = ceil(C / CL), the channels side by side (128 with four lanes along a row, 64 with eight): only
// the last row of a thread can lie beyond the channels.
template <typename S, int TG, int NR, bool LAYER>
__global__ __launch_bounds__(kThreads, NR >= 4 ? 2 : 4) void residual_norm_bwd_kernel(NormBwd p)
{
    constexpr int V = Group<S>::V, CL = kThreads / TG, TW = TG * V, NQ = LAYER ? 4 : 3;
    typedef NormBwdLds<S, TG, NR, LAYER> Lds;
    extern __shared__ __align__(16) unsigned char smem[];
    Lds &shared = *reinterpret_cast<Lds *>(smem);
    auto &lds = shared.sums;
    float *next_w = shared.vectors[0], *post_w = shared.vectors[1], *post_b = shared.vectors[2], *rscale = shared.vectors[3], *gate_of = shared.vectors[4];
    u32x4_t *fl = shared.f + threadIdx.x, *gl = reinterpret_cast<u32x4_t *>(smem + sizeof(Lds)) + threadIdx.x;  // row i: kThreads * i further
    const int tg = threadIdx.x % TG;
    const int tiles = (p.T + TW - 1) / TW;
    const int id = neighbours_together();
    if (id >= p.B * p.splits) return;
    const int b = id / p.splits, split = id - b * p.splits;
    const int len = length_of(p.len, b, p.T);
    const float per_c = 1.f / (float)p.C;
    const size_t item = (size_t)b * p.C * p.T;
    const S *dy = p.dy ? (const S *)p.dy + item : nullptr, *dn = (const S *)p.dn + item, *y = (const S *)p.y + item;
    const S *f = p.f ? (const S *)p.f + item : nullptr;
    const S *gate = p.gate_kind == NM_GATE_ELEMENT ? (const S *)p.gate + item : nullptr;
    S *dx = (S *)p.dx + item, *df = (S *)p.df + item, *dgate = gate && p.dgate ? (S *)p.dgate + item : nullptr;
    const u32x4_t zero = {0u, 0u, 0u, 0u};
    for (int c = threadIdx.x; c < p.C; c += kThreads) {
        next_w[c] = p.next_w ? p.next_w[c] : 1.f;
        post_w[c] = p.post_w ? p.post_w[c] : 1.f;
        post_b[c] = p.post_b ? p.post_b[c] : 0.f;
        rscale[c] = p.rscale ? p.rscale[c] : 1.f;
        gate_of[c] = p.gate_kind == NM_GATE_ITEM ? ((const float *)p.gate)[(size_t)b * p.C + c] : 1.f;
    }
    // (the barrier in front of their first use comes when the first tile has been asked for)
    bool filled = false;
    constexpr int kKept = (kSums + TG - 1) / TG;
    float sums[kKept][NR];  // of quantities tg, tg + TG ..
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int q = 0; q < kKept; ++q) sums[q][i] = 0.f;
    auto keep = [&](int quantity, int i, float v) {
        v = row_sum<TG>(v);
        if (tg == quantity % TG) sums[quantity / TG][i] += v;
        asm volatile("" : "+v"(sums[quantity / TG][i]));  // (added here, not at the end, which keeps all the summands)
    };

    for (int tile = split; tile < tiles; tile += p.splits) {
        int cl = threadIdx.x / TG;
        asm volatile("" : "+v"(cl));  // (what depends on it is computed where it is used: kept across tiles, it spills)
        const int t_own = tile * TW + tg * V;
        const int t0 = min(t_own, p.T - V);
        const bool store = t_own < p.T;
        // positions of the group that count in sums over time: from `first` on (the ones before are there twice), below `last`
        const int first = t_own - t0, last = store ? len - t0 : 0;
        const bool last_row = cl + (NR - 1) * CL < p.C;
        auto in = [&](int i) { return i < NR - 1 || last_row; };
        auto channel = [&](int i) { return i < NR - 1 ? cl + i * CL : min(cl + i * CL, p.C - 1); };
        auto at = [&](int i) { return (uint32_t)(channel(i) * p.T + t0) * (uint32_t)sizeof(S); };
        auto put = [&](S *to, int i, u32x4_t v) {
            if (store && in(i)) store_group<S>(to, at(i), first_positions<S>(v, len - t0));
        };
        if (min(tile * TW, p.T - V) >= len) {  // (uniform) all that the tile stores is padding
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                put(dx, i, zero);
                if (f) put(df, i, zero);
                if (dgate) put(dgate, i, zero);
            }
            continue;
        }
        u32x4_t dyr[NR], dnr[NR], yr[NR], fr[NR];
        auto load = [&](const S *from, bool there, u32x4_t (&r)[NR]) {
#pragma unroll
            for (int i = 0; i < NR; ++i) r[i] = there ? load_group<S>(from, at(i)) : zero;
            if (tile * TW + TW > len) {  // (uniform) positions in the padding: zeros, so that whatever lies there stays out of the sums
#pragma unroll
                for (int i = 0; i < NR; ++i) r[i] = first_positions<S>(r[i], len - t0);
            }
        };
        u32x4_t gr[NR];
        load(gate, gate != nullptr, gr);
        load(f, f != nullptr, fr);
        load(y, p.next, yr);
        load(dn, p.next, dnr);
        load(dy, dy != nullptr, dyr);
        if (!filled) __syncthreads();
        filled = true;
        if (gate) {
#pragma unroll
            for (int i = 0; i < NR; ++i) gl[i * kThreads] = gr[i];
        }
        if (f) {
#pragma unroll
            for (int i = 0; i < NR; ++i) fl[i * kThreads] = fr[i];
        }
        // sums over channels: of y and f, then of their squares, and those that the gradient of the norm of y takes
        float ym[V], yrs[V], fm[V], frs[V], ya[V], yb[V], s[NQ][V];
        auto clear = [&]() {
#pragma unroll
            for (int q = 0; q < NQ; ++q)
#pragma unroll
                for (int j = 0; j < V; ++j) s[q][j] = 0.f;
        };
#pragma unroll
        for (int j = 0; j < V; ++j) ym[j] = fm[j] = yb[j] = 0.f;
        if constexpr (LAYER) {
            clear();
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                asm volatile("" : "+v"(cl));
                unpack_again(yr[i]);
                unpack_again(dnr[i]);
                unpack_again(fr[i]);
                float v[V], d[V], u[V];
                const float there = in(i) ? 1.f : 0.f, w = next_w[channel(i)] * there;
                Group<S>::unpack(yr[i], v);
                Group<S>::unpack(dnr[i], d);
                Group<S>::unpack(fr[i], u);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    s[0][j] += i < NR - 1 ? v[j] : v[j] * there;
                    s[1][j] += d[j] * w;
                    s[2][j] += i < NR - 1 ? u[j] : u[j] * there;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            sum_columns(lds, s);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ym[j] = s[0][j] * per_c;
                yb[j] = s[1][j] * per_c;
                fm[j] = p.post ? s[2][j] * per_c : 0.f;
            }
        }
        clear();
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            asm volatile("" : "+v"(cl));
            unpack_again(yr[i]);
            unpack_again(dnr[i]);
            unpack_again(fr[i]);
            float v[V], d[V], u[V];
            const float there = in(i) ? 1.f : 0.f, w = next_w[channel(i)];
            Group<S>::unpack(yr[i], v);
            Group<S>::unpack(dnr[i], d);
            Group<S>::unpack(fr[i], u);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float z = v[j] - ym[j], fz = u[j] - fm[j];
                if (i == NR - 1) {
                    z *= there;
                    fz *= there;
                }
                s[0][j] += z * z;
                s[1][j] += d[j] * w * z;
                s[2][j] += fz * fz;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        sum_columns(lds, s);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            yrs[j] = p.next ? 1.f / sqrtf(s[0][j] * per_c + p.eps) : 0.f;  // (infinite without an eps, as y is zero there)
            ya[j] = s[1][j] * yrs[j] * per_c;
            frs[j] = p.post ? 1.f / sqrtf(s[2][j] * per_c + p.eps) : 1.f;
        }
        // g, in the place of dy and dn; dx and the sums over time of the norm of y.  (Without that norm y, dn and yrs are zero, and
        // all of this adds nothing to dy.)
        float g[NR][V];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            asm volatile("" : "+v"(cl));
            unpack_again(yr[i]);
            unpack_again(dnr[i]);
            unpack_again(dyr[i]);
            float hat[V], d[V];
            Group<S>::unpack(dyr[i], g[i]);
            Group<S>::unpack(yr[i], hat);
            Group<S>::unpack(dnr[i], d);
            const float w = next_w[channel(i)];
            float sw = 0.f, sb = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                hat[j] = (hat[j] - ym[j]) * yrs[j];
                g[i][j] += yrs[j] * (d[j] * w - hat[j] * ya[j] - yb[j]);
                const bool counts = j >= first && j < last;  // (hat is NaN in the padding where eps is 0)
                sw += counts ? d[j] * hat[j] : 0.f;
                sb += counts ? d[j] : 0.f;
            }
            keep(kDnw, i, sw);
            keep(kDnb, i, sb);
            put(dx, i, Group<S>::pack(g[i]));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!f) continue;
        auto gate_values = [&](int i, float (&gv)[V]) {
            if (gate) {
                Group<S>::unpack(gl[i * kThreads], gv);
            } else {
                const float of_item = gate_of[channel(i)];
#pragma unroll
                for (int j = 0; j < V; ++j) gv[j] = of_item;
            }
        };
        clear();
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int c = channel(i);
            const float rs = rscale[c], pw = post_w[c], pb = post_b[c], there = in(i) ? 1.f : 0.f;
            float gv[V], v[V];
            gate_values(i, gv);
            Group<S>::unpack(fl[i * kThreads], v);
            float srs = 0.f, spw = 0.f, spb = 0.f, sg = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float fhat = (v[j] - fm[j]) * frs[j];
                const float h = fhat * pw + pb, dh = rs * gv[j] * g[i][j], gh = g[i][j] * h;
                const float dw = i < NR - 1 ? dh * pw : dh * pw * there;
                s[0][j] += dw * fhat;
                s[1][j] += dw;
                const bool counts = j >= first && j < last;
                srs += counts ? gh * gv[j] : 0.f;
                spw += counts ? dh * fhat : 0.f;
                spb += counts ? dh : 0.f;
                sg += counts ? gh * rs : 0.f;
                v[j] = gh * rs;
            }
            keep(kDrs, i, srs);
            keep(kDpw, i, spw);
            keep(kDpb, i, spb);
            keep(kDgate, i, sg);
            if (dgate) put(dgate, i, Group<S>::pack(v));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (p.post) sum_columns(lds, s);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int c = channel(i);
            const float rs = rscale[c], pw = post_w[c];
            float gv[V], v[V];
            gate_values(i, gv);
            Group<S>::unpack(fl[i * kThreads], v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float dh = rs * gv[j] * g[i][j], fhat = (v[j] - fm[j]) * frs[j];
                v[j] = p.post ? frs[j] * (dh * pw - fhat * (s[0][j] * per_c) - (LAYER ? s[1][j] * per_c : 0.f)) : dh;
            }
            put(df, i, Group<S>::pack(v));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    const size_t rows = (size_t)p.B * p.splits;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int c = threadIdx.x / TG + i * CL;
        if (c >= p.C) break;
#pragma unroll
        for (int q = 0; q < kKept; ++q)
            if (q * TG + tg < kSums && (p.sums >> (q * TG + tg) & 1)) p.part[((q * TG + tg) * rows + id) * p.C + c] = sums[q][i];
    }
}

// Any number of channels, rows of any length, as in the forward pass; a channel's sums over time are added tile by tile in memory.
template <typename S>
__global__ __launch_bounds__(kPlainThreads) void residual_norm_bwd_plain_kernel(NormBwd p, int positions)
{
    __shared__ PlainSums lds;
    const int part = threadIdx.x / positions, parts = kPlainThreads / positions, place = threadIdx.x % positions;
    const int b = blockIdx.x / p.splits, split = blockIdx.x - b * p.splits;
    const int len = length_of(p.len, b, p.T);
    const S *dy = (const S *)p.dy, *dn = (const S *)p.dn, *y = (const S *)p.y, *f = (const S *)p.f;
    const S *gate = p.gate_kind == NM_GATE_ELEMENT ? (const S *)p.gate : nullptr;
    S *dx = (S *)p.dx, *df = (S *)p.df, *dgate = gate ? (S *)p.dgate : nullptr;
    const float per_c = 1.f / (float)p.C;
    const size_t rows = (size_t)p.B * p.splits;
    auto total = [&](float v) { return plain_total(lds, positions, v); };
    bool begun = false;
    for (int t_tile = split * positions; t_tile < p.T; t_tile += p.splits * positions) {  // (once at least: there are no more splits than tiles)
        const int t = t_tile + place, tc = min(t, p.T - 1);
        const bool valid = t < len, store = t < p.T;
        auto at = [&](int c) { return ((size_t)b * p.C + c) * p.T + tc; };
        auto read = [&](const S *q, int c) { return q && valid ? load_as_f32(q, at(c)) : 0.f; };
        auto weight = [&](const float *w, int c) { return w ? w[c] : 1.f; };
        auto statistics = [&](const S *q, float &mean, float &rstd) {
            mean = 0.f;
            float s = 0.f;
            if (p.layer) {
                for (int c = part; c < p.C; c += parts) s += read(q, c);
                mean = total(s) * per_c;
            }
            s = 0.f;
            for (int c = part; c < p.C; c += parts) s += (read(q, c) - mean) * (read(q, c) - mean);
            rstd = 1.f / sqrtf(total(s) * per_c + p.eps);
        };
        float ym = 0.f, yr = 1.f, fm = 0.f, fr = 1.f, ya = 0.f, yb = 0.f, fa = 0.f, fb = 0.f;
        if (p.next) {
            statistics(y, ym, yr);
            float s = 0.f, sb = 0.f;
            for (int c = part; c < p.C; c += parts) {
                const float d = read(dn, c) * weight(p.next_w, c);
                s += d * ((read(y, c) - ym) * yr);
                sb += d;
            }
            ya = total(s) * per_c;
            yb = p.layer ? total(sb) * per_c : 0.f;
        }
        auto gradient = [&](int c) {
            float g = read(dy, c);
            if (p.next) g += yr * (read(dn, c) * weight(p.next_w, c) - (read(y, c) - ym) * yr * ya - yb);
            return g;
        };
        auto gate_of = [&](int c) {
            return p.gate_kind == NM_GATE_ITEM ? ((const float *)p.gate)[(size_t)b * p.C + c] : gate ? read(gate, c) : 1.f;
        };
        if (f && p.post) {
            statistics(f, fm, fr);
            float s = 0.f, sb = 0.f;
            for (int c = part; c < p.C; c += parts) {
                const float d = weight(p.rscale, c) * gate_of(c) * gradient(c) * weight(p.post_w, c);
                s += d * ((read(f, c) - fm) * fr);
                sb += d;
            }
            fa = total(s) * per_c;
            fb = p.layer ? total(sb) * per_c : 0.f;
        }
        for (int c = part; c < p.C; c += parts) {
            float v[kSums] = {};
            const float g = gradient(c);
            if (store) store_from_f32(dx, at(c), valid ? g : 0.f);
            if (p.next) {
                v[kDnw] = read(dn, c) * ((read(y, c) - ym) * yr);
                v[kDnb] = read(dn, c);
            }
            if (f) {
                const float rs = weight(p.rscale, c), gt = gate_of(c), fhat = (read(f, c) - fm) * fr;
                const float pw = p.post ? weight(p.post_w, c) : 1.f;
                const float h = fhat * pw + (p.post && p.post_b ? p.post_b[c] : 0.f), dh = rs * gt * g;
                v[kDrs] = g * gt * h;
                v[kDpw] = dh * fhat;
                v[kDpb] = dh;
                v[kDgate] = g * h * rs;
                if (store) store_from_f32(df, at(c), valid ? (p.post ? fr * (dh * pw - fhat * fa - fb) : dh) : 0.f);
                if (dgate && store) store_from_f32(dgate, at(c), valid ? v[kDgate] : 0.f);
            }
#pragma unroll
            for (int q = 0; q < kSums; ++q) {
                if (!(p.sums >> q & 1)) continue;
                float s = valid ? v[q] : 0.f;
                for (int d = 1; d < positions; d <<= 1) s += __shfl_xor(s, d);
                if (place == 0) {
                    float *o = p.part + ((size_t)q * rows + blockIdx.x) * p.C + c;
                    *o = begun ? *o + s : s;
                }
            }
        }
        begun = true;
    }
}

// out[c] = sum over `rows` rows of part[rows][C], a fixed order: 32 channels by 32 shares of the rows per workgroup.
// blockIdx.y: one of up to five sums over all items, behind them an item's gate sums over its `splits` rows
struct ReduceArgs {
    const float *part;
    float *out[5];
    int quantity[5], count;
    float *dgate;
    int B, C, splits;
};
__global__ __launch_bounds__(1024) void residual_norm_sums_kernel(ReduceArgs a)
{
    __shared__ float s[32][33];
    const int cl = threadIdx.x & 31, share = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + cl, cc = min(c, a.C - 1);
    const int rows = a.B * a.splits;
    const bool item = (int)blockIdx.y >= a.count;
    const int b = (int)blockIdx.y - a.count;
    const int q = item ? (int)kDgate : a.quantity[blockIdx.y], first = item ? b * a.splits : 0, n = item ? a.splits : rows;
    const float *p = a.part + ((size_t)q * rows + first) * a.C + cc;
    float t = 0.f;
#pragma unroll 4
    for (int r = share; r < n; r += 32) t += p[(size_t)r * a.C];
    s[share][cl] = t;
    __syncthreads();
    // 32 sums of a channel: a wavefront's half adds those of one channel by exchanges
    float v = s[cl][share];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) v += __shfl_xor(v, d);
    const int co = blockIdx.x * 32 + share;
    if (cl == 0 && co < a.C) (item ? a.dgate + (size_t)b * a.C : a.out[blockIdx.y])[co] = v;
}

constexpr int kFwdTG = 4;
constexpr int kFwdLanes = kThreads / kFwdTG;  // channels side by side
constexpr int bwd_tg(int C) { return C <= kThreads / 2 ? 8 : 4; }  // 16 x 768 x 777: 63 us with four lanes along a row, 72 with two and two workgroups a CU

// Whether the kernels that hold an item's tile in registers serve a call: up to 1024 channels (four or eight groups of a tensor a
// thread), rows of a group at least, items whose byte offsets fit 32 bits.
constexpr int kMaxInRegisters = 8 * kThreads / 4;
static_assert(kMaxInRegisters == 8 * kFwdLanes, "one limit for both passes");
bool in_registers(int C, int T, size_t element) { return C <= kMaxInRegisters && T >= (int)(16 / element) && (size_t)C * T * element < (size_t)1 << 32; }

// Positions side by side in a workgroup of the plain kernels: a power of two, no more than 64
int plain_positions(int T)
{
    int n = 1;
    while (n < T && n < 64) n *= 2;
    return n;
}

// Workgroups of an item in the backward pass, each of which takes every so many-th tile: as many as fill the chip twice over,
// so that sums over time are added over several tiles before they are written.
int bwd_splits(int B, int C, int T, int dtype)
{
    const size_t element = dtype == NM_BF16 ? 2 : 4;
    const int width = in_registers(C, T, element) ? bwd_tg(C) * (int)(16 / element) : plain_positions(T);
    const int tiles = (T + width - 1) / width, want = (1024 + B - 1) / B;
    return tiles < want ? tiles : want;
}

// Workgroups of the forward pass
size_t fwd_groups(int B, int C, int T, size_t element)
{
    const int width = in_registers(C, T, element) ? kFwdTG * (int)(16 / element) : plain_positions(T);
    return (size_t)B * ((T + width - 1) / width);
}

template <typename S, int NR>
hipError_t fwd_rows(const NormFwd &p, hipStream_t s)
{
    const dim3 grid = eights(fwd_groups(p.B, p.C, p.T, sizeof(S)));
    if (p.layer)
        residual_norm_fwd_kernel<S, kFwdTG, NR, true><<<grid, dim3(kThreads), 0, s>>>(p);
    else
        residual_norm_fwd_kernel<S, kFwdTG, NR, false><<<grid, dim3(kThreads), 0, s>>>(p);
    return hipGetLastError();
}
template <typename S>
hipError_t fwd_any(const NormFwd &p, hipStream_t s)
{
    if (!in_registers(p.C, p.T, sizeof(S))) {
        residual_norm_fwd_plain_kernel<S><<<dim3((unsigned)fwd_groups(p.B, p.C, p.T, sizeof(S))), dim3(kPlainThreads), 0, s>>>(p, plain_positions(p.T));
        return hipGetLastError();
    }
    return p.C <= 4 * kFwdLanes ? fwd_rows<S, 4>(p, s) : fwd_rows<S, 8>(p, s);
}

template <typename S, int TG, int NR, bool LAYER>
hipError_t bwd_rows_of(const NormBwd &p, hipStream_t s)
{
    static LdsOptIn opt;
    constexpr int base = (int)sizeof(NormBwdLds<S, TG, NR, LAYER>), most = base + NR * kThreads * 16;
    static_assert(most <= 160 * 1024, "LDS of a CU");
    const hipError_t e = ensure_dynamic_lds(opt, (const void *)residual_norm_bwd_kernel<S, TG, NR, LAYER>, most);
    if (e != hipSuccess) return e;
    residual_norm_bwd_kernel<S, TG, NR, LAYER><<<eights((size_t)p.B * p.splits), dim3(kThreads), p.gate_kind == NM_GATE_ELEMENT ? most : base, s>>>(p);
    return hipGetLastError();
}
template <typename S, int TG>
hipError_t bwd_rows(const NormBwd &p, hipStream_t s)
{
    switch ((p.C * TG + kThreads - 1) / kThreads) {
    case 1: return p.layer ? bwd_rows_of<S, TG, 1, true>(p, s) : bwd_rows_of<S, TG, 1, false>(p, s);
    case 2: return p.layer ? bwd_rows_of<S, TG, 2, true>(p, s) : bwd_rows_of<S, TG, 2, false>(p, s);
    case 3: return p.layer ? bwd_rows_of<S, TG, 3, true>(p, s) : bwd_rows_of<S, TG, 3, false>(p, s);
    case 4: return p.layer ? bwd_rows_of<S, TG, 4, true>(p, s) : bwd_rows_of<S, TG, 4, false>(p, s);
    }
    if constexpr (TG == 4) {
        switch ((p.C * TG + kThreads - 1) / kThreads) {
        case 5: return p.layer ? bwd_rows_of<S, TG, 5, true>(p, s) : bwd_rows_of<S, TG, 5, false>(p, s);
        case 6: return p.layer ? bwd_rows_of<S, TG, 6, true>(p, s) : bwd_rows_of<S, TG, 6, false>(p, s);
        case 7: return p.layer ? bwd_rows_of<S, TG, 7, true>(p, s) : bwd_rows_of<S, TG, 7, false>(p, s);
        case 8: return p.layer ? bwd_rows_of<S, TG, 8, true>(p, s) : bwd_rows_of<S, TG, 8, false>(p, s);
        }
    }
    return hipErrorInvalidValue;  // (in_registers() lets no more through)
}
template <typename S>
hipError_t bwd_any(const NormBwd &p, hipStream_t s)
{
    if (!in_registers(p.C, p.T, sizeof(S))) {
        residual_norm_bwd_plain_kernel<S><<<dim3((unsigned)p.B * p.splits), dim3(kPlainThreads), 0, s>>>(p, plain_positions(p.T));
        return hipGetLastError();
    }
    return bwd_tg(p.C) == 8 ? bwd_rows<S, 8>(p, s) : bwd_rows<S, 4>(p, s);
}

int check_shape(int B, int C, int T, int dtype)
{
    if (B <= 0 || C <= 0 || T <= 0 || (dtype != NM_BF16 && dtype != NM_F32)) return NM_ERR_BAD_ARG;
    if ((long long)B * C * T > (1LL << 31) - 1 || C > kMaxChannels || B > 65000) return NM_ERR_UNSUPPORTED;
    return NM_OK;
}
bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    if (!a || !b) return false;
    const char *pa = (const char *)a, *pb = (const char *)b;
    return pa < pb + nb && pb < pa + na;
}
int dev(hipError_t e) { return e == hipSuccess ? NM_OK : NM_ERR_DEVICE; }

}  // namespace
}  // namespace nm

using namespace nm;

extern "C" {

int nm_residual_norm_fwd(int B, int C, int T, const void *x, const void *f, const void *gate, int gate_kind,
                         const float *rscale, const float *post_weight, const float *post_bias, const float *next_weight,
                         const float *next_bias, float eps, const int *lengths, void *y, void *n, unsigned flags, int dtype,
                         void *hip_stream)
{
    const int st = check_shape(B, C, T, dtype);
    if (st != NM_OK) return st;
    const bool post = flags & NM_NORM_POST, next = flags & NM_NORM_NEXT, layer = flags & NM_NORM_LAYER;
    if (flags & ~7u || !x || !(eps >= 0.f) || isinf(eps) || gate_kind < NM_GATE_NONE || gate_kind > NM_GATE_ELEMENT) return NM_ERR_BAD_ARG;
    if ((gate_kind != NM_GATE_NONE) != (gate != nullptr) || (f != nullptr) != (y != nullptr) || next != (n != nullptr)) return NM_ERR_BAD_ARG;
    if (!f && (!next || post || gate || rscale)) return NM_ERR_BAD_ARG;
    if ((!post && (post_weight || post_bias)) || (!next && (next_weight || next_bias)) || (!layer && (post_bias || next_bias))) return NM_ERR_BAD_ARG;
    static_assert(kThreads == 512 && kPlainThreads == 512, "the limit below");
    if (fwd_groups(B, C, T, dtype == NM_BF16 ? 2 : 4) > (1u << 23) - 8) return NM_ERR_UNSUPPORTED;  // a launch has less than 2^32 work items
    const size_t bytes = (size_t)B * C * T * (dtype == NM_BF16 ? 2 : 4), gate_bytes = gate_kind == NM_GATE_ITEM ? (size_t)B * C * 4 : bytes;
    if (overlap(y, bytes, x, bytes) || overlap(y, bytes, f, bytes) || overlap(y, bytes, gate, gate_bytes) || overlap(n, bytes, x, bytes) ||
        overlap(n, bytes, f, bytes) || overlap(n, bytes, gate, gate_bytes) || overlap(n, bytes, y, bytes))
        return NM_ERR_BAD_ARG;
    NormFwd p = {B, C, T, x, f, gate, gate_kind, rscale, post_weight, post_bias, next_weight, next_bias, eps, lengths, y, n, post, next, layer};
    return dev(dtype == NM_BF16 ? fwd_any<bf16_t>(p, (hipStream_t)hip_stream) : fwd_any<float>(p, (hipStream_t)hip_stream));
}

size_t nm_residual_norm_bwd_workspace_bytes(int B, int C, int T, int dtype)
{
    if (check_shape(B, C, T, dtype) != NM_OK) return 0;
    return align_up((size_t)kSums * B * bwd_splits(B, C, T, dtype) * C * sizeof(float), 256);
}

int nm_residual_norm_bwd(int B, int C, int T, const void *dy, const void *dn, const void *y, const void *f, const void *gate,
                         int gate_kind, const float *rscale, const float *post_weight, const float *post_bias,
                         const float *next_weight, float eps, const int *lengths, void *dx, void *df, void *dgate,
                         float *drscale, float *dpost_weight, float *dpost_bias, float *dnext_weight, float *dnext_bias,
                         unsigned flags, int dtype, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check_shape(B, C, T, dtype);
    if (st != NM_OK) return st;
    const bool post = flags & NM_NORM_POST, next = flags & NM_NORM_NEXT, layer = flags & NM_NORM_LAYER;
    if (flags & ~7u || !dx || !(eps >= 0.f) || isinf(eps) || gate_kind < NM_GATE_NONE || gate_kind > NM_GATE_ELEMENT) return NM_ERR_BAD_ARG;
    if ((gate_kind != NM_GATE_NONE) != (gate != nullptr) || (f != nullptr) != (df != nullptr) || next != (dn != nullptr) || (next && !y)) return NM_ERR_BAD_ARG;
    if (!f && (!next || post || gate || rscale || drscale)) return NM_ERR_BAD_ARG;
    if (!next && !dy) return NM_ERR_BAD_ARG;
    if ((!post && (post_weight || post_bias || dpost_weight || dpost_bias)) || (!next && (next_weight || dnext_weight || dnext_bias)) ||
        (!layer && (post_bias || dpost_bias || dnext_bias)) || (dgate && !gate))
        return NM_ERR_BAD_ARG;
    const size_t bytes = (size_t)B * C * T * (dtype == NM_BF16 ? 2 : 4), gate_bytes = gate_kind == NM_GATE_ITEM ? (size_t)B * C * 4 : bytes;
    const void *ins[5] = {dy, dn, y, f, gate};
    void *outs[3] = {dx, df, dgate};
    for (int o = 0; o < 3; ++o) {
        const size_t ob = o == 2 ? gate_bytes : bytes;
        for (int i = 0; i < 5; ++i)
            if (overlap(outs[o], ob, ins[i], i == 4 ? gate_bytes : bytes)) return NM_ERR_BAD_ARG;
        for (int q = 0; q < o; ++q)
            if (overlap(outs[o], ob, outs[q], bytes)) return NM_ERR_BAD_ARG;
    }
    const size_t need = nm_residual_norm_bwd_workspace_bytes(B, C, T, dtype);
    const bool item = gate_kind == NM_GATE_ITEM && dgate;
    float *vectors[5] = {dnext_weight, dnext_bias, drscale, dpost_weight, dpost_bias};
    const int quantity[5] = {kDnw, kDnb, kDrs, kDpw, kDpb};
    ReduceArgs r = {};
    unsigned sums = item ? 1u << kDgate : 0u;
    for (int i = 0; i < 5; ++i)
        if (vectors[i]) {
            r.out[r.count] = vectors[i];
            r.quantity[r.count++] = quantity[i];
            sums |= 1u << quantity[i];
        }
    if (sums && (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < need)) return NM_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)hip_stream;
    NormBwd p = {B, C, T, dy, dn, y, f, gate, gate_kind, rscale, post_weight, post_bias, next_weight, eps, lengths, dx, df, dgate,
                 (float *)workspace, bwd_splits(B, C, T, dtype), post, next, layer, sums};
    hipError_t e = dtype == NM_BF16 ? bwd_any<bf16_t>(p, s) : bwd_any<float>(p, s);
    if (e != hipSuccess || !sums) return dev(e);
    r.part = (const float *)workspace;
    r.dgate = (float *)dgate;
    r.B = B; r.C = C; r.splits = p.splits;
    residual_norm_sums_kernel<<<dim3((C + 31) / 32, r.count + (item ? B : 0)), dim3(1024), 0, s>>>(r);
    return dev(hipGetLastError());
}

}  // extern "C"
