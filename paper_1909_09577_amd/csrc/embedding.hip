// Lookup of tokens' embeddings and its gradient (definition: include/nm_embedding.h).
//
// Forward: a table's rows run over the channels, activations over the tokens, so a workgroup carries 64 tokens x 64 channels across LDS and
// reads and writes 128-byte pieces.  Calls of few tokens an item are copied element by element (32 items, 1024 channels, bfloat16: of 8 and 12 tokens
// each 3.9 us against 4.3 and 4.5 as tiles, of 24 4.9 against 4.6; 4 items of 256 channels: of 12 tokens 3.8 against 4.0; 32 items of 512 channels in float32: of 12
// tokens 4.2 against 3.9, of 24 4.5 against 3.8).  Single tokens of 32 items: 2.5 us, the launch.
//
// Gradient: a sum over the places of each token, which has to come out the same every time, so the places are sorted by token, without
// atomics on sums.  Three launches:
//   order  one workgroup for each range of tokens reads all token numbers, counts those of its range and of the ranges below,
//          packs the places of its range into a list in their order, and writes each to where its token's next one goes: a stable counting
//          sort.  Beside them other workgroups turn dout into rows of channels and fill dtable with zeros.
//   sums   a wavefront adds a run of eight sorted places, a lane eight channels of them; a token whose places lie in one run is finished there.
//          A frequent token's runs leave parts.
//   join   adds the parts of such a token in order.
// 16 x 1601 places, 32000 tokens of 512 channels, bfloat16: 25 + 15 + 9 us.  What has to move, 92 MB, would take 18; the turned copy of dout
// and rows that are filled and then written again are half as much once more, the order alone takes 18 us beside them.  Of the
// join's 9 us its 3200 workgroups take 7 that find no token to join (as where all tokens are equally likely); the 214 parts of the most frequent token do
// not hold it up (the same without that token).  A quarter as many workgroups, four runs each, took 8 us, and of 32 x 150 places 5.5 instead of 4.2.
#include "../../include/nm_embedding.h"
#include "token_ops.h"

namespace nm {
namespace {

// ---- forward -----------------------------------------------------------------------------------------------------
struct EmbedFwd {
    int B, V, C, U;
    Ids ids;
    const void *table;
    float scale;
    const int *len;
    void *out;
    int u_tiles, c_tiles;
};

// 64 tokens x 64 channels of an item
template <typename S>
__global__ __launch_bounds__(256) void embed_tile_kernel(EmbedFwd a)
{
    __shared__ S tile[64][64 + (sizeof(S) == 2 ? 2 : 1)];
    __shared__ int id[64];
    const int t = threadIdx.x, ct = blockIdx.x % a.c_tiles, rest = blockIdx.x / a.c_tiles;
    const int b = rest / a.u_tiles, u0 = (rest - b * a.u_tiles) * 64, c0 = ct * 64;
    const int len = length_in(a.len, b, a.U);
    if (t < 64) id[t] = u0 + t < len ? a.ids.at((size_t)b * a.U + u0 + t, a.V) : -1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // eight channels of a token
        const int u = (t >> 3) + 32 * i, c = (t & 7) * 8;
        float v[8];
        load8((const S *)a.table + (size_t)max(id[u], 0) * a.C + c0 + c, id[u] < 0 ? 0 : a.C - c0 - c, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) store_from_f32(&tile[u][c], j, v[j] * a.scale);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // eight tokens of a channel
        const int c = (t >> 3) + 32 * i, u = (t & 7) * 8;
        if (c0 + c >= a.C) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = load_as_f32(&tile[u + j][0], c);
        store8((S *)a.out + ((size_t)b * a.C + c0 + c) * a.U + u0 + u, a.U - u0 - u, v);
    }
}

// Eight neighbouring outputs of an item a thread
template <typename S>
__global__ __launch_bounds__(256) void embed_flat_kernel(EmbedFwd a)
{
    const int b = blockIdx.y, item = a.C * a.U;
    if ((blockIdx.x * 256LL + threadIdx.x) * 8 >= item) return;
    const int i0 = (blockIdx.x * 256 + threadIdx.x) * 8, rest = item - i0;
    const int len = length_in(a.len, b, a.U);
    float v[8];
    if (a.U == 1) {
        const int id = len ? a.ids.at(b, a.V) : -1;
        load8((const S *)a.table + (size_t)max(id, 0) * a.C + i0, id < 0 ? 0 : rest, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + min(j, rest - 1), c = i / a.U, u = i - c * a.U;
            const int id = u < len ? a.ids.at((size_t)b * a.U + u, a.V) : -1;
            v[j] = load_as_f32((const S *)a.table, (size_t)max(id, 0) * a.C + c);
            if (id < 0) v[j] = 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= a.scale;
    store8((S *)a.out + (size_t)b * item + i0, rest, v);
}

template <typename S>
hipError_t run_fwd(EmbedFwd a, hipStream_t s)
{
    if (a.U < 16) {
        embed_flat_kernel<S><<<dim3((unsigned)(((long long)a.C * a.U + 2047) / 2048), a.B), dim3(256), 0, s>>>(a);
    } else {
        a.u_tiles = (a.U + 63) / 64;
        a.c_tiles = (a.C + 63) / 64;
        embed_tile_kernel<S><<<dim3((unsigned)a.B * a.u_tiles * a.c_tiles), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError();
}

// ---- gradient ----------------------------------------------------------------------------------------------------
constexpr int kThreads = 512, kWaves = kThreads / 64;  // of the workgroups that sort, turn and fill
constexpr int kChunk = kWaves * 1024;                  // places that a sorting workgroup looks at at a time
constexpr int kList = 4096;                            // of its range that it can hold
constexpr int kRange = 256;                            // tokens of a sorting workgroup at most
constexpr int kRun = 8;                                // sorted places of a wavefront
constexpr int kFill = 32768;                           // floats that a workgroup fills

// A sorted place: where it is, its token, and where the token's places begin and end in the order.
struct __align__(16) Entry {
    int place, token, from, to;
};

struct EmbedBwd {
    int B, V, C, U, N;
    Ids ids;
    double per_item;  // 1 / U
    const int *len;
    const void *dout, *rows;  // rows [N][C]: dout turned, or dout itself
    void *turned;             // where to, or NULL
    float scale;
    float *dtable;
    bool add;
    Entry *order;             // [N]
    int *total;               // places that have a token
    float *parts;             // [runs][2][C]: sums of a run's first and last token
    int range, sorters, u_tiles, c_tiles, turners;
};

__device__ __forceinline__ int wave_scan(int v, int lane)  // sum of the lanes up to this one
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// The tokens of 16 places of each lane of a wavefront less v0 (negative: of a lower range), kNoToken where there is none: pairs side by side,
// place p0 + 128*i + 2*lane + s in r[2*i + s]
constexpr int kNoToken = 0x7fffffff;
__device__ __forceinline__ void tokens_at(const EmbedBwd &a, int p0, int lane, int v0, int (&r)[16])
{
    if (a.ids.wide) {
#pragma unroll
        for (int h = 0; h < 16; h += 8) {
            uint32_t lo[8], hi[8];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const int p = p0 + 64 * (h + i) + 2 * lane;
                u32x4_t w = {0u, ~0u, 0u, ~0u};
                const char *at = reinterpret_cast<const char *>(a.ids.p) + (size_t)p * 8;
                if (p + 1 < a.N) __builtin_memcpy(&w, at, 16);
                else if (p < a.N) __builtin_memcpy(&w, at, 8);
                lo[i] = w[0];
                hi[i] = w[1];
                lo[i + 1] = w[2];
                hi[i + 1] = w[3];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) r[h + i] = hi[i] == 0 && lo[i] < (uint32_t)a.V ? (int)lo[i] - v0 : kNoToken;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const int p = p0 + 64 * i + 2 * lane;
            const int *at = reinterpret_cast<const int *>(a.ids.p) + p;
            uint32_t w[2] = {~0u, ~0u};
            if (p + 1 < a.N) __builtin_memcpy(w, at, 8);
            else if (p < a.N) w[0] = (uint32_t)at[0];
#pragma unroll
            for (int s = 0; s < 2; ++s) r[i + s] = w[s] < (uint32_t)a.V ? (int)w[s] - v0 : kNoToken;
        }
    }
    if (a.len) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int p = min(p0 + 128 * (i >> 1) + 2 * lane + (i & 1), a.N - 1);
            int b = (int)((double)p * a.per_item);  // (within one of p / U)
            b -= b * a.U > p;
            b += (b + 1) * a.U <= p;
            if (p - b * a.U >= a.len[b]) r[i] = kNoToken;
        }
    }
}

// One range of tokens: which places have them, in order of the tokens and of the places.  A wavefront looks at 1024 neighbouring places
// at a time; those of the range are packed into a list in their order, of which each wavefront takes its own stretch: it counts the tokens
// there, and from what the wavefronts before it counted knows where its places go.  (Every eighth token to a wavefront, one after the other: the
// order of 25616 places took 25 us instead of 18, because a frequent token's wavefront went through the whole list.)  Where the list is too
// short for all, it is made again for the next ones.
__device__ void sort_range(const EmbedBwd &a, int which, unsigned char *smem)
{
    int *count = reinterpret_cast<int *>(smem);                    // [kRange]
    int *begin = count + kRange;                                   // [kRange]
    int *next = begin + kRange;                                    // [kRange]: where the list's first place goes
    int *ours = next + kRange;                                     // [kWaves][kRange]: a stretch's tokens; where its next place goes
    int *sums = ours + kWaves * kRange;                            // [3][kWaves]
    int *place = sums + 3 * kWaves;                                // [kList]
    uint16_t *bin = reinterpret_cast<uint16_t *>(place + kList);   // [kList]
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int v0 = which * a.range, bins = min(a.range, a.V - v0), chunks = (a.N - 1) / kChunk + 1;
    const uint64_t lower = (1ull << lane) - 1;
    for (int r = t; r < bins; r += kThreads) count[r] = 0;
    // the range's places that are number w0 .. w0+kList-1 among them go into the list; returns how many there are in all
    int less = 0;
    auto pack = [&](int w0) {
        int found = 0;
        less = 0;
        for (int k = 0; k < chunks; ++k) {
            const int p0 = k * kChunk + wave * 1024;
            int r[16], mine = 0;
            tokens_at(a, p0, lane, v0, r);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                less += __builtin_popcountll(__ballot(r[i] < 0));
                mine += __builtin_popcountll(__ballot((unsigned)r[i] < (unsigned)bins));
            }
            int *s = sums + (k & 1) * kWaves;  // (the other half may still be read)
            if (lane == 0) s[wave] = mine;
            __syncthreads();
            int at = found - w0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                at += w < wave ? s[w] : 0;
                found += s[w];
            }
            if (mine) {  // (uniform)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const bool in0 = (unsigned)r[i] < (unsigned)bins, in1 = (unsigned)r[i + 1] < (unsigned)bins;
                    const uint64_t b0 = __ballot(in0), b1 = __ballot(in1);
                    if (!(b0 | b1)) continue;
                    const int to = at + __builtin_popcountll(b0 & lower) + __builtin_popcountll(b1 & lower), p = p0 + 64 * i + 2 * lane;
                    if (in0 && (unsigned)to < (unsigned)kList) {
                        place[to] = p;
                        bin[to] = (uint16_t)r[i];
                    }
                    if (in1 && (unsigned)(to + in0) < (unsigned)kList) {
                        place[to + in0] = p + 1;
                        bin[to + in0] = (uint16_t)r[i + 1];
                    }
                    at += __builtin_popcountll(b0) + __builtin_popcountll(b1);
                }
            }
        }
        __syncthreads();
        return found;
    };
    // a wavefront's stretch of a list, a multiple of 64 places; how often every token occurs in each
    int *mine = ours + wave * kRange;
    auto stretch = [&](int listed) { return ((listed + kWaves - 1) / kWaves + 63) / 64 * 64; };
    auto tally = [&](int listed) {
        for (int r = t; r < kWaves * kRange; r += kThreads) ours[r] = 0;
        __syncthreads();
        const int side = stretch(listed), j1 = min(listed, (wave + 1) * side);
        for (int j = wave * side + lane; j < j1; j += 64) atomicAdd(&mine[bin[j]], 1);  // (whole numbers: any order gives the same)
        __syncthreads();
    };
    const int all = pack(0);
    for (int w0 = 0; w0 < all; w0 += kList) {
        if (w0) pack(w0);
        tally(min(all - w0, kList));
        for (int r = t; r < bins; r += kThreads)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) count[r] += ours[w * kRange + r];
    }
    if (lane == 0) sums[2 * kWaves + wave] = less;
    __syncthreads();
    if (wave == 0) {  // where every token's places begin
        int base = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) base += sums[2 * kWaves + w];
        for (int r0 = 0; r0 < bins; r0 += 64) {
            const int n = r0 + lane < bins ? count[r0 + lane] : 0, upto = wave_scan(n, lane);
            if (r0 + lane < bins) begin[r0 + lane] = next[r0 + lane] = base + upto - n;
            base += __shfl(upto, 63);
        }
        if (lane == 0 && v0 + bins == a.V) *a.total = base;
    }
    __syncthreads();
    for (int w0 = 0; w0 < all; w0 += kList) {
        const int listed = min(all - w0, kList);
        if (all > kList) {
            __syncthreads();
            pack(w0);
            tally(listed);
        }
        for (int r = t; r < bins; r += kThreads) {
            int at = next[r];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const int n = ours[w * kRange + r];
                ours[w * kRange + r] = at;
                at += n;
            }
            next[r] = at;
        }
        __syncthreads();
        const int side = stretch(listed), j1 = min(listed, (wave + 1) * side);
        for (int j = wave * side; j < j1; j += 64) {
            const bool is = j + lane < j1;
            const int r = is ? bin[j + lane] : 0;
            uint64_t same = __ballot(is);  // the lanes with the same token
            for (int bit = 1; bit < bins; bit <<= 1) {
                const uint64_t set = __ballot((r & bit) != 0);
                same &= r & bit ? set : ~set;
            }
            if (is) {
                const int from = begin[r], at = mine[r];
                a.order[at + __builtin_popcountll(same & lower)] = Entry{place[j + lane], v0 + r, from, from + count[r]};
                if (!(same & lower)) mine[r] = at + __builtin_popcountll(same);
            }
            __builtin_amdgcn_wave_barrier();  // (what a lane wrote, others read)
        }
    }
}

// 64 tokens x `kChannels` channels of dout as rows of channels
template <typename S>
struct Turn {
    static constexpr int kChannels = sizeof(S) == 2 ? 128 : 64, kPitch = sizeof(S) == 2 ? 66 : 65, kSteps = kChannels * 8 / kThreads;
    static constexpr int kBytes = kChannels * kPitch * sizeof(S);
};
__device__ __forceinline__ void load8_bits(const bf16_t *p, int n, bf16_t (&e)[8])
{
    const u32x4_t v = load8_any(p, n);
    __builtin_memcpy(e, &v, 16);
}
__device__ __forceinline__ void load8_bits(const float *p, int n, float (&e)[8]) { load8(p, n, e); }
__device__ __forceinline__ void store8_bits(bf16_t *p, int n, const bf16_t (&e)[8])
{
    u32x4_t v;
    __builtin_memcpy(&v, e, 16);
    store8_any(p, v, n);
}
__device__ __forceinline__ void store8_bits(float *p, int n, const float (&e)[8]) { store8(p, n, e); }

template <typename S>
__device__ void turn_tile(const EmbedBwd &a, int tile, unsigned char *smem)
{
    typedef Turn<S> T;
    S *lds = reinterpret_cast<S *>(smem);  // [kChannels][kPitch]
    const int t = threadIdx.x, ct = tile % a.c_tiles, rest = tile / a.c_tiles;
    const int b = rest / a.u_tiles, u0 = (rest - b * a.u_tiles) * 64, c0 = ct * T::kChannels;
    const int len = length_in(a.len, b, a.U);
    if (u0 >= len) return;
    S e[T::kSteps][8];
#pragma unroll
    for (int i = 0; i < T::kSteps; ++i) {
        const int c = (t >> 3) + kThreads / 8 * i, u = (t & 7) * 8;
        load8_bits((const S *)a.dout + ((size_t)b * a.C + min(c0 + c, a.C - 1)) * a.U + u0 + u, len - u0 - u, e[i]);
    }
#pragma unroll
    for (int i = 0; i < T::kSteps; ++i) {
        const int c = (t >> 3) + kThreads / 8 * i, u = (t & 7) * 8;
        __builtin_memcpy(__builtin_assume_aligned(lds + c * T::kPitch + u, 4), e[i], sizeof(e[i]));
    }
    __syncthreads();
    constexpr int kGroups = T::kChannels / 8;
#pragma unroll
    for (int i = 0; i < T::kSteps; ++i) {
        const int u = t / kGroups + kThreads / kGroups * i, c = t % kGroups * 8;
        if (u0 + u >= len) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) e[i][j] = lds[(c + j) * T::kPitch + u];
        store8_bits((S *)a.turned + ((size_t)b * a.U + u0 + u) * a.C + c0 + c, a.C - c0 - c, e[i]);
    }
}

constexpr int kSortBytes = kList * 6 + (3 + kWaves) * kRange * 4 + 3 * kWaves * 4;

template <typename S>
__global__ __launch_bounds__(kThreads, 6) void embed_order_kernel(EmbedBwd a, int first)
{
    __shared__ __align__(16) unsigned char smem[kSortBytes];
    static_assert(Turn<S>::kBytes <= kSortBytes, "");
    int w = first + blockIdx.x;
    if (w < a.sorters) {
        sort_range(a, w, smem);
        return;
    }
    w -= a.sorters;
    if (w < a.turners) {
        turn_tile<S>(a, w, smem);
        return;
    }
    const size_t all = (size_t)a.V * a.C, from = (size_t)(w - a.turners) * kFill;
#pragma unroll
    for (int i = 0; i < kFill / (kThreads * 4); ++i) {
        const size_t at = from + (i * kThreads + threadIdx.x) * 4;
        const u32x4_t zero = {0u, 0u, 0u, 0u};
        if (at + 4 <= all) {
            __builtin_memcpy(a.dtable + at, &zero, 16);
        } else {
            for (size_t k = at; k < all; ++k) a.dtable[k] = 0.f;
        }
    }
}

// A lane's channels of the gradient's row of a token
__device__ __forceinline__ void finish_row(const EmbedBwd &a, int v, int c, const float (&acc)[8], int n)
{
    float *row = a.dtable + (size_t)v * a.C + c;
    float out[8];
    if (a.add) load8(row, n, out);
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = a.add ? out[j] + acc[j] * a.scale : acc[j] * a.scale;
    store8(row, n, out);
}

template <typename S>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedBwd a, int c_waves)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = blockIdx.x * 4 + wave, run = unit / c_waves, c = (unit - run * c_waves) * 512 + lane * 8, i0 = run * kRun;
    if (i0 >= a.N) return;
    const Entry mine = a.order[min(i0 + (lane & (kRun - 1)), a.N - 1)];  // (those behind the last that there is are not used)
    const int cnt = min(kRun, *a.total - i0);
    if (cnt <= 0) return;
    const int n = a.C - c;
    const bool whole = a.C % 8 == 0;  // lanes behind the row read its last group and store nothing: no branch around a load
    const int from_c = whole ? min(c, a.C - 8) : c;
    float v[kRun][8];
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
        const size_t row = (size_t)__builtin_amdgcn_readlane(mine.place, min(k, cnt - 1)) * a.C;
        if (whole) load8((const S *)a.rows + row + from_c, 8, v[k]);
        else load8((const S *)a.rows + row + c, n, v[k]);
    }
    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = v[0][j];
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
        if (k >= cnt) break;
        const int token = __builtin_amdgcn_readlane(mine.token, k);
        if (k + 1 == cnt || __builtin_amdgcn_readlane(mine.token, k + 1 < kRun ? k + 1 : k) != token) {
            const int from = __builtin_amdgcn_readlane(mine.from, k), to = __builtin_amdgcn_readlane(mine.to, k);
            if (n > 0) {
                if (from >= i0 && to <= i0 + kRun) finish_row(a, token, c, acc, n);
                else store8(a.parts + ((size_t)run * 2 + (from < i0 ? 0 : 1)) * a.C + c, n, acc);  // (begun in an earlier run: this one's first)
            }
            if (k + 1 < kRun) {
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = v[k + 1 < kRun ? k + 1 : k][j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += v[k + 1 < kRun ? k + 1 : k][j];
        }
    }
}

// The token that begins in a run and goes beyond it: its parts in order, a wavefront every eighth of them
__global__ __launch_bounds__(512) void embed_join_kernel(EmbedBwd a, int c_waves, int first)
{
    __shared__ float sums[7][8][64];
    const uint32_t at = first + blockIdx.x;
    const int run = at / c_waves, i0 = run * kRun;
    const Entry e = a.order[i0 + kRun - 1];
    if (i0 + kRun >= *a.total || e.from < i0 || e.to <= i0 + kRun) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (at - run * c_waves) * 512 + lane * 8, n = a.C - c;
    const int last = (e.to - 1) / kRun;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int r = run + wave; r <= last; r += 8) {
        float p[8];
        load8(a.parts + ((size_t)r * 2 + (r == run ? 1 : 0)) * a.C + c, n, p);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += p[j];
    }
    if (wave) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[wave - 1][j][lane] = acc[j];
    }
    __syncthreads();
    if (wave || n <= 0) return;
#pragma unroll
    for (int w = 0; w < 7; ++w)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += sums[w][j][lane];
    finish_row(a, e.token, c, acc, n);
}

// What a call of these sizes keeps in its workspace
struct Plan {
    size_t order, total, parts, all;  // offsets, and the whole
    int runs;
};
Plan plan_of(int B, int V, int C, int U, int dtype)
{
    Plan p = {};
    const size_t N = (size_t)B * U;
    p.runs = (int)((N + kRun - 1) / kRun);
    p.order = U > 1 ? align_up(N * C * element(dtype), 256) : 0;  // (single tokens lie as rows already)
    p.total = p.order + align_up(N * sizeof(Entry), 256);
    p.parts = p.total + 256;
    p.all = p.parts + align_up((size_t)p.runs * 2 * C * 4, 256);
    return p;
}

template <typename S>
hipError_t run_bwd(EmbedBwd a, int runs, hipStream_t s)
{
    const size_t fillers = a.add ? 0 : ((size_t)a.V * a.C + kFill - 1) / kFill;
    hipError_t e = in_launches((size_t)a.sorters + a.turners + fillers,
                               [&](unsigned n, int first) { embed_order_kernel<S><<<dim3(n), dim3(kThreads), 0, s>>>(a, first); });
    if (e != hipSuccess) return e;
    const int c_waves = (a.C + 511) / 512;
    embed_sum_kernel<S><<<dim3((unsigned)(((long long)runs * c_waves + 3) / 4)), dim3(256), 0, s>>>(a, c_waves);
    e = hipGetLastError();
    if (e != hipSuccess || runs == 1) return e;
    return in_launches((size_t)(runs - 1) * c_waves, [&](unsigned n, int first) { embed_join_kernel<<<dim3(n), dim3(512), 0, s>>>(a, c_waves, first); });
}

int check(int B, int V, int C, int U, int id_bytes, float scale, int dtype)
{
    if (B <= 0 || V <= 0 || C <= 0 || U <= 0 || (id_bytes != 4 && id_bytes != 8) || !finite_float(scale) || !known_dtype(dtype)) return NM_ERR_BAD_ARG;
    const long long most = (1LL << 31) - 1;
    if ((long long)B * U > most / C || (long long)B * U > most - (1 << 14) || (long long)V * C > most) return NM_ERR_UNSUPPORTED;  // (places behind the last one are counted too)
    // what goes in one launch, below 2^32 work items: the forward pass has 256 for a tile of 64 x 64 (an item's last ones may be all but empty), the
    // gradient's sums a wavefront for eight places and 512 channels, eight for a tile at most
    if ((long long)B * ((U + 63) / 64) * ((C + 63) / 64) >= 1LL << 23 || B > 65535) return NM_ERR_UNSUPPORTED;
    return NM_OK;
}

}  // namespace
}  // namespace nm

using namespace nm;

extern "C" {

int nm_embedding_fwd(int B, int V, int C, int U, const void *ids, int id_bytes, const void *table, float scale, const int *lengths,
                     void *out, int dtype, void *hip_stream)
{
    const int st = check(B, V, C, U, id_bytes, scale, dtype);
    if (st != NM_OK) return st;
    if (!ids || !table || !out) return NM_ERR_BAD_ARG;
    const size_t places = (size_t)B * U;
    const Region in[3] = {{ids, places * id_bytes}, {table, (size_t)V * C * element(dtype)}, {lengths, (size_t)B * 4}};
    if (meets({out, places * C * element(dtype)}, in)) return NM_ERR_BAD_ARG;
    EmbedFwd a = {B, V, C, U, {ids, id_bytes == 8}, table, scale, lengths, out, 0, 0};
    return status_of(dtype == NM_BF16 ? run_fwd<bf16_t>(a, (hipStream_t)hip_stream) : run_fwd<float>(a, (hipStream_t)hip_stream));
}

size_t nm_embedding_bwd_workspace_bytes(int B, int V, int C, int U, int dtype)
{
    return check(B, V, C, U, 4, 1.f, dtype) == NM_OK ? plan_of(B, V, C, U, dtype).all : 0;
}

int nm_embedding_bwd(int B, int V, int C, int U, const void *dout, const void *ids, int id_bytes, float scale, const int *lengths,
                     float *dtable, unsigned flags, int dtype, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check(B, V, C, U, id_bytes, scale, dtype);
    if (st != NM_OK) return st;
    if (!dout || !ids || !dtable || (flags & ~(unsigned)NM_ACCUM_DW)) return NM_ERR_BAD_ARG;
    const size_t places = (size_t)B * U;
    const Region in[3] = {{ids, places * id_bytes}, {dout, places * C * element(dtype)}, {lengths, (size_t)B * 4}};
    if (meets({dtable, (size_t)V * C * 4}, in)) return NM_ERR_BAD_ARG;
    const Plan p = plan_of(B, V, C, U, dtype);
    if (workspace_missing(workspace, workspace_bytes, p.all)) return NM_ERR_WORKSPACE;
    char *ws = (char *)workspace;
    EmbedBwd a = {};
    a.B = B; a.V = V; a.C = C; a.U = U; a.N = (int)places;
    a.ids = {ids, id_bytes == 8};
    a.len = lengths;
    a.per_item = 1.0 / U;
    a.dout = dout;
    a.turned = U > 1 ? ws : nullptr;
    a.rows = U > 1 ? ws : dout;
    a.scale = scale;
    a.dtable = dtable;
    a.add = (flags & NM_ACCUM_DW) != 0;
    a.order = (Entry *)(ws + p.order);
    a.total = (int *)(ws + p.total);
    a.parts = (float *)(ws + p.parts);
    // as many ranges as there are CUs, where that leaves a range no more tokens than a workgroup has counters for
    a.range = V > 256 * kRange ? kRange : (V + 255) / 256;
    a.sorters = (V - 1) / a.range + 1;
    a.u_tiles = (U + 63) / 64;
    const int turn = dtype == NM_BF16 ? Turn<bf16_t>::kChannels : Turn<float>::kChannels;
    a.c_tiles = (C + turn - 1) / turn;
    a.turners = U > 1 ? B * a.u_tiles * a.c_tiles : 0;
    hipStream_t s = (hipStream_t)hip_stream;
    return status_of(dtype == NM_BF16 ? run_bwd<bf16_t>(a, p.runs, s) : run_bwd<float>(a, p.runs, s));
}

}  // extern "C"
