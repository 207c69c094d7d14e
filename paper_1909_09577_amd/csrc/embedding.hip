// Lookup of tokens' embeddings and its gradient (definition: include/nm_embedding.h).
//
// Forward: a table's rows run over the channels, activations over the tokens, so a workgroup carries 64 tokens x 64 channels across LDS and
// reads and writes 128-byte pieces.  Calls of few tokens an item are copied element by element.
//
// Gradient: a sum over the places of each token, which has to come out the same every time, so the places are sorted by token, without
// atomics on sums.  Three launches:
//   order  one workgroup for each range of tokens reads all token numbers, counts those of its range and of the ranges below,
//          and writes its places in order behind them (counts of a thread's own stretch of the places, summed over the threads, are where the
//          thread writes: a stable counting sort).  Beside them other workgroups turn dout into rows of channels and fill dtable
//          with zeros.
//   sums   a wavefront adds a run of 32 sorted places, a lane eight channels of them; a token whose places lie in one run is finished there.
//          A frequent token's runs leave parts.
//   join   adds the parts of such a token in order.
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
constexpr int kRange = 32;    // tokens of a sorting workgroup at most
constexpr int kChunk = 8192;  // places that it looks at at a time
constexpr int kMine = kChunk / 256;  // of a thread
constexpr int kRun = 32;      // sorted places of a wavefront
constexpr int kFill = 16384;  // floats that a workgroup fills

struct EmbedBwd {
    int B, V, C, U, N;
    Ids ids;
    const int *len;
    const void *dout, *rows;  // rows [N][C]: dout turned, or dout itself
    void *turned;             // where to, or NULL
    float scale;
    float *dtable;
    bool add;
    int *order, *token, *starts;  // places sorted by token [N], their tokens [N], where a token's begin [V+1]
    float *parts;                 // [runs][2][C]: sums of a run's first and last token
    int range, sorters, u_tiles, c_tiles, turners;
};

// the token at place p, -1 where there is none
__device__ __forceinline__ int token_at(const EmbedBwd &a, int p)
{
    if (p >= a.N) return -1;
    int id = a.ids.at(p, a.V);
    if (a.len) {
        const int b = p / a.U;
        if (p - b * a.U >= a.len[b]) id = -1;
    }
    return id;
}

__device__ __forceinline__ int wave_scan(int v, int lane)  // sum of the lanes up to this one
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

__device__ void sort_range(const EmbedBwd &a, unsigned char *smem)
{
    uint8_t *local = smem;                                                // [kChunk]: token in the range, or 255
    uint16_t *count = reinterpret_cast<uint16_t *>(smem + kChunk);        // [range][256]
    int *cursor = reinterpret_cast<int *>(smem + kChunk + kRange * 512);  // [kRange]: where a token's next place goes
    int *found = cursor + kRange;                                         // [kRange]: places of a token in the chunk
    int *below = found + kRange;                                          // [4]
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int v0 = blockIdx.x * a.range, bins = min(a.range, a.V - v0);
    if (t < kRange) cursor[t] = 0;
    __syncthreads();
    int less = 0;
    const int chunks = (a.N + kChunk - 1) / kChunk;
    auto stage = [&](int p0, bool counting) {
#pragma unroll 8
        for (int i = 0; i < kMine; ++i) {
            const int id = token_at(a, p0 + i * 256 + t), r = id - v0;
            const bool mine = id >= 0 && r >= 0 && r < bins;
            local[i * 256 + t] = mine ? (uint8_t)r : (uint8_t)255;
            if (counting) {
                less += id >= 0 && r < 0;
                if (mine) atomicAdd(&cursor[r], 1);  // (whole numbers: any order gives the same)
            }
        }
    };
    for (int k = 0; k < chunks; ++k) stage(k * kChunk, true);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) less += __shfl_xor(less, d);
    if (lane == 0) below[wave] = less;
    __syncthreads();
    if (wave == 0) {
        const int n = lane < bins ? cursor[lane] : 0, base = below[0] + below[1] + below[2] + below[3];
        const int upto = wave_scan(n, lane);
        if (lane < bins) {
            cursor[lane] = base + upto - n;
            a.starts[v0 + lane] = base + upto - n;
            if (v0 + lane == a.V - 1) a.starts[a.V] = base + upto;
        }
    }
    __syncthreads();
    for (int k = 0; k < chunks; ++k) {
        if (chunks > 1) stage(k * kChunk, false);
        for (int r = 0; r < bins; ++r) count[r * 256 + t] = 0;
        __syncthreads();
        u32x4_t w[kMine / 16];
        bool any = false;
#pragma unroll
        for (int i = 0; i < kMine / 16; ++i) {
            w[i] = *reinterpret_cast<const u32x4_t *>(local + t * kMine + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) any |= w[i][j] != 0xffffffffu;
        }
        if (any) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int r = (w[i / 16][i / 4 % 4] >> (8 * (i % 4))) & 255;
                if (r != 255) ++count[r * 256 + t];
            }
        }
        __syncthreads();
        for (int r = wave; r < bins; r += 4) {  // counts become what lies before a thread's own
            uint16_t *c = count + r * 256 + lane * 4;
            const int n0 = c[0], n1 = c[1], n2 = c[2], n3 = c[3], sum = n0 + n1 + n2 + n3;
            const int upto = wave_scan(sum, lane), from = upto - sum;
            c[0] = (uint16_t)from;
            c[1] = (uint16_t)(from + n0);
            c[2] = (uint16_t)(from + n0 + n1);
            c[3] = (uint16_t)(from + n0 + n1 + n2);
            if (lane == 63) found[r] = upto;
        }
        __syncthreads();
        if (any) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int r = (w[i / 16][i / 4 % 4] >> (8 * (i % 4))) & 255;
                if (r != 255) {
                    const int at = cursor[r] + count[r * 256 + t]++;
                    a.order[at] = k * kChunk + t * kMine + i;
                    a.token[at] = v0 + r;
                }
            }
        }
        __syncthreads();
        if (t < bins) cursor[t] += found[t];
        __syncthreads();
    }
}

// 64 tokens x 64 channels of dout as rows of channels
template <typename S>
__device__ void turn_tile(const EmbedBwd &a, int tile, unsigned char *smem)
{
    constexpr int kPitch = 64 + (sizeof(S) == 2 ? 2 : 1);
    S *lds = reinterpret_cast<S *>(smem);  // [64 channels][kPitch]
    const int t = threadIdx.x, ct = tile % a.c_tiles, rest = tile / a.c_tiles;
    const int b = rest / a.u_tiles, u0 = (rest - b * a.u_tiles) * 64, c0 = ct * 64;
    const int len = length_in(a.len, b, a.U);
    if (u0 >= len) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (t >> 3) + 32 * i, u = (t & 7) * 8;
        float v[8];
        load8((const S *)a.dout + ((size_t)b * a.C + min(c0 + c, a.C - 1)) * a.U + u0 + u, len - u0 - u, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) store_from_f32(lds + c * kPitch + u, j, v[j]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int u = (t >> 3) + 32 * i, c = (t & 7) * 8;
        if (u0 + u >= len) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = load_as_f32(lds, (c + j) * kPitch + u);
        store8((S *)a.turned + ((size_t)b * a.U + u0 + u) * a.C + c0 + c, a.C - c0 - c, v);
    }
}

template <typename S>
__global__ __launch_bounds__(256) void embed_order_kernel(EmbedBwd a)
{
    __shared__ __align__(16) unsigned char smem[kChunk + kRange * 512 + (2 * kRange + 4) * 4];
    int w = blockIdx.x;
    if (w < a.sorters) {
        sort_range(a, smem);
        return;
    }
    w -= a.sorters;
    if (w < a.turners) {
        turn_tile<S>(a, w, smem);
        return;
    }
    const size_t all = (size_t)a.V * a.C, from = (size_t)(w - a.turners) * kFill;
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kFill / 2048; ++i) {
        const size_t at = from + i * 2048 + threadIdx.x * 8;
        if (at < all) store8(a.dtable + at, (int)min(all - at, (size_t)8), zero);
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
    const int unit = blockIdx.x * 4 + wave, run = unit / c_waves, c = (unit - run * c_waves) * 512 + lane * 8;
    const int total = a.starts[a.V], i0 = run * kRun, cnt = min(kRun, total - i0);
    if (cnt <= 0) return;
    const int mine = lane < cnt ? lane : cnt - 1;
    const int place = a.order[i0 + mine], token = a.token[i0 + mine];
    const int n = a.C - c;
    const bool whole = a.C % 8 == 0;  // lanes behind the row read its last group and store nothing: no branch around a load
    const int from_c = whole ? min(c, a.C - 8) : c;
    float acc[8];
    auto leave = [&](int v) {
        if (n <= 0) return;
        const int from = a.starts[v], to = a.starts[v + 1];
        if (from >= i0 && to <= i0 + kRun) {
            finish_row(a, v, c, acc, n);
        } else {  // (where the token began in an earlier run, it is this run's first)
            store8(a.parts + ((size_t)run * 2 + (from < i0 ? 0 : 1)) * a.C + c, n, acc);
        }
    };
    int current = __builtin_amdgcn_readfirstlane(token);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    for (int i = 0; i < cnt; i += 8) {
        float v[8][8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int p = __builtin_amdgcn_readlane(place, min(i + k, cnt - 1));
            if (whole) load8((const S *)a.rows + (size_t)p * a.C + from_c, 8, v[k]);
            else load8((const S *)a.rows + (size_t)p * a.C + c, n, v[k]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (i + k >= cnt) break;
            const int id = __builtin_amdgcn_readlane(token, i + k);
            if (id != current) {
                leave(current);
                current = id;
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += v[k][j];
        }
    }
    leave(current);
}

// The token that begins in a run and goes beyond it: its parts in order, a wavefront every fourth of them
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedBwd a, int c_waves)
{
    __shared__ float sums[3][64][8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int run = blockIdx.x / c_waves, c = (blockIdx.x - run * c_waves) * 512 + lane * 8, n = a.C - c;
    const int total = a.starts[a.V], i0 = run * kRun;
    if (i0 + kRun >= total) return;  // (the last run: nothing goes beyond it)
    const int v = a.token[i0 + kRun - 1], from = a.starts[v], to = a.starts[v + 1];
    if (from < i0 || to <= i0 + kRun) return;
    const int last = (to - 1) / kRun;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int r = run + wave; r <= last; r += 4) {
        float p[8];
        load8(a.parts + ((size_t)r * 2 + (r == run ? 1 : 0)) * a.C + c, n, p);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += p[j];
    }
    if (wave) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[wave - 1][lane][j] = acc[j];
    }
    __syncthreads();
    if (wave || n <= 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += sums[w][lane][j];
    finish_row(a, v, c, acc, n);
}

// What a call of these sizes keeps in its workspace
struct Plan {
    size_t rows, order, token, starts, parts, all;  // offsets, and the whole
    int runs;
};
Plan plan_of(int B, int V, int C, int U, int dtype)
{
    Plan p = {};
    const size_t N = (size_t)B * U;
    p.runs = (int)((N + kRun - 1) / kRun);
    p.order = U > 1 ? align_up(N * C * element(dtype), 256) : 0;  // (single tokens lie as rows already)
    p.token = p.order + align_up(N * 4, 256);
    p.starts = p.token + align_up(N * 4, 256);
    p.parts = p.starts + align_up(((size_t)V + 1) * 4, 256);
    p.all = p.parts + align_up((size_t)p.runs * 2 * C * 4, 256);
    return p;
}

template <typename S>
hipError_t run_bwd(EmbedBwd a, int runs, hipStream_t s)
{
    const size_t fillers = a.add ? 0 : ((size_t)a.V * a.C + kFill - 1) / kFill;
    embed_order_kernel<S><<<dim3((unsigned)(a.sorters + a.turners + fillers)), dim3(256), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int c_waves = (a.C + 511) / 512;
    embed_sum_kernel<S><<<dim3((unsigned)(((long long)runs * c_waves + 3) / 4)), dim3(256), 0, s>>>(a, c_waves);
    e = hipGetLastError();
    if (e != hipSuccess || runs == 1) return e;
    embed_join_kernel<<<dim3((unsigned)(runs - 1) * c_waves), dim3(256), 0, s>>>(a, c_waves);
    return hipGetLastError();
}

int check(int B, int V, int C, int U, int id_bytes, float scale, int dtype)
{
    if (B <= 0 || V <= 0 || C <= 0 || U <= 0 || (id_bytes != 4 && id_bytes != 8) || !finite_float(scale) || !known_dtype(dtype)) return NM_ERR_BAD_ARG;
    const long long most = (1LL << 31) - 1;
    if ((long long)B * U > most / C || (long long)B * U > most - (1 << 14) || (long long)V * C > most) return NM_ERR_UNSUPPORTED;  // (places behind the last one are counted too)
    // the grids, below 2^32 work items: tiles of 64 x 64 (an item's last ones may be all but empty), and what is filled
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
    a.dout = dout;
    a.turned = U > 1 ? ws : nullptr;
    a.rows = U > 1 ? ws : dout;
    a.scale = scale;
    a.dtable = dtable;
    a.add = (flags & NM_ACCUM_DW) != 0;
    a.order = (int *)(ws + p.order);
    a.token = (int *)(ws + p.token);
    a.starts = (int *)(ws + p.starts);
    a.parts = (float *)(ws + p.parts);
    // as many ranges as there are CUs, where that leaves a range no more tokens than a workgroup has counters for
    a.range = (V + 255) / 256 < kRange ? (V + 255) / 256 : kRange;
    a.sorters = (V + a.range - 1) / a.range;
    a.u_tiles = (U + 63) / 64;
    a.c_tiles = (C + 63) / 64;
    a.turners = U > 1 ? B * a.u_tiles * a.c_tiles : 0;
    hipStream_t s = (hipStream_t)hip_stream;
    return status_of(dtype == NM_BF16 ? run_bwd<bf16_t>(a, p.runs, s) : run_bwd<float>(a, p.runs, s));
}

}  // extern "C"
