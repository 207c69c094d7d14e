// Attention of new tokens over a paged cache (definition: include/nm_paged_attention.h).
//
// The cache is laid out for the matrix instructions: a key is a row of channels, so that its 16 bytes are operands of the scores as they lie in
// memory; values are rows of tokens, so that theirs are operands of the second product.  Scores have places as rows and tokens as columns
// (the new tokens of all heads that share keys and values), and the places are dealt to the rows such that a lane ends up with
// those eight neighbouring places of its column that the second product wants from it: probabilities stay in the registers that they were
// made in.  One pass with a running maximum and sum for each column.
//
// Measured (bfloat16): 32 sequences of 4000 to 8001 places, 2 shared heads of 128, one token each: 46 + 5 us for 197 MB (4.3 TB/s; 8 of them before
// the first loads return and after the last).  4 x 500 tokens behind 3000 to 6000 places, 8 heads of 128 over 2: 77 + 9 us; the products alone
// would take 22, and those of the probabilities' second term half as much.  CUs are busy 63 % of the time, with one and a half wavefronts a SIMD then (LDS and
// registers have room for two): workgroups differ in what they have to do, and are dealt in one round.  While it is busy, a wavefront's products,
// exponentials and LDS reads follow one another (matrix pipes 24 % of the time, vector units 24, LDS 20).  One sequence of 2000 places: 7 + 3 us,
// two launches of few workgroups.
#include "../../include/nm_paged_attention.h"
#include "token_ops.h"

namespace nm {
namespace {

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLag = 8.f;      // powers of two that the base of the sums may lie below the maximum
constexpr int kMaxSplits = 64;
constexpr int kTile = 32;        // places that a wavefront looks at at a time
constexpr int kWaves = 4;
// columns that a workgroup reads the cache for by itself (8 sequences of 2000 places, 32 columns: 9.9 us against 11.5 for heads of 64, 13.8 against
// 12.8 for 128; 48 columns 11.8 against 13.0 and 14.2 against 14.8, but for twice the reads of a cache that is here in the caches nearby)
constexpr int kFewColumns = 32;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

struct Paged {
    int B, H, Hkv, G, D, U;
    const void *q, *k, *v;
    long long qs, os;
    int pages, log_page, max_pages;
    const int *table, *len, *q_len;
    int window;
    float c;  // |scale| * log2(e)
    uint32_t flip;  // sign bit of the scale, for the tokens' channels
    void *out;
    float *lse, *part, *part_ml;  // [splits][B*H*U][D], [splits][B*H*U][2]
    int col_tiles, splits;
};

// Products of blocks of 16 x 16, a tile of 32 places being two of them: `Mma<S>::place(m, i)` is the place of row i of block m.
template <typename S>
struct Mma;
template <>
struct Mma<bf16_t> {
    static constexpr int kChannels = 32;  // of a step of the scores
    typedef bf16x8_t Frag;
    // row i = 4*a + c of block m is place 8*a + 4*m + c: a lane's results of both blocks are eight neighbouring places
    static __device__ __forceinline__ int place(int m, int i) { return 8 * (i >> 2) + 4 * m + (i & 3); }
    static __device__ __forceinline__ int first_channel(int step, int quarter) { return 32 * step + 8 * quarter; }
    static __device__ __forceinline__ f32x4_t mul(Frag a, Frag b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma<float> {
    static constexpr int kChannels = 16;
    typedef f32x4_t Frag;  // four steps of four channels: step j takes element j of every quarter's
    static __device__ __forceinline__ int place(int m, int i) { return 16 * m + i; }
    static __device__ __forceinline__ int first_channel(int step, int quarter) { return 16 * step + 4 * quarter; }
    static __device__ __forceinline__ f32x4_t mul(Frag a, Frag b, f32x4_t c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};

__device__ __forceinline__ bf16_t flipped(bf16_t v, uint32_t flip) { return (bf16_t)(v ^ (flip >> 16)); }
__device__ __forceinline__ float flipped(float v, uint32_t flip) { return __uint_as_float(__float_as_uint(v) ^ flip); }

// The new tokens' places that a column may look at, [lo, hi)
struct Column {
    int g, u, lo, hi;
    bool exists, there;
};
__device__ __forceinline__ Column column_of(const Paged &a, int b, int m, int n, int len)
{
    Column c;
    c.exists = m < a.G * a.U;
    c.u = c.exists ? m / a.G : 0;
    c.g = m - c.u * a.G;
    if (!c.exists) c.g = 0;
    c.there = c.exists && c.u < n;
    const int at = len - n + c.u;
    c.hi = c.there ? max(0, min(at + 1, a.max_pages << a.log_page)) : 0;
    c.lo = c.there && a.window && a.window <= at ? at + 1 - a.window : 0;
    if (c.hi <= c.lo) c.there = false;
    return c;
}

// The work of a workgroup.  Neighbouring workgroups go to different XCDs; those that read the same places of the same heads to the same one, and
// the shares of a sequence to several of them, for sequences differ in length.
struct Work {
    int b, kvh, col_tile, split;
    __device__ __forceinline__ Work(const Paged &a)
    {
        const int heads = a.B * a.Hkv, i = blockIdx.x % (heads * a.splits);
        col_tile = blockIdx.x / (heads * a.splits);
        split = i / heads;
        const int bh = (int)((i - split * heads + (long long)split * a.Hkv) % heads);
        b = bh / a.Hkv;
        kvh = bh - b * a.Hkv;
    }
};

// NC blocks of 16 columns; DB blocks of 16 channels
template <typename S, int DB, int NC>
__global__ __launch_bounds__(kWaves * 64) void paged_few_kernel(Paged a)
{
    typedef Mma<S> M;
    typedef typename M::Frag Frag;
    constexpr bool kBf16 = sizeof(S) == 2;
    constexpr int KS = (DB * 16 + M::kChannels - 1) / M::kChannels;  // steps of the scores
    constexpr int VB = kBf16 ? 1 : 2;                                // value operands of 16 channels and a tile
    constexpr int kPer = 16 / sizeof(S);                             // elements of an operand's 16 bytes
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, i = lane & 15;
    const Work work(a);
    const int ct = work.col_tile, split = work.split, b = work.b, kvh = work.kvh;
    const int n_new = length_in(a.q_len, b, a.U), len = max(a.len[b], 0);

    Column col[NC];
    int first = 0x7fffffff, last = 0;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        col[n] = column_of(a, b, (ct * NC + n) * 16 + i, n_new, len);
        if (col[n].there) {
            first = min(first, col[n].lo);
            last = max(last, col[n].hi);
        }
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        first = min(first, __shfl_xor(first, d));
        last = max(last, __shfl_xor(last, d));
    }
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    const int t_first = last ? first / kTile : 0, t_last = (last + kTile - 1) / kTile, share = (t_last - t_first + a.splits - 1) / a.splits;
    const int t_begin = t_first + split * share, t_end = min(t_last, t_begin + share);

    // the tokens' channels
    Frag q[NC][KS];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        const S *p = (const S *)a.q + (size_t)b * a.qs + (size_t)(kvh * a.G + col[n].g) * a.D * a.U + col[n].u;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            S e[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int d = M::first_channel(s, quarter) + j;
                e[j] = flipped(p[(size_t)min(d, a.D - 1) * a.U], a.flip);
                if (!col[n].there || d >= a.D) e[j] = S(0);
            }
            __builtin_memcpy(&q[n][s], e, 16);
        }
    }

    // a tile's operands; a page that does not exist is read as page 0, and masked
    const int size = 1 << a.log_page;
    auto page_of = [&](int t, int part) {
        const int at = min((t * kTile + 16 * part) >> a.log_page, a.max_pages - 1);
        return a.table[(size_t)b * a.max_pages + at];
    };
    Frag kf[2][KS], vf[DB][VB];
    auto load_k = [&](int t, int pg0, int pg1) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int place = M::place(m, i), pg = place < 16 ? pg0 : pg1, row = (t * kTile + place) & (size - 1);
            const S *p = (const S *)a.k + (((size_t)pg * a.Hkv + kvh) * size + row) * a.D;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int d = M::first_channel(s, quarter);
                kf[m][s] = *reinterpret_cast<const Frag *>(p + min(d, a.D - kPer));
                if (DB * 16 % M::kChannels && s == KS - 1 && d >= a.D) kf[m][s] = Frag{};
            }
        }
    };
    auto load_v = [&](int t, int pg0, int pg1) {
#pragma unroll
        for (int h = 0; h < VB; ++h) {
            const int place = kBf16 ? 8 * quarter : 16 * h + 4 * quarter, pg = place < 16 ? pg0 : pg1, row = (t * kTile + place) & (size - 1);
            const S *p = (const S *)a.v + (((size_t)pg * a.Hkv + kvh) * a.D + i) * size + row;
#pragma unroll
            for (int d = 0; d < DB; ++d) vf[d][h] = *reinterpret_cast<const Frag *>(p + (size_t)d * 16 * size);
        }
    };

    float mx[NC], sum[NC];
    f32x4_t acc[NC][DB];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        mx[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[n][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    auto there = [&](int pg) { return (unsigned)pg < (unsigned)a.pages; };
    auto usable = [&](int pg) { return there(pg) ? pg : 0; };

    int t = t_begin + wave, pg0 = 0, pg1 = 0, next0 = 0, next1 = 0;
    if (t < t_end) {
        pg0 = page_of(t, 0);
        pg1 = page_of(t, 1);
        load_k(t, usable(pg0), usable(pg1));
        load_v(t, usable(pg0), usable(pg1));
        next0 = page_of(t + kWaves, 0);
        next1 = page_of(t + kWaves, 1);
    }
    for (; t < t_end; t += kWaves) {
        const int t0 = t * kTile;
        f32x4_t s[NC][2];
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                s[n][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int st = 0; st < KS; ++st) s[n][m] = M::mul(kf[m][st], q[n][st], s[n][m]);
            }
        const bool more = t + kWaves < t_end;
        if (more) load_k(t + kWaves, usable(next0), usable(next1));
        const bool whole = there(pg0) && there(pg1);
        bool inside = whole;
#pragma unroll
        for (int n = 0; n < NC; ++n) inside = inside && (!col[n].there || (col[n].lo <= t0 && t0 + kTile <= col[n].hi));
        const bool edge = !__all(inside);
        Frag p[NC][2];  // bfloat16: the probabilities and what their rounding leaves; float: of the two blocks
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            // (as plain floats: with ROCm 7.2's compiler a form that set elements of the matrix result under the branch gave wrong outputs in the tests of
            // masked tiles; why was not found)
            float z[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = s[n][j >> 2][j & 3];
            if (edge) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int place = M::place(j >> 2, 4 * quarter + (j & 3)), pos = t0 + place;
                    const bool seen = (pos >= col[n].lo) & (pos < col[n].hi) & there(place < 16 ? pg0 : pg1);
                    z[j] = seen ? z[j] : -INFINITY;
                }
            }
            float top = z[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) top = fmaxf(top, z[j]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32)) * a.c;
            if (__any(top > mx[n] + kLag)) {
                top = fmaxf(top, mx[n]);
                const float shrink = __builtin_amdgcn_exp2f(mx[n] - (top == -INFINITY ? 0.f : top));
                sum[n] *= shrink;
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[n][d] *= shrink;
                mx[n] = top;
            }
            const float base = mx[n] == -INFINITY ? 0.f : mx[n];
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j], a.c, -base));
                sum[n] += e[j];
            }
            if constexpr (kBf16) {
                u32x4_t hi, lo;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    hi[j] = pack_bf16x2(e[2 * j], e[2 * j + 1]);
                    lo[j] = pack_bf16x2(e[2 * j] - __uint_as_float(hi[j] << 16), e[2 * j + 1] - __uint_as_float(hi[j] & 0xffff0000u));
                }
                p[n][0] = __builtin_bit_cast(Frag, hi);
                p[n][1] = __builtin_bit_cast(Frag, lo);
            } else {
                __builtin_memcpy(&p[n][0], e, 16);
                __builtin_memcpy(&p[n][1], e + 4, 16);
            }
        }
        if (t0 < first || t0 + kTile > last || !whole) {  // (uniform) values that no token looks at may hold anything
#pragma unroll
            for (int h = 0; h < VB; ++h) {
                const int place = kBf16 ? 8 * quarter : 16 * h + 4 * quarter, from = first - t0 - place, to = last - t0 - place;
                const bool exists = there(place < 16 ? pg0 : pg1);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    S e[kPer];
                    __builtin_memcpy(e, &vf[d][h], 16);
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        if (!exists || j < from || j >= to) e[j] = S(0);
                    __builtin_memcpy(&vf[d][h], e, 16);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                if constexpr (kBf16) {
                    acc[n][d] = M::mul(vf[d][0], p[n][1], acc[n][d]);
                    acc[n][d] = M::mul(vf[d][0], p[n][0], acc[n][d]);
                } else {
                    acc[n][d] = M::mul(vf[d][0], p[n][0], acc[n][d]);
                    acc[n][d] = M::mul(vf[d][VB - 1], p[n][1], acc[n][d]);
                }
            }
        if (more) {
            load_v(t + kWaves, usable(next0), usable(next1));
            pg0 = next0;
            pg1 = next1;
            next0 = page_of(t + 2 * kWaves, 0);
            next1 = page_of(t + 2 * kWaves, 1);
        }
    }

    // the wavefronts' maxima, sums and products are joined through LDS
    float *sums = reinterpret_cast<float *>(smem);          // [kWaves][NC][2][16]
    float *prod = sums + kWaves * NC * 32;                  // [kWaves][NC][DB][64][4]
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        float all = sum[n];
        all += __shfl_xor(all, 16);
        all += __shfl_xor(all, 32);
        if (quarter == 0) {
            sums[(wave * NC + n) * 32 + i] = mx[n];
            sums[(wave * NC + n) * 32 + 16 + i] = all;
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4_t *>(prod + (((wave * NC + n) * DB + d) * 64 + lane) * 4) = acc[n][d];
    }
    __syncthreads();
    const size_t rows = (size_t)a.B * a.H * a.U;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        float top = -INFINITY, total = 0.f, weight[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sums[(w * NC + n) * 32 + i]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            weight[w] = __builtin_amdgcn_exp2f(sums[(w * NC + n) * 32 + i] - (top == -INFINITY ? 0.f : top));
            total += weight[w] * sums[(w * NC + n) * 32 + 16 + i];
        }
        if (!col[n].exists) continue;
        const int head = kvh * a.G + col[n].g;
        const size_t row = ((size_t)b * a.H + head) * a.U + col[n].u;
        const bool some = col[n].there && total != 0.f;
        if (wave == 0 && quarter == 0) {
            if (a.splits > 1) {
                float *ml = a.part_ml + ((size_t)split * rows + row) * 2;
                ml[0] = some ? top : -INFINITY;
                ml[1] = some ? total : 0.f;
            } else if (a.lse) {
                a.lse[row] = some ? (top + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
            }
        }
        const float inv = some ? (a.splits > 1 ? 1.f : 1.f / total) : 0.f;
        for (int d = wave; d < DB; d += kWaves) {
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v += weight[w] * *reinterpret_cast<const f32x4_t *>(prod + (((w * NC + n) * DB + d) * 64 + lane) * 4);
            const int ch = 16 * d + 4 * quarter;
            if (!some) v = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (a.splits > 1) {
                *reinterpret_cast<f32x4_t *>(a.part + ((size_t)split * rows + row) * a.D + ch) = v;
            } else {
                S *o = (S *)a.out + (size_t)b * a.os + ((size_t)head * a.D + ch) * a.U + col[n].u;
#pragma unroll
                for (int r = 0; r < 4; ++r) store_from_f32(o, (size_t)r * a.U, v[r] * inv);
            }
        }
    }
}


// Many columns: four wavefronts with 32 columns each share tiles of 64 places, which go from memory through registers to LDS, the next one
// while this one is worked on.  Blocks of 32 x 32; bfloat16 alone.  Rows in LDS are 16 bytes longer than their contents, so that 16 lanes that
// read 16 rows meet every bank once.
constexpr int kManyTile = 64, kManyColumns = 128;
typedef float f32x16_t __attribute__((ext_vector_type(16)));

template <int DB>
struct ManyLds {
    static constexpr int kPitchK = DB * 32 + 16, kPitchV = kManyTile * 2 + 16, kRowsV = (DB + 1) / 2 * 32;
    static constexpr int kBuffer = kManyTile * kPitchK + kRowsV * kPitchV, kBytes = 2 * kBuffer;
};

template <int DB>
__global__ __launch_bounds__(256, 2) void paged_many_kernel(Paged a)
{
    typedef ManyLds<DB> L;
    typedef bf16x8_t Frag;
    constexpr int D = DB * 16, ND = (DB + 1) / 2, kGran = D / 8, kLoads = (kManyTile * kGran + 255) / 256, kAll = kManyTile * kGran;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, i32 = lane & 31;
    const Work work(a);
    const int ct = work.col_tile, split = work.split, b = work.b, kvh = work.kvh;
    const int n_new = length_in(a.q_len, b, a.U), len = max(a.len[b], 0);
    const Column col = column_of(a, b, ct * kManyColumns + wave * 32 + i32, n_new, len);
    int first = col.there ? col.lo : 0x7fffffff, last = col.there ? col.hi : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        first = min(first, __shfl_xor(first, d));
        last = max(last, __shfl_xor(last, d));
    }
    const int wave_first = __builtin_amdgcn_readfirstlane(first), wave_last = __builtin_amdgcn_readfirstlane(last);
    int *range = reinterpret_cast<int *>(smem);
    if (lane == 0) {
        range[wave] = wave_first;
        range[4 + wave] = wave_last;
    }
    __syncthreads();
    first = min(min(range[0], range[1]), min(range[2], range[3]));
    last = max(max(range[4], range[5]), max(range[6], range[7]));
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    __syncthreads();
    const int t_first = last ? first / kManyTile : 0, t_last = (last + kManyTile - 1) / kManyTile, share = (t_last - t_first + a.splits - 1) / a.splits;
    const int t_begin = t_first + split * share, t_end = min(t_last, t_begin + share);

    const int size = 1 << a.log_page;
    const int *table = a.table + (size_t)b * a.max_pages;
    const bf16_t *kbase = (const bf16_t *)a.k + (size_t)kvh * size * D, *vbase = (const bf16_t *)a.v + (size_t)kvh * size * D;
    const size_t page_stride = (size_t)a.Hkv * size * D;
    auto there = [&](int pg) { return (unsigned)pg < (unsigned)a.pages; };
    // the pages of a tile's four groups of 16 places
    struct Pages {
        int p0, p1, p2, p3;
        __device__ __forceinline__ int of(int j) const  // (of values: a choice between members would put them into scratch memory)
        {
            const int lower = j & 1 ? +p1 : +p0, upper = j & 1 ? +p3 : +p2;
            return j & 2 ? +upper : +lower;
        }
    };
    auto page_at = [&](int place) { return table[min(place >> a.log_page, a.max_pages - 1)]; };
    auto pages_of = [&](int t) {
        const int p = t * kManyTile;
        return Pages{page_at(p), page_at(p + 16), page_at(p + 32), page_at(p + 48)};
    };
    auto all_there = [&](const Pages &p) { return there(p.p0) && there(p.p1) && there(p.p2) && there(p.p3); };
    Pages pg = {}, next_pg = {};
    u32x4_t kr[kLoads], vr[kLoads];
    const int vg = tid & 7;  // the thread's group of eight places of the values' rows
    // where this thread's parts of a tile lie: from its first place on, where one page has them all
    const uint32_t k_off = (uint32_t)tid * 16, v_off = ((uint32_t)(tid >> 3) * (uint32_t)size + 8 * vg) * 2;
    auto load = [&](int t, const Pages &p) {
        if (a.log_page >= 6) {  // (uniform)
            const size_t page = (size_t)(there(p.p0) ? p.p0 : 0) * page_stride;
            const int row0 = (t * kManyTile) & (size - 1);
            const char *kp = reinterpret_cast<const char *>(kbase + page + (size_t)row0 * D), *vp = reinterpret_cast<const char *>(vbase + page + row0);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                kr[i] = *reinterpret_cast<const u32x4_t *>(kp + i * 4096 + (kAll % 256 == 0 || i + 1 < kLoads ? k_off : min(k_off, (uint32_t)(kAll - 1 - i * 256) * 16)));
                const uint32_t row = (uint32_t)i * 64 * (uint32_t)size;  // 32 rows of values
                vr[i] = *reinterpret_cast<const u32x4_t *>(vp + row + (D % 32 == 0 || i + 1 < kLoads ? v_off : min(v_off, (uint32_t)((D - 1 - i * 32) * size + 8 * vg) * 2)));
            }
            return;
        }
        const Pages q = {there(p.p0) ? p.p0 : 0, there(p.p1) ? p.p1 : 0, there(p.p2) ? p.p2 : 0, there(p.p3) ? p.p3 : 0};
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int e = min(i * 256 + tid, kAll - 1), row = e / kGran, g = e - row * kGran;
            const int page = q.of(row >> 4);
            kr[i] = *reinterpret_cast<const u32x4_t *>(kbase + page * page_stride + (size_t)((t * kManyTile + row) & (size - 1)) * D + g * 8);
        }
        const int page = q.of(vg >> 1);
        const bf16_t *v = vbase + page * page_stride + ((t * kManyTile + 8 * vg) & (size - 1));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) vr[i] = *reinterpret_cast<const u32x4_t *>(v + (size_t)min(i * 32 + (tid >> 3), D - 1) * size);
    };
    auto write = [&](unsigned char *buf, int t, const Pages &p) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int e = i * 256 + tid, row = e / kGran, g = e - row * kGran;
            if (kAll % 256 == 0 || e < kAll) *reinterpret_cast<u32x4_t *>(buf + row * L::kPitchK + g * 16) = kr[i];
        }
        const int t0 = t * kManyTile, pos = t0 + 8 * vg;
        if (t0 < first || t0 + kManyTile > last || !all_there(p)) {  // (uniform) values that no token looks at
            const bool exists = there(p.of(vg >> 1));
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                bf16_t e[8];
                __builtin_memcpy(e, &vr[i], 16);
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = exists && pos + j >= first && pos + j < last ? e[j] : (bf16_t)0;
                __builtin_memcpy(&vr[i], e, 16);
            }
        }
        unsigned char *v = buf + kManyTile * L::kPitchK + vg * 16;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = i * 32 + (tid >> 3);
            if (D % 32 == 0 || row < D) *reinterpret_cast<u32x4_t *>(v + row * L::kPitchV) = vr[i];
        }
    };

    if (t_begin < t_end) {
        pg = pages_of(t_begin);
        load(t_begin, pg);
    }
    Frag q[DB];
    {
        const bf16_t *p = (const bf16_t *)a.q + (size_t)b * a.qs + (size_t)(kvh * a.G + col.g) * D * a.U + col.u;
#pragma unroll
        for (int s = 0; s < DB; ++s) {
            bf16_t e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = flipped(p[(size_t)(16 * s + 8 * half + j) * a.U], a.flip);
                if (!col.there) e[j] = 0;
            }
            __builtin_memcpy(&q[s], e, 16);
        }
    }
    float mx = -INFINITY, sum = 0.f;
    f32x16_t acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
    // places are dealt to the rows of the scores such that a lane's register r is place 16*(r/8) + 8*half + r%8 of a block
    const int k_row = (i32 & 16) | (i32 & 4) << 1 | (i32 & 8) >> 1 | (i32 & 3);

    auto compute = [&](const unsigned char *buf, int t0, bool whole) {
        const unsigned char *kp = buf + k_row * L::kPitchK + half * 16, *vp = buf + kManyTile * L::kPitchK + i32 * L::kPitchV + half * 16;
        f32x16_t s[2];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[n][r] = 0.f;
#pragma unroll
        for (int st = 0; st < DB; ++st)
#pragma unroll
            for (int n = 0; n < 2; ++n)
                s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const Frag *>(kp + n * 32 * L::kPitchK + st * 32), q[st], s[n], 0, 0, 0);
        float z[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) z[j] = s[j >> 4][j & 15];
        if (!__all(whole && (!col.there || (col.lo <= t0 && t0 + kManyTile <= col.hi)))) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const int pos = t0 + 32 * (j >> 4) + 16 * ((j >> 3) & 1) + 8 * half + (j & 7);
                const bool seen = (pos >= col.lo) & (pos < col.hi) & there(pg.of(j >> 3));
                z[j] = seen ? z[j] : -INFINITY;
            }
        }
        float top = z[0];
#pragma unroll
        for (int j = 1; j < 32; ++j) top = fmaxf(top, z[j]);
        top = fmaxf(top, __shfl_xor(top, 32)) * a.c;
        if (__any(top > mx + kLag)) {
            top = fmaxf(top, mx);
            const float shrink = __builtin_amdgcn_exp2f(mx - (top == -INFINITY ? 0.f : top));
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] *= shrink;
            mx = top;
        }
        const float base = mx == -INFINITY ? 0.f : mx;
        // two bfloat16 terms: what one alone leaves, up to 2^-9 of a probability, is more than the result's own rounding where values cancel (error
        // of chunks of 500 tokens against 64 bits 2.3e-3 with one term, 1.7e-3 with two, the result's rounding; 66 and 79 us)
        Frag p0[4], p1[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float e[8], part = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[8 * k + j], a.c, -base));
                part += e[j];
            }
            sum += part;
            u32x4_t hi, lo;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                hi[j] = pack_bf16x2(e[2 * j], e[2 * j + 1]);
                lo[j] = pack_bf16x2(e[2 * j] - __uint_as_float(hi[j] << 16), e[2 * j + 1] - __uint_as_float(hi[j] & 0xffff0000u));
            }
            p0[k] = __builtin_bit_cast(Frag, hi);
            p1[k] = __builtin_bit_cast(Frag, lo);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            Frag v[ND];
#pragma unroll
            for (int d = 0; d < ND; ++d) v[d] = *reinterpret_cast<const Frag *>(vp + d * 32 * L::kPitchV + k * 32);
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[d], p1[k], acc[d], 0, 0, 0);
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[d], p0[k], acc[d], 0, 0, 0);
        }
    };
    for (int t = t_begin, turn = 0; t < t_end; ++t, turn ^= 1) {
        unsigned char *buf = smem + turn * L::kBuffer;
        write(buf, t, pg);
        const bool more = t + 1 < t_end;
        if (more) next_pg = pages_of(t + 1);
        __syncthreads();  // (the other buffer is written next: all are through with it before they pass here again)
        if (more) load(t + 1, next_pg);
        const int t0 = t * kManyTile;
        if (t0 < wave_last && t0 + kManyTile > wave_first) compute(buf, t0, all_there(pg));
        pg = next_pg;
    }
    float total = sum;
    total += __shfl_xor(total, 32);
    if (!col.exists) return;
    const int head = kvh * a.G + col.g;
    const size_t rows = (size_t)a.B * a.H * a.U, row = ((size_t)b * a.H + head) * a.U + col.u;
    const bool some = col.there && total != 0.f;
    if (half == 0) {
        if (a.splits > 1) {
            float *ml = a.part_ml + ((size_t)split * rows + row) * 2;
            ml[0] = some ? mx : -INFINITY;
            ml[1] = some ? total : 0.f;
        } else if (a.lse) {
            a.lse[row] = some ? (mx + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
        }
    }
    const float inv = some ? (a.splits > 1 ? 1.f : 1.f / total) : 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int ch = 32 * d + 2 * r + 4 * half;
            if (D % 32 && ch >= D) continue;
            f32x4_t v = {acc[d][r], acc[d][r + 1], acc[d][r + 2], acc[d][r + 3]};
            if (!some) v = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (a.splits > 1) {
                *reinterpret_cast<f32x4_t *>(a.part + ((size_t)split * rows + row) * D + ch) = v;
            } else {
                bf16_t *o = (bf16_t *)a.out + (size_t)b * a.os + ((size_t)head * D + ch) * a.U + col.u;
#pragma unroll
                for (int j = 0; j < 4; ++j) store_from_f32(o, (size_t)j * a.U, v[j] * inv);
            }
        }
}

// ROWS rows of outputs from row0 on (there are fewer than 2^30), by EACH threads for a row: neighbouring lanes store neighbouring tokens.
template <typename S, int ROWS, int EACH>
__device__ __forceinline__ void store_rows(const Paged &a, const float (&tile)[ROWS][128 + 1], size_t row0)
{
    const uint32_t r = threadIdx.x % ROWS, to = (uint32_t)row0 + r, U = (uint32_t)a.U, bh = to / U, u = to - bh * U, b = bh / (uint32_t)a.H, h = bh - b * (uint32_t)a.H;
    if (to >= (uint32_t)a.B * (uint32_t)a.H * U) return;
    S *out = (S *)a.out + (size_t)b * a.os + (size_t)h * a.D * U + u;
    for (int d = threadIdx.x / ROWS; d < a.D; d += EACH) store_from_f32(out, (size_t)d * U, tile[r][d]);
}

// Joins the sums of `splits` workgroups in order: a wavefront takes a row (a token of a head), a lane one split's maximum and sum, and then
// eight channels of every fourth split.  (One thread for a row's maxima, split after split, took 17 us for 512 rows of 16 splits.)
template <typename S, int ROWS>
__global__ __launch_bounds__(ROWS * 64) void paged_join_kernel(Paged a)
{
    __shared__ float tile[ROWS][128 + 1];
    const size_t rows = (size_t)a.B * a.H * a.U, row0 = (size_t)blockIdx.x * ROWS;
    const int lane = threadIdx.x & 63, r = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slice = lane >> 4, d0 = (lane & 15) * 8;
    const size_t row = min(row0 + r, rows - 1);
    float2 ml = {-INFINITY, 0.f};
    if (lane < a.splits) ml = *reinterpret_cast<const float2 *>(a.part_ml + ((size_t)lane * rows + row) * 2);
    const float *part = a.part + row * a.D + min(d0, a.D - 8);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float top = ml.x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float w = __builtin_amdgcn_exp2f(ml.x - (top == -INFINITY ? 0.f : top));
    float total = w * ml.y;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    for (int s0 = 0; s0 < a.splits; s0 += 16) {  // (four splits' loads of a lane at a time)
        float p[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k) load8(part + (size_t)min(s0 + 4 * k + slice, a.splits - 1) * rows * a.D, 8, p[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int s = s0 + 4 * k + slice;
            const float ws = __shfl(w, min(s, 63));  // (0 from the last split on)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += s < a.splits ? ws * p[k][j] : 0.f;
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] += __shfl_xor(v[j], 16);
        v[j] += __shfl_xor(v[j], 32);
        v[j] *= inv;
    }
    if (a.lse && lane == 0 && row0 + r < rows) a.lse[row] = total != 0.f ? (top + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
    if (a.U == 1) {  // a head's channels side by side
        const size_t b = row / a.H, h = row - b * a.H;
        if (slice == 0 && d0 < a.D && row0 + r < rows) store8((S *)a.out + b * a.os + h * a.D + d0, 8, v);
        return;
    }
    if (slice == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[r][d0 + j] = v[j];
    }
    __syncthreads();
    store_rows<S, ROWS, 64>(a, tile, row0);
}

// The same for few splits and many tokens: a thread takes eight channels of a row, one split after the other.  (16000 rows of 4 splits: 9 us
// against 15, for 37 MB.)
constexpr int kFewSplits = 4, kJoinRows = 32;
template <typename S>
__global__ __launch_bounds__(kJoinRows * 16) void paged_join_few_kernel(Paged a)
{
    __shared__ float tile[kJoinRows][128 + 1];
    const size_t rows = (size_t)a.B * a.H * a.U, row0 = (size_t)blockIdx.x * kJoinRows;
    const int r = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * 8;
    const size_t row = min(row0 + r, rows - 1);
    float2 ml[kFewSplits];
    float p[kFewSplits][8];
    const float *part = a.part + row * a.D + min(d0, a.D - 8);
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {  // (those behind the last split read it again, and count for nothing)
        const int of = min(s, a.splits - 1);
        ml[s] = *reinterpret_cast<const float2 *>(a.part_ml + (of * rows + row) * 2);
        load8(part + of * rows * a.D, 8, p[s]);
    }
    float top = ml[0].x;
#pragma unroll
    for (int s = 1; s < kFewSplits; ++s) top = fmaxf(top, ml[s].x);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, total = 0.f;
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
        if (s >= a.splits) continue;
        const float w = __builtin_amdgcn_exp2f(ml[s].x - (top == -INFINITY ? 0.f : top));
        total += w * ml[s].y;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += w * p[s][j];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    if (a.lse && d0 == 0 && row0 + r < rows) a.lse[row] = total != 0.f ? (top + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[r][d0 + j] = v[j] * inv;
    __syncthreads();
    store_rows<S, kJoinRows, 16>(a, tile, row0);
}

struct Plan {
    bool many;
    int blocks, col_tiles, splits;  // blocks: of 16 columns of a workgroup with few of them
    size_t part_bytes, ml_bytes;
};
Plan plan_of(int B, int H, int Hkv, int D, int U, int page_size, int max_pages, int dtype)
{
    Plan p = {};
    const long long columns = (long long)(H / Hkv) * U, room = (long long)max_pages * page_size;
    p.many = dtype == NM_BF16 && columns > kFewColumns;
    p.blocks = columns > 16 ? 2 : 1;
    const int of_group = p.many ? kManyColumns : 16 * p.blocks, of_round = p.many ? kManyTile : kTile * kWaves;
    p.col_tiles = (int)((columns + of_group - 1) / of_group);
    // workgroups share a token's places where there are fewer than two a CU, of few columns one (two 47 us instead of 45 for 32 sequences of
    // 4000 to 8000 places; of many columns one a CU 100 + 7 us for chunks of 500 tokens behind 3000 to 6000 places, two 78 + 9, four 82 + 17; chunks of 200 of
    // two sequences 24 + 4, 24 + 7, 24 + 10), but look at two rounds of places at least.  The shares are those of the longest sequence that
    // there may be and of all U tokens: shorter sequences have shorter ones, and columns behind q_lengths workgroups without work.
    const long long groups = (long long)B * Hkv * p.col_tiles, rounds = (room + of_round - 1) / of_round, wanted = p.many ? 512 : 256;
    long long splits = wanted / groups;
    if (splits > rounds / 2) splits = rounds / 2;
    if (splits > kMaxSplits) splits = kMaxSplits;
    p.splits = splits < 1 ? 1 : (int)splits;
    const size_t rows = (size_t)B * H * U;
    p.part_bytes = p.splits > 1 ? align_up(p.splits * rows * D * 4, 256) : 0;
    p.ml_bytes = p.splits > 1 ? align_up(p.splits * rows * 2 * 4, 256) : 0;
    return p;
}

template <int DB>
hipError_t run_many(const Paged &a, hipStream_t s)
{
    static LdsOptIn opt;
    auto *fn = paged_many_kernel<DB>;
    const hipError_t e = ensure_dynamic_lds(opt, (const void *)fn, ManyLds<DB>::kBytes);
    if (e != hipSuccess) return e;
    fn<<<dim3((unsigned)(a.B * a.Hkv) * a.col_tiles * a.splits), dim3(256), ManyLds<DB>::kBytes, s>>>(a);
    return hipGetLastError();
}

template <typename S, int DB, int NC>
hipError_t run_few(const Paged &a, hipStream_t s)
{
    static LdsOptIn opt;
    constexpr int bytes = kWaves * NC * (32 + DB * 256) * 4;
    auto *fn = paged_few_kernel<S, DB, NC>;
    const hipError_t e = ensure_dynamic_lds(opt, (const void *)fn, bytes);
    if (e != hipSuccess) return e;
    fn<<<dim3((unsigned)(a.B * a.Hkv) * a.col_tiles * a.splits), dim3(kWaves * 64), bytes, s>>>(a);
    return hipGetLastError();
}
template <typename S, int DB>
hipError_t run_blocks(const Paged &a, const Plan &p, hipStream_t s)
{
    if constexpr (sizeof(S) == 2) {
        if (p.many) return run_many<DB>(a, s);
    }
    return p.blocks == 1 ? run_few<S, DB, 1>(a, s) : run_few<S, DB, 2>(a, s);
}
template <typename S>
hipError_t run(const Paged &a, const Plan &p, hipStream_t s)
{
    hipError_t e;
    switch (a.D / 16) {
    case 1: e = run_blocks<S, 1>(a, p, s); break;
    case 2: e = run_blocks<S, 2>(a, p, s); break;
    case 3: e = run_blocks<S, 3>(a, p, s); break;
    case 4: e = run_blocks<S, 4>(a, p, s); break;
    case 5: e = run_blocks<S, 5>(a, p, s); break;
    case 6: e = run_blocks<S, 6>(a, p, s); break;
    case 7: e = run_blocks<S, 7>(a, p, s); break;
    default: e = run_blocks<S, 8>(a, p, s); break;
    }
    if (e != hipSuccess || a.splits == 1) return e;
    const size_t rows = (size_t)a.B * a.H * a.U;
    if (a.splits <= kFewSplits && a.U >= kJoinRows) paged_join_few_kernel<S><<<dim3((unsigned)((rows + kJoinRows - 1) / kJoinRows)), dim3(kJoinRows * 16), 0, s>>>(a);
    else if (a.U >= 16) paged_join_kernel<S, 16><<<dim3((unsigned)((rows + 15) / 16)), dim3(1024), 0, s>>>(a);
    else paged_join_kernel<S, 4><<<dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

int check(int B, int H, int Hkv, int D, int U, int page_size, int max_pages, int dtype)
{
    if (B <= 0 || H <= 0 || Hkv <= 0 || D <= 0 || U <= 0 || page_size <= 0 || max_pages <= 0 || H % Hkv || !known_dtype(dtype)) return NM_ERR_BAD_ARG;
    const long long most = (1LL << 31) - 1;
    if (D % 16 || D > 128 || page_size < 16 || page_size > 256 || (page_size & (page_size - 1))) return NM_ERR_UNSUPPORTED;
    if ((long long)max_pages * page_size > most - 512 || (long long)B * max_pages > most) return NM_ERR_UNSUPPORTED;
    if ((long long)H * D > most / U || (long long)B * H > most / 2 / U) return NM_ERR_UNSUPPORTED;
    // the grid, of 256 work items for 16 columns or more and a split: below 2^32 (from 2^10 workgroups on nothing is split)
    if ((long long)B * Hkv >= 1LL << 23 || (long long)B * Hkv * (((long long)H / Hkv * U + 15) / 16) >= 1LL << 23) return NM_ERR_UNSUPPORTED;
    return NM_OK;
}

}  // namespace
}  // namespace nm

using namespace nm;

extern "C" {

size_t nm_paged_attn_workspace_bytes(int B, int heads, int kv_heads, int D, int U, int page_size, int max_pages, int dtype)
{
    if (check(B, heads, kv_heads, D, U, page_size, max_pages, dtype) != NM_OK) return 0;
    const Plan p = plan_of(B, heads, kv_heads, D, U, page_size, max_pages, dtype);
    return p.part_bytes + p.ml_bytes;
}

int nm_paged_attn_fwd(int B, int heads, int kv_heads, int D, int U, const void *q, long long q_stride, const void *k_cache,
                      const void *v_cache, int pages, int page_size, const int *page_table, int max_pages, const int *lengths,
                      const int *q_lengths, int window, float scale, void *o, long long o_stride, float *lse, int dtype, void *workspace,
                      size_t workspace_bytes, void *hip_stream)
{
    const int st = check(B, heads, kv_heads, D, U, page_size, max_pages, dtype);
    if (st != NM_OK) return st;
    const long long item = (long long)heads * D * U;
    if (!q || !k_cache || !v_cache || !page_table || !lengths || !o || pages <= 0 || window < 0 || !finite_float(scale) || !stride_ok(q_stride, item) ||
        !stride_ok(o_stride, item) || (uintptr_t)k_cache % 16 || (uintptr_t)v_cache % 16)
        return NM_ERR_BAD_ARG;
    const int size = (int)element(dtype);
    if ((long long)pages * kv_heads > (1LL << 40) / (page_size * D)) return NM_ERR_UNSUPPORTED;
    const size_t cache = (size_t)pages * kv_heads * page_size * D * size;
    const Items to = {o, o_stride, item, B, size}, from = {q, q_stride, item, B, size};
    const Region l = {lse, (size_t)B * heads * U * 4};
    const Region in[5] = {{k_cache, cache}, {v_cache, cache}, {page_table, (size_t)B * max_pages * 4}, {lengths, (size_t)B * 4}, {q_lengths, (size_t)B * 4}};
    if (meet(to, from) || meets(to.region(), in) || meets(l, in) || meet(l, from.region()) || meet(l, to.region())) return NM_ERR_BAD_ARG;
    const Plan p = plan_of(B, heads, kv_heads, D, U, page_size, max_pages, dtype);
    if (workspace_missing(workspace, workspace_bytes, p.part_bytes + p.ml_bytes)) return NM_ERR_WORKSPACE;
    Paged a = {};
    a.B = B; a.H = heads; a.Hkv = kv_heads; a.G = heads / kv_heads; a.D = D; a.U = U;
    a.q = q; a.k = k_cache; a.v = v_cache; a.qs = q_stride; a.os = o_stride;
    a.pages = pages; a.max_pages = max_pages;
    while (1 << a.log_page < page_size) ++a.log_page;
    a.table = page_table; a.len = lengths; a.q_len = q_lengths;
    a.window = window;
    const float c = (scale < 0.f ? -scale : scale) * 1.4426950408889634f;
    a.c = c < 1e-37f ? 1e-37f : c;  // (not zero: masked scores are -infinity times this)
    a.flip = scale < 0.f ? 0x80000000u : 0u;
    a.out = o; a.lse = lse;
    a.part = (float *)workspace;
    a.part_ml = (float *)((char *)workspace + p.part_bytes);
    a.col_tiles = p.col_tiles; a.splits = p.splits;
    hipStream_t s = (hipStream_t)hip_stream;
    return status_of(dtype == NM_BF16 ? run<bf16_t>(a, p, s) : run<float>(a, p, s));
}

}  // extern "C"
