// What the kernels of cross attention share: tiles of channel-major tensors in LDS and the matrix-core operands cut from them.
//
// Everything here multiplies blocks of 32 x 32.  A tile holds DP channels (D rounded up to a multiple of 32, zeros behind) of
// 32 * NB neighbouring positions as they lie in memory: blocks [DP rows][32 positions].  Two kinds of operand are read from it:
//   across  rows of the product = positions, reduction = channels (scores and their gradients): a lane needs consecutive
//           channels of one position, a column of the block, which the transposing LDS read delivers in bfloat16; in float a
//           lane needs one value;
//   along   rows of the product = channels, reduction = positions (the products with probabilities): a lane needs consecutive
//           positions of one channel, 16 bytes of a row.
// The second product's other operand is the result of the first one, which stays in the registers it was made in: a lane then
// holds, for its column, rows 8*(r/4) + 4*(lane/32) + r%4 (r = 0..15).  In bfloat16 the next product wants eight consecutive rows
// per lane, so the positions are dealt to the rows of the first product such that register r holds position
// 16*(r/8) + 8*(lane/32) + r%8 instead; the transposing read does that by the order of its addresses alone.  In float a register
// is an operand as it is.
// 16-byte granules of a row are stored in an order that depends on the row, so that both kinds of reads touch every bank once.
#pragma once

#include "nm_common.h"

namespace nm {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename S>
struct Mma;

template <>
struct Mma<bf16_t> {
    static constexpr int kRow = 64;       // bytes of a block's row
    static constexpr int kPerGranule = 8; // elements of 16 bytes
    static constexpr int kSteps = 16;     // channels of a step of the first product
    typedef bf16x8_t Frag;                // operand of one step
    struct Probs {                        // operand of the second product: a block's 32 positions
        bf16x8_t s[2];
    };
    static __device__ __forceinline__ int granule(int row, int g) { return row * kRow + ((g ^ ((row >> 2) & 3)) << 4); }
    // position of register r in the block
    static __device__ __forceinline__ int position(int r, int half) { return 16 * (r >> 3) + 8 * half + (r & 7); }

    // byte offset of the lane's `across` operand of step 0; step k is 1024 bytes further.  order: of the positions, as above
    template <bool ORDER>
    static __device__ __forceinline__ void across_offsets(int lane, int (&off)[2])
    {
        const int half = lane >> 5, i = lane & 15, g16 = (lane >> 4) & 1, j = i & 3;
        const int group = ORDER ? ((j & 1) << 1 | j >> 1) : j;  // of four positions
        const int row = 8 * half + (i >> 2), g = 2 * g16 + (group >> 1);
        off[0] = granule(row, g) + (group & 1) * 8;
        off[1] = granule(row + 4, g) + (group & 1) * 8;
    }
    static __device__ __forceinline__ Frag across(const unsigned char *block, const int (&off)[2], int step)
    {
        union {
            s16x4_t h[2];
            bf16x8_t v;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(block + off[0] + step * 1024));
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(block + off[1] + step * 1024));
        return u.v;
    }
    // the same operand of 32 columns straight from memory: channels d0.. of the lane's column, `pitch` elements apart
    static __device__ __forceinline__ Frag column(const bf16_t *p, int step, int half, int D, size_t pitch, bool there, uint32_t flip)
    {
        union {
            bf16_t e[8];
            bf16x8_t v;
        } u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int d = 16 * step + 8 * half + j;
            u.e[j] = there && d < D ? (bf16_t)(p[(size_t)d * pitch] ^ (flip >> 16)) : (bf16_t)0;
        }
        return u.v;
    }
    static __device__ __forceinline__ f32x16_t mul(Frag a, Frag b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

    static __device__ __forceinline__ Probs probs(const f32x16_t &p)  // rounds to bfloat16
    {
        Probs out;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const u32x4_t w = {pack_bf16x2(p[8 * s], p[8 * s + 1]), pack_bf16x2(p[8 * s + 2], p[8 * s + 3]),
                               pack_bf16x2(p[8 * s + 4], p[8 * s + 5]), pack_bf16x2(p[8 * s + 6], p[8 * s + 7])};
            out.s[s] = __builtin_bit_cast(bf16x8_t, w);
        }
        return out;
    }
    // the `along` operand of 32 channels from row d0 on, and its product with up to NC columns' probabilities
    struct Along {
        bf16x8_t s[2];
    };
    static __device__ __forceinline__ Along along(const unsigned char *block, int d0, int lane)
    {
        Along a;
        const int row = d0 + (lane & 31), half = lane >> 5;
        a.s[0] = *reinterpret_cast<const bf16x8_t *>(block + granule(row, half));
        a.s[1] = *reinterpret_cast<const bf16x8_t *>(block + granule(row, 2 + half));
        return a;
    }
    static __device__ __forceinline__ f32x16_t mul(const Along &a, const Probs &p, f32x16_t c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.s[0], p.s[0], c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.s[1], p.s[1], c, 0, 0, 0);
    }
    static __device__ __forceinline__ u32x4_t first(u32x4_t v, int n) { return first_of8(v, n); }
    static __device__ __forceinline__ u32x4_t down(u32x4_t v, int t, int len) { return shift8_down(v, t, len); }
};

template <>
struct Mma<float> {
    static constexpr int kRow = 128;
    static constexpr int kPerGranule = 4;
    static constexpr int kSteps = 2;
    typedef float Frag;
    typedef f32x16_t Probs;
    static __device__ __forceinline__ int granule(int row, int g) { return row * kRow + ((g ^ ((row >> 1) & 7)) << 4); }
    static __device__ __forceinline__ int position(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

    template <bool ORDER>
    static __device__ __forceinline__ void across_offsets(int lane, int (&off)[2])
    {
        const int n = lane & 31;
        off[0] = (lane >> 5) * kRow + (n & 3) * 4;
        off[1] = (n >> 2) << 4;
    }
    static __device__ __forceinline__ Frag across(const unsigned char *block, const int (&off)[2], int step)
    {
        return *reinterpret_cast<const float *>(block + off[0] + (off[1] ^ ((step & 7) << 4)) + step * 2 * kRow);
    }
    static __device__ __forceinline__ Frag column(const float *p, int step, int half, int D, size_t pitch, bool there, uint32_t flip)
    {
        const int d = 2 * step + half;
        return there && d < D ? __uint_as_float(__float_as_uint(p[(size_t)d * pitch]) ^ flip) : 0.f;
    }
    static __device__ __forceinline__ f32x16_t mul(Frag a, Frag b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ Probs probs(const f32x16_t &p) { return p; }
    struct Along {
        f32x4_t s[4];
    };
    static __device__ __forceinline__ Along along(const unsigned char *block, int d0, int lane)
    {
        Along a;
        const int row = d0 + (lane & 31), half = lane >> 5;
#pragma unroll
        for (int s = 0; s < 4; ++s) a.s[s] = *reinterpret_cast<const f32x4_t *>(block + granule(row, 2 * s + half));
        return a;
    }
    static __device__ __forceinline__ f32x16_t mul(const Along &a, const Probs &p, f32x16_t c)
    {
#pragma unroll
        for (int r = 0; r < 16; ++r) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.s[r >> 2][r & 3], p[r], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ u32x4_t first(u32x4_t v, int n)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < n ? v[j] : 0u;
        return v;
    }
    // of a row of at least four elements: the group at step t was read from its last four where it runs over the end
    static __device__ __forceinline__ u32x4_t down(u32x4_t v, int t, int len)
    {
        const int s = t + 4 - len;
        if (s <= 0) return v;
        if (s & 1) v = u32x4_t{v[1], v[2], v[3], 0u};
        if (s & 2) v = u32x4_t{v[2], v[3], 0u, 0u};
        return s < 4 ? v : u32x4_t{0u, 0u, 0u, 0u};
    }
};

// A tile of NB blocks, loaded by NT threads: `count` granules each, held in registers between the load and the write.
template <typename S, int DP, int NB, int NT>
struct Tile {
    typedef Mma<S> M;
    static constexpr int kBlock = DP * M::kRow + (NB > 1 ? 128 : 0);  // (blocks side by side begin at other banks)
    static constexpr int kBytes = NB * kBlock;
    static constexpr int kPerRow = NB * M::kRow / 16;  // granules
    static constexpr int kCount = DP * kPerRow / NT;
    static_assert(DP * kPerRow % NT == 0, "whole granules per thread");
    u32x4_t r[kCount];

    // rows: channel 0 at step 0 of the sequence, `len` elements a row, D rows; t0: the tile's first position
    __device__ __forceinline__ void load(const S *rows, int D, int len, int t0, int thread)
    {
        constexpr int G = M::kPerGranule;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int e = i * NT + thread, row = min(e / kPerRow, D - 1), t = t0 + (e % kPerRow) * G;
            if (len >= G) {  // (uniform)
                __builtin_memcpy(&r[i], rows + (size_t)row * len + min(t, len - G), 16);
            } else {
                S v[G];
#pragma unroll
                for (int j = 0; j < G; ++j) v[j] = t + j < len ? rows[(size_t)row * len + t + j] : S(0);
                __builtin_memcpy(&r[i], v, 16);
            }
        }
    }
    // zeros for rows from D on and positions from `valid` (<= len) on
    __device__ __forceinline__ void write(unsigned char *tile, int D, int len, int valid, int t0, int thread)
    {
        constexpr int G = M::kPerGranule;
        const bool ends = t0 + NB * 32 > valid;  // (uniform)
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int e = i * NT + thread, row = e / kPerRow, gi = e % kPerRow, t = t0 + gi * G;
            u32x4_t v = r[i];
            if (ends) {
                if (len >= G) v = M::down(v, t, len);
                v = M::first(v, valid - t);
            }
            if (row >= D) v = u32x4_t{0u, 0u, 0u, 0u};
            constexpr int GB = M::kRow / 16;
            *reinterpret_cast<u32x4_t *>(tile + (gi / GB) * kBlock + M::granule(row, gi % GB)) = v;
        }
    }
};

// A wavefront's result, 32 * (DP / 32) channels x 32 positions with the positions as columns, to rows of `len` elements in memory:
// through LDS (`block`, DP rows, the wavefront's own), so that a lane stores 16 bytes of a row and four or eight lanes a whole
// block's row.  Straight from the registers a store covers two bytes of a lane, and the address unit is what the kernel waits for.
template <typename S, int DP>
__device__ __forceinline__ void store_block(unsigned char *block, const f32x16_t (&acc)[DP / 32], float scale, S *rows, int D, int len, int t0, int valid,
                                            int lane)
{
    typedef Mma<S> M;
    constexpr int G = M::kPerGranule, GB = M::kRow / 16;
    const int t = lane & 31, half = lane >> 5;
    const bool there = t0 + t < valid;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int ch = d * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
            store_from_f32(reinterpret_cast<S *>(block + M::granule(ch, t / G)), t % G, there ? acc[d][r] * scale : 0.f);
        }
    wave_fence();
#pragma unroll
    for (int i = 0; i < DP * GB / 64; ++i) {
        const int row = i * (64 / GB) + lane / GB, g = lane % GB, n = len - (t0 + g * G);
        if (row >= D || n <= 0) continue;
        const u32x4_t v = *reinterpret_cast<const u32x4_t *>(block + M::granule(row, g));
        S *p = rows + (size_t)row * len + t0 + g * G;
        if (n >= G) {
            __builtin_memcpy(p, &v, 16);
        } else {
            S e[G];
            __builtin_memcpy(e, &v, 16);
#pragma unroll
            for (int j = 0; j < G - 1; ++j)
                if (j < n) p[j] = e[j];
        }
    }
}

__device__ __forceinline__ int clipped(int v, int hi) { return v < 0 ? 0 : (v > hi ? hi : v); }

// Arguments of the kernels, forward and backward.
struct AttnArgs {
    int B, H, Hkv, G, D, U, T;
    const void *q, *k, *v, *o, *dout;
    long long qs, ks, vs, os, dos;
    const int *len, *q_len, *windows;
    float c;        // |scale| * log2(e): scores in units of powers of two
    float scale;
    uint32_t flip;  // sign bit of scale: one operand of the scores changes its sign instead
    void *out, *dq, *dk, *dv;
    long long dqs, dks, dvs;
    float *lse;
    float *part, *part_ml;  // sums of the workgroups that share tokens, their maxima and sums
    float *delta;           // [B][H][U]
    int col_tiles, splits, tiles_per_split;
};

// The frames a token may look at, [lo, hi).
__device__ __forceinline__ void frames_of(const AttnArgs &a, int b, int u, int len, int &lo, int &hi)
{
    lo = 0;
    hi = len;
    if (a.windows) {
        const int *w = a.windows + ((size_t)b * a.U + u) * 2;
        lo = max(lo, w[0]);
        hi = min(hi, w[1]);
    }
}
__device__ __forceinline__ float half_max(float v) { return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float half_sum(float v) { return v + __shfl_xor(v, 32); }

}  // namespace nm
