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
    // the same operand of 32 columns straight from memory: channels of the lane's column p, `pitch` elements apart (a head's
    // rows span less than 4 GiB); zeros unless `there`.  Every load is made, from a channel that exists: a branch around each is what
    // the call would wait for.
    static __device__ __forceinline__ Frag column(const bf16_t *p, int step, int half, int D, uint32_t pitch, bool there)
    {
        bf16_t e[8];
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = *reinterpret_cast<const bf16_t *>(reinterpret_cast<const char *>(p) + (size_t)((uint32_t)min(16 * step + 8 * half + j, D - 1) * pitch * 2u));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = 16 * step + 8 * half + 2 * j;
            w[j] = (uint32_t)e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
            w[j] &= !there || d >= D ? 0u : (d + 1 < D ? 0xffffffffu : 0xffffu);
        }
        return __builtin_bit_cast(bf16x8_t, u32x4_t{w[0], w[1], w[2], w[3]});
    }
    static __device__ __forceinline__ f32x16_t mul(Frag a, Frag b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ Frag flipped(Frag a, uint32_t flip)
    {
        const uint32_t both = flip | flip >> 16;
        u32x4_t w = __builtin_bit_cast(u32x4_t, a);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] ^= both;
        return __builtin_bit_cast(bf16x8_t, w);
    }
    static __device__ __forceinline__ float dot(Frag a, Frag b)
    {
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) t += (float)a[j] * (float)b[j];
        return t;
    }

    // Rounds to bfloat16, which is what the matrix instruction takes.  Outputs are then off from 64 bits by 0.0018 to 0.0024 of their rms, against
    // 0.0017 of the rounding of the stored result alone; two terms of p would be half as many matrix instructions again in the forward pass.
    static __device__ __forceinline__ Probs probs(const f32x16_t &p)
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
    // Twice as many bits: what the rounding leaves is a second operand.  ds takes this form: it is made with the delta of rounded outputs,
    // and the two errors together would be a third more than those that the stored outputs have anyway.
    // Products of channels with the block's values, eight of a lane's at a time, so that few operands are in registers at once.
    template <int ND>
    static __device__ __forceinline__ void add_in_two_terms(f32x16_t (&acc)[ND], const unsigned char *block, int lane, const f32x16_t &p)
    {
        const int row = lane & 31, half = lane >> 5;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            u32x4_t hi, lo;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = p[8 * s + 2 * j], b = p[8 * s + 2 * j + 1];
                hi[j] = pack_bf16x2(a, b);
                lo[j] = pack_bf16x2(a - __uint_as_float(hi[j] << 16), b - __uint_as_float(hi[j] & 0xffff0000u));
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const bf16x8_t rows = *reinterpret_cast<const bf16x8_t *>(block + granule(32 * d + row, 2 * s + half));
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows, __builtin_bit_cast(bf16x8_t, lo), acc[d], 0, 0, 0);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows, __builtin_bit_cast(bf16x8_t, hi), acc[d], 0, 0, 0);
            }
        }
    }
    // the `along` operand of 32 channels from row d0 on, and its product with a block's probabilities
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
    static __device__ __forceinline__ Frag column(const float *p, int step, int half, int D, uint32_t pitch, bool there)
    {
        const int d = 2 * step + half;
        const float v = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p) + (size_t)((uint32_t)min(d, D - 1) * pitch * 4u));
        return there && d < D ? v : 0.f;
    }
    static __device__ __forceinline__ f32x16_t mul(Frag a, Frag b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ Frag flipped(Frag a, uint32_t flip) { return __uint_as_float(__float_as_uint(a) ^ flip); }
    static __device__ __forceinline__ float dot(Frag a, Frag b) { return a * b; }
    static __device__ __forceinline__ Probs probs(const f32x16_t &p) { return p; }
    template <int ND>
    static __device__ __forceinline__ void add_in_two_terms(f32x16_t (&acc)[ND], const unsigned char *block, int lane, const f32x16_t &p)
    {
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] = mul(along(block, d * 32, lane), p, acc[d]);
    }
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

// A tile of NB blocks, loaded by NT threads: kCount granules each, held in registers between the load and the write.
template <typename S, int DP, int NB, int NT>
struct Tile {
    typedef Mma<S> M;
    static constexpr int kBlock = DP * M::kRow + (NB > 1 ? 128 : 0);  // (blocks side by side begin at other banks)
    static constexpr int kBytes = NB * kBlock;
    static constexpr int kPerRow = NB * M::kRow / 16;  // granules
    static constexpr int kAll = DP * kPerRow, kCount = (kAll + NT - 1) / NT;  // (beyond the last granule a thread loads a row that is there)

    // A thread's places in the tiles of a sequence: byte offsets from channel 0 of a tile's first position, in 32 bits beside a base
    // that all threads share (a head's rows span less than 4 GiB).  Sequences of equal shape have the same.
    struct Places {
        uint32_t off[kCount];
        __device__ __forceinline__ void set(int D, int len, int thread)
        {
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                const int e = i * NT + thread, row = min(e / kPerRow, D - 1);
                off[i] = ((uint32_t)row * (uint32_t)len + (uint32_t)(e % kPerRow) * M::kPerGranule) * (uint32_t)sizeof(S);
            }
        }
    };
    u32x4_t r[kCount];

    // rows: channel 0 at step 0 of the sequence, `len` elements a row; t0: the tile's first position (below len)
    __device__ __forceinline__ void load(const S *rows, const Places &at, int len, int t0, int thread)
    {
        constexpr int G = M::kPerGranule;
        const char *base = reinterpret_cast<const char *>(rows + t0);
        if (t0 + NB * 32 <= len) {  // (uniform)
#pragma unroll
            for (int i = 0; i < kCount; ++i) __builtin_memcpy(&r[i], base + at.off[i], 16);
        } else if (len >= G) {  // groups that reach over the end are read from the row's last whole one
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                const int t = t0 + (i * NT + thread) % kPerRow * G;
                __builtin_memcpy(&r[i], reinterpret_cast<const char *>(rows) + (at.off[i] + (uint32_t)(t0 + min(len - G - t, 0)) * (uint32_t)sizeof(S)), 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                const int t = (i * NT + thread) % kPerRow * G;  // (t0 is 0)
                S v[G];
#pragma unroll
                for (int j = 0; j < G; ++j) v[j] = t + j < len ? *reinterpret_cast<const S *>(base + at.off[i] + j * sizeof(S)) : S(0);
                __builtin_memcpy(&r[i], v, 16);
            }
        }
    }
    // zeros for rows from D on and positions from `valid` (<= len) on
    __device__ __forceinline__ void write(unsigned char *tile, int D, int len, int valid, int t0, int thread)
    {
        constexpr int G = M::kPerGranule, GB = M::kRow / 16;
        if (t0 + NB * 32 > valid) {  // (uniform)
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                const int t = t0 + (i * NT + thread) % kPerRow * G;
                if (len >= G) r[i] = M::down(r[i], t, len);
                r[i] = M::first(r[i], valid - t);
            }
        }
        if (D < DP) {  // (uniform)
#pragma unroll
            for (int i = 0; i < kCount; ++i)
                if ((i * NT + thread) / kPerRow >= D) r[i] = u32x4_t{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int e = i * NT + thread, row = e / kPerRow, gi = e % kPerRow;
            if (kAll % NT == 0 || e < kAll) *reinterpret_cast<u32x4_t *>(tile + (gi / GB) * kBlock + M::granule(row, gi % GB)) = r[i];
        }
    }
};

// A wavefront's result, 32 * (DP / 32) channels x 32 positions with the positions as columns, to rows of `len` elements in memory:
// through LDS (`block`, DP rows, the wavefront's own), so that a lane stores 16 bytes of a row and four or eight lanes a whole
// block's row.  `scale` may differ from lane to lane (a lane is a position).  Straight from the registers a store covers two bytes of a lane, and the address unit is what the kernel waits for.
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
        for (int r = 0; r < 16; r += 2) {
            const int ch = d * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
            const float v0 = there ? acc[d][r] * scale : 0.f, v1 = there ? acc[d][r + 1] * scale : 0.f;
            S *p0 = reinterpret_cast<S *>(block + M::granule(ch, t / G)) + t % G, *p1 = reinterpret_cast<S *>(block + M::granule(ch + 1, t / G)) + t % G;
            if constexpr (sizeof(S) == 2) {
                const uint32_t w = pack_bf16x2(v0, v1);
                *p0 = (S)(w & 0xffffu);
                *p1 = (S)(w >> 16);
            } else {
                *p0 = v0;
                *p1 = v1;
            }
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
    int col_tiles, splits;
    int head_tiles;  // column tiles of a head, or 0: tiles run over the heads that share keys and values
    int head_waves_log;  // log2 of the heads whose tokens a workgroup's wavefronts take side by side
    float *kv_part;  // [parts][2][B][Hkv][D][T]: sums of the workgroups that share positions
    int pos_tiles, parts, units_per_part;
    int dq_first;  // the workgroups of dq come before those of dk and dv
};

// A workgroup's NW blocks of a head's tokens or positions as operands of its wavefronts, through LDS (`smem`).  All that a kernel wants
// is loaded before the first is taken: taking waits.
template <typename S, int DP, int NW>
struct OwnColumns {
    typedef Tile<S, DP, NW, NW * 64> Own;
    typedef Mma<S> M;
    Own own;
    __device__ __forceinline__ void load(const S *rows, int D, int len, int t0)
    {
        typename Own::Places at;
        at.set(D, len, threadIdx.x);
        own.load(rows, at, len, t0, threadIdx.x);
    }
    template <int KS>
    __device__ __forceinline__ void take(unsigned char *smem, int D, int len, int valid, int t0, int wave, int lane, typename M::Frag (&f)[KS])
    {
        int off[2];
        M::template across_offsets<false>(lane, off);
        own.write(smem, D, len, valid, t0, threadIdx.x);
        __syncthreads();
#pragma unroll
        for (int s = 0; s < KS; ++s) f[s] = M::across(smem + wave * Own::kBlock, off, s);
        __syncthreads();
    }
    // the same, and the operands of a second tensor's blocks, which were written behind these
    template <int KS>
    __device__ __forceinline__ void take(unsigned char *smem, int D, int len, int valid, int t0, int wave, int lane, typename M::Frag (&f)[KS],
                                         typename M::Frag (&second)[KS])
    {
        int off[2];
        M::template across_offsets<false>(lane, off);
        own.write(smem, D, len, valid, t0, threadIdx.x);
        __syncthreads();
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            f[s] = M::across(smem + wave * Own::kBlock, off, s);
            second[s] = M::across(smem + Own::kBytes + wave * Own::kBlock, off, s);
        }
        __syncthreads();
    }
};

// The same for a wavefront with a block of its own, through LDS of its own.  (Rows of a group at least: shorter ones have no tiles
// of several heads.)
template <typename S, int DP>
struct WaveColumns {
    typedef Tile<S, DP, 1, 64> Own;
    typedef Mma<S> M;
    Own own;
    __device__ __forceinline__ void load(const S *rows, int D, int len, int t0, int lane)
    {
        typename Own::Places at;
        at.set(D, len, lane);
        own.load(rows, at, len, t0, lane);
    }
    template <int KS>
    __device__ __forceinline__ void take(unsigned char *block, int D, int len, int valid, int t0, int lane, typename M::Frag (&f)[KS])
    {
        int off[2];
        M::template across_offsets<false>(lane, off);
        wave_fence();
        own.write(block, D, len, valid, t0, lane);
        wave_fence();
#pragma unroll
        for (int s = 0; s < KS; ++s) f[s] = M::across(block, off, s);
        wave_fence();
    }
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
