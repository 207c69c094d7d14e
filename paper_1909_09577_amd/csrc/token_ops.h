// What the operators on a decoder's tokens share (embedding, heads' norms and rotation, paged attention, token scores).
#pragma once

#include "../../include/nm_conv1d.h"
#include "nm_common.h"

namespace nm {

// Eight consecutive elements of a tensor as floats: the first n of them at p, zeros behind (p needs its element's alignment only).
__device__ __forceinline__ void load8(const bf16_t *p, int n, float (&v)[8])
{
    const u32x4_t r = load8_any(p, n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(r[j] << 16);
        v[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, int n, float (&v)[8])
{
    if (n >= 8) {
        __builtin_memcpy(v, p, 32);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : 0.f;
    }
}
__device__ __forceinline__ void store8(bf16_t *p, int n, const float (&v)[8])
{
    store8_any(p, u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])}, n);
}
__device__ __forceinline__ void store8(float *p, int n, const float (&v)[8])
{
    if (n >= 8) {
        __builtin_memcpy(p, v, 32);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = v[j];
    }
}

// Token numbers of four or eight bytes; -1 for what is no class.
struct Ids {
    const void *p;
    int wide;
    __device__ __forceinline__ int at(size_t i, int V) const
    {
        if (wide) {
            const long long v = reinterpret_cast<const long long *>(p)[i];
            return v < 0 || v >= V ? -1 : (int)v;
        }
        const int v = reinterpret_cast<const int *>(p)[i];
        return v < 0 || v >= V ? -1 : v;
    }
};

__device__ __forceinline__ int length_in(const int *len, int b, int n)
{
    if (!len) return n;
    const int v = len[b];
    return v < 0 ? 0 : (v > n ? n : v);
}

// Sums over lanes by the vector unit alone (an exchange through LDS takes the LDS unit of all wavefronts of a CU as long as a dozen
// additions take a SIMD).
template <int N>
__device__ __forceinline__ float turned_in_row(float v)  // lane i of 16 gets lane i - N
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum_of_rows(float v)  // over the four rows of 16 lanes
{
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float pair = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const uint32_t p = __float_as_uint(pair);
    const auto b = __builtin_amdgcn_permlane32_swap(p, p, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
template <int N>
__device__ __forceinline__ float sum_of_every(float v)  // over the lanes whose number is this lane's modulo N (2 or 4)
{
    if constexpr (N == 2) v += turned_in_row<2>(v);
    if constexpr (N <= 4) v += turned_in_row<4>(v);
    v += turned_in_row<8>(v);
    return sum_of_rows(v);
}

// ---- host ----------------------------------------------------------------------------------------------------------
inline bool known_dtype(int dtype) { return dtype == NM_BF16 || dtype == NM_F32; }
inline size_t element(int dtype) { return dtype == NM_BF16 ? 2 : 4; }
inline int status_of(hipError_t e) { return e == hipSuccess ? NM_OK : NM_ERR_DEVICE; }
// A launch has fewer than 2^32 work items: more workgroups go in several launches, whose first one's number the kernel gets.  (A grid with a second
// side takes its 3200 short workgroups 9.1 us in the embedding gradient's join instead of 8.5.)
template <typename F>
hipError_t in_launches(size_t workgroups, F launch)
{
    constexpr size_t most = (size_t)1 << 22;
    for (size_t first = 0; first < workgroups; first += most) {
        launch((unsigned)(workgroups - first < most ? workgroups - first : most), (int)first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
inline bool finite_float(float v) { return v - v == 0.f; }

struct Region {
    const void *p;
    size_t bytes;
};
inline bool meet(const Region &a, const Region &b)
{
    if (!a.p || !b.p) return false;
    const char *pa = (const char *)a.p, *pb = (const char *)b.p;
    return pa < pb + b.bytes && pb < pa + a.bytes;
}
// Whether a region meets one of the others
template <int N>
bool meets(const Region &a, const Region (&others)[N])
{
    for (const Region &o : others)
        if (meet(a, o)) return true;
    return false;
}
// A tensor of B items of `item` elements each, `stride` elements apart
struct Items {
    const void *p;
    long long stride, item;
    int B, size;
    Region region() const { return {p, (size_t)((B - 1) * stride + item) * size}; }
};
// Items that lie between another tensor's (the parts of one projection's output) overlap as regions but not as tensors.
inline bool meet(const Items &a, const Items &b)
{
    if (!meet(a.region(), b.region())) return false;
    if (a.B == 1 || a.stride != b.stride || a.size != b.size) return true;
    const long long stride = a.stride * a.size;
    long long d = ((const char *)b.p - (const char *)a.p) % stride;  // of b's items behind a's
    if (d < 0) d += stride;
    return d < a.item * a.size || d + b.item * b.size > stride;
}
inline bool stride_ok(long long stride, long long item) { return stride >= item && stride < 1LL << 40; }
inline bool workspace_missing(const void *ws, size_t have, size_t need) { return need && (!ws || have < need || (uintptr_t)ws % 256); }

}  // namespace nm
