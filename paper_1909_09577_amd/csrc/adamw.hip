// AdamW over the tensors of a plan in one launch (definition: include/nm_adamw.h).
//
// Bound by memory: 30 bytes an element with float states (parameter, both moments in and out, gradient in, bfloat16 copy
// out), 18 with 8-bit states, whose 64-bit arithmetic takes about as long: roots and reciprocals come from the float instructions
// and steps of Newton's iteration (library roots and divisions: 1530 us instead of 1190 to 1205 over 322 million weights; with
// float states 1590 to 1845 us, 5.2 to 6.1 TB/s).  A wavefront owns a block of 256 elements, four neighbours per lane, so that every access is
// 16 bytes (float), 8 (copy) or 4 (codes) per lane and contiguous over the wavefront, and so that the maximum of a block of
// 8-bit states needs no LDS.  A workgroup takes kChunkBlocks blocks of one tensor; the plan names the tensor of every chunk.
#include "../../include/nm_adamw.h"
#include "../../include/nm_conv1d.h"
#include "nm_common.h"

#include <math.h>
#include <string.h>

namespace nm {
namespace {

constexpr int kBlock = 256;       // elements of a block
constexpr int kChunkBlocks = 16;  // blocks of a workgroup: four per wavefront
constexpr uint32_t kMagic = 0x4e4d4157u;

struct PlanHeader {  // the first 64 bytes of a plan; the records and then the chunks' tensors (int32) follow
    uint32_t magic;
    int state_bits, count, chunks;
    unsigned long long bytes;
    unsigned char zeros[40];
};
struct Record {
    float *param;
    const float *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    bf16_t *copy;
    uint32_t n;
    float weight_decay;
    uint32_t first_block;  // of the plan
    int first_chunk;
    int aligned;  // 16-byte groups of every tensor can be read and written as such
    int zero;
};
static_assert(sizeof(PlanHeader) == 64 && sizeof(Record) == 80, "the plan's layout");

struct StepArgs {
    float lr, step_size, beta1, one_minus_beta1, beta2, one_minus_beta2, root_correction, eps;
    double beta1_d, beta2_d, one_minus_beta1_d, one_minus_beta2_d;
    const float *grad_scale;
    uint32_t seed;
};

// Four neighbouring elements, the first n of them there.
template <typename V, typename T>
__device__ __forceinline__ void load4(const T *p, int n, bool whole, T (&out)[4])
{
    if (whole) {
        const V v = *reinterpret_cast<const V *>(p);
        __builtin_memcpy(out, &v, sizeof(V));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = j < n ? p[j] : T(0);
    }
}
template <typename V, typename T>
__device__ __forceinline__ void store4(T *p, int n, bool whole, const T (&in)[4])
{
    if (whole) {
        V v;
        __builtin_memcpy(&v, in, sizeof(V));
        *reinterpret_cast<V *>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = in[j];
    }
}

// A pointer that was read from the plan: to global memory (taken for a generic one, every access would go by the path that also serves LDS).
template <typename T>
__device__ __forceinline__ T *global(T *p)
{
    return (T *)(__attribute__((address_space(1))) T *)p;
}

// times_element: the element's number * 0x9E3779B9
__device__ __forceinline__ uint32_t mixed(uint32_t times_element, uint32_t seed)
{
    uint32_t h = times_element ^ seed;
    h = (h ^ (h >> 16)) * 0x6A09E667u;
    h = (h ^ (h >> 13)) * 0xBB67AE85u;
    return h ^ (h >> 16);
}

constexpr double kLargest = 448.0 * 0x1.fffffep127;  // moment whose scale is a float; larger ones count as infinite

// The scale of a block from each lane's largest finite magnitude: rounding to float and the division keep the order, so the
// lanes' own scales are reduced.
__device__ __forceinline__ float block_scale(double amax)
{
    double q = amax * (1.0 / 448.0);
    q = __builtin_fma(__builtin_fma(-q, 448.0, amax), 1.0 / 448.0, q);  // amax / 448, rounded as a division is
    float s = (float)q;
    s = amax > 0.0 ? fmaxf(s, 0x1p-126f) : 0.f;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s = fmaxf(s, __shfl_xor(s, d));
    return s > 0.f ? s : 1.f;
}

// 1/s to a double's precision or an ulp of it, s a float from 2^-126 on: two steps of Newton's iteration from the float reciprocal.
__device__ __forceinline__ double reciprocal(float s)
{
    double y = (double)__builtin_amdgcn_rcpf(s);
    y = __builtin_fma(__builtin_fma(-(double)s, y, 1.0), y, y);
    return __builtin_fma(__builtin_fma(-(double)s, y, 1.0), y, y);
}
// The root of v to some 1e-14: one step of Newton's iteration from the float root, for v that is a normal float with room around it.
__device__ __forceinline__ double quick_root(double v)
{
    const float r = __builtin_amdgcn_sqrtf((float)v);
    const double d = (double)r;
    return __builtin_fma(__builtin_fma(-d, d, v), (double)(0.5f * __builtin_amdgcn_rcpf(r)), d);
}

// E4M3 code of magnitude z (>= 0, in units of the scale) rounded by the 16 bits u.  With e the exponent of z (at least that of
// the smallest normal value, -6), z * 2^(3-e) counts steps, eight to sixteen of them in a binade; a code counts the steps from
// zero.
__device__ __forceinline__ uint32_t e4m3_steps(double z, uint32_t u)
{
    const int e = max((int)((__double_as_longlong(z) >> 52) & 0x7ff) - 1023, -6);
    const double per_step = __longlong_as_double((long long)(1023 + 3 - e) << 52);
    const int steps = (int)floor(z * per_step + (double)u * 0x1p-16) + 8 * (e + 6);
    return (uint32_t)min(steps, 126);
}

template <int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(const Record *__restrict__ records, const int *__restrict__ chunk_tensor,
                                                    StepArgs a)
{
    const Record &rec = records[chunk_tensor[blockIdx.x]];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n = rec.n;
    const float decay = 1.f - a.lr * rec.weight_decay;
    const float gs = a.grad_scale ? a.grad_scale[0] : 1.f;
    float *__restrict__ param = global(rec.param);
    const float *__restrict__ grad = global(rec.grad);
    bf16_t *__restrict__ copy = global(rec.copy);
    const uint32_t block0 = (uint32_t)((int)blockIdx.x - rec.first_chunk) * kChunkBlocks + wave;
#pragma unroll
    for (int i = 0; i < kChunkBlocks / 4; ++i) {
        const uint32_t block = block0 + 4 * i;  // of the tensor
        const uint32_t at = block * kBlock + 4 * lane;
        if (block * kBlock >= n) break;  // (uniform)
        const int left = at < n ? (int)min(n - at, 4u) : 0;
        const bool whole = left == 4 && rec.aligned;
        float p[4], g[4], update[4];
        load4<float4>(param + at, left, whole, p);
        load4<float4>(grad + at, left, whole, g);
        if constexpr (BITS == 32) {
            float *mp = global((float *)rec.m) + at, *vp = global((float *)rec.v) + at;
            float m[4], v[4];
            load4<float4>(mp, left, whole, m);
            load4<float4>(vp, left, whole, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float gj = g[j] * gs;
                m[j] = a.beta1 * m[j] + a.one_minus_beta1 * gj;
                v[j] = a.beta2 * v[j] + a.one_minus_beta2 * (gj * gj);
                update[j] = m[j] / (sqrtf(v[j]) * a.root_correction + a.eps);
            }
            store4<float4>(mp, left, whole, m);
            store4<float4>(vp, left, whole, v);
        } else {
            unsigned char *mp = global((unsigned char *)rec.m) + at, *rp = global((unsigned char *)rec.v) + at;
            float *m_scales = global(rec.m_scale), *r_scales = global(rec.v_scale);
            unsigned char mc[4], rc[4];
            load4<uint32_t>(mp, left, whole, mc);
            load4<uint32_t>(rp, left, whole, rc);
            const double ms = m_scales[block], rs = r_scales[block];
            double m[4], r[4], m_max = 0.0, r_max = 0.0;
            const uint32_t mw = mc[0] | mc[1] << 8 | mc[2] << 16 | (uint32_t)mc[3] << 24;
            const uint32_t rw = rc[0] | rc[1] << 8 | rc[2] << 16 | (uint32_t)rc[3] << 24;
            const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(mw, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(mw, true);
            const auto r01 = __builtin_amdgcn_cvt_pk_f32_fp8(rw, false), r23 = __builtin_amdgcn_cvt_pk_f32_fp8(rw, true);
            const float mf[4] = {m01[0], m01[1], m23[0], m23[1]}, rf[4] = {r01[0], r01[1], r23[0], r23[1]};
            double v[4];
            bool plain = true;  // all of the lane's v have a float root
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const double gj = (double)g[j] * (double)gs;
                m[j] = a.beta1_d * ((double)mf[j] * ms) + a.one_minus_beta1_d * gj;
                const double rj = (double)rf[j] * rs;
                v[j] = a.beta2_d * (rj * rj) + a.one_minus_beta2_d * (gj * gj);
                if (j >= left) m[j] = v[j] = 0.0;
                plain = plain && v[j] < 0x1p100 && (v[j] > 0x1p-100 || v[j] == 0.0);
            }
            if (__all(plain)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = v[j] > 0.0 ? quick_root(v[j]) : 0.0;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = sqrt(v[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                update[j] = (float)m[j] * __builtin_amdgcn_rcpf((float)r[j] * a.root_correction + a.eps);  // (an ulp or two; the denominator is no subnormal)
                // (comparisons are false for a NaN)
                const double ma = fabs(m[j]);
                if (ma <= kLargest) m_max = fmax(m_max, ma);
                if (r[j] <= kLargest) r_max = fmax(r_max, r[j]);
            }
            const float m_scale = block_scale(m_max), r_scale = block_scale(r_max);
            const double per_m = reciprocal(m_scale), per_r = reciprocal(r_scale);
            const uint32_t element = ((rec.first_block + block) * kBlock + 4 * lane) * 0x9E3779B9u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t u = mixed(element + j * 0x9E3779B9u, a.seed);
                const double ma = fabs(m[j]);
                uint32_t cm = e4m3_steps(ma * per_m, u & 0xffffu) | (m[j] < 0.0 ? 0x80u : 0u);
                uint32_t cr = e4m3_steps(r[j] * per_r, u >> 16);
                if (cr == 0 && r[j] > 0.0) cr = 1;
                if (!(ma <= kLargest)) cm = 0x7fu;
                if (!(r[j] <= kLargest)) cr = 0x7fu;
                mc[j] = (unsigned char)cm;
                rc[j] = (unsigned char)cr;
            }
            store4<uint32_t>(mp, left, whole, mc);
            store4<uint32_t>(rp, left, whole, rc);
            if (lane == 0) {
                m_scales[block] = m_scale;
                r_scales[block] = r_scale;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = p[j] * decay - a.step_size * update[j];
        store4<float4>(param + at, left, whole, p);
        if (copy) {
            bf16_t c[4];
            const uint32_t w[2] = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3])};
            __builtin_memcpy(c, w, 8);
            store4<uint2>(copy + at, left, whole, c);
        }
    }
}

bool check_tensors(const nm_adamw_tensor *t, int count, int bits, long long *blocks, long long *chunks)
{
    if (!t || count <= 0 || count > (1 << 20) || (bits != 8 && bits != 32)) return false;
    *blocks = *chunks = 0;
    for (int i = 0; i < count; ++i) {
        const nm_adamw_tensor &a = t[i];
        if (!a.param || !a.grad || !a.m || !a.v || a.n < 1 || a.n >= (1LL << 31)) return false;
        if ((bits == 8) != (a.m_scale != nullptr) || (bits == 8) != (a.v_scale != nullptr)) return false;
        if (!(a.weight_decay >= 0.f) || isinf(a.weight_decay)) return false;
        if (((uintptr_t)a.param | (uintptr_t)a.grad | (uintptr_t)a.m_scale | (uintptr_t)a.v_scale) % 4 || (uintptr_t)a.copy % 2) return false;
        if (bits == 32 && ((uintptr_t)a.m | (uintptr_t)a.v) % 4) return false;
        if ((void *)a.param == (const void *)a.grad || a.param == a.m || a.param == a.v || a.m == a.v || a.m == (const void *)a.grad ||
            a.v == (const void *)a.grad || (bits == 8 && a.m_scale == a.v_scale))
            return false;
        const long long b = (a.n + kBlock - 1) / kBlock;
        *blocks += b;
        *chunks += (b + kChunkBlocks - 1) / kChunkBlocks;
    }
    return *chunks < (1LL << 24);  // workgroups of 256: a launch has less than 2^32 work items
}
size_t plan_size(int count, long long chunks)
{
    return align_up(sizeof(PlanHeader) + (size_t)count * sizeof(Record) + (size_t)chunks * sizeof(int), 256);
}

}  // namespace
}  // namespace nm

using namespace nm;

extern "C" {

size_t nm_adamw_plan_bytes(const nm_adamw_tensor *tensors, int count, int state_bits)
{
    long long blocks, chunks;
    return check_tensors(tensors, count, state_bits, &blocks, &chunks) ? plan_size(count, chunks) : 0;
}

int nm_adamw_plan(const nm_adamw_tensor *tensors, int count, int state_bits, void *plan, size_t plan_bytes)
{
    long long blocks, chunks;
    if (!check_tensors(tensors, count, state_bits, &blocks, &chunks) || !plan) return NM_ERR_BAD_ARG;
    if (plan_bytes < plan_size(count, chunks) || (uintptr_t)plan % 8) return NM_ERR_WORKSPACE;
    memset(plan, 0, plan_size(count, chunks));
    PlanHeader *h = (PlanHeader *)plan;
    h->magic = kMagic;
    h->state_bits = state_bits;
    h->count = count;
    h->chunks = (int)chunks;
    h->bytes = plan_size(count, chunks);
    Record *rec = (Record *)(h + 1);
    int *chunk_tensor = (int *)(rec + count);
    long long block = 0;
    int chunk = 0;
    for (int i = 0; i < count; ++i) {
        const nm_adamw_tensor &t = tensors[i];
        Record &r = rec[i];
        r.param = t.param; r.grad = t.grad; r.m = t.m; r.v = t.v;
        r.m_scale = t.m_scale; r.v_scale = t.v_scale; r.copy = (bf16_t *)t.copy;
        r.n = (uint32_t)t.n;
        r.weight_decay = t.weight_decay;
        r.first_block = (uint32_t)block;
        r.first_chunk = chunk;
        const uintptr_t state = (uintptr_t)t.m | (uintptr_t)t.v;
        r.aligned = ((uintptr_t)t.param | (uintptr_t)t.grad) % 16 == 0 && state % (state_bits == 32 ? 16 : 4) == 0 && (uintptr_t)t.copy % 8 == 0;
        const long long b = (t.n + kBlock - 1) / kBlock;
        block += b;
        for (long long c = 0; c < b; c += kChunkBlocks) chunk_tensor[chunk++] = i;
    }
    return NM_OK;
}

int nm_adamw_step(const void *plan, const void *plan_device, size_t plan_bytes, double lr, double beta1, double beta2,
                  double eps, long long step, const float *grad_scale, unsigned seed, void *hip_stream)
{
    if (!plan || !plan_device || plan_bytes < sizeof(PlanHeader) || (uintptr_t)plan % 8 || (uintptr_t)plan_device % 256) return NM_ERR_BAD_ARG;
    const PlanHeader *h = (const PlanHeader *)plan;
    if (h->magic != kMagic || h->bytes > plan_bytes || h->count <= 0 || h->chunks <= 0 || h->bytes != plan_size(h->count, h->chunks)) return NM_ERR_BAD_ARG;
    if (!isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0x1p-126) || isinf(eps) || step < 1) return NM_ERR_BAD_ARG;
    StepArgs a;
    a.lr = (float)lr;
    a.step_size = (float)(lr / (1.0 - pow(beta1, (double)step)));
    a.root_correction = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    a.beta1 = (float)beta1; a.one_minus_beta1 = (float)(1.0 - beta1);
    a.beta2 = (float)beta2; a.one_minus_beta2 = (float)(1.0 - beta2);
    a.eps = (float)eps;
    a.beta1_d = beta1; a.one_minus_beta1_d = 1.0 - beta1;
    a.beta2_d = beta2; a.one_minus_beta2_d = 1.0 - beta2;
    a.grad_scale = grad_scale;
    a.seed = seed;
    const Record *rec = (const Record *)((const char *)plan_device + sizeof(PlanHeader));
    const int *chunk_tensor = (const int *)(rec + h->count);
    const hipStream_t s = (hipStream_t)hip_stream;
    if (h->state_bits == 8)
        adamw_kernel<8><<<dim3(h->chunks), dim3(256), 0, s>>>(rec, chunk_tensor, a);
    else
        adamw_kernel<32><<<dim3(h->chunks), dim3(256), 0, s>>>(rec, chunk_tensor, a);
    return hipGetLastError() == hipSuccess ? NM_OK : NM_ERR_DEVICE;
}

}  // extern "C"
