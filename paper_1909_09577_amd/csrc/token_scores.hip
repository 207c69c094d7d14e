// Log-probabilities of given tokens, entropies, the likeliest classes, and the scores' gradient (definition: include/nm_token_scores.h).
//
// Forward: one pass over the scores with a running maximum m, s = sum exp(z - m) and t = sum exp(z - m) * (z - m), of which
// lse = m + log s and entropy = log s - t/s, in powers of two throughout.  Places lie side by side in memory, so lanes are places (64 of
// them, or fewer places times several classes); wavefronts, workgroups and spare lanes share the classes, and join what they found in pairs.
//
// The largest scores in order: a lane takes eight classes at a time and keeps a list of the largest of their maxima.  The K largest scores lie in
// the eights of the K largest maxima (an eight that is not among them has K scores before all of its own), so that one insertion is
// made for eight classes at most, and at the end the K eights are read again and sorted.  Of two sorted lists a_i and b_i of K the K largest of
// all are the larger ones of a_i and b_(K-1-i), which are in order again after log K exchanges.
//
// Backward: element by element from the saved lse and entropy, a thread on the same eight places of every so many classes.
#include "../../include/nm_token_scores.h"
#include "token_ops.h"

namespace nm {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr int kNone = 0x7fffffff;  // class of an empty place in a list: behind all others
constexpr int kMaxSplits = 64;
constexpr int kRounds = 32;  // of classes side by side that a wavefront does at least where workgroups share a place's classes

struct ScoresFwd {
    int B, V, U;
    const void *scores;
    Ids targets;  // (p NULL: none)
    const int *len;
    float *logp, *entropy, *lse, *top_logp;
    int *top_ids;
    int top;
    int log_lanes;  // log2 of the places that a wavefront has side by side
    int u_tiles, splits, per;  // classes of a wavefront
    float *part;    // [splits][3][B*U]: m, s, t
    float *part_z;  // [splits][K][B*U]
    int *part_id;
};

template <int K>
struct State {
    float m, s, t;  // in powers of two
    float z[K ? K : 1];
    int id[K ? K : 1];
    __device__ __forceinline__ void clear_list()
    {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            z[i] = -INFINITY;
            id[i] = kNone;
        }
    }
    __device__ __forceinline__ void clear()
    {
        m = -INFINITY;
        s = t = 0.f;
        clear_list();
    }
    static __device__ __forceinline__ bool before(float za, int ia, float zb, int ib) { return za > zb || (za == zb && ia < ib); }
    // sums are taken to `top` from here on
    __device__ __forceinline__ void rebase(float top)
    {
        if (s != 0.f) {
            const float d = m - top, f = __builtin_amdgcn_exp2f(d);
            t = f * (t + d * s);
            s *= f;
        }
        m = top;
    }
    __device__ __forceinline__ void insert(float v, int c)
    {
#pragma unroll
        for (int i = K - 1; i >= 0; --i) {
            // place i takes the newcomer, its upper neighbour or stays
            const bool here = before(v, c, z[i], id[i]), above = i > 0 && before(v, c, z[i ? i - 1 : 0], id[i ? i - 1 : 0]);
            z[i] = here ? (above ? z[i ? i - 1 : 0] : v) : z[i];
            id[i] = here ? (above ? id[i ? i - 1 : 0] : c) : id[i];
        }
    }
    __device__ __forceinline__ void join_sums(float om, float os, float ot)
    {
        const float top = fmaxf(m, om);
        if (m < top) rebase(top);
        if (om < top && os != 0.f) {
            const float d = om - top, f = __builtin_amdgcn_exp2f(d);
            ot = f * (ot + d * os);
            os *= f;
        }
        s += os;
        t += ot;
    }
    __device__ __forceinline__ void join_list(const float (&oz)[K ? K : 1], const int (&oid)[K ? K : 1])
    {
        if constexpr (K > 0) {
            float nz[K];
            int ni[K];
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const bool mine = before(z[i], id[i], oz[K - 1 - i], oid[K - 1 - i]);
                nz[i] = mine ? z[i] : oz[K - 1 - i];
                ni[i] = mine ? id[i] : oid[K - 1 - i];
            }
#pragma unroll
            for (int d = K / 2; d >= 1; d >>= 1)
#pragma unroll
                for (int i = 0; i < K; ++i)
                    if (!(i & d)) {
                        const bool swap = before(nz[i + d], ni[i + d], nz[i], ni[i]);
                        const float zl = swap ? nz[i + d] : nz[i], zh = swap ? nz[i] : nz[i + d];
                        const int il = swap ? ni[i + d] : ni[i], ih = swap ? ni[i] : ni[i + d];
                        nz[i] = zl;
                        nz[i + d] = zh;
                        ni[i] = il;
                        ni[i + d] = ih;
                    }
#pragma unroll
            for (int i = 0; i < K; ++i) {
                z[i] = nz[i];
                id[i] = ni[i];
            }
        }
    }
    __device__ __forceinline__ void join_list_of_lane(int mask)
    {
        float oz[K ? K : 1];
        int oi[K ? K : 1];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            oz[i] = __shfl_xor(z[i], mask);
            oi[i] = __shfl_xor(id[i], mask);
        }
        join_list(oz, oi);
    }
    __device__ __forceinline__ void join_lane(int mask)
    {
        join_sums(__shfl_xor(m, mask), __shfl_xor(s, mask), __shfl_xor(t, mask));
        join_list_of_lane(mask);
    }
};

// Eights: a wavefront has classes c0 .. c1-1, a lane of it every step-th of them from c0 + (lane's number) on, eight at a time.  The classes of
// the eight that holds class c, in order.
struct Eight {
    int first, step, end;
    __device__ __forceinline__ Eight(const ScoresFwd &a, int c)
    {
        step = 64 >> a.log_lanes;
        const int c0 = c / a.per * a.per, round = (c - c0) / step;
        first = c - (round & 7) * step;
        end = min(a.V, c0 + a.per);
    }
};
// The sorted scores of one of the listed eights are added to `list`
template <typename S, int K>
__device__ __forceinline__ void read_again(const ScoresFwd &a, const S *column, float top, int id, State<K> &list)
{
    const Eight e(a, id == kNone ? 0 : id);
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = load_as_f32(column, (size_t)min(e.first + i * e.step, a.V - 1) * a.U);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = e.first + i * e.step;
        const bool is = id != kNone && c < e.end;
        const float v = is && z[i] == z[i] ? z[i] : -INFINITY;
        const int vc = is ? c : kNone;
        if (__any(State<K>::before(v, vc, list.z[K ? K - 1 : 0], list.id[K ? K - 1 : 0]))) list.insert(v, vc);
    }
}

// The results of a place, but for its alternatives; the log-sum-exp
template <typename S>
__device__ __forceinline__ float finish_sums(const ScoresFwd &a, int b, int u, bool there, float m, float s, float t)
{
    const size_t at = (size_t)b * a.U + u;
    const float log_s = __builtin_amdgcn_logf(s), lse = ((m == -INFINITY ? 0.f : m) + log_s) * kLn2;
    if (a.lse) a.lse[at] = there ? lse : 0.f;
    if (a.entropy) a.entropy[at] = there && s != 0.f ? (log_s - t / s) * kLn2 : 0.f;
    if (a.logp) {
        const int target = there ? a.targets.at(at, a.V) : -1;
        const float z = target < 0 ? 0.f : load_as_f32((const S *)a.scores, ((size_t)b * a.V + target) * a.U + u);
        a.logp[at] = target < 0 ? 0.f : (lse == -INFINITY ? lse : z - lse);
    }
    return lse;
}
__device__ __forceinline__ void finish_alternative(const ScoresFwd &a, int b, int u, bool there, int i, float z, int id, float lse)
{
    const size_t to = ((size_t)b * a.top + i) * a.U + u;
    a.top_ids[to] = there ? id : -1;
    a.top_logp[to] = there ? (lse == -INFINITY ? lse : z - lse) : 0.f;
}

template <typename S, int K>
__global__ __launch_bounds__(256, K > 8 ? 2 : 4) void scores_fwd_kernel(ScoresFwd a)
{
    constexpr int kAhead = 16;
    __shared__ float sums[4][3][64];
    __shared__ float list_z[K ? 4 : 1][K ? K : 1][64];
    __shared__ int list_id[K ? 4 : 1][K ? K : 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ut = blockIdx.x % a.u_tiles, rest = blockIdx.x / a.u_tiles, split = rest % a.splits, b = rest / a.splits;
    const int lanes = 1 << a.log_lanes, u = ut * lanes + (lane & (lanes - 1)), step = 64 >> a.log_lanes;
    const int len = length_in(a.len, b, a.U);
    const int c0 = (split * 4 + wave) * a.per, c1 = min(a.V, c0 + a.per);
    const bool there = u < len;
    State<K> st;
    st.clear();
    const S *column = (const S *)a.scores + (size_t)b * a.V * a.U + min(u, a.U - 1);
    if (ut * lanes < len) {  // (uniform)
        // rows of `step` classes, kAhead of them at a time; a lane's bytes from a row's first element are of 32 bits
        const uint32_t mine = ((uint32_t)(lane >> a.log_lanes) * (uint32_t)a.U + (uint32_t)min(u, a.U - 1)) * (uint32_t)sizeof(S);
        const size_t row = (size_t)step * a.U;
        auto take = [&](const float (&z)[kAhead], int c) {  // c: this lane's first class
            float top = z[0];
#pragma unroll
            for (int i = 1; i < kAhead; ++i) top = fmaxf(top, z[i]);
            if (top * kLog2e > st.m) st.rebase(top * kLog2e);
            const float base = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const float y = __builtin_fmaf(z[i], kLog2e, -base), e = __builtin_amdgcn_exp2f(y);
                st.s += e;
                st.t = __builtin_fmaf(e, fmaxf(y, -1e30f), st.t);  // (zero times what is barred)
            }
            if constexpr (K > 0) {
#pragma unroll
                for (int h = 0; h < kAhead; h += 8) {
                    float best = z[h];
#pragma unroll
                    for (int i = 1; i < 8; ++i) best = fmaxf(best, z[h + i]);
                    best = fmaxf(best, -INFINITY);  // (of eight NaN)
                    if (__any(best > st.z[K - 1] || st.id[K - 1] == kNone)) {
                        int at = kNone;  // the first class that has it
#pragma unroll
                        for (int i = 7; i >= 0; --i) {
                            const int ci = c + (h + i) * step;
                            at = ci < c1 && (z[h + i] == best || best == -INFINITY) ? ci : at;
                        }
                        st.insert(best == best ? best : -INFINITY, at);
                    }
                }
            }
        };
        const S *p = (const S *)a.scores + (size_t)b * a.V * a.U + (size_t)c0 * a.U;
        int c = c0;
        for (; c + kAhead * step <= c1; c += kAhead * step, p += kAhead * row) {
            float z[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) z[i] = load_as_f32(reinterpret_cast<const S *>(reinterpret_cast<const char *>(p + i * row) + mine), 0);
            if (!there) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) z[i] = -INFINITY;
            }
            take(z, c + (lane >> a.log_lanes));
        }
        if (c < c1) {
            const int first = c + (lane >> a.log_lanes);
            float z[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) z[i] = load_as_f32(column, (size_t)min(first + i * step, a.V - 1) * a.U);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) z[i] = there && first + i * step < c1 ? z[i] : -INFINITY;
            take(z, first);
        }
        for (int d = lanes; d < 64; d <<= 1) st.join_lane(d);
    }
    auto leave = [&](int w) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            list_z[w][i][lane] = st.z[i];
            list_id[w][i][lane] = st.id[i];
        }
    };
    auto join_list_of = [&](int w) {
        float oz[K ? K : 1];
        int oi[K ? K : 1];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            oz[i] = list_z[w][i][lane];
            oi[i] = list_id[w][i][lane];
        }
        st.join_list(oz, oi);
    };
    sums[wave][0][lane] = st.m;
    sums[wave][1][lane] = st.s;
    sums[wave][2][lane] = st.t;
    leave(wave);
    __syncthreads();
    if (a.splits > 1) {
        if (wave) return;
        for (int w = 1; w < 4; ++w) {
            st.join_sums(sums[w][0][lane], sums[w][1][lane], sums[w][2][lane]);
            join_list_of(w);
        }
        if (lane >= lanes || u >= a.U) return;
        const size_t all = (size_t)a.B * a.U, at = (size_t)b * a.U + u;
        float *p = a.part + (size_t)split * 3 * all + at;
        p[0] = st.m;
        p[all] = st.s;
        p[2 * all] = st.t;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            a.part_z[((size_t)split * K + i) * all + at] = st.z[i];
            a.part_id[((size_t)split * K + i) * all + at] = st.id[i];
        }
        return;
    }
    // every wavefront has the eights of all four, reads a fourth of them again, and the first one joins what they find
    if constexpr (K > 0) {
        for (int w = 0; w < 4; ++w)
            if (w != wave) join_list_of(w);
        State<K> best;
        best.clear_list();
        if (ut * lanes < len) {
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (i % 4 == wave) read_again<S, K>(a, column, st.z[i], st.id[i], best);
        }
#pragma unroll
        for (int i = 0; i < K; ++i) {
            st.z[i] = best.z[i];
            st.id[i] = best.id[i];
        }
        __syncthreads();
        leave(wave);
        __syncthreads();
    }
    if (wave) return;
    for (int w = 1; w < 4; ++w) {
        st.join_sums(sums[w][0][lane], sums[w][1][lane], sums[w][2][lane]);
        join_list_of(w);
    }
    if (lane >= lanes || u >= a.U) return;
    const float lse = finish_sums<S>(a, b, u, there, st.m, st.s, st.t);
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i < a.top) finish_alternative(a, b, u, there, i, st.z[i], st.id[i], lse);
}

// Joins what `splits` workgroups found: neighbouring lanes take a place's splits, and then a share of its eights
template <typename S, int K>
__global__ __launch_bounds__(256) void scores_join_kernel(ScoresFwd a, int log_splits)
{
    const int t = blockIdx.x * 256 + threadIdx.x, group = 1 << log_splits, split = t & (group - 1), all = a.B * a.U, at = min(t >> log_splits, all - 1);
    const bool exists = t >> log_splits < all;
    State<K> st;
    st.clear();
    if (split < a.splits) {
        const float *p = a.part + (size_t)split * 3 * all + at;
        st.m = p[0];
        st.s = p[all];
        st.t = p[2 * (size_t)all];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            st.z[i] = a.part_z[((size_t)split * K + i) * all + at];
            st.id[i] = a.part_id[((size_t)split * K + i) * all + at];
        }
    }
    for (int d = 1; d < group; d <<= 1) st.join_lane(d);
    const int b = at / a.U, u = at - b * a.U;
    const bool there = u < length_in(a.len, b, a.U);
    float lse = 0.f;
    if (split == 0 && exists) lse = finish_sums<S>(a, b, u, there, st.m, st.s, st.t);
    if constexpr (K > 0) {
        State<K> best;
        best.clear_list();
        for (int i0 = 0; i0 < K; i0 += group) {
            float z = -INFINITY;
            int id = kNone;
#pragma unroll
            for (int i = 0; i < K; ++i) {  // (a list is in registers: no index of a lane's own)
                z = i == i0 + split ? st.z[i] : z;
                id = i == i0 + split ? st.id[i] : id;
            }
            read_again<S, K>(a, (const S *)a.scores + (size_t)b * a.V * a.U + u, z, there ? id : kNone, best);
        }
        for (int d = 1; d < group && d < K; d <<= 1) best.join_list_of_lane(d);
        if (split || !exists) return;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i < a.top) finish_alternative(a, b, u, there, i, best.z[i], best.id[i], lse);
    }
}

// The lists' length that serves `top`: of two a power
int list_of(int top) { return top <= 1 ? top : top <= 4 ? 4 : top <= 8 ? 8 : 16; }

struct Plan {
    int log_lanes, u_tiles, splits, per;
    size_t part_bytes, list_bytes;  // of the sums, of the scores of the lists
};
Plan plan_of(int B, int V, int U, int top)
{
    Plan p = {};
    while (p.log_lanes < 6 && (1 << p.log_lanes) < U) ++p.log_lanes;
    const int lanes = 1 << p.log_lanes, step = 64 >> p.log_lanes;
    p.u_tiles = (U + lanes - 1) / lanes;
    // four workgroups a CU, but a wavefront has 32 rounds of classes to do at least: what follows them takes about as long
    const long long groups = (long long)B * p.u_tiles;
    long long splits = 1024 / groups;
    const long long most = V / (4LL * step * kRounds);
    if (splits > most) splits = most;
    if (splits > kMaxSplits) splits = kMaxSplits;
    if (splits < 1) splits = 1;
    p.per = (int)((V + 4 * splits - 1) / (4 * splits));
    p.splits = (int)((V + 4LL * p.per - 1) / (4LL * p.per));
    const size_t all = (size_t)B * U;
    p.part_bytes = p.splits > 1 ? align_up((size_t)p.splits * 3 * all * 4, 256) : 0;
    p.list_bytes = p.splits > 1 ? align_up((size_t)p.splits * list_of(top) * all * 4, 256) : 0;
    return p;
}

template <typename S, int K>
hipError_t run_list(const ScoresFwd &a, hipStream_t s)
{
    scores_fwd_kernel<S, K><<<dim3((unsigned)a.B * a.u_tiles * a.splits), dim3(256), 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    int log_splits = 0;
    while ((1 << log_splits) < a.splits) ++log_splits;
    const long long threads = ((long long)a.B * a.U) << log_splits;
    scores_join_kernel<S, K><<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s>>>(a, log_splits);
    return hipGetLastError();
}
template <typename S>
hipError_t run_fwd(const ScoresFwd &a, hipStream_t s)
{
    switch (list_of(a.top)) {
    case 0: return run_list<S, 0>(a, s);
    case 1: return run_list<S, 1>(a, s);
    case 4: return run_list<S, 4>(a, s);
    case 8: return run_list<S, 8>(a, s);
    default: return run_list<S, 16>(a, s);
    }
}

// ---- backward ----------------------------------------------------------------------------------------------------
struct ScoresBwd {
    int B, V, U;
    const void *scores;
    Ids targets;
    const int *len;
    const float *lse, *entropy, *dlogp, *dentropy;
    void *out;
    int groups, group_tiles, side, rows, rounds;  // of eight places; tiles of `side` of them; classes side by side in a workgroup, and one after the other
};

struct Place {
    float lse, entropy, dl, dh;
    int target;
    bool there;
};
__device__ __forceinline__ Place place_of(const ScoresBwd &a, int b, int u, int len)
{
    Place p;
    const size_t at = (size_t)b * a.U + u;
    p.lse = a.lse[at];
    p.there = u < len && p.lse != -INFINITY;
    p.target = p.there && a.dlogp ? a.targets.at(at, a.V) : -1;
    p.dl = p.target >= 0 ? a.dlogp[at] : 0.f;
    p.dh = a.dentropy ? a.dentropy[at] : 0.f;
    p.entropy = a.dentropy ? a.entropy[at] : 0.f;
    return p;
}
__device__ __forceinline__ float gradient(const Place &p, float z, int c)
{
    const float x = z - p.lse, q = __builtin_amdgcn_exp2f(x * kLog2e);
    const float g = p.dl * ((c == p.target ? 1.f : 0.f) - q) - p.dh * q * (fmaxf(x, -1e30f) + p.entropy);
    return p.there ? g : 0.f;
}

// Rows of eight places at least: the last group of a row begins eight before its end, and what two groups share is made twice.
template <typename S, typename G>
__global__ __launch_bounds__(256) void scores_bwd_kernel(ScoresBwd a)
{
    const int gt = blockIdx.x % a.group_tiles, rest = blockIdx.x / a.group_tiles, tiles = (a.V + a.rows * a.rounds - 1) / (a.rows * a.rounds);
    const int vt = rest % tiles, b = rest / tiles;
    const int r = threadIdx.x / a.side, group = gt * a.side + threadIdx.x - r * a.side;
    if (r >= a.rows || group >= a.groups) return;
    const int u = min(group * 8, a.U - 8), len = length_in(a.len, b, a.U);
    Place p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = place_of(a, b, u + j, len);
    const int c0 = vt * a.rows * a.rounds + r;
    const size_t base = (size_t)b * a.V * a.U + u;
    const bool any = u < len;
    for (int i = 0; i < a.rounds; i += 4) {
        float z[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (any) load8((const S *)a.scores + base + (size_t)min(c0 + (i + k) * a.rows, a.V - 1) * a.U, 8, z[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = c0 + (i + k) * a.rows;
            if (i + k >= a.rounds || c >= a.V) return;
            float g[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = any ? gradient(p[j], z[k][j], c) : 0.f;
            store8((G *)a.out + base + (size_t)c * a.U, 8, g);
        }
    }
}

// Shorter rows: eight neighbouring elements of an item a thread
template <typename S, typename G>
__global__ __launch_bounds__(256) void scores_bwd_flat_kernel(ScoresBwd a)
{
    const int per_item = ((long long)a.V * a.U + 2047) / 2048, b = blockIdx.x / per_item;
    const long long item = (long long)a.V * a.U, i0 = ((long long)(blockIdx.x - b * per_item) * 256 + threadIdx.x) * 8;
    if (i0 >= item) return;
    const int len = length_in(a.len, b, a.U), n = (int)min(item - i0, 8LL);
    float z[8], g[8];
    load8((const S *)a.scores + (size_t)b * item + i0, n, z);
    int c = (int)(i0 / a.U), u = (int)(i0 - (long long)c * a.U);
    Place p = place_of(a, b, u, len);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] = gradient(p, z[j], c);
        if (++u == a.U) {
            u = 0;
            ++c;
        }
        if (a.U > 1) p = place_of(a, b, u, len);
    }
    store8((G *)a.out + (size_t)b * item + i0, n, g);
}

template <typename S, typename G>
hipError_t run_bwd(ScoresBwd a, hipStream_t s)
{
    if (a.U < 8) {
        const long long per_item = ((long long)a.V * a.U + 2047) / 2048;
        scores_bwd_flat_kernel<S, G><<<dim3((unsigned)(per_item * a.B)), dim3(256), 0, s>>>(a);
        return hipGetLastError();
    }
    a.groups = (a.U + 7) / 8;
    a.group_tiles = (a.groups + 255) / 256;
    a.side = (a.groups + a.group_tiles - 1) / a.group_tiles;
    a.rows = 256 / a.side;
    a.rounds = 16;
    const long long tiles = (a.V + a.rows * a.rounds - 1) / (a.rows * a.rounds);
    scores_bwd_kernel<S, G><<<dim3((unsigned)(tiles * a.group_tiles * a.B)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

int check(int B, int V, int U, int dtype)
{
    if (B <= 0 || V <= 0 || U <= 0 || !known_dtype(dtype)) return NM_ERR_BAD_ARG;
    const long long most = (1LL << 31) - 1;
    if ((long long)B * V > most / U || V > most - (1 << 16) || U > 1 << 29) return NM_ERR_UNSUPPORTED;  // (classes behind the last one are counted too)
    // the grids, below 2^32 work items: a workgroup of the backward pass has 2048 elements, or one item's rest
    if ((long long)B * ((U + 63) / 64) >= 1LL << 23 || (long long)B * (((long long)V * U + 2047) / 2048) >= 1LL << 24) return NM_ERR_UNSUPPORTED;
    return NM_OK;
}
int check_top(int V, int top)
{
    return top < 0 || top > V ? NM_ERR_BAD_ARG : top > NM_MOST_ALTERNATIVES ? NM_ERR_UNSUPPORTED : NM_OK;
}

}  // namespace
}  // namespace nm

using namespace nm;

extern "C" {

size_t nm_token_scores_workspace_bytes(int B, int V, int U, int top, int dtype)
{
    if (check(B, V, U, dtype) != NM_OK || check_top(V, top) != NM_OK) return 0;
    const Plan p = plan_of(B, V, U, top);
    return p.part_bytes + 2 * p.list_bytes;
}

int nm_token_scores_fwd(int B, int V, int U, const void *scores, const void *targets, int target_bytes, const int *lengths, int top,
                        float *logp, float *entropy, float *lse, int *top_ids, float *top_logp, int dtype, void *workspace,
                        size_t workspace_bytes, void *hip_stream)
{
    int st = check(B, V, U, dtype);
    if (st == NM_OK) st = check_top(V, top);
    if (st != NM_OK) return st;
    if (!scores || (logp == nullptr) != (targets == nullptr) || (top == 0) != (top_ids == nullptr) || (top == 0) != (top_logp == nullptr) ||
        (targets && target_bytes != 4 && target_bytes != 8) || (!logp && !entropy && !lse && !top))
        return NM_ERR_BAD_ARG;
    const size_t places = (size_t)B * U;
    const Region in[3] = {{scores, places * V * element(dtype)}, {targets, places * target_bytes}, {lengths, (size_t)B * 4}};
    const Region out[5] = {{logp, places * 4}, {entropy, places * 4}, {lse, places * 4}, {top_ids, places * top * 4}, {top_logp, places * top * 4}};
    for (int i = 0; i < 5; ++i) {
        if (meets(out[i], in)) return NM_ERR_BAD_ARG;
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return NM_ERR_BAD_ARG;
    }
    const Plan p = plan_of(B, V, U, top);
    if (workspace_missing(workspace, workspace_bytes, p.part_bytes + 2 * p.list_bytes)) return NM_ERR_WORKSPACE;
    ScoresFwd a = {};
    a.B = B; a.V = V; a.U = U;
    a.scores = scores;
    a.targets = {targets, target_bytes == 8};
    a.len = lengths;
    a.logp = logp; a.entropy = entropy; a.lse = lse; a.top_logp = top_logp; a.top_ids = top_ids;
    a.top = top;
    a.log_lanes = p.log_lanes; a.u_tiles = p.u_tiles; a.splits = p.splits; a.per = p.per;
    a.part = (float *)workspace;
    a.part_z = (float *)((char *)workspace + p.part_bytes);
    a.part_id = (int *)((char *)workspace + p.part_bytes + p.list_bytes);
    hipStream_t s = (hipStream_t)hip_stream;
    return status_of(dtype == NM_BF16 ? run_fwd<bf16_t>(a, s) : run_fwd<float>(a, s));
}

int nm_token_scores_bwd(int B, int V, int U, const void *scores, const void *targets, int target_bytes, const int *lengths,
                        const float *lse, const float *entropy, const float *dlogp, const float *dentropy, void *dscores, int dtype,
                        int grad_dtype, void *hip_stream)
{
    const int st = check(B, V, U, dtype);
    if (st != NM_OK) return st;
    if (!known_dtype(grad_dtype) || !scores || !lse || !dscores || (dlogp == nullptr) != (targets == nullptr) || (!dlogp && !dentropy) ||
        (dentropy && !entropy) || (targets && target_bytes != 4 && target_bytes != 8))
        return NM_ERR_BAD_ARG;
    const size_t places = (size_t)B * U;
    const Region in[7] = {{scores, places * V * element(dtype)}, {targets, places * target_bytes}, {lengths, (size_t)B * 4}, {lse, places * 4},
                          {entropy, places * 4}, {dlogp, places * 4}, {dentropy, places * 4}};
    if (meets({dscores, places * V * element(grad_dtype)}, in)) return NM_ERR_BAD_ARG;
    ScoresBwd a = {};
    a.B = B; a.V = V; a.U = U;
    a.scores = scores;
    a.targets = {targets, target_bytes == 8};
    a.len = lengths;
    a.lse = lse; a.entropy = entropy; a.dlogp = dlogp; a.dentropy = dentropy;
    a.out = dscores;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == NM_BF16) return status_of(grad_dtype == NM_BF16 ? run_bwd<bf16_t, bf16_t>(a, s) : run_bwd<bf16_t, float>(a, s));
    return status_of(grad_dtype == NM_BF16 ? run_bwd<float, bf16_t>(a, s) : run_bwd<float, float>(a, s));
}

}  // extern "C"
