// Log-probabilities of given tokens, entropies, the likeliest classes, and the scores' gradient (definition: include/nm_token_scores.h).
//
// Forward: one pass over the scores with a running maximum m, s = sum exp(z - m) and t = sum exp(z - m) * (z - m), of which
// lse = m + log s and entropy = log s - t/s.  m is subtracted before anything is scaled to powers of two (0.4 us of 25 at 32 x 150 places of
// 5000 classes): scores may be of any finite size, and places filled with a type's lowest value.  Places lie side by side in memory, so lanes are places (64 of
// them, or fewer places times several classes); wavefronts, workgroups and spare lanes share the classes, and join what they found in pairs.
//
// The largest scores in order: a lane takes 16 neighbouring classes at a time and keeps a list of the largest maxima of eights of them (of all 16,
// for four alternatives: 1 us less, and 2 more where the groups are read again).  The K largest scores lie in the groups of the K largest maxima (a group that is not among them has K scores
// before all of its own; of equal maxima the lower group comes first, and with it its classes), so that one insertion is made for a
// group at most, and at the end the K groups are read again and put in order.  Of two sorted lists a_i and b_i of K the K largest
// of all are the larger ones of a_i and b_(K-1-i), which are in order again after log K exchanges.
//
// Backward: element by element from the saved lse and entropy, a thread on the same eight places of every so many classes.
//
// Measured: 32 x 150 places of 5000 classes, four alternatives, bfloat16: 19 + 8 us; the scores that count, 36 MB, would take 7.  The vector units
// are busy 38 % of the time (an exponential, a maximum and two sums a score), and the join reads 32 lines of memory a place again.  16 single
// places of 32000 classes, eight alternatives, float32: 11 + 6 us, chains of exchanges between lanes.  Backward of 16 x 333 places of 5000
// classes, float32 to bfloat16: 37 us for 160 MB, 4.3 TB/s.
#include "../../include/nm_token_scores.h"
#include "token_ops.h"

namespace nm {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr int kNone = 0x7fffffff;  // class of an empty place in a list: behind all others

struct ScoresFwd {
    int B, V, U;
    const void *scores;
    Ids targets;  // (p NULL: none)
    const int *len;
    float *logp, *entropy, *lse, *top_logp;
    int *top_ids;
    int top;
    int log_lanes;  // log2 of the places that a wavefront has side by side
    int u_tiles, splits, per;  // per: classes of a wavefront, a multiple of kAhead
    float *part;    // [splits][3][B*U]: m, s, t
    uint64_t *part_keys;  // [splits][K][B*U]
};

// A score and its class as one number: the larger one comes first in order, of equal scores the lower class (0.0 and -0.0 are equal), a NaN
// with the -infinities.
typedef uint64_t key_t;
__device__ __forceinline__ key_t key_of(float z, int c)
{
    const uint32_t u = __float_as_uint((z == z ? z : -INFINITY) + 0.f);
    const uint32_t ordered = u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
    return (key_t)ordered << 32 | (uint32_t)~c;
}
__device__ __forceinline__ int class_of(key_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float score_of(key_t k)
{
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float(o >> 31 ? o ^ 0x80000000u : ~o);
}
constexpr key_t kEmpty = (key_t)0x007fffffu << 32 | 0x80000000u;  // -infinity of class 2^31 - 1: behind all others

__device__ __forceinline__ key_t shuffled(key_t k, int mask)
{
    return (key_t)(uint32_t)__shfl_xor((int)(k >> 32), mask) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)k, mask);
}
__device__ __forceinline__ key_t of_lane(key_t k, int lane)  // (the same lane for all)
{
    return (key_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}

// A difference of scores in powers of two, a finite one (what it is an exponent of is zero long before)
__device__ __forceinline__ float twos(float d) { return fmaxf(d * kLog2e, -1e30f); }

struct Sums {
    float m = -INFINITY, s = 0.f, t = 0.f;  // t in powers of two
    // sums are taken to `top` from here on
    __device__ __forceinline__ void rebase(float top)
    {
        if (s != 0.f) {
            const float d = twos(m - top), f = __builtin_amdgcn_exp2f(d);
            t = f * (t + d * s);
            s *= f;
        }
        m = top;
    }
    __device__ __forceinline__ void join(float om, float os, float ot)
    {
        const float top = fmaxf(m, om);
        if (m < top) rebase(top);
        if (om < top && os != 0.f) {
            const float d = twos(om - top), f = __builtin_amdgcn_exp2f(d);
            ot = f * (ot + d * os);
            os *= f;
        }
        s += os;
        t += ot;
    }
    __device__ __forceinline__ void join_lane(int mask) { join(__shfl_xor(m, mask), __shfl_xor(s, mask), __shfl_xor(t, mask)); }
};

constexpr int kAhead = 16;                                       // classes that a lane takes at a time
constexpr int G = 8, kGroups = kAhead / G;                       // classes that a list's entry stands for

template <int K>
struct List {  // the K largest, in order
    key_t k[K ? K : 1];
    __device__ __forceinline__ List()
    {
#pragma unroll
        for (int i = 0; i < K; ++i) k[i] = kEmpty;
    }
    __device__ __forceinline__ void insert(key_t v)
    {
        bool here[K ? K : 1];
#pragma unroll
        for (int i = 0; i < K; ++i) here[i] = v > k[i];
#pragma unroll
        for (int i = K - 1; i >= 0; --i)  // place i takes the newcomer, its upper neighbour or stays
            k[i] = here[i] ? (i > 0 && here[i ? i - 1 : 0] ? k[i ? i - 1 : 0] : v) : k[i];
    }
    __device__ __forceinline__ void join(const key_t (&o)[K ? K : 1])
    {
#pragma unroll
        for (int i = 0; i < K; ++i) k[i] = k[i] > o[K - 1 - i] ? k[i] : o[K - 1 - i];
#pragma unroll
        for (int d = K / 2; d >= 1; d >>= 1)
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (!(i & d)) {
                    const key_t hi = k[i] > k[i + d] ? k[i] : k[i + d], lo = k[i] > k[i + d] ? k[i + d] : k[i];
                    k[i] = hi;
                    k[i + d] = lo;
                }
    }
    __device__ __forceinline__ void join_lane(int mask)
    {
        key_t o[K ? K : 1];
#pragma unroll
        for (int i = 0; i < K; ++i) o[i] = shuffled(k[i], mask);
        join(o);
    }
};

// A place's log-sum-exp in two parts, the largest score and the logarithm of the sum: together they would leave nothing of the latter where scores
// are large.  Differences with it are made in double.
struct Lse {
    float m, log_s;  // (0 and -infinity where nothing is left)
    __device__ __forceinline__ double log_sum() const { return (double)log_s * 0.69314718055994530942; }
    __device__ __forceinline__ double whole() const { return (double)m + log_sum(); }
    __device__ __forceinline__ float logq(float z) const { return log_s == -INFINITY ? -INFINITY : (float)(((double)z - m) - log_sum()); }
};

// The results of a place, but for its alternatives
template <typename S>
__device__ __forceinline__ Lse finish_sums(const ScoresFwd &a, int b, int u, bool there, const Sums &v)
{
    const size_t at = (size_t)b * a.U + u;
    const Lse lse = {v.m == -INFINITY ? 0.f : v.m, __builtin_amdgcn_logf(v.s)};  // (powers of two)
    if (a.lse) a.lse[at] = there ? (float)lse.whole() : 0.f;
    if (a.entropy) a.entropy[at] = there && v.s != 0.f ? (lse.log_s - v.t / v.s) * kLn2 : 0.f;
    if (a.logp) {
        const int target = there ? a.targets.at(at, a.V) : -1;
        const float z = target < 0 ? 0.f : load_as_f32((const S *)a.scores, ((size_t)b * a.V + target) * a.U + u);
        a.logp[at] = target < 0 ? 0.f : lse.logq(z);
    }
    return lse;
}

template <typename S, int K>
__global__ __launch_bounds__(256, K > 8 ? 2 : 4) void scores_fwd_kernel(ScoresFwd a)
{
    __shared__ float sums[3][3][64];
    __shared__ key_t lists[K ? 3 : 1][K ? K : 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // neighbouring workgroups go to different XCDs: tiles of the same rows, which share lines of memory, are as many apart as there are others
    const int others = a.B * a.splits, ut = blockIdx.x / others, rest = blockIdx.x - ut * others, split = rest % a.splits, b = rest / a.splits;
    const int lanes = 1 << a.log_lanes, u = ut * lanes + (lane & (lanes - 1)), step = 64 >> a.log_lanes;
    const int len = length_in(a.len, b, a.U);
    // (the last wavefronts' shares may end beyond 2^31)
    const int c0 = (int)min((long long)(split * 4 + wave) * a.per, (long long)a.V), c1 = (int)min((long long)c0 + a.per, (long long)a.V);
    const bool there = u < len;
    Sums st;
    List<K> list;
    if (ut * lanes < len) {  // (uniform)
        // A lane's classes: kAhead of c + kAhead * (its number among those with its place); bytes from there are of 32 bits.  (Places behind the
        // item's end are worked on like others where a tile has one that counts.)
        const int r = lane >> a.log_lanes, round = kAhead * step;
        const uint32_t mine = ((uint32_t)(r * kAhead) * (uint32_t)a.U + (uint32_t)min(u, a.U - 1)) * (uint32_t)sizeof(S);
        auto take = [&](const float (&z)[kAhead], int c) {  // c: this lane's first class
            float best[kGroups];
#pragma unroll
            for (int h = 0; h < kGroups; ++h) {
                best[h] = z[G * h];
#pragma unroll
                for (int i = 1; i < G; ++i) best[h] = fmaxf(best[h], z[G * h + i]);
            }
            const float top = fmaxf(best[0], best[kGroups - 1]);
            if (top > st.m) st.rebase(top);
            const float base = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const float y = (z[i] - base) * kLog2e, e = __builtin_amdgcn_exp2f(y);
                st.s += e;
                st.t = __builtin_fmaf(e, fmaxf(y, -1e30f), st.t);  // (zero times what is barred)
            }
            if constexpr (K > 0) {
#pragma unroll
                for (int h = 0; h < kGroups; ++h) {
                    const key_t k = c + G * h < c1 ? key_of(best[h], c + G * h) : kEmpty;
                    if (__any(k > list.k[K - 1])) list.insert(k);
                }
            }
        };
        const char *p = reinterpret_cast<const char *>((const S *)a.scores + (size_t)b * a.V * a.U + (size_t)c0 * a.U);
        const size_t row = (size_t)a.U * sizeof(S);
        int c = c0;
        S ahead[kAhead];  // the next classes' are on their way while these are worked on
        auto request = [&]() {
            if (a.U == 1) {  // (side by side)
                __builtin_memcpy(ahead, p + mine, sizeof(ahead));
            } else {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) ahead[i] = *reinterpret_cast<const S *>(p + i * row + mine);
            }
            p += round * row;
        };
        if (c + round <= c1) request();
        for (; c + round <= c1; c += round) {
            float z[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) z[i] = load_as_f32(ahead, i);
            if (c + 2 * round <= c1) request();
            take(z, c + r * kAhead);
        }
        if (c < c1) {
            const S *column = (const S *)a.scores + (size_t)b * a.V * a.U + min(u, a.U - 1);
            const int first = c + r * kAhead;
            float z[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) z[i] = load_as_f32(column, (size_t)min(first + i, a.V - 1) * a.U);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) z[i] = first + i < c1 ? z[i] : -INFINITY;
            take(z, first);
        }
        for (int d = lanes; d < 64; d <<= 1) {
            st.join_lane(d);
            list.join_lane(d);
        }
    }
    if (wave) {
        sums[wave - 1][0][lane] = st.m;
        sums[wave - 1][1][lane] = st.s;
        sums[wave - 1][2][lane] = st.t;
#pragma unroll
        for (int i = 0; i < K; ++i) lists[wave - 1][i][lane] = list.k[i];
    }
    __syncthreads();
    if (wave) return;
    for (int w = 0; w < 3; ++w) {
        st.join(sums[w][0][lane], sums[w][1][lane], sums[w][2][lane]);
        key_t o[K ? K : 1];
#pragma unroll
        for (int i = 0; i < K; ++i) o[i] = lists[w][i][lane];
        list.join(o);
    }
    if (lane >= lanes || u >= a.U) return;
    if (K == 0 && a.splits == 1) {
        finish_sums<S>(a, b, u, there, st);
        return;
    }
    const size_t all = (size_t)a.B * a.U, at = (size_t)b * a.U + u;
    float *p = a.part + (size_t)split * 3 * all + at;
    p[0] = st.m;
    p[all] = st.s;
    p[2 * all] = st.t;
#pragma unroll
    for (int i = 0; i < K; ++i) a.part_keys[((size_t)split * K + i) * all + at] = list.k[i];
}

// How many of the first n lanes' `others` come before this lane's number (those behind the n-th are empty, up to a multiple of eight)
__device__ __forceinline__ int rank_of(key_t k, key_t others, int n)
{
    int rank = 0;
    for (int j = 0; j < n; j += 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) rank += of_lane(others, j + i) > k;
    return rank;
}

// A wavefront joins what `splits` workgroups found of a place.  A lane has one of their lists' entries, and finds its place in order by
// comparing it with all others; then one of the classes of the K eights that come first, read again, and the same.
template <typename S, int K>
__global__ __launch_bounds__(256) void scores_join_kernel(ScoresFwd a, int first)
{
    const int lane = threadIdx.x & 63, all = a.B * a.U;
    const int at = (first + (int)blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (at >= all) return;
    const int b = at / a.U, u = at - b * a.U;
    const bool there = u < length_in(a.len, b, a.U);
    Sums st;
    key_t mine = kEmpty;
    if (lane < a.splits) {
        const float *p = a.part + (size_t)lane * 3 * all + at;
        st.m = p[0];
        st.s = p[all];
        st.t = p[2 * (size_t)all];
    }
    if (K && lane < a.splits * K) mine = a.part_keys[(size_t)lane * all + at];
    for (int d = 1; d < a.splits; d <<= 1) st.join_lane(d);  // (to lane 0 all; lanes behind the last split have nothing to add)
    Lse lse = {0.f, 0.f};
    if (lane == 0) lse = finish_sums<S>(a, b, u, there, st);
    if constexpr (K > 0) {
        lse.m = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(lse.m)));
        lse.log_s = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(lse.log_s)));
        constexpr int kAll = K * G, kEach = (kAll + 63) / 64, kAtOnce = 64 / G;  // classes of all groups, of a lane; groups of 64 lanes
        const S *column = (const S *)a.scores + (size_t)b * a.V * a.U + u;
        key_t found[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) found[e] = kEmpty;
        if (there) {  // (uniform)
            int rank = rank_of(mine, mine, a.splits * K);
            if (mine == kEmpty) rank = 64;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                int c = kNone;
#pragma unroll
                for (int j = 0; j < kAtOnce && kAtOnce * e + j < K; ++j) {  // lanes G*j .. G*j+G-1: the group in place kAtOnce*e + j
                    const uint64_t has = __ballot(rank == kAtOnce * e + j);
                    const int id = has ? class_of(of_lane(mine, __builtin_ctzll(has))) : kNone;
                    c = lane / G == j ? id : c;
                }
                if (c != kNone && c + lane % G < a.V) found[e] = key_of(load_as_f32(column, (size_t)(c + lane % G) * a.U), c + lane % G);
            }
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            int rank = 0;
#pragma unroll
            for (int f = 0; f < kEach; ++f) rank += rank_of(found[e], found[f], kAll < 64 ? kAll : 64);
            if (there && found[e] != kEmpty && rank < a.top) {
                const size_t to = ((size_t)b * a.top + rank) * a.U + u;
                a.top_ids[to] = class_of(found[e]);
                a.top_logp[to] = lse.logq(score_of(found[e]));
            }
        }
        if (!there && lane < a.top) {
            const size_t to = ((size_t)b * a.top + lane) * a.U + u;
            a.top_ids[to] = -1;
            a.top_logp[to] = 0.f;
        }
    }
}

// The lists' length that serves `top`: of two a power
int list_of(int top) { return top <= 1 ? top : top <= 4 ? 4 : top <= 8 ? 8 : 16; }

struct Plan {
    int log_lanes, u_tiles, splits, per;
    size_t part_bytes, list_bytes;
};
Plan plan_of(int B, int V, int U, int top)
{
    Plan p = {};
    // places side by side: as many as there are, and of long rows 32 where the last 64 would be less than half full (32 items of 5000 classes, four
    // alternatives, both launches: 65 places 20 us against 22 with 64, 150 27 against 29, 280 41 against 42, 800 99 against 97; 4 x 150 places of 32000 classes
    // 26 against 32; 32 x 150 of 1000, eight alternatives, 21 against 22), but not from 2^24 places on: a lane's first class lies up to 16 rows behind a wavefront's, in bytes of 32 bits
    while (p.log_lanes < 6 && (1 << p.log_lanes) < U) ++p.log_lanes;
    if (U > 32 && U < 1 << 24 && U % 64 > 0 && U % 64 <= 32) p.log_lanes = 5;
    const int lanes = 1 << p.log_lanes, step = 64 >> p.log_lanes, list = list_of(top);
    p.u_tiles = (U + lanes - 1) / lanes;
    // four workgroups a CU (32 items of 5000 classes, both launches: 65 places 20.0 us, with two a CU 19.7, 90 21 and 20, 150 27 and 28, 280 41 and 53), but a wavefront has a whole round of classes to do, and a
    // wavefront joins all lists of a place
    const long long groups = (long long)B * p.u_tiles;
    long long splits = 1024 / groups;
    const long long most = (V + 4LL * step * kAhead - 1) / (4LL * step * kAhead), joined = 64 / (list ? list : 1);
    if (splits > most) splits = most;
    if (splits > joined) splits = joined;
    if (splits < 1) splits = 1;
    const long long whole = kAhead * step, per = ((V + 4 * splits - 1) / (4 * splits) + whole - 1) / whole * whole;  // whole rounds of a wavefront
    p.per = (int)(per < V ? per : (V + kAhead - 1) / kAhead * kAhead);
    p.splits = (int)((V + 4LL * p.per - 1) / (4LL * p.per));
    const size_t all = (size_t)B * U;
    const bool parts = p.splits > 1 || list;
    p.part_bytes = parts ? align_up((size_t)p.splits * 3 * all * 4, 256) : 0;
    p.list_bytes = align_up((size_t)p.splits * list * all * sizeof(key_t), 256);
    return p;
}

template <typename S, int K>
hipError_t run_list(const ScoresFwd &a, hipStream_t s)
{
    scores_fwd_kernel<S, K><<<dim3((unsigned)a.B * a.u_tiles * a.splits), dim3(256), 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (K == 0 && a.splits == 1)) return e;
    return in_launches(((size_t)a.B * a.U + 3) / 4, [&](unsigned n, int first) { scores_join_kernel<S, K><<<dim3(n), dim3(256), 0, s>>>(a, first); });
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

// The forward pass's log-sum-exp is rounded to float: up to this magnitude a probability is off by 2^-13 of itself for it.  Beyond, to where nothing is left
// of the logarithm of the sum, a workgroup adds up exp(z - lse) over the classes itself for its places (16 x 333 places of 5000 classes, float32: 42 us,
// all of them such places 345).
constexpr float kCoarse = 4096.f;

struct Place {
    float lse, rest, entropy, dl, dh;  // rest: what lse lacks
    int target;
    bool there;
    __device__ __forceinline__ bool coarse() const { return there && fabsf(lse) > kCoarse; }
};
__device__ __forceinline__ Place place_of(const ScoresBwd &a, int b, int u, int len)
{
    Place p;
    const size_t at = (size_t)b * a.U + u;
    p.lse = a.lse[at];
    p.rest = 0.f;
    p.there = u < len && p.lse != -INFINITY;
    p.target = p.there && a.dlogp ? a.targets.at(at, a.V) : -1;
    p.dl = p.target >= 0 ? a.dlogp[at] : 0.f;
    p.dh = a.dentropy ? a.dentropy[at] : 0.f;
    p.entropy = a.dentropy ? a.entropy[at] : 0.f;
    return p;
}
__device__ __forceinline__ float gradient(const Place &p, float z, int c)
{
    const float x = (z - p.lse) - p.rest, q = __builtin_amdgcn_exp2f(x * kLog2e);
    const float g = p.dl * ((c == p.target ? 1.f : 0.f) - q) - p.dh * q * (fmaxf(x, -1e30f) + p.entropy);
    return p.there ? g : 0.f;
}

// Rows of eight places at least: the last group of a row begins eight before its end, and what two groups share is made twice.
template <typename S, typename G>
__global__ __launch_bounds__(256) void scores_bwd_kernel(ScoresBwd a)
{
    const int gt = blockIdx.x % a.group_tiles, rest = blockIdx.x / a.group_tiles, tiles = (a.V + a.rows * a.rounds - 1) / (a.rows * a.rounds);
    const int vt = rest % tiles, b = rest / tiles;
    const int r = threadIdx.x / a.side, g = threadIdx.x - r * a.side, group = gt * a.side + g;
    const bool mine = r < a.rows && group < a.groups;
    const int u = min(min(group, a.groups - 1) * 8, a.U - 8), len = length_in(a.len, b, a.U);
    Place p[8];
    bool coarse = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        p[j] = place_of(a, b, u + j, len);
        coarse |= p[j].coarse();
    }
    if (__syncthreads_or(mine && coarse)) {
        __shared__ float sums[256][8];
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int c = r; mine && c < a.V; c += a.rows) {
            float z[8];
            load8((const S *)a.scores + ((size_t)b * a.V + c) * a.U + u, 8, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += __builtin_amdgcn_exp2f((z[j] - p[j].lse) * kLog2e);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[threadIdx.x][j] = s[j];
        __syncthreads();
        if (mine) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float all = 0.f;
                for (int i = 0; i < a.rows; ++i) all += sums[i * a.side + g][j];
                if (p[j].coarse()) p[j].rest = __builtin_amdgcn_logf(all) * kLn2;
            }
        }
    }
    if (!mine) return;
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
    const int len = length_in(a.len, b, a.U), n = (int)max(min(item - i0, 8LL), 0LL);
    float z[8], g[8];
    load8((const S *)a.scores + (size_t)b * item + (n ? i0 : 0), n, z);
    __shared__ float rests[8];
    const bool any = __syncthreads_or(threadIdx.x < a.U && place_of(a, b, threadIdx.x, len).coarse());
    if (any) {
        __shared__ float sums[4];
        for (int u = 0; u < a.U; ++u) {
            const Place p = place_of(a, b, u, len);
            float s = 0.f;
            if (p.coarse()) {  // (uniform)
                for (int c = threadIdx.x; c < a.V; c += 256)
                    s += __builtin_amdgcn_exp2f((load_as_f32((const S *)a.scores, (size_t)b * item + (size_t)c * a.U + u) - p.lse) * kLog2e);
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
            }
            if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
            __syncthreads();
            if (threadIdx.x == 0) rests[u] = p.coarse() ? __builtin_amdgcn_logf(sums[0] + sums[1] + sums[2] + sums[3]) * kLn2 : 0.f;
            __syncthreads();
        }
    }
    if (!n) return;
    int c = (int)((uint32_t)i0 / (uint32_t)a.U), u = (int)i0 - c * a.U;  // (an item has fewer than 2^31)
    auto place = [&]() {
        Place p = place_of(a, b, u, len);
        if (any) p.rest = rests[u];
        return p;
    };
    Place p = place();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] = gradient(p, z[j], c);
        if (++u == a.U) {
            u = 0;
            ++c;
        }
        if (a.U > 1) p = place();
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
    // two workgroups a CU: what a thread reads of its places takes as long as some rounds (16 x 5000 x 333: 16 rounds 45 us, 32 37)
    const long long rounds = ((long long)a.V * a.B * a.group_tiles / a.rows + 511) / 512;
    a.rounds = (int)((rounds < 4 ? 4 : rounds > 64 ? 64 : rounds) + 3) / 4 * 4;
    const long long tiles = (a.V + a.rows * a.rounds - 1) / (a.rows * a.rounds);
    scores_bwd_kernel<S, G><<<dim3((unsigned)(tiles * a.group_tiles * a.B)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

int check(int B, int V, int U, int dtype)
{
    if (B <= 0 || V <= 0 || U <= 0 || !known_dtype(dtype)) return NM_ERR_BAD_ARG;
    const long long most = (1LL << 31) - 1;
    if ((long long)B * V > most / U || V > most - (1 << 16) || U > 1 << 29) return NM_ERR_UNSUPPORTED;  // (classes behind the last one are counted too)
    // the grids, below 2^32 work items (the join has several where need be): a workgroup of the backward pass has 2048 elements, or one item's rest
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
    return p.part_bytes + p.list_bytes;
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
    if (workspace_missing(workspace, workspace_bytes, p.part_bytes + p.list_bytes)) return NM_ERR_WORKSPACE;
    ScoresFwd a = {};
    a.B = B; a.V = V; a.U = U;
    a.scores = scores;
    a.targets = {targets, target_bytes == 8};
    a.len = lengths;
    a.logp = logp; a.entropy = entropy; a.lse = lse; a.top_logp = top_logp; a.top_ids = top_ids;
    a.top = top;
    a.log_lanes = p.log_lanes; a.u_tiles = p.u_tiles; a.splits = p.splits; a.per = p.per;
    a.part = (float *)workspace;
    a.part_keys = (uint64_t *)((char *)workspace + p.part_bytes);
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
