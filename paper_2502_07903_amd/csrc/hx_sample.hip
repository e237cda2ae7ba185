// hx_sample.hip -- one draw from every row of scores: temperature, top-k, top-p, min-p (hx_sample).
//
// Weights are w = exp((x - m) / T) in binary64, m the row's largest score (Exponent).  A row is read in
// groups of 16 bytes (Row); a region is a run of groups that one wavefront walks, 64 groups at a time, and
// the regions of a row follow each other in index order.  A draw is then: the regions' weights, their sum S
// in order, the first region at which they pass t = u S, and the first entry of that region (Pick).
//
// Without filters (all_kernel) the row is read once: a wavefront keeps its own largest score so far, sums
// weights relative to it, and scales the sums when it grows (the ratio of two maxima is an exponential of
// their difference); the regions' sums meet at the end.  Few rows are split over several workgroups, and a
// second launch (finish_kernel) joins them.
//
// With filters (cut_kernel, a workgroup per row): all three keep a prefix of the order (descending score,
// ascending index), so the kept set is everything up to one entry's place in it.  That entry is found by
// counting, for top-k, and by adding whole-number weights, for top-p (no order of addition changes their
// sums, and each bin has a unit of its own, as fine as 64 bits allow for weights of its size), in 1,024 bins
// of the distance from m.  The entries of the bin in which the cut falls, if at most kList, go to a list in
// LDS, which is split by the bits of their places until a wavefront can rank the rest; a longer bin is split
// again by the keys' bits over the row.  min-p's bound is a search over the keys.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "hx_internal.h"

namespace hx {
namespace {

using u64 = unsigned long long;
using u128 = unsigned __int128;

// ------------------------------------------------------------------ scores

// A score's 32-bit key has the scores' order; V: entries of 16 bytes; X: a score in registers.
template <int kType>
struct Scores;
template <>
struct Scores<HX_SCORE_I32> {
    using T = int32_t;
    using X = int32_t;
    static constexpr int V = 4;
    static constexpr X kMasked = INT32_MIN, kLeast = INT32_MIN + 1;  // the lowest score that is none
    static __device__ __forceinline__ X clean(X x) { return x; }
    static __device__ __forceinline__ X widen(T x) { return x; }
    static __device__ __forceinline__ void unpack(const uint4& q, X (&v)[V]) {
        v[0] = (int32_t)q.x, v[1] = (int32_t)q.y, v[2] = (int32_t)q.z, v[3] = (int32_t)q.w;
    }
    static __device__ __forceinline__ X larger(X a, X b) { return a > b ? a : b; }
    static __device__ __forceinline__ uint32_t key(X x) { return (uint32_t)x ^ 0x80000000u; }
    static __device__ __forceinline__ X value(uint32_t k) { return (int32_t)(k ^ 0x80000000u); }
    static __device__ __forceinline__ X value_up(uint32_t k) { return value(k); }
    static __device__ __forceinline__ float below(X m, X x) { return (float)((uint32_t)m - (uint32_t)x); }
};
// Floats: NaN is masked (clean makes it -inf; unpack leaves it); keys are sign and magnitude in two's-complement
// order, -0 as +0.
struct FloatScores {
    using X = float;
    static constexpr X kMasked = -INFINITY, kLeast = -FLT_MAX;
    static __device__ __forceinline__ X clean(float x) { return x > -INFINITY ? x : -INFINITY; }
    static __device__ __forceinline__ X larger(X a, X b) { return fmaxf(a, b); }
    static __device__ __forceinline__ uint32_t key(X x) {
        const uint32_t b = __float_as_uint(x + 0.0f);
        return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    }
    static __device__ __forceinline__ X value(uint32_t k) {
        return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
    }
    // The largest score whose key is at most k: the key of -0, which no score has, would compare equal to +0.
    static __device__ __forceinline__ X value_up(uint32_t k) { return value(k == 0x7FFFFFFFu ? k - 1 : k); }
    static __device__ __forceinline__ float below(X m, X x) { return m - x; }
};
template <>
struct Scores<HX_SCORE_F32> : FloatScores {
    using T = float;
    static constexpr int V = 4;
    static __device__ __forceinline__ X widen(T x) { return clean(x); }
    static __device__ __forceinline__ void unpack(const uint4& q, X (&v)[V]) {
        v[0] = __uint_as_float(q.x), v[1] = __uint_as_float(q.y);
        v[2] = __uint_as_float(q.z), v[3] = __uint_as_float(q.w);
    }
};
template <>
struct Scores<HX_SCORE_F16> : FloatScores {
    using T = uint16_t;
    static constexpr int V = 8;
    static __device__ __forceinline__ X raw(T x) {
        _Float16 h;
        __builtin_memcpy(&h, &x, 2);
        return (float)h;
    }
    static __device__ __forceinline__ X widen(T x) { return clean(raw(x)); }
    static __device__ __forceinline__ void unpack(const uint4& q, X (&v)[V]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = raw((T)w[i]), v[2 * i + 1] = raw((T)(w[i] >> 16));
    }
};
template <>
struct Scores<HX_SCORE_BF16> : FloatScores {
    using T = uint16_t;
    static constexpr int V = 8;
    static __device__ __forceinline__ X widen(T x) { return clean(__uint_as_float((uint32_t)x << 16)); }
    static __device__ __forceinline__ void unpack(const uint4& q, X (&v)[V]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
};

// w = exp((x - m) / T) as 2^(d c), d = x - m, c = log2(e) / T: d c = n + f with n whole and |f| <= 1/2, and
// 2^f = 1 + f q(f), q the interpolation of (2^f - 1) / f at the ten Chebyshev nodes of [-1/2, 1/2] (computed
// in 80 digits; 2^f is off by 6e-16 at most).  Masked scores (-inf) end at d c = -2000, whose weight is 0.
// n comes from adding 1.5 2^52, which leaves it in the sum's low bits.  18 binary64 operations; several scores
// are worked on side by side, step by step, since one's steps depend on each other.
struct Exponent {
    double m, c, least;  // least: d where d c = -2000
    double lead;         // q's first coefficient, kept in vector registers: an fma reads one scalar operand
    int infinite;        // m = +inf: entries equal to it have d = 0
    template <class X>
    __device__ __forceinline__ void set(X top, double scale) {
        m = (double)top;
        c = scale;
        infinite = __builtin_amdgcn_readfirstlane(m > DBL_MAX);
        if (infinite) m = 0x1p200;  // every finite score is infinitely far below
        least = -2000.0 / scale;
        lead = 0x1.e5e9f548e5725p-28;
        asm("" : "+v"(lead));
    }
    // kAbove: scores may be above m, to weights of infinity.
    template <bool kAbove = false, int N, class X>
    __device__ __forceinline__ void weights(const X (&x)[N], double (&w)[N]) const {
        constexpr int M = N < 4 ? N : 4;  // side by side
#pragma unroll
        for (int b = 0; b < N; b += M) some_weights<kAbove, M>(x + b, w + b);
    }
    template <bool kAbove, int M, class X>
    __device__ __forceinline__ void some_weights(const X* x, double* w) const {
        double d[M], t[M], q[M];
#pragma unroll
        for (int e = 0; e < M; ++e) d[e] = fmax((double)x[e] - m, least);
        if (kAbove) {
#pragma unroll
            for (int e = 0; e < M; ++e) d[e] = fmin(d[e], -least);
        }
        if (__builtin_amdgcn_readfirstlane(infinite)) {  // the same in every lane: a branch, not a mask
#pragma unroll
            for (int e = 0; e < M; ++e) d[e] = fmin(d[e], 0.0);
        }
#pragma unroll
        for (int e = 0; e < M; ++e) t[e] = fma(d[e], c, 0x1.8p52);
#pragma unroll
        for (int e = 0; e < M; ++e) d[e] = fma(d[e], c, -(t[e] - 0x1.8p52));
        constexpr double k[9] = {0x1.b6571de2f2351p-24, 0x1.62bfe46117445p-20, 0x1.ffcb76789860fp-17,
                                 0x1.4309130378460p-13, 0x1.5d87fe908f88ap-10, 0x1.3b2ab6fba385fp-7,
                                 0x1.c6b08d7044119p-5,  0x1.ebfbdff82c590p-3,  0x1.62e42fefa39f7p-1};
#pragma unroll
        for (int e = 0; e < M; ++e) q[e] = lead;
#pragma unroll
        for (int i = 0; i < 9; ++i) {
#pragma unroll
            for (int e = 0; e < M; ++e) q[e] = fma(q[e], d[e], k[i]);
        }
#pragma unroll
        for (int e = 0; e < M; ++e) {
            w[e] = ldexp(fma(q[e], d[e], 1.0), (int)(uint32_t)__double_as_longlong(t[e]));
            if (std::is_same<X, int32_t>::value) w[e] = x[e] == (X)INT32_MIN ? 0.0 : w[e];
        }
    }
    template <class X>
    __device__ __forceinline__ double weight(X x) const {
        const X one[1] = {x};
        double w[1];
        weights(one, w);
        return w[0];
    }
};

// ------------------------------------------------------------------ a row

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

__device__ const uint4 kNoEntries = {};
// Said to be global memory: a load that could be of LDS waits for both kinds.
typedef uint32_t Words __attribute__((ext_vector_type(4)));
using Group = const __attribute__((address_space(1))) Words;

template <class S>
struct Row {
    static constexpr int V = S::V;
    using X = typename S::X;
    const typename S::T* x;
    int n, lead;  // entries; those of the first 16 bytes that precede the row
    int groups;   // of 16 aligned bytes (n is at most 2^30: indices of groups and entries fit 32 bits)
    int whole_lo, whole_hi;  // groups [whole_lo, whole_hi] lie within the row
    Group* from;             // group 0; kNoEntries for a row without a whole group
    __device__ __forceinline__ Row(const SampleArgs& a, int64_t r) {
        x = static_cast<const typename S::T*>(a.data) + r * a.stride;
        n = a.N;
        lead = (int)(((uintptr_t)x & 15) / sizeof(typename S::T));
        groups = (n + lead + V - 1) / V;
        whole_lo = lead > 0 ? 1 : 0;
        whole_hi = (n + lead) / V - 1;
        from = (Group*)((uintptr_t)x & ~(uintptr_t)15);
        if (whole_hi < whole_lo) from = (Group*)(uintptr_t)&kNoEntries;
    }
    __device__ __forceinline__ int first(int g) const { return g * V - lead; }  // index of its first entry
    // The 16 bytes of group g, or of the whole group nearest to it: a load that no branch surrounds, so that it can be
    // in flight while the group before it is worked on.
    __device__ __forceinline__ uint4 fetch(int g) const {
        const int w = g > whole_hi ? whole_hi : g;
        const auto q = from[whole_hi < whole_lo ? 0 : w < whole_lo ? whole_lo : w];
        return uint4{q.x, q.y, q.z, q.w};
    }
    // Entries of group g, fetched as q, of a region that ends at hi; those outside the row and the region are masked,
    // and not read.
    template <bool kClean = true>
    __device__ __forceinline__ void entries(int g, int hi, const uint4& q, X (&v)[V]) const {
        S::unpack(q, v);
        if (kClean) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = S::clean(v[e]);
        }
        if (g >= hi || g < whole_lo || g > whole_hi) {
            const int i = first(g);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = g < hi && i + e >= 0 && i + e < n ? S::widen(x[i + e]) : S::kMasked;
        }
    }
    // body(entries, index of the first) for a wavefront's groups [lo, hi), 64 at a time and all lanes together (masked
    // entries where a lane has no group).  The next kAhead times 64 groups are fetched meanwhile: one where the body is
    // long, four where the loads' latency would be the time.  Without kClean, NaN stays.
    template <int kAhead, bool kClean = true, class B>
    __device__ __forceinline__ void walk(int lo, int hi, B body) const {
        const int lane = threadIdx.x & 63;
        uint4 next[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) next[k] = fetch(lo + 64 * k + lane);
        for (int g = lo + lane; g - lane < hi; g += 64 * kAhead) {
            uint4 q[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                q[k] = next[k];
                next[k] = fetch(g + 64 * (kAhead + k));
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (k > 0 && g - lane + 64 * k >= hi) continue;
                X v[V];
                entries<kClean>(g + 64 * k, hi, q[k], v);
                body(v, first(g + 64 * k));
            }
        }
    }
};

// Groups [lo, hi) of region k of a row's `regions`: whole wavefronts' worth, in index order.
struct Region {
    int lo, hi;
    __device__ __forceinline__ Region(int groups, int regions, int k) {
        const int per = (groups + regions * 64 - 1) / (regions * 64) * 64;
        lo = k < (groups + per - 1) / per ? per * k : groups;
        hi = groups - lo > per ? lo + per : groups;
    }
};

struct Parameters {
    float T, p, q;
    int32_t k;
    bool bad;
    __device__ __forceinline__ Parameters(const SampleArgs& a, int64_t r) {
        T = a.temperature ? a.temperature[r] : 1.0f;
        k = a.top_k ? a.top_k[r] : 0;
        p = a.top_p ? a.top_p[r] : 1.0f;
        q = a.min_p ? a.min_p[r] : 0.0f;
        bad = !(T >= 0.0f) || !(T <= FLT_MAX) || isnan(p) || isnan(q);
    }
    __device__ __forceinline__ double scale() const { return 0x1.71547652b82fep+0 / (double)T; }  // log2(e) / T
};

__device__ __forceinline__ void write_nothing(const SampleArgs& a, int64_t r) {
    a.pick[r] = -1;
    if (a.logp) a.logp[r] = -INFINITY;
    if (a.kept) a.kept[r] = 0;
}

// ------------------------------------------------------------------ wavefront sums

// Sums and maxima over the lanes by data-parallel moves (rows of 16 lanes shifted by 1, 2, 4 and 8, then the rows'
// last lanes broadcast on), which take a tenth of the time of moves through LDS.  A lane without a source gets `idle`.
template <int kControl, int kRows, class A>
__device__ __forceinline__ A move(A v, A idle) {
    static_assert(sizeof(A) == 4 || sizeof(A) == 8, "whole registers");
    int from[sizeof(A) / 4], none[sizeof(A) / 4], to[sizeof(A) / 4];
    __builtin_memcpy(from, &v, sizeof(A));
    __builtin_memcpy(none, &idle, sizeof(A));
#pragma unroll
    for (int k = 0; k < (int)sizeof(A) / 4; ++k)
        to[k] = __builtin_amdgcn_update_dpp(none[k], from[k], kControl, kRows, 0xf, false);
    A r;
    __builtin_memcpy(&r, to, sizeof(A));
    return r;
}
template <class A>
__device__ __forceinline__ A last_lane(A v) {
    int w[sizeof(A) / 4];
    __builtin_memcpy(w, &v, sizeof(A));
#pragma unroll
    for (int k = 0; k < (int)sizeof(A) / 4; ++k) w[k] = __builtin_amdgcn_readlane(w[k], 63);
    __builtin_memcpy(&v, w, sizeof(A));
    return v;
}
// A value that all lanes have, to scalar registers.
template <class A>
__device__ __forceinline__ A scalar(A v) {
    int w[sizeof(A) / 4];
    __builtin_memcpy(w, &v, sizeof(A));
#pragma unroll
    for (int k = 0; k < (int)sizeof(A) / 4; ++k) w[k] = __builtin_amdgcn_readfirstlane(w[k]);
    __builtin_memcpy(&v, w, sizeof(A));
    return v;
}
template <class A>
__device__ __forceinline__ A wave_scan(A v) {  // inclusive
    v += move<0x111, 0xf>(v, A(0));
    v += move<0x112, 0xf>(v, A(0));
    v += move<0x114, 0xf>(v, A(0));
    v += move<0x118, 0xf>(v, A(0));
    v += move<0x142, 0xa>(v, A(0));
    v += move<0x143, 0xc>(v, A(0));
    return v;
}
template <class A>
__device__ __forceinline__ A wave_sum(A v) {
    return last_lane(wave_scan(v));
}
// The sum of the first `number` words of x, at most eight, each lane of a wavefront reading one.
template <class A>
__device__ __forceinline__ A sum_of_first(const A* x, int number) {
    const int lane = threadIdx.x & 63;
    A v = lane < number ? x[lane] : A(0);
    v += move<0x111, 0xf>(v, A(0));
    v += move<0x112, 0xf>(v, A(0));
    v += move<0x114, 0xf>(v, A(0));
    int w[sizeof(A) / 4];
    __builtin_memcpy(w, &v, sizeof(A));
#pragma unroll
    for (int k = 0; k < (int)sizeof(A) / 4; ++k) w[k] = __builtin_amdgcn_readlane(w[k], 7);
    __builtin_memcpy(&v, w, sizeof(A));
    return v;
}
template <class A>
__device__ __forceinline__ A wave_max(A v) {
    const auto larger = [](A a, A b) { return b > a ? b : a; };
    v = larger(v, move<0x111, 0xf>(v, v));
    v = larger(v, move<0x112, 0xf>(v, v));
    v = larger(v, move<0x114, 0xf>(v, v));
    v = larger(v, move<0x118, 0xf>(v, v));
    v = larger(v, move<0x142, 0xa>(v, v));
    v = larger(v, move<0x143, 0xc>(v, v));
    return last_lane(v);
}

// ------------------------------------------------------------------ the draw

// What a region adds: the weight of its entries, relative to the score of `key`, and their number.
struct Part {
    double weight;
    uint32_t key, count;
};

// The end of a row's draw: the entry found, the kept entries' weight and number.
struct Draw {
    const SampleArgs& a;
    int64_t r;
    double m, T, sum;
    u64 kept;
    __device__ __forceinline__ void write(int index, double v) const {
        a.pick[r] = index;
        if (a.kept) a.kept[r] = (int32_t)kept;
        if (a.logp) a.logp[r] = T == 0.0 ? 0.0f : (float)((v == m ? 0.0 : (v - m) / T) - log(sum));
    }
};

template <int kLanes>
struct PickShared {
    double wave[kLanes / 64];
    int found[kLanes / 64], last[kLanes / 64];
    double before;
    int target;
};

// The region in which the draw u falls, given each lane's region's weight (lanes in index order, at most one region a
// lane, some weight above 0): the weight of all to *sum, of the regions before it to *before.  one: the first region
// with weight.
template <int kLanes>
__device__ int target_region(double mine, double u, bool one, double* sum, double* before, PickShared<kLanes>& sh) {
    constexpr int kWaves = kLanes / 64;
    const int wave = wave_index(), lane = threadIdx.x & 63;
    const double scan = wave_scan(mine);
    const u64 has = __ballot(mine > 0.0);
    if (lane == 63) {
        sh.wave[wave] = scan;
        sh.last[wave] = has ? wave * 64 + 63 - __clzll(has) : -1;
    }
    __syncthreads();
    double ahead = 0.0, all = 0.0;
    int last = 0;
    for (int k = 0; k < kWaves; ++k) {
        if (k == wave) ahead = all;
        all += sh.wave[k];
        last = sh.last[k] >= 0 ? sh.last[k] : last;
    }
    const double t = one ? 0.0 : u * all;
    const u64 past = __ballot(mine > 0.0 && ahead + scan > t);
    if (lane == 0) sh.found[wave] = past ? wave * 64 + __ffsll(past) - 1 : kLanes;
    __syncthreads();
    int target = last;  // where rounding leaves t unreached
    for (int k = kWaves - 1; k >= 0; --k) target = sh.found[k] < kLanes ? sh.found[k] : target;
    if ((int)threadIdx.x == target) sh.before = ahead + (scan - mine);
    __syncthreads();
    *sum = all;
    *before = sh.before;
    return target;
}

// The first entry of groups [lo, hi) up to which the weights sum to more than t, or the last one with weight
// (which rounding can leave as the only choice), to the row's outputs; false if none has weight.  weights(entries, index
// of the first, w): 0 for entries that are not kept.  Every lane of the workgroup calls it.
template <int kLanes, class S, class W>
__device__ bool pick_in_region(const Row<S>& row, const Region& g, double t, const Draw& draw, W weights,
                               PickShared<kLanes>& sh) {
    constexpr int kWaves = kLanes / 64;
    const int wave = wave_index(), lane = threadIdx.x & 63;
    double run = 0.0;
    int last = -1;
    for (int g0 = g.lo; g0 < g.hi; g0 += kLanes) {
        const int at = g0 + (int)threadIdx.x;
        typename S::X v[S::V];
        double w[S::V], mine = 0.0;
        int own = -1;
        row.entries(at, g.hi, row.fetch(at), v);
        weights(v, row.first(at), w);
#pragma unroll
        for (int e = 0; e < S::V; ++e) {
            mine += w[e];
            if (w[e] > 0.0) own = e;
        }
        const double scan = wave_scan(mine);
        const u64 has = __ballot(own >= 0);
        const int top = has ? 63 - __clzll(has) : 0;
        const int top_e = __shfl(own, top, 64);
        if (lane == 63) {
            sh.wave[wave] = scan;
            sh.last[wave] = has ? row.first(g0 + wave * 64 + top) + top_e : -1;
        }
        __syncthreads();
        for (int k = 0; k < wave; ++k) run += sh.wave[k];
        double sum = run + (scan - mine);
        int e_found = -1;
        if (own >= 0) {
#pragma unroll
            for (int e = 0; e < S::V; ++e) {
                sum += w[e];
                if (e_found < 0 && w[e] > 0.0 && sum > t) e_found = e;
            }
        }
        for (int k = wave; k < kWaves; ++k) run += sh.wave[k];
        const u64 past = __ballot(e_found >= 0);
        const int first = past ? __ffsll(past) - 1 : 64;
        if (lane == 0) sh.found[wave] = first;
        __syncthreads();
        int hit = kWaves;
        for (int k = kWaves - 1; k >= 0; --k) {
            if (sh.found[k] < 64) hit = k;
        }
        for (int k = 0; k < kWaves; ++k)
            if (sh.last[k] >= 0) last = sh.last[k];
        if (hit < kWaves) {
            if (wave == hit && lane == first) {
                double value = 0.0;
#pragma unroll
                for (int e = 0; e < S::V; ++e)
                    if (e == e_found) value = (double)v[e];
                draw.write(row.first(at) + e_found, value);
            }
            return true;
        }
        __syncthreads();
    }
    if (last < 0) return false;
    if (threadIdx.x == 0) draw.write(last, (double)S::widen(row.x[last]));
    return true;
}

// ------------------------------------------------------------------ no filters

constexpr int kAllLanes = 256, kAllWaves = kAllLanes / 64;
// Regions of a wavefront where the workgroup has the whole row, since the draw reads one of them again; a short row's
// is small as it is.
constexpr int kAllRegions = 8, kShortRow = 8192;
constexpr int kFinishLanes = 256;
constexpr int kMaxSplits = 64;

// The largest of the lanes' entries.  Cleaned first: of a signalling NaN and a number the maximum is NaN.
template <class S>
__device__ __forceinline__ typename S::X wave_most(const typename S::X (&v)[S::V]) {
    typename S::X most = S::kMasked;
#pragma unroll
    for (int e = 0; e < S::V; ++e) most = S::larger(most, S::clean(v[e]));
    return wave_max(most);
}

// Weights of a wavefront's regions k0 .. k0 + n - 1 in one pass, to parts: relative to one of its own scores (Part's
// key), the largest of the first 64 groups that hold any, and a larger one from where the weights pass 2^500.
template <class S>
__device__ void sum_regions(const Row<S>& row, int regions, int k0, int n, const Parameters& par, Part* parts) {
    using X = typename S::X;
    const Region first(row.groups, regions, k0), last(row.groups, regions, k0 + n - 1);
    const int per = first.hi - first.lo, lane = threadIdx.x & 63;
    const bool greedy = par.T == 0.0f;
    const double scale = greedy ? 1.0 : par.scale();
    X ref = S::kMasked;
    Exponent ex;
    ex.set(ref, scale);
    double sum = 0.0;
    uint32_t count = 0;  // of the wavefront
    int k = 0, end = first.hi, g0 = first.lo;
    const auto close = [&] {  // region k is done
        if (greedy) ref = wave_max(ref);
        const double total = greedy ? 1.0 : wave_sum(sum);
        if (lane == 0) parts[k] = Part{total, S::key(ref), count};
        if (greedy) ref = S::kMasked;
        sum = 0.0;
        count = 0;
        ++k;
        end += per;
    };
    row.template walk<1, false>(first.lo, last.hi, [&](const X (&v)[S::V], int) {
        if (g0 >= end) close();
        g0 += 64;
#pragma unroll
        for (int e = 0; e < S::V; ++e) count += __popcll(__ballot(v[e] >= S::kLeast));  // false for NaN
        if (greedy) {
#pragma unroll
            for (int e = 0; e < S::V; ++e) ref = v[e] > ref ? v[e] : ref;
            return;
        }
        if (ref == S::kMasked) {
            ref = wave_most<S>(v);
            if (ref == S::kMasked) return;
            ex.set(ref, scale);
        }
        double w[S::V], here = 0.0;
        ex.template weights<true>(v, w);
#pragma unroll
        for (int e = 0; e < S::V; ++e) here += w[e];
        if (__any(!(here < 0x1p500))) {
            // the earlier regions' parts keep their own score
            const X old = ref;
            ref = wave_most<S>(v);
            ex.set(ref, scale);
            sum *= ex.weight(old);
            ex.weights(v, w);
            here = 0.0;
#pragma unroll
            for (int e = 0; e < S::V; ++e) here += w[e];
        }
        sum += here;
    });
    while (k < n) close();
}

// The row's draw from its regions' parts, at most kLanes.
template <int kLanes, class S>
__device__ void finish_row(const SampleArgs& a, int64_t r, const Row<S>& row, const Parameters& par, const Part* parts,
                           int regions, PickShared<kLanes>& sh) {
    using X = typename S::X;
    uint32_t top_key = 0;
    u64 count = 0;
    for (int k = 0; k < regions; ++k) {
        top_key = parts[k].key > top_key ? parts[k].key : top_key;
        count += parts[k].count;
    }
    if (count == 0 || par.bad) {
        if (threadIdx.x == 0) write_nothing(a, r);
        return;
    }
    const X top = S::value(top_key);
    if (par.T == 0.0f) {
        int first = 0;
        while (parts[first].key != top_key) ++first;
        pick_in_region<kLanes>(
            row, Region(row.groups, regions, first), 0.5, Draw{a, r, (double)top, 0.0, 1.0, 1},
            [&](const X (&v)[S::V], int, double (&w)[S::V]) {
#pragma unroll
                for (int e = 0; e < S::V; ++e) w[e] = v[e] == top ? 1.0 : 0.0;
            },
            sh);
        return;
    }
    Exponent ex;
    double mine = 0.0;
    if ((int)threadIdx.x < regions) {
        // by half the exponent twice: a part's weight can be up to 2^524, and its score's 0
        const Part p = parts[threadIdx.x];
        ex.set(top, 0.5 * par.scale());
        const double half = p.count ? ex.weight(S::value(p.key)) : 0.0;
        mine = p.weight * half * half;
    }
    ex.set(top, par.scale());
    const double u = (double)(a.rnd[r] >> 11) * 0x1p-53;
    double sum, before;
    int target = target_region<kLanes>(mine, u, false, &sum, &before, sh);
    const Draw draw{a, r, (double)top, (double)par.T, sum, count};
    const auto weights = [&](const X (&v)[S::V], int, double (&w)[S::V]) { ex.weights(v, w); };
    if (pick_in_region<kLanes>(row, Region(row.groups, regions, target), u * sum - before, draw, weights, sh)) return;
    // Entries that weigh 0 each and something together, where the draw is 0 or an earlier region's end but for rounding:
    // the next region with weight, or behind the last the last entry of a region whose entries do weigh something.
    double all, ahead;
    while (__syncthreads_or((int)threadIdx.x > target && mine > 0.0)) {
        target = target_region<kLanes>((int)threadIdx.x > target ? mine : 0.0, 0.0, true, &all, &ahead, sh);
        if (pick_in_region<kLanes>(row, Region(row.groups, regions, target), 0.0, draw, weights, sh)) return;
    }
    target = target_region<kLanes>(mine >= 0x1p-900 ? mine : 0.0, 2.0, false, &all, &ahead, sh);
    pick_in_region<kLanes>(row, Region(row.groups, regions, target), INFINITY, draw, weights, sh);
}

// A row's split s of `splits`: workgroup r * splits + s.  With one split the row ends here.
// Bound by the exponentials' binary64 operations, 26 vector instructions an entry in all: 1,024 rows of 131,072 bf16
// 112 us a call, 2.4 TB/s, of which reading the 268 MB once is 52 us; a row of 256 i32 4.4 us, the launch.
template <int kType>
__global__ void __launch_bounds__(kAllLanes) all_kernel(SampleArgs a, int splits, Part* parts) {
    using S = Scores<kType>;
    constexpr int kRegions = kAllWaves * kAllRegions;
    __shared__ Part own[kRegions];
    __shared__ PickShared<kAllLanes> sh;
    const int64_t r = a.row0 + blockIdx.x / splits;
    const int s = blockIdx.x % splits, wave = wave_index();
    const Row<S> row(a, r);
    const Parameters par(a, r);
    if (splits > 1) {
        sum_regions(row, splits * kAllWaves, s * kAllWaves + wave, 1, par, parts + (r * splits + s) * kAllWaves + wave);
        return;
    }
    const int each = a.N <= kShortRow ? 1 : kAllRegions;
    sum_regions(row, kAllWaves * each, wave * each, each, par, own + wave * each);
    __syncthreads();
    finish_row<kAllLanes>(a, r, row, par, own, kAllWaves * each, sh);
}

template <int kType>
__global__ void __launch_bounds__(kFinishLanes) finish_kernel(SampleArgs a, int splits, const Part* parts) {
    using S = Scores<kType>;
    __shared__ Part own[kMaxSplits * kAllWaves];
    __shared__ PickShared<kFinishLanes> sh;
    const int64_t r = a.row0 + blockIdx.x;
    const int regions = splits * kAllWaves;
    for (int k = threadIdx.x; k < regions; k += kFinishLanes) own[k] = parts[r * regions + k];
    __syncthreads();
    finish_row<kFinishLanes>(a, r, Row<S>(a, r), Parameters(a, r), own, regions, sh);
}

// ------------------------------------------------------------------ filters

// Lanes of a row: 512 with at most 128 registers, so that two rows share a CU and one computes while the other waits
// (1,024 rows of 32,768 bf16 with top-p and min-p: 139 us; 1,024 lanes, one row a CU: 207; 256 lanes: 154).
constexpr int kCutLanes = 512, kCutWaves = kCutLanes / 64;
constexpr int kBinBits = 10, kBins = 1 << kBinBits;
constexpr int kList = 2048;
constexpr int kRank = 256;

// x as a whole number, rounded towards zero: NaN to 0, what is too large to the largest, as the instruction has it and
// the language does not say.
__device__ __forceinline__ uint32_t saturate(float x) {
    uint32_t r;
    asm("v_cvt_u32_f32 %0, %1" : "=v"(r) : "v"(x));
    return r;
}

// An entry's place in the order (descending score, ascending index): smaller is earlier.
__device__ __forceinline__ u64 place_of(uint32_t key, uint32_t index) { return ((u64)~key << 32) | index; }
__device__ __forceinline__ uint32_t key_at(u64 place) { return ~(uint32_t)(place >> 32); }

// The smallest key in (lo, hi] for which reached() holds (it holds for hi, and for every key above one for which it
// does), by 64 probes a round; every lane of a wavefront calls it.
template <class F>
__device__ __forceinline__ uint32_t least_key(uint32_t lo, uint32_t hi, F reached) {
    const int lane = threadIdx.x & 63;
    while (hi - lo > 1) {
        const uint32_t step = ((hi - lo - 1) >> 6) + 1;  // 64 steps reach hi
        const u64 probe = (u64)lo + (u64)step * (lane + 1);
        const u64 m = __ballot(probe >= hi || reached((uint32_t)probe));
        const int first = __ffsll(m) - 1;
        const u64 up = (u64)lo + (u64)step * (first + 1);
        lo += step * first;
        hi = up < hi ? (uint32_t)up : hi;
    }
    return hi;
}

template <int kLanes, bool kLists = true>
struct CutShared {
    static constexpr int kWaves = kLanes / 64;
    uint32_t count[kBins];
    u64 weight[kBins];
    u64 list[kLists ? kList : 1], list_w[kLists ? kList : 1];
    ulonglong2 some[kRank];  // place, weight
    u64 wave_c[kWaves], wave_w[kWaves], wave_h[kWaves];
    u128 above_w;
    u64 above_c, in_bin, found, found_w, lo64, hi64;
    uint32_t bin, listed, lo, hi;
    Part part[kWaves];
    PickShared<kLanes> pick;
};

// Weights of several bins are whole numbers of up to 97 bits: those of a bin shifted to the last bin's unit.  Sums go
// over lanes in two parts, of 48 bits and the rest.
constexpr int kPart = 48;
__device__ __forceinline__ u64 low_part(u128 v) { return (u64)v & (((u64)1 << kPart) - 1); }
__device__ __forceinline__ u64 high_part(u128 v) { return (u64)(v >> kPart); }
// The same of w << shift: w below 2^63, shift at most 48.
__device__ __forceinline__ u64 low_part(u64 w, int shift) { return (w << shift) & (((u64)1 << kPart) - 1); }
__device__ __forceinline__ u64 high_part(u64 w, int shift) { return w >> (kPart - shift); }
__device__ __forceinline__ u128 joined(u64 low, u64 high) { return ((u128)high << kPart) + low; }
// The least whole number, from 1 up, that is at least p times v (both rounded to binary64).
__device__ __forceinline__ u128 share_of(double p, u128 v) {
    const double x = ceil(p * ((double)high_part(v) * 0x1p48 + (double)low_part(v)));
    const double high = trunc(x * 0x1p-48);
    const u128 r = joined((u64)(x - high * 0x1p48), (u64)high);
    return r ? r : 1;
}

// A row's extent: its largest and smallest score's keys and the number of its entries.
struct Extent {
    uint32_t top, low, count, unused;
};

// What a row's filters ask for.
template <class S>
struct Goal {
    using X = typename S::X;
    bool nothing;     // no entries, or parameters out of range
    bool one;         // the first of the largest scores is all that is kept
    bool by_k, by_p;  // top-k leaves something out, top-p does
    u64 k;
    double p, q;
    X top;
    uint32_t top_key;
    Exponent ex;
    float bins_per;  // distance bins per unit of score
    // A weight of bin b is a whole number of 2^-(unit + more), more = b finer / 2^20 rounded up.  No weight of the bin
    // is above 2^-(b finer / 2^20) (finer is a thousandth less than the bins' width has it, for the roundings of a
    // distance): the whole numbers are at most 2^(unit + 1), their sums below 2^62, and down to the last bin, in which
    // more is 35 at most, each is off by 2^-(unit + 1) of itself, or 3% more.
    int unit, finer;
    __device__ __forceinline__ Goal(const Parameters& par, const Extent& e, int n) {
        nothing = e.count == 0 || par.bad;
        one = par.T == 0.0f || par.q > 1.0f || par.p <= 0.0f || par.k == 1;
        by_k = !nothing && !one && par.k > 0 && (uint32_t)par.k < e.count;
        by_p = !nothing && !one && par.p < 1.0f;
        k = (u64)par.k;
        p = (double)par.p;
        q = (double)par.q;
        top_key = e.top;
        top = S::value(e.top);
        ex.set(top, par.T == 0.0f ? 1.0 : par.scale());
        // weights past 24 T below the top add less than 4e-11 each: their bins need no width of their own; a count
        // alone goes by the scores' range
        const float reach = 24.0f * par.T, spread = S::below(top, S::value(e.low));
        const float range = par.p < 1.0f && reach < spread ? reach : spread;
        bins_per = (float)(kBins - 1) / range;
        // range / T is at most 24; a range so short that bins_per is infinite has no bins but the first and the last
        const float bits_in_bins = fminf(range / par.T, 24.0f) * 1.44125f;
        finer = by_p && bins_per <= FLT_MAX ? (int)(bits_in_bins * (1048576.0f / (kBins - 1))) : 0;
        const int bits = n > 1 ? 32 - __clz(n - 1) : 0;
        unit = bits < 11 ? 50 : 61 - bits;
    }
    // The last place whose weight is at least min-p; every lane of a wavefront calls it.
    __device__ __forceinline__ u64 last_by_weight() const {
        if (one) return place_of(top_key, 0xFFFFFFFFu);
        if (!(q > 0.0)) return ~(u64)0;
        const uint32_t k_ = least_key(S::key(S::kMasked), top_key,
                                      [&](uint32_t c) { return ex.weight(S::value(c)) >= q; });
        return place_of(k_, 0xFFFFFFFFu);
    }
};

// Where a row's filters end: the place of the last kept entry.
template <int kLanes, class S, bool kLists = true>
struct Cutter {
    using X = typename S::X;
    static constexpr int kWaves = kLanes / 64, kOwn = kBins / kLanes;  // bins of a lane
    static_assert(kWaves <= 8, "sum_of_first");
    const Row<S>& row;
    Region mine;  // this wavefront's
    const Exponent& ex;
    X top;
    uint32_t top_key;
    float bins_per;
    int finer, first_one;
    bool weights;  // top-p is on
    bool filled;   // the bins hold the row's distances
    CutShared<kLanes, kLists>& sh;
    __device__ __forceinline__ Cutter(const Row<S>& r, const Region& g, const Goal<S>& goal,
                                      CutShared<kLanes, kLists>& shared)
        : row(r), mine(g), ex(goal.ex), top(goal.top), top_key(goal.top_key), bins_per(goal.bins_per),
          finer(goal.finer), first_one((1075 - goal.unit) << 20), weights(goal.by_p), filled(false), sh(shared) {}

    // Upper half of 2^(52 - u), 2^-u bin b's unit: what stays of its low bits after adding w is w 2^u, rounded.
    __device__ __forceinline__ int one_of(uint32_t b) const {
        return (__mul24((int)b, -finer) + first_one) & 0x7FF00000;
    }
    // How many bits the last bin's unit is finer.
    __device__ __forceinline__ int shift_of(uint32_t b) const { return (one_of(b) - one_of(kBins - 1)) >> 20; }
    __device__ __forceinline__ u64 fixed(double w, uint32_t b) const {
        const int one = one_of(b);
        return (u64)__double_as_longlong(w + __hiloint2double(one, 0)) - ((u64)(uint32_t)one << 32);
    }
    __device__ __forceinline__ u64 fixed_of(X v, uint32_t b) const { return weights ? fixed(ex.weight(v), b) : 0; }
    // Distance bins: equal scores share one, and a lower score is never in an earlier one.  NaN (inf - inf, or the
    // top itself where bins_per is infinite) goes to the first bin, what is past the range to the last.
    __device__ __forceinline__ uint32_t bin_of(X v) const {
        const uint32_t b = saturate(S::below(top, v) * bins_per);
        return b < kBins - 1 ? b : kBins - 1;
    }
    // The keys of bins b0 to b1: from the smallest whose bin is at most b1 to the last before those whose bin is below
    // b0.  Both ends at once, by 32 probes a round each; every lane of a wavefront calls it.
    __device__ __forceinline__ void keys_of(uint32_t b0, uint32_t b1, uint32_t* first, uint32_t* last) const {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        const uint32_t want = half ? b0 : b1 + 1;  // bins below this one (none is below bin 0)
        uint32_t lo = S::key(S::kMasked), hi = half && b0 == 0 ? top_key + 1 : top_key;
        if (half && b0 == 0) lo = top_key;
        while (__any(hi - lo > 1)) {
            const uint32_t step = hi - lo > 1 ? ((hi - lo - 1) >> 5) + 1 : 1;
            const u64 probe = (u64)lo + (u64)step * ((lane & 31) + 1);
            const u64 m = __ballot(probe >= hi || bin_of(S::value((uint32_t)probe)) < want);
            const int at = __ffs((unsigned)(m >> (32 * half))) - 1;
            const u64 up = (u64)lo + (u64)step * (at + 1);
            lo += step * at;
            hi = up < hi ? (uint32_t)up : hi;
        }
        *first = (uint32_t)__builtin_amdgcn_readlane((int)hi, 0);
        *last = (uint32_t)__builtin_amdgcn_readlane((int)hi, 32) - 1;
    }
    template <int kAhead, class B>
    __device__ __forceinline__ void walk(B body) const {
        row.template walk<kAhead>(mine.lo, mine.hi, body);
    }

    __device__ __forceinline__ void clear_bins() {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            sh.count[threadIdx.x + i * kLanes] = 0;
            sh.weight[threadIdx.x + i * kLanes] = 0;
        }
        filled = false;
        __syncthreads();
    }

    // Counts (of every entry, masked ones last) and weights by distance bin.  The last bin's are summed in registers:
    // most entries can be there.
    __device__ void fill_bins(bool counts) {
        clear_bins();
        const int lane = threadIdx.x & 63;
        uint32_t far = 0;
        u64 far_w = 0;
        if (weights) {
            walk<1>([&](const X (&v)[S::V], int) {
                double w[S::V];
                ex.weights(v, w);
#pragma unroll
                for (int e = 0; e < S::V; ++e) {
                    const uint32_t b = bin_of(v[e]);
                    const u64 f = fixed(w[e], b);
                    if (b == kBins - 1) {
                        far_w += f;
                        ++far;
                    } else {
                        atomicAdd(&sh.weight[b], f);
                        if (counts) atomicAdd(&sh.count[b], 1u);
                    }
                }
            });
        } else {
            walk<2>([&](const X (&v)[S::V], int) {
#pragma unroll
                for (int e = 0; e < S::V; ++e) {
                    const uint32_t b = bin_of(v[e]);
                    if (b == kBins - 1) ++far;
                    else atomicAdd(&sh.count[b], 1u);
                }
            });
        }
        far = wave_sum(far);
        far_w = wave_sum(far_w);
        if (lane == 0) {
            atomicAdd(&sh.count[kBins - 1], far);
            atomicAdd(&sh.weight[kBins - 1], far_w);
        }
        filled = true;
        __syncthreads();
    }

    // The bin, from 0 up, in which the count reaches want or the weight goal; above_c and above_w are those of what
    // precedes the bins.  Leaves bin, in_bin, above_c and above_w (with kFar of the distance bins, each shifted by its
    // own; otherwise of 64 bits, in one bin's unit) in LDS.  Returns goal: with p, its share of all distance bins'
    // weight.
    template <bool kFar>
    __device__ u128 cross(bool by_weight, u64 want, u128 goal, u64 above_c, u64 above_w, double p = 0.0) {
        const int wave = wave_index(), lane = threadIdx.x & 63;
        uint32_t c[kOwn], sum_c = 0;
        u64 w[kOwn], high[kOwn], sum_w = 0, sum_h = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const uint32_t b = kOwn * threadIdx.x + i;
            c[i] = sh.count[b];
            w[i] = weights ? sh.weight[b] : 0;
            high[i] = 0;
            if (kFar) {
                const int shift = shift_of(b);
                high[i] = high_part(w[i], shift);
                w[i] = low_part(w[i], shift);
            }
            sum_c += c[i];
            sum_w += w[i];
            sum_h += high[i];
        }
        const uint32_t sc = wave_scan(sum_c);
        const u64 sw = weights ? wave_scan(sum_w) : 0, su = kFar && weights ? wave_scan(sum_h) : 0;
        if (lane == 63) {
            sh.wave_c[wave] = sc;
            sh.wave_w[wave] = sw;
            if (kFar) sh.wave_h[wave] = su;
        }
        __syncthreads();
        u64 ec = above_c + sum_of_first(sh.wave_c, wave) + sc - sum_c, ew = above_w + sw - sum_w, eh = 0;
        if (weights) {
            ew += sum_of_first(sh.wave_w, wave);
            if (kFar) eh = sum_of_first(sh.wave_h, wave) + su - sum_h;
            if (kFar && p > 0.0)
                goal = share_of(p, joined(sum_of_first(sh.wave_w, kWaves), sum_of_first(sh.wave_h, kWaves)));
        }
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const bool here = !by_weight ? ec < want && ec + c[i] >= want
                              : kFar     ? joined(ew, eh) < goal && joined(ew + w[i], eh + high[i]) >= goal
                                         : ew < (u64)goal && ew + w[i] >= (u64)goal;
            if (here) {
                sh.bin = kOwn * threadIdx.x + i;
                sh.in_bin = c[i];
                sh.above_c = ec;
                sh.above_w = kFar ? joined(ew, eh) : ew;
            }
            ec += c[i];
            ew += w[i];
            eh += high[i];
        }
        __syncthreads();
        return goal;
    }
    // What goal leaves to add, in units of that shift.
    __device__ __forceinline__ u64 left_for(int shift, u128 goal, u128 above_w) const {
        return (u64)((goal - above_w + (((u128)1 << shift) - 1)) >> shift);
    }

    // Place of the number-th entry (from 1) whose score is v, in index order.
    __device__ u64 nth_equal(X v, u64 number) {
        const int wave = wave_index(), lane = threadIdx.x & 63;
        u64 n = 0;
        walk<2>([&](const X (&x)[S::V], int) {
#pragma unroll
            for (int e = 0; e < S::V; ++e) n += __popcll(__ballot(x[e] == v));
        });
        if (lane == 0) sh.wave_c[wave] = n;
        __syncthreads();
        u64 before = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const u64 c = sh.wave_c[k];
            before += k < wave ? c : 0;
        }
        if (before < number && before + n >= number) {
            u64 seen = before;
            walk<1>([&](const X (&x)[S::V], int first) {
                if (seen >= number) return;
                uint32_t here = 0;
#pragma unroll
                for (int e = 0; e < S::V; ++e) here += x[e] == v;
                const uint32_t scan = wave_scan(here);
                u64 at = seen + scan - here;
                if (at < number && at + here >= number) {
#pragma unroll
                    for (int e = 0; e < S::V; ++e)
                        if (x[e] == v && ++at == number) sh.found = place_of(S::key(v), (uint32_t)(first + e));
                }
                seen += last_lane(scan);
            });
        }
        __syncthreads();
        const u64 r = sh.found;
        __syncthreads();
        return r;
    }

    // How many of `number` entries of the same score v, of weight w, the cut takes.
    __device__ u64 equal_needed(u64 w, u64 number, bool by_weight, u64 want, u64 goal, u64 above_c, u64 above_w,
                                u64* up_to) const {
        u64 r = want - above_c;
        if (by_weight) r = (goal - above_w + w - 1) / w;  // w > 0: the weight reaches goal here
        r = r < number ? r : number;
        *up_to = above_w + r * w;
        return r;
    }

    // The cut among the listed entries, their weights in list_w: split by the bits of their places until at most kRank
    // are left, which are ranked.  Sums of whole numbers cross in every round; one that did not would leave in_bin 0
    // and end the loop.
    __device__ u64 cut_list(uint32_t number, bool by_weight, u64 want, u64 goal, u64 above_c, u64 above_w, u64* up_to) {
        const int tid = threadIdx.x;
        u64 lo = 0, hi = ~(u64)0;  // places still in question
        if (tid == 0) sh.in_bin = number;
        __syncthreads();
        while (sh.in_bin > kRank) {
            if (tid == 0) {
                sh.lo64 = ~(u64)0;
                sh.hi64 = 0;
            }
            clear_bins();
            if (tid == 0) sh.in_bin = 0;
            u64 least = ~(u64)0, most = 0;
            for (uint32_t i = tid; i < number; i += kLanes) {
                const u64 p = sh.list[i];
                if (p < lo || p > hi) continue;
                least = p < least ? p : least;
                most = p > most ? p : most;
            }
            least = ~wave_max(~least);
            most = wave_max(most);
            if ((tid & 63) == 0 && most >= least) {
                atomicMin(&sh.lo64, least);
                atomicMax(&sh.hi64, most);
            }
            __syncthreads();
            lo = sh.lo64;
            hi = sh.hi64;
            const u64 spread = (hi - lo) >> kBinBits;
            const int shift = spread ? 64 - __clzll(spread) : 0;
            for (uint32_t i = tid; i < number; i += kLanes) {
                const u64 p = sh.list[i];
                if (p < lo || p > hi) continue;
                const uint32_t b = (uint32_t)((p - lo) >> shift);
                atomicAdd(&sh.count[b], 1u);
                if (weights) atomicAdd(&sh.weight[b], sh.list_w[i]);
            }
            __syncthreads();
            cross<false>(by_weight, want, goal, above_c, above_w);
            above_c = scalar(sh.above_c);
            above_w = scalar((u64)sh.above_w);
            lo += (u64)sh.bin << shift;
            const u64 span = ((u64)1 << shift) - 1;  // lo + span can pass 2^64, where the lowest ints' places end
            hi = hi - lo > span ? lo + span : hi;
        }
        // at most kRank entries: each against all
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        for (uint32_t i = tid; i < number; i += kLanes) {
            const u64 p = sh.list[i];
            if (p < lo || p > hi) continue;
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < kRank) sh.some[at] = ulonglong2{p, sh.list_w[i]};
        }
        __syncthreads();
        const uint32_t left = sh.listed < kRank ? sh.listed : kRank;
        if ((uint32_t)tid < left) {
            const u64 p = sh.some[tid].x, w = sh.some[tid].y;
            u64 before = above_c, before_w = above_w;
#pragma unroll 4
            for (uint32_t j = 0; j < left; ++j) {
                const ulonglong2 other = sh.some[j];
                const bool earlier = other.x < p;
                before += earlier;
                before_w += earlier ? other.y : 0;
            }
            if (by_weight ? before_w < goal && before_w + w >= goal : before + 1 == want) {
                sh.found = p;
                sh.found_w = before_w + w;
            }
        }
        __syncthreads();
        const u64 r = scalar(sh.found);
        *up_to = scalar(sh.found_w);
        __syncthreads();
        return r;
    }

    // The entry at which the count reaches want (by_weight false) or the weight reaches goal, or with p that share of
    // all, in the order; the distance bins hold their sums.  *up_to: the weight up to and with it (where weights are
    // summed).
    __device__ u64 cut(bool by_weight, u64 want, u128 goal, double p, u128* up_to) {
        const int tid = threadIdx.x;
        goal = cross<true>(by_weight, want, goal, 0, 0, p);
        uint32_t lo, hi;
        const uint32_t bin = scalar(sh.bin);
        u64 above_c = scalar(sh.above_c), above_w = 0, with = 0, at;  // from here on weights are of this bin's unit
        const u128 far_w = scalar(sh.above_w);
        const u64 need = by_weight ? left_for(shift_of(bin), goal, far_w) : 0;
        keys_of(bin, bin, &lo, &hi);
        for (;;) {
            __syncthreads();
            if (tid == 0) {
                sh.listed = 0;
                sh.lo = 0xFFFFFFFFu;
                sh.hi = 0;
            }
            __syncthreads();
            // the entries with these keys into the list, and the range they take
            const X from = S::value(lo), to = S::value_up(hi);
            X least = to, most = from;
            uint32_t any = 0;
            walk<2>([&](const X (&v)[S::V], int first) {
                bool reach = false;
#pragma unroll
                for (int e = 0; e < S::V; ++e) reach = reach || v[e] >= from;
                if (!__any(reach)) return;
#pragma unroll
                for (int e = 0; e < S::V; ++e) {
                    if (v[e] >= from && v[e] <= to) {
                        least = v[e] < least ? v[e] : least;
                        most = v[e] > most ? v[e] : most;
                        any = 1;
                        const uint32_t at = atomicAdd(&sh.listed, 1u);
                        if (at < kList) sh.list[at] = place_of(S::key(v[e]), (uint32_t)(first + e));
                    }
                }
            });
            if (any) {
                atomicMin(&sh.lo, S::key(least));
                atomicMax(&sh.hi, S::key(most));
            }
            __syncthreads();
            lo = sh.lo;
            hi = sh.hi;
            const uint32_t number = sh.listed;
            if (number <= kList) {
                for (uint32_t i = tid; i < number; i += kLanes)
                    sh.list_w[i] = fixed_of(S::value(key_at(sh.list[i])), bin);
                at = cut_list(number, by_weight, want, need, above_c, above_w, &with);
                break;
            }
            if (lo == hi) {  // equal scores: as many of them as it takes, in index order
                const X v = S::value(lo);
                at = nth_equal(v, equal_needed(fixed_of(v, bin), number, by_weight, want, need, above_c, above_w,
                                               &with));
                break;
            }
            // split the range of keys: bins from the largest key down
            const int shift = 32 - __clz((hi - lo) >> kBinBits);
            clear_bins();
            walk<1>([&](const X (&v)[S::V], int) {
#pragma unroll
                for (int e = 0; e < S::V; ++e) {
                    const uint32_t k = S::key(v[e]);
                    if (k < lo || k > hi) continue;
                    const uint32_t b = (hi - k) >> shift;
                    atomicAdd(&sh.count[b], 1u);
                    if (weights) atomicAdd(&sh.weight[b], fixed_of(v[e], bin));
                }
            });
            __syncthreads();
            cross<false>(by_weight, want, need, above_c, above_w);
            above_c = scalar(sh.above_c);
            above_w = scalar((u64)sh.above_w);
            const uint32_t b = sh.bin, span = (1u << shift) - 1;
            hi -= b << shift;
            lo = hi - lo > span ? hi - span : lo;
        }
        *up_to = far_w + ((u128)with << shift_of(bin));
        return at;
    }

    // The last kept place by all filters.
    __device__ u64 last_kept(const Goal<S>& goal) {
        u64 last = ~(u64)0;
        u128 total = 0;
#pragma unroll 1
        for (int by_weight = goal.by_k ? 0 : 1; by_weight <= (goal.by_p ? 1 : 0); ++by_weight) {
            // top-k's cut first: top-p goes by the weight of the first k, and reaches its share of that before the last
            // of them
            if (!filled) fill_bins(goal.by_k && !by_weight);
            const u64 at = cut(by_weight != 0, goal.k, share_of(goal.p, total),
                               by_weight && !goal.by_k ? goal.p : 0.0, &total);
            last = at < last ? at : last;
        }
        const u64 at = goal.last_by_weight();
        return at < last ? at : last;
    }
};

// Whether an entry is kept: everything up to a place.
template <class S>
struct Kept {
    using X = typename S::X;
    X edge;
    int edge_at;
    __device__ __forceinline__ explicit Kept(u64 last) {
        edge = last == ~(u64)0 ? S::kMasked : S::value(key_at(last));
        edge_at = (uint32_t)last > 0x7FFFFFFFu ? INT32_MAX : (int)(uint32_t)last;
    }
    __device__ __forceinline__ bool operator()(X v, int i) const {
        return v > edge || (v == edge && i <= edge_at && v != S::kMasked);
    }
    // Weights of a lane's entries, 0 for those not kept; skipped where no lane of the wavefront keeps one.
    __device__ __forceinline__ bool weights(const Exponent& ex, bool one, const X (&v)[S::V], int first,
                                            double (&w)[S::V], uint32_t* count) const {
        bool keep[S::V], some = false;
#pragma unroll
        for (int e = 0; e < S::V; ++e) {
            keep[e] = (*this)(v[e], first + e);
            some = some || keep[e];
        }
#pragma unroll
        for (int e = 0; e < S::V; ++e) w[e] = 0.0;
        if (!__any(some)) return false;
        if (!one) ex.weights(v, w);
#pragma unroll
        for (int e = 0; e < S::V; ++e) {
            w[e] = !keep[e] ? 0.0 : one ? 1.0 : w[e];
            *count += __popcll(__ballot(keep[e]));
        }
        return true;
    }
};

// The extent of a wavefront's groups.
template <class S>
__device__ Extent extent_of(const Row<S>& row, const Region& g) {
    using X = typename S::X;
    X most = S::kMasked, least = S::value(0xFFFFFFFFu - (std::is_same<X, float>::value ? 0x7FFFFFu : 0u));
    uint32_t count = 0;
    row.template walk<4>(g.lo, g.hi, [&](const X (&v)[S::V], int) {
#pragma unroll
        for (int e = 0; e < S::V; ++e) {
            most = S::larger(most, v[e]);
            least = v[e] != S::kMasked && v[e] < least ? v[e] : least;
            count += __popcll(__ballot(v[e] != S::kMasked));
        }
    });
    return Extent{wave_max(S::key(most)), ~wave_max(~S::key(least)), count, 0u};
}

// Weight and number of a wavefront's kept entries.
template <class S>
__device__ Part sum_kept(const Row<S>& row, const Region& g, const Kept<S>& kept, const Goal<S>& goal) {
    double sum = 0.0;
    uint32_t number = 0;
    row.template walk<2>(g.lo, g.hi, [&](const typename S::X (&v)[S::V], int first) {
        double w[S::V];
        if (!kept.weights(goal.ex, goal.one, v, first, w, &number)) return;
#pragma unroll
        for (int e = 0; e < S::V; ++e) sum += w[e];
    });
    return Part{wave_sum(sum), 0u, number};
}

// The row's draw among its kept entries, from its regions' parts, at most kLanes.
template <int kLanes, class S>
__device__ void draw_kept(const SampleArgs& a, int64_t r, const Row<S>& row, const Parameters& par, const Kept<S>& kept,
                          const Goal<S>& goal, const Part* parts, int regions, PickShared<kLanes>& sh) {
    u64 count = 0;
    if (!goal.one) {
        // each wavefront for itself
        for (int k = threadIdx.x & 63; k < regions; k += 64) count += parts[k].count;
        count = wave_sum(count);
    }
    const double u = (double)(a.rnd[r] >> 11) * 0x1p-53;
    double sum, before;
    const int target = target_region<kLanes>((int)threadIdx.x < regions ? parts[threadIdx.x].weight : 0.0, u, goal.one,
                                             &sum, &before, sh);
    const double t = goal.one ? 0.0 : u * sum;  // one: the first of equal weights
    const Draw draw{a, r, (double)goal.top, (double)par.T, goal.one ? 1.0 : sum, goal.one ? 1 : count};
    pick_in_region<kLanes>(
        row, Region(row.groups, regions, target), t - before, draw,
        [&](const typename S::X (&v)[S::V], int first, double (&w)[S::V]) {
            uint32_t n = 0;
            kept.weights(goal.ex, goal.one, v, first, w, &n);
        },
        sh);
}

// A row by one workgroup.
template <class S>
__device__ void cut_row(const SampleArgs& a, int64_t r, const Row<S>& row, const Parameters& par,
                        CutShared<kCutLanes>& sh) {
    const int tid = threadIdx.x, wave = wave_index(), lane = tid & 63;
    const Region mine(row.groups, kCutWaves, wave);
    const Extent own = extent_of(row, mine);
    if (tid == 0) {
        sh.listed = sh.hi = 0;
        sh.lo = 0xFFFFFFFFu;
    }
    __syncthreads();
    if (own.count && lane == 0) {
        atomicAdd(&sh.listed, own.count);
        atomicMax(&sh.hi, own.top);
        atomicMin(&sh.lo, own.low);
    }
    __syncthreads();
    const Goal<S> goal(par, Extent{sh.hi, sh.lo, sh.listed, 0u}, row.n);
    if (goal.nothing) {
        if (tid == 0) write_nothing(a, r);
        return;
    }
    __syncthreads();
    Cutter<kCutLanes, S> cut(row, mine, goal, sh);
    const Kept<S> kept(cut.last_kept(goal));
    const Part p = sum_kept(row, mine, kept, goal);
    if (lane == 0) sh.part[wave] = p;
    __syncthreads();
    draw_kept<kCutLanes>(a, r, row, par, kept, goal, sh.part, kCutWaves, sh.pick);
}

// 256 rows of 50,257 f16 with top-p and min-p: 77 us, of which a row takes 4 for its extent, 22 for the bins' weights
// (an exponential and an LDS atomic of 64 bits an entry), 7 to 25 for the cut, 8 for the kept entries' sums and 4 for the draw.
// The later passes find the row in the caches; every pass ends in a barrier that waits for the slowest wavefront.
template <int kType>
__global__ void __launch_bounds__(kCutLanes, 4) cut_kernel(SampleArgs a) {  // four wavefronts a SIMD: 128 registers
    using S = Scores<kType>;
    __shared__ CutShared<kCutLanes> sh;
    const int64_t r = a.row0 + blockIdx.x;
    cut_row(a, r, Row<S>(a, r), Parameters(a, r), sh);
}

// ------------------------------------------------------------------ filters, a row split over workgroups
//
// The same steps, each a launch of its own over all splits of all rows; what the splits find meets in the
// row's SplitRow, and each workgroup works out for itself what follows from that:
//   extent_kernel  the splits' extents; clears the row's bins and lists
//   fill_kernel    counts and weights of the distance bins, summed in the row's
//   gather_kernel  the entries of the bins in which the cuts fall, into the row's lists
//   sum_kernel     the cuts, from the lists; weight and number of the regions' kept entries
//   draw_kernel    a workgroup per row: the draw
// 16 rows of 131,072 i32 with top-p: 4.5, 8.5, 10.5, 13 and 6 us.  Each launch is bound by its chain: the first
// loads, the row's state from the other workgroups, one pass over 4,096 entries or more, the reduction.
// The draw as the last step of the row's last workgroup of sum_kernel, a device-wide fence in each, takes 104 us
// instead of 42.
// A bin with more entries than a list holds is of one score as a rule (16-bit scores): the cut is then a number of
// them, and the split in which the last one is finds it.  A row with a longer list of different scores is cut as a
// whole by draw_kernel.

constexpr int kSplitLanes = 512, kSplitWaves = kSplitLanes / 64;

struct SplitRow {
    uint32_t count[kBins];
    u64 weight[kBins];
    u64 list[2][kList];  // places: of top-k's bin, of top-p's
    u128 above_w[2];  // before those bins: weight
    u64 above_c;      // and entries (top-k)
    u128 share;       // top-p's goal (without top-k)
    u64 last;                 // place of the last kept entry
    uint32_t listed[2], lo[2], hi[2];  // entries of those bins, their range of keys
    uint32_t found[2][kMaxSplits];     // entries of each split
    Extent extent[kMaxSplits];
    Part part[kMaxSplits * kSplitWaves];
    __device__ __forceinline__ bool fits(int c) const { return listed[c] <= kList; }
    __device__ __forceinline__ bool cut_here() const {
        return (fits(0) || lo[0] == hi[0]) && (fits(1) || lo[1] == hi[1]);
    }
};

template <class S>
__device__ __forceinline__ Extent row_extent(const SplitRow& w, int splits) {
    const int lane = threadIdx.x & 63;  // kMaxSplits lanes
    Extent e{0u, 0xFFFFFFFFu, 0u, 0u};
    if (lane < splits) e = w.extent[lane];
    if (e.count == 0) e = Extent{0u, 0xFFFFFFFFu, 0u, 0u};
    return Extent{wave_max(e.top), ~wave_max(~e.low), wave_sum(e.count), 0u};
}

template <int kType>
__global__ void __launch_bounds__(kSplitLanes) extent_kernel(SampleArgs a, int splits, SplitRow* rows) {
    using S = Scores<kType>;
    __shared__ Extent own[kSplitWaves];
    const int64_t i = blockIdx.x / splits, r = a.row0 + i;
    const int s = blockIdx.x % splits, wave = wave_index();
    SplitRow& w = rows[i];
    for (int b = s * kSplitLanes + threadIdx.x; b < kBins; b += splits * kSplitLanes) {
        w.count[b] = 0;
        w.weight[b] = 0;
    }
    if (s == 0 && threadIdx.x < 2) {
        w.listed[threadIdx.x] = w.hi[threadIdx.x] = 0;
        w.lo[threadIdx.x] = 0xFFFFFFFFu;
    }
    const Row<S> row(a, r);
    const Extent e = extent_of(row, Region(row.groups, splits * kSplitWaves, s * kSplitWaves + wave));
    if ((threadIdx.x & 63) == 0) own[wave] = e.count ? e : Extent{0u, 0xFFFFFFFFu, 0u, 0u};
    __syncthreads();
    if (threadIdx.x == 0) {
        Extent all = own[0];
        for (int k = 1; k < kSplitWaves; ++k) {
            all.top = own[k].top > all.top ? own[k].top : all.top;
            all.low = own[k].low < all.low ? own[k].low : all.low;
            all.count += own[k].count;
        }
        w.extent[s] = all;
    }
}

template <int kType>
__global__ void __launch_bounds__(kSplitLanes) fill_kernel(SampleArgs a, int splits, SplitRow* rows) {
    using S = Scores<kType>;
    __shared__ CutShared<kSplitLanes, false> sh;
    const int64_t i = blockIdx.x / splits, r = a.row0 + i;
    const int s = blockIdx.x % splits;
    SplitRow& w = rows[i];
    const Row<S> row(a, r);
    const Goal<S> goal(Parameters(a, r), row_extent<S>(w, splits), row.n);
    if (!goal.by_k && !goal.by_p) return;
    const Region mine(row.groups, splits * kSplitWaves, s * kSplitWaves + wave_index());
    Cutter<kSplitLanes, S, false> cut(row, mine, goal, sh);
    cut.fill_bins(goal.by_k);
    for (int b = threadIdx.x; b < kBins; b += kSplitLanes) {
        const uint32_t c = sh.count[b];
        const u64 v = sh.weight[b];
        if (c) atomicAdd(&w.count[b], c);
        if (v) atomicAdd(&w.weight[b], v);
    }
}

template <int kType>
__global__ void __launch_bounds__(kSplitLanes) gather_kernel(SampleArgs a, int splits, SplitRow* rows) {
    using S = Scores<kType>;
    using X = typename S::X;
    __shared__ CutShared<kSplitLanes> sh;
    __shared__ uint32_t listed[2], base[2], ends[4];  // ends: least keys, largest keys
    const int64_t i = blockIdx.x / splits, r = a.row0 + i;
    const int s = blockIdx.x % splits, tid = threadIdx.x;
    SplitRow& w = rows[i];
    const Row<S> row(a, r);
    const Goal<S> goal(Parameters(a, r), row_extent<S>(w, splits), row.n);
    if (!goal.by_k && !goal.by_p) return;
    Cutter<kSplitLanes, S> cut(row, Region(row.groups, splits * kSplitWaves, s * kSplitWaves + wave_index()), goal, sh);
    for (int b = tid; b < kBins; b += kSplitLanes) {
        sh.count[b] = w.count[b];
        sh.weight[b] = w.weight[b];
    }
    if (tid < 2) {
        listed[tid] = ends[2 + tid] = 0;
        ends[tid] = 0xFFFFFFFFu;
    }
    __syncthreads();
    // keys [lo, hi] of the bins of either cut; none: an empty range
    uint32_t lo[2] = {0xFFFFFFFFu, 0xFFFFFFFFu}, hi[2] = {0u, 0u};
    u128 least = 0, most = 0;  // bounds of the first k's weight
    if (goal.by_k) {
        cut.template cross<true>(false, goal.k, 0, 0, 0);
        const uint32_t bin = sh.bin;
        cut.keys_of(bin, bin, &lo[0], &hi[0]);
        least = sh.above_w;
        most = least + ((u128)sh.weight[bin] << cut.shift_of(bin));
        if (s == 0 && tid == 0) {
            w.above_c = sh.above_c;
            w.above_w[0] = least;
        }
        __syncthreads();
    }
    if (goal.by_p) {
        // after top-k its cut is between the goals that these bounds give (at least one unit: a weight reaches it)
        const u128 share = cut.template cross<true>(true, 0, share_of(goal.p, least), 0, 0, goal.by_k ? 0.0 : goal.p);
        const uint32_t bin = sh.bin;
        if (s == 0 && tid == 0) {
            w.share = share;
            w.above_w[1] = sh.above_w;
        }
        __syncthreads();
        if (goal.by_k) cut.template cross<true>(true, 0, share_of(goal.p, most), 0, 0);
        cut.keys_of(bin, sh.bin, &lo[1], &hi[1]);
        __syncthreads();
    }
    // sh.list and sh.list_w hold the two lists until they are copied
    const X from[2] = {S::value(lo[0]), S::value(lo[1])}, to[2] = {S::value_up(hi[0]), S::value_up(hi[1])};
    const bool on[2] = {goal.by_k, goal.by_p};
    X low[2] = {to[0], to[1]}, high[2] = {from[0], from[1]};
    bool any[2] = {false, false};
    cut.template walk<4>([&](const X (&v)[S::V], int first) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (!on[c]) continue;
            u64* list = c ? sh.list_w : sh.list;
            bool reach = false;
#pragma unroll
            for (int e = 0; e < S::V; ++e) reach = reach || v[e] >= from[c];
            if (!__any(reach)) continue;
#pragma unroll
            for (int e = 0; e < S::V; ++e) {
                if (v[e] >= from[c] && v[e] <= to[c]) {
                    low[c] = v[e] < low[c] ? v[e] : low[c];
                    high[c] = v[e] > high[c] ? v[e] : high[c];
                    any[c] = true;
                    const uint32_t at = atomicAdd(&listed[c], 1u);
                    if (at < kList) list[at] = place_of(S::key(v[e]), (uint32_t)(first + e));
                }
            }
        }
    });
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        if (!__any(any[c])) continue;
        const uint32_t k0 = ~wave_max(any[c] ? ~S::key(low[c]) : 0u), k1 = wave_max(any[c] ? S::key(high[c]) : 0u);
        if ((tid & 63) == 0) {
            atomicMin(&ends[c], k0);
            atomicMax(&ends[2 + c], k1);
        }
    }
    __syncthreads();
    if (tid < 2) {  // one set of the row's atomics a workgroup: they wait for each other
        w.found[tid][s] = listed[tid];
        base[tid] = 0u;
        if (listed[tid]) {
            base[tid] = atomicAdd(&w.listed[tid], listed[tid]);
            atomicMin(&w.lo[tid], ends[tid]);
            atomicMax(&w.hi[tid], ends[2 + tid]);
        }
    }
    __syncthreads();
    for (int c = 0; c < 2; ++c) {
        const uint32_t n = listed[c] < kList ? listed[c] : kList, at = base[c];
        const u64* list = c ? sh.list_w : sh.list;
        for (uint32_t k = tid; k < n && at + k < kList; k += kSplitLanes) w.list[c][at + k] = list[k];
    }
}

template <int kType>
__global__ void __launch_bounds__(kSplitLanes, 4) sum_kernel(SampleArgs a, int splits, SplitRow* rows) {
    using S = Scores<kType>;
    using X = typename S::X;
    __shared__ CutShared<kSplitLanes> sh;
    const int64_t i = blockIdx.x / splits, r = a.row0 + i;
    const int s = blockIdx.x % splits, tid = threadIdx.x, region = s * kSplitWaves + wave_index();
    SplitRow& w = rows[i];
    const Row<S> row(a, r);
    const Goal<S> goal(Parameters(a, r), row_extent<S>(w, splits), row.n);
    if (goal.nothing || !w.cut_here()) return;
    const Region mine(row.groups, splits * kSplitWaves, region);
    Cutter<kSplitLanes, S> cut(row, mine, goal, sh);
    const u64 q = goal.last_by_weight();
    u64 last = q;
    u128 share = w.share;  // top-k's cut has another
    int writer = 0;  // the split that knows the row's last place: all do, but of equal scores
#pragma unroll 1
    for (int c = goal.by_k ? 0 : 1; c <= (goal.by_p ? 1 : 0); ++c) {
        uint32_t number = w.listed[c], bin = cut.bin_of(S::value(w.lo[c]));
        const u64 above_c = c ? 0 : w.above_c;
        u128 above_w = w.above_w[c];
        // Top-p's list after top-k's cut is of all bins that the cut can be in: where their units are further apart
        // than the sums have bits for, those of the cut's own bin are ranked.
        const bool several = c && goal.by_k && number <= kList &&
                             cut.shift_of(cut.bin_of(S::value(w.hi[c]))) > cut.shift_of(bin) + 1;
        if (several) {
            for (int b = tid; b < kBins; b += kSplitLanes) sh.weight[b] = w.weight[b];
            __syncthreads();
            cut.template cross<true>(true, 0, share, 0, 0);
            bin = scalar(sh.bin);
            above_w = scalar(sh.above_w);
            if (tid == 0) sh.listed = 0;
            __syncthreads();
        }
        const int shift = cut.shift_of(bin);
        const u64 need = c ? cut.left_for(shift, share, above_w) : 0;
        u64 with = 0, at;
        if (number <= kList) {
            for (uint32_t k = tid; k < number; k += kSplitLanes) {
                const u64 p = w.list[c][k];
                const X v = S::value(key_at(p));
                const uint32_t own = cut.bin_of(v);
                if (several && own != bin) continue;
                const uint32_t to = several ? atomicAdd(&sh.listed, 1u) : k;
                sh.list[to] = p;
                sh.list_w[to] = cut.fixed_of(v, own) << (cut.shift_of(own) - shift);
            }
            if (several) {
                __syncthreads();
                number = sh.listed;
            }
            at = cut.cut_list(number, c != 0, goal.k, need, above_c, 0, &with);
            writer = 0;
        } else {
            // the earlier splits keep all of these, the later ones none
            const uint32_t key = w.lo[c];
            const X v = S::value(key);
            const u64 taken = cut.equal_needed(cut.fixed_of(v, bin), number, c != 0, goal.k, need, above_c, 0, &with);
            const int lane = tid & 63;  // kMaxSplits lanes
            const uint32_t here = lane < splits ? w.found[c][lane] : 0;
            const u64 to = wave_scan((u64)here);
            const int split = __ffsll(__ballot(to >= taken)) - 1;
            at = place_of(key, s < split ? 0xFFFFFFFFu : 0u);
            if (s == split) at = cut.nth_equal(v, taken - (u64)__shfl(to - here, split, 64));
            writer = q < place_of(key, 0u) ? 0 : split;
        }
        last = at < last ? at : last;
        share = share_of(goal.p, above_w + ((u128)with << shift));
    }
    if (s == writer && tid == 0) w.last = last;
    const Part p = sum_kept(row, mine, Kept<S>(last), goal);
    if ((tid & 63) == 0) w.part[region] = p;
}

template <int kType>
__global__ void __launch_bounds__(kCutLanes, 4) draw_kernel(SampleArgs a, int splits, const SplitRow* rows) {
    using S = Scores<kType>;
    __shared__ CutShared<kCutLanes> sh;
    const int64_t r = a.row0 + blockIdx.x;
    const SplitRow& w = rows[blockIdx.x];
    const Row<S> row(a, r);
    const Parameters par(a, r);
    const Goal<S> goal(par, row_extent<S>(w, splits), row.n);
    if (goal.nothing) {
        if (threadIdx.x == 0) write_nothing(a, r);
        return;
    }
    if (!w.cut_here()) {
        cut_row(a, r, row, par, sh);
        return;
    }
    static_assert(kMaxSplits * kSplitWaves <= kCutLanes, "a lane for every region");
    Part* parts = reinterpret_cast<Part*>(sh.list);
    static_assert(sizeof(sh.list) >= sizeof(w.part), "the parts fit the list's room");
    const int regions = splits * kSplitWaves;
    if ((int)threadIdx.x < regions) parts[threadIdx.x] = w.part[threadIdx.x];
    __syncthreads();
    draw_kept<kCutLanes>(a, r, row, par, Kept<S>(w.last), goal, parts, regions, sh.pick);
}

// Workgroups a row without filters is split into: until the chip has two for every CU, with 4,096 entries
// left to each.
int splits_of(int32_t R, int32_t N) {
    int64_t s = 512 / R, most = N / 4096;
    if (s > most) s = most;
    if (s > kMaxSplits) s = kMaxSplits;
    return s < 1 ? 1 : (int)s;
}

constexpr int32_t kSplitRows = 192;  // of more rows none is split

// Workgroups a row with filters is split into, 4,096 entries or more to each; 0: one workgroup and a single launch.
// Splitting takes five launches, in which every split works out the row's cuts for itself, and pays while the rows
// alone leave most of the chip idle: 16 rows of 131,072 i32 with top-p 43 against 154 us, 64 of 32,768 41 against 50,
// 192 of 131,072 f32 with top-k and top-p 133 against 164, one of 8,388,608 121 against 7,825; but one of 16,384 27
// against 22, 128 of 32,768 56 against 49, 260 of 131,072 215 against 192, 512 of 262,144 1,297 against 572.  Where
// more scores than a list holds share the bin of a cut, not all equal, it costs an eighth more: 16 rows of 262,144 f32
// with top-p 442 against 389, 64 of 1,048,576 1,805 against 1,593.
int cut_splits_of(int32_t R, int32_t N) {
    if (N < 24576 || R > kSplitRows || (int64_t)R * 500 > N) return 0;
    int64_t s = 1024 / R, most = N / 4096;
    if (s > most) s = most;
    return (int)(s < kMaxSplits ? s : kMaxSplits);
}

constexpr int32_t kRowsPerLaunch = 1 << 20;  // a grid has fewer than 2^32 lanes; split rows are far fewer

size_t cut_workspace(int32_t R, int32_t N) { return cut_splits_of(R, N) ? sizeof(SplitRow) * R : 0; }

template <int kType>
hipError_t launch(SampleArgs a, void* workspace, hipStream_t s) {
    const bool filters = a.top_k || a.top_p || a.min_p;
    const int splits = filters ? cut_splits_of(a.R, a.N) : splits_of(a.R, a.N);
    for (int64_t r0 = 0; r0 < a.R; r0 += kRowsPerLaunch) {
        const unsigned rows = (unsigned)(a.R - r0 < kRowsPerLaunch ? a.R - r0 : kRowsPerLaunch);
        a.row0 = r0;
        if (!filters) {
            Part* parts = static_cast<Part*>(workspace);  // more splits than one: few rows
            hipLaunchKernelGGL(all_kernel<kType>, dim3(rows * splits), dim3(kAllLanes), 0, s, a, splits, parts);
            if (splits > 1)
                hipLaunchKernelGGL(finish_kernel<kType>, dim3(rows), dim3(kFinishLanes), 0, s, a, splits, parts);
        } else if (!splits) {
            hipLaunchKernelGGL(cut_kernel<kType>, dim3(rows), dim3(kCutLanes), 0, s, a);
        } else {
            SplitRow* w = static_cast<SplitRow*>(workspace);
            const dim3 grid(rows * splits), block(kSplitLanes);
            hipLaunchKernelGGL(extent_kernel<kType>, grid, block, 0, s, a, splits, w);
            if (a.top_k || a.top_p) {
                hipLaunchKernelGGL(fill_kernel<kType>, grid, block, 0, s, a, splits, w);
                hipLaunchKernelGGL(gather_kernel<kType>, grid, block, 0, s, a, splits, w);
            }
            hipLaunchKernelGGL(sum_kernel<kType>, grid, block, 0, s, a, splits, w);
            hipLaunchKernelGGL(draw_kernel<kType>, dim3(rows), dim3(kCutLanes), 0, s, a, splits, w);
        }
    }
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int32_t R, int32_t N) {
    const int splits = splits_of(R, N);
    const size_t parts = splits > 1 ? (size_t)R * splits * kAllWaves * sizeof(Part) : 0, cuts = cut_workspace(R, N);
    return ((parts > cuts ? parts : cuts) + 511) & ~(size_t)255;
}

hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s) {
    prof_mark(kKSample, false, s);
    const hipError_t e = a.type == HX_SCORE_I32   ? launch<HX_SCORE_I32>(a, workspace, s)
                         : a.type == HX_SCORE_F32 ? launch<HX_SCORE_F32>(a, workspace, s)
                         : a.type == HX_SCORE_F16 ? launch<HX_SCORE_F16>(a, workspace, s)
                                                  : launch<HX_SCORE_BF16>(a, workspace, s);
    prof_mark(kKSample, true, s);
    return e;
}

}  // namespace hx
