// hx_sample.hip -- one draw from every row of scores: temperature, top-k, top-p, min-p (hx_sample).
//
// Weights are w = exp((x - m) / T) in binary64, m the row's largest score (Exponent).  A row is read in
// groups of 16 bytes (Row); a region is a run of groups that one wavefront walks, 64 groups at a time, and
// the regions of a row follow each other in index order.  A draw is then: the regions' weights, their sum S
// in order, the first region at which they pass t = u S, and the first entry of that region (pick_in_region).
//
// Without filters (all_kernel) the row is read once: a wavefront keeps its own largest score so far, sums
// weights relative to it, and scales the sums when it grows (the ratio of two maxima is an exponential of
// their difference); the regions' sums meet at the end.  Few rows are split over several workgroups, and a
// second launch (finish_kernel) joins them.
//
// With filters (cut_kernel, a workgroup per row): all three keep a prefix of the order (descending score,
// ascending index), so the kept set is everything up to one entry (Cut).  That entry is found by counting,
// for top-k, and by adding whole-number weights, for top-p (64-bit sums: no order of addition changes
// them), in 2,048 bins of the distance from m; the entries of the bin in which the cut falls, if at most
// kList, are ranked against each other in LDS, and otherwise the bin is split again by the keys' bits.
// min-p's bound is a search over the keys.
#include <float.h>
#include <math.h>

#include "hx_internal.h"

namespace hx {
namespace {

using u64 = unsigned long long;

// ------------------------------------------------------------------ scores

// A score's 32-bit key has the scores' order (0: below all); V: entries of 16 bytes.
template <int kType>
struct Scores;
template <>
struct Scores<HX_SCORE_I32> {
    using T = int32_t;
    using X = int32_t;  // a score in registers
    static constexpr int V = 4;
    static constexpr X kMasked = INT32_MIN;
    static __device__ __forceinline__ X widen(T x) { return x; }
    static __device__ __forceinline__ void unpack(const uint4& q, X (&v)[V]) {
        v[0] = (int32_t)q.x, v[1] = (int32_t)q.y, v[2] = (int32_t)q.z, v[3] = (int32_t)q.w;
    }
    static __device__ __forceinline__ uint32_t key(X x) { return (uint32_t)x ^ 0x80000000u; }
    static __device__ __forceinline__ X value(uint32_t k) { return (int32_t)(k ^ 0x80000000u); }
    static __device__ __forceinline__ float below(X m, X x) { return (float)((uint32_t)m - (uint32_t)x); }
};
// Floats: NaN is masked (-inf) as it is read; keys are sign and magnitude in two's-complement order, -0 as +0.
struct FloatScores {
    using X = float;
    static constexpr X kMasked = -INFINITY;
    static __device__ __forceinline__ X clean(float x) { return x > -INFINITY ? x : -INFINITY; }
    static __device__ __forceinline__ uint32_t key(X x) {
        const uint32_t b = __float_as_uint(x + 0.0f);
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    static __device__ __forceinline__ X value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
    static __device__ __forceinline__ float below(X m, X x) { return m - x; }
};
template <>
struct Scores<HX_SCORE_F32> : FloatScores {
    using T = float;
    static constexpr int V = 4;
    static __device__ __forceinline__ X widen(T x) { return clean(x); }
    static __device__ __forceinline__ void unpack(const uint4& q, X (&v)[V]) {
        v[0] = clean(__uint_as_float(q.x)), v[1] = clean(__uint_as_float(q.y));
        v[2] = clean(__uint_as_float(q.z)), v[3] = clean(__uint_as_float(q.w));
    }
};
template <>
struct Scores<HX_SCORE_F16> : FloatScores {
    using T = uint16_t;
    static constexpr int V = 8;
    static __device__ __forceinline__ X widen(T x) {
        _Float16 h;
        __builtin_memcpy(&h, &x, 2);
        return clean((float)h);
    }
    static __device__ __forceinline__ void unpack(const uint4& q, X (&v)[V]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = widen((T)w[i]), v[2 * i + 1] = widen((T)(w[i] >> 16));
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
            v[2 * i] = clean(__uint_as_float(w[i] << 16)), v[2 * i + 1] = clean(__uint_as_float(w[i] & 0xffff0000u));
    }
};

// w = exp((x - m) / T) as 2^(d c), d = x - m, c = log2(e) / T: d c = n + f with n whole and |f| <= 1/2, and
// 2^f = 1 + f q(f), q the interpolation of (2^f - 1) / f at the ten Chebyshev nodes of [-1/2, 1/2] (computed
// in 80 digits; 2^f is off by 6e-16 at most).  Masked scores (-inf) get n = -2000 and weight 0.
struct Exponent {
    double m, c;
    bool infinite;  // m = +inf: entries equal to it have d = 0
    template <class X>
    __device__ __forceinline__ void set(X top, double scale) {
        m = (double)top;
        c = scale;
        infinite = m > DBL_MAX;
        if (infinite) m = 0x1p200;  // every finite score is infinitely far below
    }
    static __device__ __forceinline__ double pow2(double y) {
        y = fmax(y, -2000.0);
        const double n = rint(y), f = y - n;
        double q = 0x1.e5e9f548e5725p-28;
        q = fma(q, f, 0x1.b6571de2f2351p-24);
        q = fma(q, f, 0x1.62bfe46117445p-20);
        q = fma(q, f, 0x1.ffcb76789860fp-17);
        q = fma(q, f, 0x1.4309130378460p-13);
        q = fma(q, f, 0x1.5d87fe908f88ap-10);
        q = fma(q, f, 0x1.3b2ab6fba385fp-7);
        q = fma(q, f, 0x1.c6b08d7044119p-5);
        q = fma(q, f, 0x1.ebfbdff82c590p-3);
        q = fma(q, f, 0x1.62e42fefa39f7p-1);
        return ldexp(fma(q, f, 1.0), (int)n);
    }
    __device__ __forceinline__ double weight(float x) const {
        double d = (double)x - m;
        if (infinite) d = fmin(d, 0.0);
        return pow2(d * c);
    }
    __device__ __forceinline__ double weight(int32_t x) const {
        const double w = pow2(((double)x - m) * c);
        return x == INT32_MIN ? 0.0 : w;
    }
};

// ------------------------------------------------------------------ a row

template <class S>
struct Row {
    static constexpr int V = S::V;
    const typename S::T* x;
    int n, lead;     // entries; those of the first 16 bytes that precede the row
    int64_t groups;  // of 16 aligned bytes
    __device__ __forceinline__ Row(const SampleArgs& a, int64_t r) {
        x = static_cast<const typename S::T*>(a.data) + r * a.stride;
        n = a.N;
        lead = (int)(((uintptr_t)x & 15) / sizeof(typename S::T));
        groups = ((int64_t)n + lead + V - 1) / V;
    }
    __device__ __forceinline__ int64_t first(int64_t g) const { return g * V - lead; }  // index of its first entry
    // Entries of group g; those outside the row are masked, and not read.
    __device__ __forceinline__ void load(int64_t g, typename S::X (&v)[V]) const {
        const int64_t i = first(g);
        if (i >= 0 && i + V <= n) {
            S::unpack(*reinterpret_cast<const uint4*>(x + i), v);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = i + e >= 0 && i + e < n ? S::widen(x[i + e]) : S::kMasked;
        }
    }
};

// Groups [lo, hi) of region k of a row's `regions`: whole wavefronts' worth, in index order.
struct Region {
    int64_t lo, hi;
    __device__ __forceinline__ Region(int64_t groups, int regions, int k) {
        const int64_t per = (groups + (int64_t)regions * 64 - 1) / ((int64_t)regions * 64) * 64;
        lo = per * k < groups ? per * k : groups;
        hi = lo + per < groups ? lo + per : groups;
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

// ------------------------------------------------------------------ wavefront and workgroup sums

__device__ __forceinline__ double wave_sum(double v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
    for (int o = 32; o > 0; o >>= 1) v += (uint32_t)__shfl_xor((int)v, o, 64);
    return v;
}
template <class X>
__device__ __forceinline__ X wave_max(X v) {
    for (int o = 32; o > 0; o >>= 1) {
        const X p = __shfl_xor(v, o, 64);
        v = p > v ? p : v;
    }
    return v;
}
template <class A>
__device__ __forceinline__ A wave_scan(A v) {  // inclusive
    for (int o = 1; o < 64; o <<= 1) {
        const A p = __shfl_up(v, o, 64);
        if ((int)(threadIdx.x & 63) >= o) v += p;
    }
    return v;
}

// ------------------------------------------------------------------ the draw

// What a region adds: its largest score's key, the weight relative to that score (to the row's in
// cut_kernel), and the number of entries.
struct Part {
    double weight;
    uint32_t key, count;
};

template <int kLanes>
struct PickShared {
    double wave[kLanes / 64];
    int found[kLanes / 64], last[kLanes / 64];
};

// The first kept entry of groups [lo, hi) up to which the weights sum to more than t, or the last one with
// weight (which rounding can leave as the only choice).  weight(v, index): 0 for entries that are not kept.
// Every lane of the workgroup calls it, and gets the answer.
template <int kLanes, class S, class W>
__device__ int64_t pick_in_region(const Row<S>& row, const Region& g, double t, W weight, PickShared<kLanes>& sh) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    double run = 0.0;
    int64_t last = -1;
    for (int64_t g0 = g.lo; g0 < g.hi; g0 += kLanes) {
        typename S::X v[S::V];
        double w[S::V], mine = 0.0;
        const int64_t at = row.first(g0 + tid);
        int own = -1;
        if (g0 + tid < g.hi) {
            row.load(g0 + tid, v);
#pragma unroll
            for (int e = 0; e < S::V; ++e) {
                w[e] = weight(v[e], at + e);
                mine += w[e];
                if (w[e] > 0.0) own = e;
            }
        }
        const double scan = wave_scan(mine);
        if (lane == 63) sh.wave[wave] = scan;
        const u64 has = __ballot(own >= 0);
        const int top = has ? 63 - __clzll(has) : 0;
        const int top_e = __shfl(own, top, 64);
        if (lane == 0) sh.last[wave] = has ? (wave * 64 + top) * S::V + top_e : -1;
        __syncthreads();
        double before = run;
        for (int k = 0; k < wave; ++k) before += sh.wave[k];
        double total = run;
        for (int k = 0; k < kLanes / 64; ++k) total += sh.wave[k];
        // an entry is past t when the sum up to it is; the first lane that holds one
        int e_found = -1;
        double sum = before + (scan - mine);
        if (own >= 0) {
#pragma unroll
            for (int e = 0; e < S::V; ++e) {
                sum += w[e];
                if (e_found < 0 && w[e] > 0.0 && sum > t) e_found = e;
            }
        }
        const u64 past = __ballot(e_found >= 0);
        const int first = past ? __ffsll(past) - 1 : 0;
        const int first_e = __shfl(e_found, first, 64);
        if (lane == 0) sh.found[wave] = past ? (wave * 64 + first) * S::V + first_e : -1;
        __syncthreads();
        const int64_t base = row.first(g0);
        int64_t found = -1;
        for (int k = kLanes / 64 - 1; k >= 0; --k) {
            if (sh.found[k] >= 0) found = base + sh.found[k];
        }
        for (int k = 0; k < kLanes / 64; ++k)
            if (sh.last[k] >= 0) last = base + sh.last[k];
        __syncthreads();
        if (found >= 0) return found;
        run = total;
    }
    return last;
}

// ------------------------------------------------------------------ no filters

constexpr int kAllLanes = 256, kAllWaves = kAllLanes / 64;
constexpr int kFinishLanes = 256;

// Sum of a wavefront's groups [lo, hi) relative to the largest of them, in one pass.
template <class S>
__device__ Part sum_region(const Row<S>& row, const Region& g, double scale) {
    const int lane = threadIdx.x & 63;
    typename S::X top = S::kMasked;
    Exponent ex;
    ex.set(top, scale);
    double sum = 0.0;
    uint32_t count = 0;
    for (int64_t g0 = g.lo; g0 < g.hi; g0 += 64) {
        typename S::X v[S::V];
        if (g0 + lane < g.hi) {
            row.load(g0 + lane, v);
        } else {
#pragma unroll
            for (int e = 0; e < S::V; ++e) v[e] = S::kMasked;
        }
        typename S::X most = v[0];
#pragma unroll
        for (int e = 1; e < S::V; ++e) most = v[e] > most ? v[e] : most;
        if (__any(most > top)) {
            const typename S::X grown = wave_max(most);
            ex.set(grown, scale);
            if (top != S::kMasked) sum *= ex.weight(top);
            top = grown;
        }
#pragma unroll
        for (int e = 0; e < S::V; ++e) {
            sum += ex.weight(v[e]);
            count += v[e] != S::kMasked;
        }
    }
    return Part{wave_sum(sum), S::key(top), wave_sum(count)};
}

// The row's draw from its regions' parts, in parts[0 .. regions).  parts' weights are scaled to the row's
// largest score by the lanes, in place in scaled[].
template <int kLanes, class S>
__device__ void finish_row(const SampleArgs& a, int64_t r, const Row<S>& row, const Parameters& par, const Part* parts,
                           int regions, double* scaled, PickShared<kLanes>& sh) {
    const int tid = threadIdx.x;
    uint32_t top = 0;
    uint64_t count = 0;
    for (int k = 0; k < regions; ++k) {
        top = parts[k].key > top ? parts[k].key : top;
        count += parts[k].count;
    }
    if (count == 0 || par.bad) {
        if (tid == 0) write_nothing(a, r);
        return;
    }
    if (par.T == 0.0f) {
        int first = 0;
        while (parts[first].key != top) ++first;
        const typename S::X best = S::value(top);
        const int64_t found = pick_in_region<kLanes>(
            row, Region(row.groups, regions, first), 0.5,
            [&](typename S::X v, int64_t) { return v == best ? 1.0 : 0.0; }, sh);
        if (tid == 0) {
            a.pick[r] = (int32_t)found;
            if (a.logp) a.logp[r] = 0.0f;
            if (a.kept) a.kept[r] = 1;
        }
        return;
    }
    Exponent ex;
    ex.set(S::value(top), par.scale());
    for (int k = tid; k < regions; k += kLanes)
        scaled[k] = parts[k].count ? parts[k].weight * ex.weight(S::value(parts[k].key)) : 0.0;
    __syncthreads();
    double sum = 0.0;
    int target = 0;
    for (int k = 0; k < regions; ++k) {
        sum += scaled[k];
        if (scaled[k] > 0.0) target = k;
    }
    const double t = ((double)(a.rnd[r] >> 11) * 0x1p-53) * sum;
    double before = 0.0;
    for (int k = 0; k < regions; ++k) {
        if (before + scaled[k] > t) {
            target = k;
            break;
        }
        if (k == target) break;
        before += scaled[k];
    }
    const int64_t found = pick_in_region<kLanes>(
        row, Region(row.groups, regions, target), t - before,
        [&](typename S::X v, int64_t) { return ex.weight(v); }, sh);
    if (tid == 0) {
        a.pick[r] = (int32_t)found;
        if (a.logp) {
            const double v = (double)S::widen(row.x[found]), m = (double)S::value(top);
            const double z = v == m ? 0.0 : (v - m) / (double)par.T;
            a.logp[r] = (float)(z - log(sum));
        }
        if (a.kept) a.kept[r] = (int32_t)count;
    }
}

// A row's split s of `splits`: workgroup r * splits + s.  With one split the row ends here.
template <int kType>
__global__ void __launch_bounds__(kAllLanes) all_kernel(SampleArgs a, int splits, Part* parts) {
    using S = Scores<kType>;
    __shared__ Part own[kAllWaves];
    __shared__ double scaled[kAllWaves];
    __shared__ PickShared<kAllLanes> sh;
    const int64_t r = a.row0 + blockIdx.x / splits;
    const int s = blockIdx.x % splits, wave = threadIdx.x >> 6;
    const Row<S> row(a, r);
    const Parameters par(a, r);
    const Part p = sum_region(row, Region(row.groups, splits * kAllWaves, s * kAllWaves + wave),
                              par.T > 0.0f ? par.scale() : 0.0);
    if (splits > 1) {
        if ((threadIdx.x & 63) == 0) parts[(r * splits + s) * kAllWaves + wave] = p;
        return;
    }
    if ((threadIdx.x & 63) == 0) own[wave] = p;
    __syncthreads();
    finish_row<kAllLanes>(a, r, row, par, own, kAllWaves, scaled, sh);
}

constexpr int kMaxSplits = 64;

template <int kType>
__global__ void __launch_bounds__(kFinishLanes) finish_kernel(SampleArgs a, int splits, const Part* parts) {
    using S = Scores<kType>;
    __shared__ Part own[kMaxSplits * kAllWaves];
    __shared__ double scaled[kMaxSplits * kAllWaves];
    __shared__ PickShared<kFinishLanes> sh;
    const int64_t r = a.row0 + blockIdx.x;
    const int regions = splits * kAllWaves;
    for (int k = threadIdx.x; k < regions; k += kFinishLanes) own[k] = parts[r * regions + k];
    __syncthreads();
    finish_row<kFinishLanes>(a, r, Row<S>(a, r), Parameters(a, r), own, regions, scaled, sh);
}

// ------------------------------------------------------------------ filters

constexpr int kCutLanes = 1024, kCutWaves = kCutLanes / 64;
constexpr int kBins = 2048;
constexpr int kList = 512;

struct CutShared {
    uint32_t count[kBins];
    u64 weight[kBins];
    u64 list[kList];
    u64 list_w[kList];
    u64 wave_c[kCutWaves], wave_w[kCutWaves];
    u64 above_c, above_w, total_w, found, found_w;
    uint32_t bin, in_bin, listed, lo, hi;
    Part part[kCutWaves];
    PickShared<kCutLanes> pick;
};

// An entry's place in the order (descending score, ascending index): smaller is earlier.
__device__ __forceinline__ u64 place_of(uint32_t key, int64_t index) {
    return ((u64)~key << 32) | (u64)(uint32_t)index;
}

template <class S>
struct Cutter {
    using X = typename S::X;
    const Row<S>& row;
    Region mine;  // this wavefront's
    Exponent ex;
    X top;
    float bins_per;  // level-0 bins per unit of score
    double unit;     // whole-number weights are w * unit, rounded: sums below 2^62
    bool weights;    // top-p is on
    CutShared& sh;

    __device__ __forceinline__ u64 fixed(X v) const { return (u64)rint(ex.weight(v) * unit); }
    // Distance bins: equal scores share one, and a lower score is never in an earlier one.  NaN (inf - inf, or the
    // top itself where bins_per is infinite) goes to the first bin, what is past the range to the last.
    __device__ __forceinline__ uint32_t bin_of(X v) const {
        const float b = S::below(top, v) * bins_per;
        return b >= (float)(kBins - 1) ? kBins - 1 : b > 0.0f ? (uint32_t)b : 0u;
    }
    // body(v, index) for every entry of this wavefront's region that is not masked.
    template <class B>
    __device__ __forceinline__ void walk(B body) const {
        const int lane = threadIdx.x & 63;
        for (int64_t g = mine.lo + lane; g < mine.hi; g += 64) {
            X v[S::V];
            row.load(g, v);
            const int64_t i = row.first(g);
#pragma unroll
            for (int e = 0; e < S::V; ++e)
                if (v[e] != S::kMasked) body(v[e], i + e);
        }
    }

    __device__ void clear_bins() {
        for (int b = threadIdx.x; b < kBins; b += kCutLanes) {
            sh.count[b] = 0;
            sh.weight[b] = 0;
        }
        __syncthreads();
    }

    // The bin, from 0 up, in which the count passes want or the weight reaches goal; above_c and above_w of the
    // earlier ones are added to those of the call.
    template <bool kByWeight>
    __device__ void cross(u64 want, double goal, u64 above_c, u64 above_w) {
        const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
        const u64 c0 = sh.count[2 * tid], c1 = sh.count[2 * tid + 1];
        const u64 w0 = sh.weight[2 * tid], w1 = sh.weight[2 * tid + 1];
        const u64 sc = wave_scan(c0 + c1), sw = wave_scan(w0 + w1);
        if (lane == 63) {
            sh.wave_c[wave] = sc;
            sh.wave_w[wave] = sw;
        }
        __syncthreads();
        u64 ec = above_c + sc - (c0 + c1), ew = above_w + sw - (w0 + w1);
        for (int k = 0; k < wave; ++k) {
            ec += sh.wave_c[k];
            ew += sh.wave_w[k];
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const u64 c = q ? c1 : c0, w = q ? w1 : w0;
            const bool here = kByWeight ? (double)ew < goal && (double)(ew + w) >= goal : ec < want && ec + c >= want;
            if (here) {
                sh.bin = 2 * tid + q;
                sh.in_bin = (uint32_t)c;
                sh.above_c = ec;
                sh.above_w = ew;
            }
            ec += c;
            ew += w;
        }
        __syncthreads();
    }

    // Index place of the number-th entry (from 1) whose score is v, in index order.
    __device__ u64 nth_equal(X v, u64 number) {
        const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
        uint32_t n = 0;
        walk([&](X x, int64_t) { n += x == v; });
        const uint32_t in_region = wave_sum(n);
        if (lane == 0) sh.wave_c[wave] = in_region;
        __syncthreads();
        u64 before = 0;
        for (int k = 0; k < wave; ++k) before += sh.wave_c[k];
        if (before < number && before + in_region >= number) {
            u64 seen = before;
            for (int64_t g0 = mine.lo; g0 < mine.hi; g0 += 64) {
                X x[S::V];
                uint32_t here = 0;
                if (g0 + lane < mine.hi) {
                    row.load(g0 + lane, x);
#pragma unroll
                    for (int e = 0; e < S::V; ++e) here += x[e] == v;
                }
                const uint32_t scan = wave_scan(here);
                u64 at = seen + scan - here;
                if (here > 0 && at < number && at + here >= number) {
                    for (int e = 0; e < S::V; ++e)
                        if (x[e] == v && ++at == number) sh.found = place_of(S::key(v), row.first(g0 + lane) + e);
                }
                seen += (uint32_t)__shfl((int)scan, 63, 64);
                if (seen >= number) break;
            }
        }
        __syncthreads();
        const u64 r = sh.found;
        __syncthreads();
        return r;
    }

    // The entry at which the count reaches want (kByWeight false) or the weight reaches goal, in the order; the
    // level-0 bins hold their sums.  *up_to: the weight up to and with it (where weights are summed).
    template <bool kByWeight>
    __device__ u64 cut(u64 want, double goal, u64* up_to) {
        const int tid = threadIdx.x;
        cross<kByWeight>(want, goal, 0, 0);
        bool level0 = true;
        uint32_t lo = 0, hi = 0;  // keys of the bin, after level 0
        for (;;) {
            const uint32_t bin = sh.bin;
            const u64 above_c = sh.above_c, above_w = sh.above_w;
            __syncthreads();
            if (tid == 0) {
                sh.listed = 0;
                sh.lo = 0xFFFFFFFFu;
                sh.hi = 0;
            }
            __syncthreads();
            // the bin's entries into the list, and their range of keys
            uint32_t least = 0xFFFFFFFFu, most = 0;
            walk([&](X v, int64_t i) {
                const uint32_t k = S::key(v);
                if (level0 ? bin_of(v) != bin : k < lo || k > hi) return;
                least = k < least ? k : least;
                most = k > most ? k : most;
                const uint32_t at = atomicAdd(&sh.listed, 1u);
                if (at < kList) sh.list[at] = place_of(k, i);
            });
            if (most >= least) {
                atomicMin(&sh.lo, least);
                atomicMax(&sh.hi, most);
            }
            __syncthreads();
            level0 = false;
            lo = sh.lo;
            hi = sh.hi;
            const uint32_t number = sh.listed;
            if (number <= kList) {
                // each lane's entry against all: how many come before it, and their weight
                u64 mine_at = 0, w = 0;
                if (tid < (int)number) {
                    mine_at = sh.list[tid];
                    w = weights ? fixed(S::value(~(uint32_t)(mine_at >> 32))) : 0;
                    sh.list_w[tid] = w;
                }
                __syncthreads();
                if (tid < (int)number) {
                    u64 before = 0, before_w = above_w;
                    for (uint32_t j = 0; j < number; ++j) {
                        const bool earlier = sh.list[j] < mine_at;
                        before += earlier;
                        before_w += earlier ? sh.list_w[j] : 0;
                    }
                    const bool here = kByWeight ? (double)before_w < goal && (double)(before_w + w) >= goal
                                                : above_c + before + 1 == want;
                    if (here) {
                        sh.found = mine_at;
                        sh.found_w = before_w + w;
                    }
                }
                __syncthreads();
                const u64 r = sh.found;
                *up_to = sh.found_w;
                __syncthreads();
                return r;
            }
            if (lo == hi) {  // equal scores: as many of them as it takes, in index order
                const X v = S::value(lo);
                const u64 w = weights ? fixed(v) : 0;
                u64 r;
                if (kByWeight) {
                    const double q = (goal - (double)above_w) / (double)w;  // w > 0: the weight passes goal in this bin
                    r = q < 1.0 ? 1 : q >= (double)number ? number : (u64)q;
                    while (r > 1 && (double)(above_w + (r - 1) * w) >= goal) --r;
                    while (r < number && (double)(above_w + r * w) < goal) ++r;
                } else {
                    r = want - above_c;
                }
                *up_to = above_w + r * w;
                return nth_equal(v, r);
            }
            // split the range of keys: 2,048 bins from the largest key down
            const int shift = 32 - __clz((hi - lo) >> 11);
            clear_bins();
            walk([&](X v, int64_t) {
                const uint32_t k = S::key(v);
                if (k < lo || k > hi) return;
                const uint32_t b = (hi - k) >> shift;
                atomicAdd(&sh.count[b], 1u);
                if (weights) atomicAdd(&sh.weight[b], fixed(v));
            });
            __syncthreads();
            cross<kByWeight>(want, goal, above_c, above_w);
            const uint32_t b = sh.bin;
            const uint32_t top_key = hi - (b << shift);
            const uint32_t span = (1u << shift) - 1;
            lo = top_key - lo > span ? top_key - span : lo;
            hi = top_key;
        }
    }
    __device__ void fill_bins(bool counts) {
        clear_bins();
        walk([&](X v, int64_t) {
            const uint32_t b = bin_of(v);
            if (counts) atomicAdd(&sh.count[b], 1u);
            if (weights) atomicAdd(&sh.weight[b], fixed(v));
        });
        __syncthreads();
    }
    __device__ u64 total_weight() {
        const int wave = threadIdx.x >> 6;
        u64 w = sh.weight[2 * threadIdx.x] + sh.weight[2 * threadIdx.x + 1];
        w = wave_scan(w);
        if ((threadIdx.x & 63) == 63) sh.wave_w[wave] = w;
        __syncthreads();
        w = 0;
        for (int k = 0; k < kCutWaves; ++k) w += sh.wave_w[k];
        __syncthreads();
        return w;
    }
};

// The smallest key whose weight is at least q, by 64 probes a round; every lane of a wavefront calls it.
template <class S>
__device__ uint32_t key_of_weight(const Exponent& ex, typename S::X top, double q) {
    const int lane = threadIdx.x & 63;
    uint32_t lo = S::key(S::kMasked), hi = S::key(top);  // weight(lo) < q <= weight(hi)
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo) / 65 + 1;
        const u64 probe = (u64)lo + (u64)step * (lane + 1);
        const bool reached = probe >= hi || ex.weight(S::value((uint32_t)probe)) >= q;
        const u64 m = __ballot(reached);  // never 0 in the last lane: lo + 64 step >= hi - step
        const int first = m ? __ffsll(m) - 1 : 64;
        const u64 up = (u64)lo + (u64)step * (first + 1);
        lo += step * first;
        hi = up < hi ? (uint32_t)up : hi;
    }
    return hi;
}

template <int kType>
__global__ void __launch_bounds__(kCutLanes) cut_kernel(SampleArgs a) {
    using S = Scores<kType>;
    using X = typename S::X;
    __shared__ CutShared sh;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t r = a.row0 + blockIdx.x;
    const Row<S> row(a, r);
    const Parameters par(a, r);
    const Region mine(row.groups, kCutWaves, wave);

    // the largest score, the smallest one, the number of entries
    X top = S::kMasked, low = S::value(0xFFFFFFFFu - (kType == HX_SCORE_I32 ? 0u : 0x7FFFFFu));
    uint32_t eligible = 0;
    for (int64_t g = mine.lo + lane; g < mine.hi; g += 64) {
        X v[S::V];
        row.load(g, v);
#pragma unroll
        for (int e = 0; e < S::V; ++e) {
            top = v[e] > top ? v[e] : top;
            low = v[e] != S::kMasked && v[e] < low ? v[e] : low;
            eligible += v[e] != S::kMasked;
        }
    }
    if (tid == 0) sh.listed = sh.hi = 0;
    if (tid == 0) sh.lo = 0xFFFFFFFFu;
    __syncthreads();
    eligible = wave_sum(eligible);
    if (eligible) {
        const uint32_t most = wave_max(S::key(top)), least = ~wave_max(~S::key(low));
        if (lane == 0) {
            atomicAdd(&sh.listed, eligible);
            atomicMax(&sh.hi, most);
            atomicMin(&sh.lo, least);
        }
    }
    __syncthreads();
    eligible = sh.listed;
    if (eligible == 0 || par.bad) {
        if (tid == 0) write_nothing(a, r);
        return;
    }
    top = S::value(sh.hi);
    low = S::value(sh.lo);
    __syncthreads();

    const bool greedy = par.T == 0.0f;
    // weights past 24 T below the top add less than 4e-11 each: their bins need no width of their own
    const float reach = 24.0f * par.T, spread = S::below(top, low);
    Exponent ex;
    ex.set(top, greedy ? 0.0 : par.scale());
    Cutter<S> cut{row, mine, ex, top, (float)(kBins - 1) / (reach < spread ? reach : spread), 0.0, false, sh};
    u64 last = ~(u64)0;  // place of the last kept entry
    if (greedy || par.q > 1.0f || par.p <= 0.0f) {
        last = cut.nth_equal(top, 1);  // one entry is kept always
    } else {
        const bool by_k = par.k > 0 && (uint32_t)par.k < eligible, by_p = par.p < 1.0f;
        cut.weights = by_p;
        cut.unit = ldexp(1.0, 62 - (row.n > 1 ? 32 - __clz(row.n - 1) : 0));
        if (by_k || by_p) {
            cut.fill_bins(by_k);
            u64 total = by_p ? cut.total_weight() : 0, up_to = 0;
            if (by_k) {
                last = cut.template cut<false>((u64)par.k, 0.0, &up_to);
                total = up_to;
            }
            if (by_p) {
                // within the first k: their weight reaches p of itself before the last of them does
                if (by_k) cut.fill_bins(true);
                const u64 at = cut.template cut<true>(0, (double)par.p * (double)total, &up_to);
                last = at < last ? at : last;
            }
        }
        if (par.q > 0.0f) {
            const u64 at = place_of(key_of_weight<S>(ex, top, (double)par.q), 0xFFFFFFFFll);
            last = at < last ? at : last;
        }
    }

    // weight and number of the kept entries, by region
    const bool all = last == ~(u64)0;
    const X edge = all ? S::kMasked : S::value(~(uint32_t)(last >> 32));
    const int64_t edge_at = (int64_t)(uint32_t)last;
    const auto weight = [&](X v, int64_t i) {
        const bool kept = v != S::kMasked && (v > edge || (v == edge && i <= edge_at));
        return !kept ? 0.0 : greedy ? 1.0 : ex.weight(v);
    };
    double sum = 0.0;
    uint32_t number = 0;
    for (int64_t g = mine.lo + lane; g < mine.hi; g += 64) {
        X v[S::V];
        row.load(g, v);
        const int64_t i = row.first(g);
#pragma unroll
        for (int e = 0; e < S::V; ++e) {
            if (v[e] == S::kMasked || v[e] < edge || (v[e] == edge && i + e > edge_at)) continue;
            sum += greedy ? 1.0 : ex.weight(v[e]);
            ++number;
        }
    }
    sum = wave_sum(sum);
    number = wave_sum(number);
    if (lane == 0) sh.part[wave] = Part{sum, 0u, number};
    __syncthreads();
    double S_all = 0.0;
    u64 kept = 0;
    int target = 0;
    for (int k = 0; k < kCutWaves; ++k) {
        S_all += sh.part[k].weight;
        kept += sh.part[k].count;
        if (sh.part[k].weight > 0.0) target = k;
    }
    const double t = ((double)(a.rnd[r] >> 11) * 0x1p-53) * S_all;
    double before = 0.0;
    for (int k = 0; k < target; ++k) {
        if (before + sh.part[k].weight > t) {
            target = k;
            break;
        }
        before += sh.part[k].weight;
    }
    const int64_t found = pick_in_region<kCutLanes>(row, Region(row.groups, kCutWaves, target), t - before, weight, sh.pick);
    if (tid == 0) {
        a.pick[r] = (int32_t)found;
        if (a.logp) {
            const double v = (double)S::widen(row.x[found]), m = (double)top;
            const double z = v == m ? 0.0 : (v - m) / (double)par.T;
            a.logp[r] = greedy ? 0.0f : (float)(z - log(S_all));
        }
        if (a.kept) a.kept[r] = (int32_t)kept;
    }
}

// Workgroups a row without filters is split into: until the chip has two for every CU, with 4,096 entries
// left to each.
int splits_of(int32_t R, int32_t N) {
    int64_t s = 512 / R, most = N / 4096;
    if (s > most) s = most;
    if (s > kMaxSplits) s = kMaxSplits;
    return s < 1 ? 1 : (int)s;
}

constexpr int32_t kRowsPerLaunch = 1 << 20;  // a grid has fewer than 2^32 lanes

template <int kType>
hipError_t launch(SampleArgs a, void* workspace, hipStream_t s) {
    const int splits = splits_of(a.R, a.N);  // 1 where a second launch is needed
    Part* parts = static_cast<Part*>(workspace);
    for (int64_t r0 = 0; r0 < a.R; r0 += kRowsPerLaunch) {
        const unsigned rows = (unsigned)(a.R - r0 < kRowsPerLaunch ? a.R - r0 : kRowsPerLaunch);
        a.row0 = r0;
        if (a.top_k || a.top_p || a.min_p) {
            hipLaunchKernelGGL(cut_kernel<kType>, dim3(rows), dim3(kCutLanes), 0, s, a);
            continue;
        }
        hipLaunchKernelGGL(all_kernel<kType>, dim3(rows * splits), dim3(kAllLanes), 0, s, a, splits, parts);
        if (splits > 1)
            hipLaunchKernelGGL(finish_kernel<kType>, dim3(rows), dim3(kFinishLanes), 0, s, a, splits, parts);
    }
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int32_t R, int32_t N) {
    const int splits = splits_of(R, N);
    const size_t parts = splits > 1 ? (size_t)R * splits * kAllWaves * sizeof(Part) : 0;
    return (parts + 511) & ~(size_t)255;
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
