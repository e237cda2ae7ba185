// hx_sample.hip -- one draw from every row of scores: temperature, top-k, top-p, min-p (hx_sample).
//
// A score becomes a 32-bit key whose order is the scores' order (key_of; 0 = masked), and back.  All three
// filters keep a prefix of the order (descending score, ascending index), so a row's kept set is one pair
// (tau, r): every key above tau, and the first r entries whose key is tau.  The pairs are found by radix
// selection over the key's digits, with counts for top-k and with whole-number weights for top-p (64-bit
// sums: no order of addition changes them); min-p's is a bisection over the keys.  The draw is then the
// first entry, in index order, at which the kept weights pass t = u S.
//
// One workgroup per row; the row is read again for every step.
#include <float.h>
#include <math.h>

#include "hx_internal.h"

namespace hx {
namespace {

constexpr int kLanes = 1024, kWaves = kLanes / 64;
constexpr int kBins = 2048;

// ------------------------------------------------------------------ keys

template <int kType>
struct Scores;
template <>
struct Scores<HX_SCORE_I32> {
    using T = int32_t;
    static __device__ __forceinline__ uint32_t key(T x) { return (uint32_t)x ^ 0x80000000u; }
    static __device__ __forceinline__ double value(uint32_t k) { return (double)(int32_t)(k ^ 0x80000000u); }
};
// Floats: sign and magnitude to two's-complement order; -0 as +0, NaN and -inf as 0 (masked).
struct FloatScores {
    static __device__ __forceinline__ uint32_t key_f(float x) {
        if (!(x > -INFINITY)) return 0u;
        const uint32_t b = __float_as_uint(x + 0.0f);
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    static __device__ __forceinline__ double value(uint32_t k) {
        return (double)__uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
    }
};
template <>
struct Scores<HX_SCORE_F32> : FloatScores {
    using T = float;
    static __device__ __forceinline__ uint32_t key(T x) { return key_f(x); }
};
template <>
struct Scores<HX_SCORE_F16> : FloatScores {
    using T = uint16_t;
    static __device__ __forceinline__ uint32_t key(T x) {
        _Float16 h;
        __builtin_memcpy(&h, &x, 2);
        return key_f((float)h);
    }
};
template <>
struct Scores<HX_SCORE_BF16> : FloatScores {
    using T = uint16_t;
    static __device__ __forceinline__ uint32_t key(T x) { return key_f(__uint_as_float((uint32_t)x << 16)); }
};

// ------------------------------------------------------------------ a row

template <class S>
struct Row {
    const typename S::T* x;
    int n;
    uint32_t top;  // largest key
    double m, T;   // its value, the temperature
    double scale;  // whole-number weights are w * scale, rounded: 2^(62 - ceil(log2 n))
    __device__ __forceinline__ uint32_t key(int i) const { return S::key(x[i]); }
    __device__ __forceinline__ double z(uint32_t k) const { return k == top ? 0.0 : (S::value(k) - m) / T; }
    __device__ __forceinline__ double w(uint32_t k) const { return exp(z(k)); }
    __device__ __forceinline__ uint64_t fixed(uint32_t k) const { return (uint64_t)rint(w(k) * scale); }
};

struct Shared {
    uint32_t count[kBins];
    unsigned long long weight[kBins];
    unsigned long long wave64[2][kWaves];
    double waved[kWaves];
    uint32_t wave32[kWaves];
    unsigned long long out_w, out_above;
    uint32_t out_bin, out_count, out_seen;
    int pick;
};

__device__ __forceinline__ uint32_t block_max(uint32_t v, Shared& sh) {
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    if ((threadIdx.x & 63) == 0) sh.wave32[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int k = 0; k < kWaves; ++k) v = max(v, sh.wave32[k]);
    __syncthreads();
    return v;
}

__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared& sh) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor((unsigned long long)v, o, 64);
    if ((threadIdx.x & 63) == 0) sh.wave64[0][threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int k = 0; k < kWaves; ++k) v += sh.wave64[0][k];
    __syncthreads();
    return v;
}

// Where a prefix of the order ends: at key tau, of whose entries the prefix holds r; above: the
// entries with larger keys and their whole-number weight.
struct Cut {
    uint32_t tau;
    uint64_t r;
    uint64_t above_count, above_weight;
};

// The first key, in descending order, at which the count reaches want (kByWeight false) or the weight
// reaches goal.  Three radix digits of 11, 11 and 10 bits.
template <bool kByWeight, class S>
__device__ Cut select(const Row<S>& row, uint64_t want, double goal, bool weights, Shared& sh) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    uint64_t above_c = 0, above_w = 0;
    uint32_t at_tau = 0;
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0;
        const int bits = level == 2 ? 10 : 11;
        for (int b = tid; b < kBins; b += kLanes) {
            sh.count[b] = 0;
            sh.weight[b] = 0;
        }
        if (tid == 0) sh.out_bin = 0;
        __syncthreads();
        for (int i = tid; i < row.n; i += kLanes) {
            const uint32_t k = row.key(i);
            if (k == 0 || (level > 0 && (k >> (shift + bits)) != prefix)) continue;
            const uint32_t b = (k >> shift) & ((1u << bits) - 1);
            atomicAdd(&sh.count[b], 1u);
            if (weights) atomicAdd(&sh.weight[b], (unsigned long long)row.fixed(k));
        }
        __syncthreads();
        // lane t holds the t-th pair of bins from the top; an exclusive scan over the lanes
        const int hi_bin = kBins - 1 - 2 * tid, lo_bin = hi_bin - 1;
        const uint32_t c0 = sh.count[hi_bin], c1 = sh.count[lo_bin];
        const uint64_t w0 = sh.weight[hi_bin], w1 = sh.weight[lo_bin];
        uint64_t sc = c0 + c1, sw = w0 + w1;
        for (int o = 1; o < 64; o <<= 1) {
            const uint64_t pc = __shfl_up((unsigned long long)sc, o, 64), pw = __shfl_up((unsigned long long)sw, o, 64);
            if ((tid & 63) >= o) {
                sc += pc;
                sw += pw;
            }
        }
        if ((tid & 63) == 63) {
            sh.wave64[0][tid >> 6] = sc;
            sh.wave64[1][tid >> 6] = sw;
        }
        __syncthreads();
        uint64_t bc = above_c, bw = above_w;
        for (int k = 0; k < tid >> 6; ++k) {
            bc += sh.wave64[0][k];
            bw += sh.wave64[1][k];
        }
        uint64_t ec = bc + sc - (c0 + c1), ew = bw + sw - (w0 + w1);
        for (int q = 0; q < 2; ++q) {
            const uint32_t c = q ? c1 : c0;
            const uint64_t w = q ? w1 : w0;
            // the first bin with an entry that reaches the goal: later bins find it reached before them
            const bool reached = kByWeight ? (double)(ew + w) >= goal : ec + c >= want;
            const bool before = kByWeight ? ec > 0 && (double)ew >= goal : ec >= want;
            if (c > 0 && reached && !before) {
                sh.out_bin = q ? lo_bin : hi_bin;
                sh.out_count = c;
                sh.out_above = ec;
                sh.out_w = ew;
            }
            ec += c;
            ew += w;
        }
        __syncthreads();
        prefix = (prefix << bits) | sh.out_bin;
        at_tau = sh.out_count;
        above_c = sh.out_above;
        above_w = sh.out_w;
        __syncthreads();
    }
    Cut cut{prefix, 0, above_c, above_w};
    if (kByWeight) {
        const uint64_t wt = row.fixed(prefix);
        uint64_t r = 1;
        if (wt > 0 && goal > (double)above_w) {
            const double q = (goal - (double)above_w) / (double)wt;
            r = q < 1.0 ? 1 : q >= (double)at_tau ? at_tau : (uint64_t)q;
            while (r > 1 && (double)(above_w + (r - 1) * wt) >= goal) --r;
            while (r < at_tau && (double)(above_w + r * wt) < goal) ++r;
        }
        cut.r = r;
    } else {
        cut.r = want - above_c;
    }
    return cut;
}

template <int kType>
__global__ void __launch_bounds__(kLanes) sample_kernel(SampleArgs a) {
    using S = Scores<kType>;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r = blockIdx.x;
    Row<S> row;
    row.x = static_cast<const typename S::T*>(a.data) + r * a.stride;
    row.n = a.N;
    const float tf = a.temperature ? a.temperature[r] : 1.0f;
    const int32_t kf = a.top_k ? a.top_k[r] : 0;
    const float pf = a.top_p ? a.top_p[r] : 1.0f;
    const float qf = a.min_p ? a.min_p[r] : 0.0f;

    uint32_t top = 0;
    uint64_t some = 0;
    for (int i = tid; i < row.n; i += kLanes) {
        const uint32_t k = row.key(i);
        top = max(top, k);
        some += k != 0;
    }
    top = block_max(top, sh);
    const uint64_t eligible = block_sum(some, sh);
    if (top == 0 || !(tf >= 0.0f) || !(tf <= FLT_MAX) || isnan(pf) || isnan(qf)) {
        if (tid == 0) {
            a.pick[r] = -1;
            if (a.logp) a.logp[r] = -INFINITY;
            if (a.kept) a.kept[r] = 0;
        }
        return;
    }
    row.top = top;
    row.m = S::value(top);
    row.T = (double)tf;
    row.scale = ldexp(1.0, 62 - (row.n > 1 ? 32 - __clz(row.n - 1) : 0));

    // the kept set: keys above tau, and the first ties entries at tau
    uint32_t tau = 0;
    uint64_t ties = 0;
    if (tf == 0.0f) {
        tau = top;
        ties = 1;
    } else {
        const bool by_k = kf > 0 && (uint64_t)kf < eligible, by_p = pf < 1.0f;
        Cut ck{1u, 0, 0, 0};
        if (by_k) {
            ck = select<false>(row, (uint64_t)kf, 0.0, by_p, sh);
            tau = ck.tau;
            ties = ck.r;
        }
        if (by_p) {
            uint64_t total = 0;
            if (by_k) {
                total = ck.above_weight + ck.r * row.fixed(ck.tau);
            } else {
                for (int i = tid; i < row.n; i += kLanes) {
                    const uint32_t k = row.key(i);
                    if (k) total += row.fixed(k);
                }
                total = block_sum(total, sh);
            }
            // a prefix that reaches p of the first K lies within them
            const Cut cp = select<true>(row, 0, (double)pf * (double)total, true, sh);
            if (cp.tau > tau) {
                tau = cp.tau;
                ties = cp.r;
            } else if (cp.tau == tau && cp.r < ties) {
                ties = cp.r;
            }
        }
        if (qf > 1.0f) {  // no entry reaches it: the first one is kept
            tau = top;
            ties = 1;
        } else if (qf > 0.0f) {
            // the smallest key whose weight reaches min-p
            uint32_t lo = 0, hi = top;
            while (hi - lo > 1) {
                const uint32_t mid = lo + (hi - lo) / 2;
                // keys between the masked one and the lowest score have no value of their own: below every score
                if (S::value(mid) <= row.m && row.w(mid) >= (double)qf) hi = mid;
                else lo = mid;
            }
            if (hi > tau) {
                tau = hi;
                ties = UINT64_MAX;
            }
        }
    }

    // the index of the last kept entry at tau: wavefront w reads region [w per, (w + 1) per)
    const int per = (int)((((int64_t)row.n + kLanes - 1) / kLanes) * 64);
    const int64_t lo = (int64_t)wave * per, hi = lo + per < row.n ? lo + per : row.n;
    int64_t last_tie = -1;
    if (tau > 0) {
        uint64_t mine = 0;
        for (int64_t i = lo; i < hi; i += 64) {
            const bool at = i + lane < hi && row.key((int)(i + lane)) == tau;
            mine += __popcll(__ballot(at));
        }
        if (lane == 0) sh.wave64[0][wave] = mine;
        if (tid == 0) sh.pick = row.n;  // every tie is kept
        __syncthreads();
        uint64_t before = 0;
        for (int k = 0; k < wave; ++k) before += sh.wave64[0][k];
        if (before < ties && before + mine >= ties) {
            uint64_t seen = before;
            for (int64_t i = lo; i < hi; i += 64) {
                const unsigned long long at = __ballot(i + lane < hi && row.key((int)(i + lane)) == tau);
                const uint64_t here = __popcll(at & ((lane == 63 ? 0ull : 1ull << (lane + 1)) - 1ull));
                if (((at >> lane) & 1) && seen + here == ties) sh.pick = (int)(i + lane);
                seen += __popcll(at);
                if (seen >= ties) break;
            }
        }
        __syncthreads();
        last_tie = sh.pick;
        __syncthreads();
    }
    const auto kept = [&](uint32_t k, int64_t i) { return k != 0 && (k > tau || (k == tau && i <= last_tie)); };

    // weight and number of the kept entries, by region
    double mine = 0.0;
    uint64_t number = 0;
    for (int64_t i = lo + lane; i < hi; i += 64) {
        const uint32_t k = row.key((int)i);
        if (!kept(k, i)) continue;
        mine += tf == 0.0f ? 1.0 : row.w(k);
        ++number;
    }
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
    if (lane == 0) sh.waved[wave] = mine;
    number = block_sum(number, sh);  // also orders waved
    double sum = 0.0;
    int last_wave = 0;
    for (int k = 0; k < kWaves; ++k) {
        sum += sh.waved[k];
        if (sh.waved[k] > 0.0) last_wave = k;
    }
    const double t = ((double)(a.rnd[r] >> 11) * 0x1p-53) * sum;
    double before = 0.0;
    int target = last_wave;
    for (int k = 0; k < kWaves; ++k) {
        if (before + sh.waved[k] > t) {
            target = k;
            break;
        }
        before += sh.waved[k];
    }
    if (wave != target) return;
    // the target wavefront walks its region; rounding may leave t unreached, then the last entry with weight
    int64_t found = -1, last = -1;
    double run = 0.0;
    for (int k = 0; k < target; ++k) run += sh.waved[k];
    for (int64_t i = lo; i < hi && found < 0; i += 64) {
        const uint32_t k = i + lane < hi ? row.key((int)(i + lane)) : 0u;
        double v = kept(k, i + lane) ? (tf == 0.0f ? 1.0 : row.w(k)) : 0.0;
        const unsigned long long has = __ballot(v > 0.0);
        if (has) last = i + 63 - __clzll(has);
        for (int o = 1; o < 64; o <<= 1) {
            const double p = __shfl_up(v, o, 64);
            if (lane >= o) v += p;
        }
        const unsigned long long past = __ballot(run + v > t) & has;
        if (past) found = i + __ffsll(past) - 1;
        run += __shfl(v, 63, 64);
    }
    if (found < 0) found = last;
    if (lane == 0) {
        a.pick[r] = (int32_t)found;
        if (a.logp) a.logp[r] = tf == 0.0f ? 0.0f : (float)(row.z(row.key((int)found)) - log(sum));
        if (a.kept) a.kept[r] = (int32_t)number;
    }
}

}  // namespace

size_t sample_workspace_bytes(int32_t, int32_t) { return 256; }

hipError_t launch_sample(const SampleArgs& a, void*, hipStream_t s) {
    prof_mark(kKSample, false, s);
    const dim3 grid((unsigned)a.R), block(kLanes);
    if (a.type == HX_SCORE_I32) hipLaunchKernelGGL(sample_kernel<HX_SCORE_I32>, grid, block, 0, s, a);
    else if (a.type == HX_SCORE_F32) hipLaunchKernelGGL(sample_kernel<HX_SCORE_F32>, grid, block, 0, s, a);
    else if (a.type == HX_SCORE_F16) hipLaunchKernelGGL(sample_kernel<HX_SCORE_F16>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(sample_kernel<HX_SCORE_BF16>, grid, block, 0, s, a);
    prof_mark(kKSample, true, s);
    return hipGetLastError();
}

}  // namespace hx
