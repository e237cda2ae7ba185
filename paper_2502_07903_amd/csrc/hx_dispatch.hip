// hx_dispatch.hip -- from a flow assignment to the replicas' paged KV memory: routes of requests
// (hx_route_requests), blocks and token slots of their KV caches (hx_kv_place), and the blocks back to the
// free lists (hx_kv_release).
//
// All of it is whole-number work around one pattern: rows in ascending order, each with a key (its node or
// replica) and an amount, need the sum of the amounts of the earlier rows with the same key.  A wavefront
// gets it from ballots alone (Peers), a workgroup by a scan of the wavefronts' per-key totals in LDS.
#include "hx_internal.h"

namespace hx {
namespace {

constexpr int kLanes = 1024, kWaves = kLanes / 64;
constexpr int kKeys = 256;  // nodes or replicas: at most 255

using u64 = unsigned long long;

// The lanes of a wavefront with this lane's key (0..255): eight ballots.  Lanes with has false have no key.
struct Peers {
    u64 mask, below;
    __device__ __forceinline__ Peers(int key, bool has) {
        mask = __ballot(has);
        for (int b = 0; b < 8; ++b) {
            const u64 m = __ballot((key >> b) & 1);
            mask &= (key >> b) & 1 ? m : ~m;
        }
        if (!has) mask = 0;
        below = mask & (((u64)1 << (threadIdx.x & 63)) - 1);
    }
    __device__ __forceinline__ bool first() const { return mask != 0 && below == 0; }
};

// Sums over the peers below this lane and over all of them: one ballot per bit of the amounts.
__device__ __forceinline__ void peer_sums(const Peers& p, uint32_t amount, u64* below, u64* all) {
    u64 b = 0, a = 0;
    for (int bit = 0; __ballot(amount >> bit != 0); ++bit) {
        const u64 m = __ballot((amount >> bit) & 1);
        b += (u64)__popcll(m & p.below) << bit;
        a += (u64)__popcll(m & p.mask) << bit;
        if (bit == 31) break;
    }
    *below = b;
    *all = a;
}

struct KeySums {
    u64 wave[kWaves][kKeys];  // per-key totals of a wavefront's rows, then the sums before it
    u64 run[kKeys];           // per-key totals of the tiles before
};

// Sum of amount over the earlier rows with this lane's key, tiles before included; every lane of the
// workgroup calls it.  The tile's totals are added to run.
__device__ u64 key_prefix(KeySums& s, int key, bool has, uint32_t amount) {
    const int tid = threadIdx.x, wave = tid >> 6;
    for (int i = tid; i < kWaves * kKeys; i += kLanes) (&s.wave[0][0])[i] = 0;
    __syncthreads();
    const Peers p(has ? key : 0, has);
    u64 below, all;
    peer_sums(p, has ? amount : 0u, &below, &all);
    if (p.first()) s.wave[wave][key] = all;
    __syncthreads();
    if (tid < kKeys) {
        u64 at = s.run[tid];
        for (int w = 0; w < kWaves; ++w) {
            const u64 v = s.wave[w][tid];
            s.wave[w][tid] = at;
            at += v;
        }
        s.run[tid] = at;
    }
    __syncthreads();
    const u64 r = has ? s.wave[wave][key] + below : 0;
    __syncthreads();
    return r;
}

// Inclusive scan over the workgroup's lanes.
__device__ u64 block_scan(u64 v, u64* wave_sum) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const u64 p = __shfl_up(v, o, 64);
        if (lane >= o) v += p;
    }
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += wave_sum[w];
    __syncthreads();
    return v;
}

// ------------------------------------------------------------------ routes

struct RouteArgs {
    int32_t max_p, max_d, max_pd, nets, cand, n_req;
    const int32_t *n_p, *n_d, *kv_flow;
    const uint64_t* rnd;
    hx_routes o;
    u64* ends;  // [max_pd] running sum of the flows
};

__device__ void group(KeySums& s, u64* wave_sum, int nodes, int n_req, const int32_t* node, int32_t* order,
                      int32_t* base) {
    const int tid = threadIdx.x;
    if (tid < kKeys) s.run[tid] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < n_req; i0 += kLanes) {
        const int v = i0 + tid < n_req ? node[i0 + tid] : -1;
        key_prefix(s, v, v >= 0, 1u);
    }
    // where each node's run starts; requests without a route follow the last
    const u64 mine = tid < nodes ? s.run[tid] : 0;
    const u64 end = block_scan(mine, wave_sum);
    if (tid < nodes) base[tid] = (int32_t)(end - mine);
    if (tid == nodes) base[nodes] = (int32_t)end;
    __syncthreads();
    if (tid < kKeys) s.run[tid] = tid <= nodes ? end - mine : 0;
    __syncthreads();
    for (int i0 = 0; i0 < n_req; i0 += kLanes) {
        const bool in = i0 + tid < n_req;
        const int v = in ? node[i0 + tid] : 0;
        const u64 at = key_prefix(s, v < 0 ? nodes : v, in, 1u);
        if (in) order[at] = i0 + tid;
    }
}

__global__ void __launch_bounds__(kLanes) route_kernel(RouteArgs a) {
    __shared__ KeySums s;
    __shared__ u64 wave_sum[kWaves];
    __shared__ u64 carry;
    const int tid = threadIdx.x;
    const int P = a.n_p[a.cand], D = a.n_d[a.cand];
    const bool ok = P >= 0 && D >= 0 && P <= a.max_p && D <= a.max_d && (int64_t)P * D <= a.max_pd;
    const int edges = ok ? P * D : 0;
    if (tid == 0) carry = 0;
    __syncthreads();
    for (int e0 = 0; e0 < edges; e0 += kLanes) {
        const int e = e0 + tid;
        const int32_t f = e < edges ? a.kv_flow[(int64_t)e * a.nets + a.cand] : 0;
        const u64 v = block_scan(f > 0 ? (u64)f : 0, wave_sum) + carry;
        if (e < edges) a.ends[e] = v;
        __syncthreads();
        if (tid == kLanes - 1) carry = v;
        __syncthreads();
    }
    const u64 total = carry;
    for (int i = tid; i < a.n_req; i += kLanes) {
        int p = -1, d = -1;
        if (total > 0) {
            const u64 t = __umul64hi((u64)a.rnd[i], total);
            int lo = 0, hi = edges - 1;  // the first edge whose end is past t
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (a.ends[mid] > t) hi = mid;
                else lo = mid + 1;
            }
            p = lo / D;
            d = lo - p * D;
        }
        a.o.prefill[i] = p;
        a.o.decode[i] = d;
    }
    __syncthreads();
    if (a.o.p_order) group(s, wave_sum, a.max_p, a.n_req, a.o.prefill, a.o.p_order, a.o.p_base);
    __syncthreads();
    if (a.o.d_order) group(s, wave_sum, a.max_d, a.n_req, a.o.decode, a.o.d_order, a.o.d_base);
}

// ------------------------------------------------------------------ KV memory

struct PlaceArgs {
    hx_kv_pool p;
    hx_kv_rows r;
    const int32_t* n_new;
    int64_t *tok_base, *slots;
    int64_t max_slots;
    uint8_t* placed;
};

// Entries of replica q's part of the free list, and how many of them are free.
__device__ __forceinline__ int64_t room_of(const hx_kv_pool& p, int q) {
    const int64_t c = (int64_t)p.base[q + 1] - p.base[q];
    return c < 0 ? 0 : c;
}
__device__ __forceinline__ int64_t free_of(const hx_kv_pool& p, int q) {
    const int64_t c = room_of(p, q), f = p.free_count[q];
    return f < 0 ? 0 : f > c ? c : f;
}

__global__ void __launch_bounds__(kLanes) place_kernel(PlaceArgs a) {
    __shared__ KeySums s;
    __shared__ u64 wave_sum[kWaves], carry;
    __shared__ int64_t free0[kKeys];
    __shared__ u64 taken[kKeys];
    const int tid = threadIdx.x, R = a.p.n_replicas;
    const int64_t bs = a.p.block_size;
    if (tid < kKeys) {
        s.run[tid] = 0;
        taken[tid] = 0;
        free0[tid] = tid < R ? free_of(a.p, tid) : 0;
    }
    if (tid == 0) carry = 0;
    __syncthreads();
    for (int i0 = 0; i0 < a.r.n_rows; i0 += kLanes) {
        const int i = i0 + tid;
        const bool in = i < a.r.n_rows;
        const int64_t held = in ? a.r.held[i] : 0, raw = in ? a.n_new[i] : 0;
        const int q = in ? a.r.replica[i] : -1;
        const int64_t add = raw < 0 ? 0 : raw;
        const u64 end = block_scan((u64)add, wave_sum) + carry;
        __syncthreads();
        if (tid == kLanes - 1) carry = end;
        const int64_t tok = (int64_t)(end - (u64)add);
        if (in && i == 0) a.tok_base[0] = 0;
        if (in) a.tok_base[i + 1] = (int64_t)end;
        const int64_t b0 = (held + bs - 1) / bs, b1 = (held + add + bs - 1) / bs;
        const bool fits = in && q >= 0 && q < R && held >= 0 && raw >= 0 && held + add <= INT32_MAX &&
                          b1 <= a.r.max_blocks && (int64_t)end <= a.max_slots;
        const uint32_t need = fits ? (uint32_t)(b1 - b0) : 0u;
        const u64 at = key_prefix(s, q, fits, need);
        const bool served = fits && (need == 0 || (int64_t)(at + need) <= free0[q]);
        if (in) {
            a.placed[i] = served;
            a.r.held_out[i] = (int32_t)(served ? held + add : held);
        }
        if (served && need > 0) atomicMax(&taken[q], at + need);
        if (in) {
            int32_t* table = a.r.block_table + (int64_t)i * a.r.table_stride;
            const int32_t* top = served && need > 0 ? a.p.free_list + a.p.base[q] + free0[q] - 1 - (int64_t)at : nullptr;
            if (served)
                for (uint32_t c = 0; c < need; ++c) table[b0 + c] = top[-(int64_t)c];
            for (int64_t t = 0; t < add && tok + t < a.max_slots; ++t) {
                const int64_t pos = held + t;
                a.slots[tok + t] = served ? table[pos / bs] * bs + pos % bs : -1;
            }
        }
        __syncthreads();
    }
    if (tid < R) a.p.free_out[tid] = (int32_t)(free0[tid] - (int64_t)taken[tid]);
}

struct ReleaseArgs {
    hx_kv_pool p;
    hx_kv_rows r;
    const uint8_t* done;
};

// Rows in descending order: the last row's last block lands lowest.
__global__ void __launch_bounds__(kLanes) release_kernel(ReleaseArgs a) {
    __shared__ KeySums s;
    __shared__ int64_t free0[kKeys], room[kKeys];
    __shared__ u64 given[kKeys];
    const int tid = threadIdx.x, R = a.p.n_replicas;
    const int64_t bs = a.p.block_size;
    if (tid < kKeys) {
        s.run[tid] = 0;
        given[tid] = 0;
        free0[tid] = tid < R ? free_of(a.p, tid) : 0;
        room[tid] = tid < R ? room_of(a.p, tid) - free0[tid] : 0;
    }
    __syncthreads();
    for (int i0 = 0; i0 < a.r.n_rows; i0 += kLanes) {
        const int i = a.r.n_rows - 1 - (i0 + tid);
        const bool in = i >= 0;
        const int64_t held = in ? a.r.held[i] : 0;
        const int q = in ? a.r.replica[i] : -1;
        const int64_t nb = (held + bs - 1) / bs;
        const bool fits = in && a.done[i] && q >= 0 && q < R && held >= 0 && nb <= a.r.max_blocks;
        const uint32_t blocks = fits ? (uint32_t)nb : 0u;
        const u64 at = key_prefix(s, q, fits, blocks);
        const bool goes = fits && (blocks == 0 || (int64_t)(at + blocks) <= room[q]);
        if (in) a.r.held_out[i] = goes ? 0 : (int32_t)held;
        if (goes && blocks > 0) {
            atomicMax(&given[q], at + blocks);
            const int32_t* table = a.r.block_table + (int64_t)i * a.r.table_stride;
            int32_t* to = a.p.free_list + a.p.base[q] + free0[q] + (int64_t)at;
            for (uint32_t c = 0; c < blocks; ++c) to[c] = table[blocks - 1 - c];
        }
        __syncthreads();
    }
    if (tid < R) a.p.free_out[tid] = (int32_t)(free0[tid] + (int64_t)given[tid]);
}

}  // namespace

size_t route_workspace_bytes(int32_t, int32_t, int32_t max_pd, int32_t) {
    return ((size_t)max_pd * sizeof(u64) + 255) & ~(size_t)255;
}

hipError_t launch_route(const FlowNet& f, int32_t cand, const int32_t* kv_flow, const uint64_t* rnd, const hx_routes& o,
                        void* workspace, hipStream_t s) {
    const RouteArgs a{f.max_p, f.max_d, f.max_pd, f.N, cand, o.n_req, f.n_p, f.n_d, kv_flow, rnd, o,
                      static_cast<u64*>(workspace)};
    prof_mark(kKRoute, false, s);
    hipLaunchKernelGGL(route_kernel, dim3(1), dim3(kLanes), 0, s, a);
    prof_mark(kKRoute, true, s);
    return hipGetLastError();
}

size_t kv_workspace_bytes(int32_t, int32_t) { return 256; }

hipError_t launch_place(const hx_kv_pool& p, const hx_kv_rows& r, const int32_t* n_new, int64_t* tok_base,
                        int64_t* slots, int64_t max_slots, uint8_t* placed, void*, hipStream_t s) {
    const PlaceArgs a{p, r, n_new, tok_base, slots, max_slots, placed};
    prof_mark(kKPlace, false, s);
    hipLaunchKernelGGL(place_kernel, dim3(1), dim3(kLanes), 0, s, a);
    prof_mark(kKPlace, true, s);
    return hipGetLastError();
}

hipError_t launch_release(const hx_kv_pool& p, const hx_kv_rows& r, const uint8_t* done, void*, hipStream_t s) {
    const ReleaseArgs a{p, r, done};
    prof_mark(kKRelease, false, s);
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kLanes), 0, s, a);
    prof_mark(kKRelease, true, s);
    return hipGetLastError();
}

}  // namespace hx
