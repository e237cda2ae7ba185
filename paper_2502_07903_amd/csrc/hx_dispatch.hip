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
    u64 run[kKeys];           // per-key totals of the rows before
};

// Sum of amount over the earlier rows with this lane's key, the rows before (run) included; every lane of the
// workgroup calls it, keys are below `keys`.  The 1,024 rows' totals are added to run.
__device__ u64 key_prefix(KeySums& s, int keys, int key, bool has, uint32_t amount) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    for (int k = lane; k < keys; k += 64) s.wave[wave][k] = 0;
    const Peers p(has ? key : 0, has);
    u64 below, all;
    peer_sums(p, has ? amount : 0u, &below, &all);
    __builtin_amdgcn_wave_barrier();  // one wavefront's LDS accesses keep their order: the clearing is before this
    if (p.first()) s.wave[wave][key] = all;
    __syncthreads();
    if (tid < keys) {
        u64 at = s.run[tid];
#pragma unroll
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
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (w < wave) v += wave_sum[w];
    __syncthreads();
    return v;
}

// Sums over the chunks (of `number`, rows of kKeys words) of this lane's key, tid mod kKeys: those before chunk `at`
// and all.  Four lanes share a key's chunks, with eight loads in flight each; part: LDS.
template <class W>
__device__ void chunk_sums(const W* words, int keys, int number, int at, u64 (*part)[2][kKeys], u64* before, u64* all) {
    const int key = threadIdx.x % kKeys, share = threadIdx.x / kKeys;
    constexpr int kShares = kLanes / kKeys, kFlight = 8;
    u64 b = 0, a = 0;
    if (key < keys) {
        for (int t0 = share; t0 < number; t0 += kShares * kFlight) {
            W v[kFlight];
#pragma unroll
            for (int k = 0; k < kFlight; ++k) {
                const int t = t0 + k * kShares;
                v[k] = t < number ? words[(int64_t)t * kKeys + key] : 0;
            }
#pragma unroll
            for (int k = 0; k < kFlight; ++k) {
                a += v[k];
                b += t0 + k * kShares < at ? v[k] : 0;
            }
        }
    }
    part[share][0][key] = b;
    part[share][1][key] = a;
    __syncthreads();
    b = a = 0;
#pragma unroll
    for (int k = 0; k < kShares; ++k) {
        b += part[k][0][key];
        a += part[k][1][key];
    }
    __syncthreads();
    *before = b;
    *all = a;
}

// Rows are worked on by chunks of whole 1,024s, a workgroup each, and at most kChunks of them, so that a chunk
// can add up what the others counted by itself.
constexpr int kChunks = 128;
struct Chunks {
    int32_t number, rows;
    explicit Chunks(int32_t n) {
        const int64_t tiles = ((int64_t)n + kLanes - 1) / kLanes;
        const int64_t per = (tiles + kChunks - 1) / kChunks;
        number = (int32_t)((tiles + per - 1) / per);
        rows = (int32_t)(per * kLanes < n ? per * kLanes : n);
    }
};

// ------------------------------------------------------------------ routes

// Running sums of up to so many edges are kept in LDS, by every workgroup (in 32 of the 64 KB that a launch has
// without asking for more); the networks of two sides of 64 nodes fit.
constexpr int kEdgesLds = 4096;

struct RouteArgs {
    int32_t max_p, max_d, max_pd, nets, cand, n_req, chunk;
    const int32_t *n_p, *n_d, *kv_flow;
    const uint64_t* rnd;
    hx_routes o;
    u64* ends;          // [max_pd] running sum of the flows, past kEdgesLds edges
    uint32_t* counts;   // [2][chunks][kKeys] requests of each prefill and decode node, more chunks than one
};

// Running sums of the flows, each lane summing edges next to each other.  Returns their total; D: decode nodes.
__device__ u64 flow_ends(const RouteArgs& a, u64* ends, u64* wave_sum, int* edges_out, int* d_out) {
    const int tid = threadIdx.x;
    const int P = a.n_p[a.cand], D = a.n_d[a.cand];
    const bool ok = P >= 0 && D >= 0 && P <= a.max_p && D <= a.max_d && (int64_t)P * D <= a.max_pd;
    const int edges = ok ? P * D : 0;
    const int per = (edges + kLanes - 1) / kLanes;
    const int lo = tid * per < edges ? tid * per : edges, hi = lo + per < edges ? lo + per : edges;
    u64 mine = 0;
    constexpr int kAhead = kEdgesLds / kLanes;  // loads in flight
    for (int e0 = lo; e0 < hi; e0 += kAhead) {
        int32_t f[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) f[k] = e0 + k < hi ? a.kv_flow[(int64_t)(e0 + k) * a.nets + a.cand] : 0;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            mine += f[k] > 0 ? (u64)f[k] : 0;
            if (e0 + k < hi) ends[e0 + k] = mine;
        }
    }
    const u64 scan = block_scan(mine, wave_sum);
    for (int e = lo; e < hi; ++e) ends[e] += scan - mine;
    __shared__ u64 total;
    if (tid == kLanes - 1) total = scan;
    __syncthreads();
    *edges_out = edges;
    *d_out = D;
    return total;
}

// Request i's edge: the first one whose running sum is past floor(rnd F / 2^64).
__device__ __forceinline__ void route_one(const RouteArgs& a, int i, const u64* ends, int edges, int D, u64 total,
                                          int* p, int* d) {
    *p = *d = -1;
    if (total > 0) {
        const u64 t = __umul64hi((u64)a.rnd[i], total);
        int lo = 0, hi = edges - 1;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (ends[mid] > t) hi = mid;
            else lo = mid + 1;
        }
        *p = lo / D;
        *d = lo - *p * D;
    }
    a.o.prefill[i] = *p;
    a.o.decode[i] = *d;
}

// Where each node's run starts, from the nodes' totals (run): base, and the starts in run; requests without a
// route (key `nodes`) follow the last.
__device__ void run_starts(KeySums& s, u64* wave_sum, int nodes, int32_t* base) {
    const int tid = threadIdx.x;
    const u64 mine = tid < nodes ? s.run[tid] : 0;
    const u64 end = block_scan(mine, wave_sum);
    if (base && tid <= nodes) base[tid] = (int32_t)(end - mine);
    __syncthreads();
    if (tid <= nodes) s.run[tid] = end - mine;
    __syncthreads();
}

// All of it by one workgroup, up to 1,024 requests: 256 requests over 4 x 4 nodes 8 us, a chain of loads, scans and
// barriers; a call 9 us.
template <bool kLds>
__global__ void __launch_bounds__(kLanes) route_kernel(RouteArgs a) {
    __shared__ u64 wave_sum[kWaves];
    extern __shared__ u64 lds[];  // the running sums, and after them the lists' KeySums
    u64* ends = kLds ? lds : a.ends;
    KeySums& s = *reinterpret_cast<KeySums*>(lds);
    const int tid = threadIdx.x;
    int edges, D, p = -1, d = -1;
    const u64 total = flow_ends(a, ends, wave_sum, &edges, &D);
    const bool in = tid < a.n_req;
    if (in) route_one(a, tid, ends, edges, D, total, &p, &d);
    __syncthreads();
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int nodes = side ? a.max_d : a.max_p, node = side ? d : p;
        int32_t* order = side ? a.o.d_order : a.o.p_order;
        if (!order) continue;
        if (tid <= nodes) s.run[tid] = 0;
        __syncthreads();
        // a first count gives the starts, after which a lane's place is its start and its rank
        const u64 rank = key_prefix(s, nodes + 1, node < 0 ? nodes : node, in, 1u);
        run_starts(s, wave_sum, nodes, side ? a.o.d_base : a.o.p_base);
        if (in) order[s.run[node < 0 ? nodes : node] + rank] = tid;
        __syncthreads();
    }
}

// More requests: a chunk's edges and its counts of every node (65,536 over 64 x 64: 9 us, the edges' running sums in
// every workgroup and twelve steps of search a request),
template <bool kLds>
__global__ void __launch_bounds__(kLanes) route_edges_kernel(RouteArgs a) {
    __shared__ uint32_t count[2][kKeys];
    __shared__ u64 wave_sum[kWaves];
    extern __shared__ u64 lds_ends[];
    const int tid = threadIdx.x;
    int edges, D;
    u64 total;
    if (kLds) {
        total = flow_ends(a, lds_ends, wave_sum, &edges, &D);
    } else {
        // written by the launch before; counts outside the arrays have no edges there either
        const int P = a.n_p[a.cand];
        D = a.n_d[a.cand];
        edges = P >= 0 && D >= 0 && P <= a.max_p && D <= a.max_d && (int64_t)P * D <= a.max_pd ? P * D : 0;
        total = edges ? a.ends[edges - 1] : 0;
    }
    if (tid < 2 * kKeys) (&count[0][0])[tid] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t i1 = i0 + a.chunk < a.n_req ? i0 + a.chunk : a.n_req;
    for (int64_t i = i0 + tid; i < i1; i += kLanes) {
        int p, d;
        route_one(a, (int)i, kLds ? lds_ends : a.ends, edges, D, total, &p, &d);
        if (p >= 0) {
            atomicAdd(&count[0][p], 1u);
            atomicAdd(&count[1][d], 1u);
        }
    }
    __syncthreads();
    if (tid < 2 * kKeys) {
        const int side = tid / kKeys, k = tid % kKeys;
        a.counts[((int64_t)side * gridDim.x + blockIdx.x) * kKeys + k] = count[side][k];
    }
}

__global__ void __launch_bounds__(kLanes) route_ends_kernel(RouteArgs a) {
    __shared__ u64 wave_sum[kWaves];
    int edges, D;
    flow_ends(a, a.ends, wave_sum, &edges, &D);
}

// then its requests to their places: after all requests of earlier nodes, and the earlier chunks' of the same (8 us).
__global__ void __launch_bounds__(kLanes) route_lists_kernel(RouteArgs a) {
    __shared__ KeySums s;
    __shared__ u64 wave_sum[kWaves];
    const int tid = threadIdx.x, side = blockIdx.y;
    const int nodes = side ? a.max_d : a.max_p;
    const int32_t* node = side ? a.o.decode : a.o.prefill;
    int32_t* order = side ? a.o.d_order : a.o.p_order;
    if (!order) return;
    u64 before, all;
    chunk_sums(a.counts + (int64_t)side * gridDim.x * kKeys, nodes, (int)gridDim.x, (int)blockIdx.x,
               reinterpret_cast<u64(*)[2][kKeys]>(s.wave), &before, &all);
    if (tid >= nodes) before = all = 0;
    if (tid <= nodes) s.run[tid] = all;
    __syncthreads();
    run_starts(s, wave_sum, nodes, blockIdx.x == 0 ? (side ? a.o.d_base : a.o.p_base) : nullptr);
    const int64_t i0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t i1 = i0 + a.chunk < a.n_req ? i0 + a.chunk : a.n_req;
    // requests without a route: those of earlier chunks are what their nodes leave of i0
    const u64 earlier = block_scan(before, wave_sum);
    if (tid < nodes) s.run[tid] += before;
    if (tid == kLanes - 1) s.run[nodes] += (u64)i0 - earlier;
    __syncthreads();
    for (int64_t i = i0; i < i1; i += kLanes) {
        const bool in = i + tid < i1;
        const int v = in ? node[i + tid] : 0;
        const u64 at = key_prefix(s, nodes + 1, v < 0 ? nodes : v, in, 1u);
        if (in) order[at] = (int32_t)(i + tid);
    }
}

// ------------------------------------------------------------------ KV memory

// A row of a call, as its tokens or blocks need it.
struct KvRow {
    int64_t top;   // place: free-list index of its first new block (the next ones below it); release: of its last
    int32_t held;  // tokens before the call
    int32_t number;  // place: 1 where served; release: blocks that go
};

struct KvArgs {
    hx_kv_pool p;
    hx_kv_rows r;
    int32_t chunk, chunks;
    const int32_t* n_new;
    int64_t *tok_base, *slots;
    int64_t max_slots;
    uint8_t* placed;
    const uint8_t* done;
    uint32_t factor, shift;  // x / block_size = (x factor >> 32) >> shift for x < 2^31, block_size > 1
    KvRow* row;    // [n_rows]
    u64* total;    // [chunks][kKeys] blocks of each replica's rows
    u64* tokens;   // [chunks]
    u64* moved;    // [kKeys] blocks taken or given
    int64_t *free0, *room;  // [kKeys] entries free before, and left above them
};

struct Replica {
    int64_t free0, room;
    __device__ __forceinline__ Replica(int64_t f, int64_t r) : free0(f), room(r) {}
    __device__ __forceinline__ Replica(const hx_kv_pool& p, int q) {
        const int64_t c = (int64_t)p.base[q + 1] - p.base[q], f = p.free_count[q];
        const int64_t cap = c < 0 ? 0 : c;
        free0 = f < 0 ? 0 : f > cap ? cap : f;
        room = cap - free0;
    }
};

// Row i's lengths and blocks.  place: need; release: the blocks that would go (rows count from the last).
struct Demand {
    int64_t held, add;
    int q;
    uint32_t blocks;
    bool fits;
    template <bool kPlace>
    __device__ __forceinline__ void read(const KvArgs& a, int64_t i, bool in) {
        const int64_t bs = a.p.block_size;
        held = in ? a.r.held[i] : 0;
        q = in ? a.r.replica[i] : -1;
        fits = in && q >= 0 && q < a.p.n_replicas && held >= 0;
        if (kPlace) {
            const int64_t raw = in ? a.n_new[i] : 0;
            add = raw < 0 ? 0 : raw;
            fits = fits && raw >= 0 && held + add <= INT32_MAX;
            // 32-bit divisions: held + add is below 2^31 wherever the quotient counts
            const uint32_t b = (uint32_t)bs;
            const uint32_t b0 = ((uint32_t)held + b - 1) / b, b1 = ((uint32_t)(held + add) + b - 1) / b;
            fits = fits && b1 <= (uint32_t)a.r.max_blocks;
            blocks = fits ? b1 - b0 : 0u;
        } else {
            add = 0;
            const uint32_t nb = ((uint32_t)held + (uint32_t)bs - 1) / (uint32_t)bs;
            fits = fits && a.done[i] && nb <= (uint32_t)a.r.max_blocks;
            blocks = fits ? nb : 0u;
        }
    }
};

// Totals of every chunk: blocks by replica, and tokens (4,096 rows: 3 us, the launch and one chain of loads).
template <bool kPlace>
__global__ void __launch_bounds__(kLanes) kv_totals_kernel(KvArgs a) {
    __shared__ u64 sum[kKeys], wave_sum[kWaves];
    const int tid = threadIdx.x;
    if (tid < kKeys) {
        sum[tid] = 0;
        if (blockIdx.x == 0 && tid < a.p.n_replicas) {
            const Replica q(a.p, tid);
            a.moved[tid] = 0;
            a.free0[tid] = q.free0;
            a.room[tid] = q.room;
        }
    }
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t i1 = i0 + a.chunk < a.r.n_rows ? i0 + a.chunk : a.r.n_rows;
    u64 tokens = 0;
    for (int64_t i = i0 + tid; i < i1; i += kLanes) {
        Demand d;
        d.read<kPlace>(a, kPlace ? i : a.r.n_rows - 1 - i, true);
        tokens += (u64)d.add;
        if (d.blocks) atomicAdd(&sum[d.q], (u64)d.blocks);
    }
    tokens = block_scan(tokens, wave_sum);
    if (tid == kLanes - 1) a.tokens[blockIdx.x] = tokens;
    __syncthreads();
    if (tid < a.p.n_replicas) a.total[(int64_t)blockIdx.x * kKeys + tid] = sum[tid];
}

// x / block_size for x < 2^31.  With 2^(l-1) < b <= 2^l and factor = ceil(2^(31+l) / b), factor b is above 2^(31+l) by
// less than b <= 2^l, so that x factor / 2^(31+l) is above x / b by less than 1 / b, and has the same whole part.
__device__ __forceinline__ uint32_t over_block(const KvArgs& a, uint32_t x) {
    return a.p.block_size == 1 ? x : __umulhi(x, a.factor) >> a.shift;
}

// Slot of token t (counted over all rows) of row i, which starts at token first: its block is the table's, or new
// and entered into it by its first token.
__device__ __forceinline__ int64_t slot_of(const KvArgs& a, int64_t i, const KvRow& row, int64_t t, int64_t first) {
    if (!row.number) return -1;
    const uint32_t b = (uint32_t)a.p.block_size, pos = (uint32_t)(row.held + (int32_t)(t - first));
    const uint32_t col = over_block(a, pos), off = pos - col * b;
    const uint32_t b0 = row.held ? over_block(a, (uint32_t)row.held - 1) + 1 : 0;
    int32_t* entry = a.r.block_table + i * a.r.table_stride + col;
    int32_t block;
    if (col < b0) {
        block = *entry;
    } else {
        block = a.p.free_list[row.top - (int64_t)(col - b0)];
        if (off == 0) *entry = block;
    }
    return (int64_t)block * b + off;
}

constexpr int kFillHere = 4096;  // tokens that place's one workgroup fills in itself

// The rows of a chunk, with the sums of the chunks before (kOne: the only one).  Fills the slots too where fill.
// 256 rows of one token 6 us, 4,096 prompts 8 us: chains of loads, eight ballots for the peers and one for every bit of
// the amounts.
template <bool kPlace, bool kOne>
__global__ void __launch_bounds__(kLanes) kv_rows_kernel(KvArgs a, int fill) {
    __shared__ KeySums s;
    __shared__ u64 wave_sum[kWaves], carry;
    __shared__ int64_t free0[kKeys], limit[kKeys];
    __shared__ u64 moved[kKeys];
    __shared__ int32_t start[kOne ? kLanes : 1];  // kOne: the rows' first tokens and data, for the fill
    __shared__ KvRow own[kOne ? kLanes : 1];
    const int tid = threadIdx.x, R = a.p.n_replicas;
    u64 before = 0, total;
    if (!kOne)
        chunk_sums(a.total, R, (int)blockIdx.x, (int)blockIdx.x, reinterpret_cast<u64(*)[2][kKeys]>(s.wave), &before,
                   &total);
    if (tid < R) {
        const Replica q = kOne ? Replica(a.p, tid) : Replica(a.free0[tid], a.room[tid]);
        s.run[tid] = before;
        moved[tid] = 0;
        free0[tid] = q.free0;
        limit[tid] = kPlace ? q.free0 : q.room;
    }
    if (tid == 0) carry = 0;
    if (!kOne && kPlace) {
        const u64 tokens = block_scan(tid < (int)blockIdx.x ? a.tokens[tid] : 0, wave_sum);  // kChunks <= kLanes
        if (tid == kLanes - 1) carry = tokens;
    }
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t i1 = i0 + a.chunk < a.r.n_rows ? i0 + a.chunk : a.r.n_rows;
    for (int64_t i = i0; i < i1; i += kLanes) {
        const bool in = i + tid < i1;
        const int64_t at_row = kPlace ? i + tid : a.r.n_rows - 1 - (i + tid);
        Demand d;
        d.read<kPlace>(a, at_row, in);
        u64 end = 0;
        if (kPlace) {
            end = block_scan((u64)d.add, wave_sum) + carry;
            __syncthreads();
            if (tid == kLanes - 1) carry = end;
            if (in) a.tok_base[at_row + 1] = (int64_t)end;
            if (in && at_row == 0) a.tok_base[0] = 0;
            // rows past the slots: the rows after them are too, so what those would count does not matter
            d.fits = d.fits && (int64_t)end <= a.max_slots;
            d.blocks = d.fits ? d.blocks : 0u;
        }
        const u64 at = key_prefix(s, R, d.q, d.fits, d.blocks);
        const bool served = d.fits && (d.blocks == 0 || (int64_t)(at + d.blocks) <= limit[d.q]);
        if (served && d.blocks) atomicMax(&moved[d.q], at + d.blocks);
        if (in) {
            const int64_t first = d.fits ? a.p.base[d.q] + free0[d.q] : 0;
            KvRow row;
            row.held = (int32_t)d.held;
            if (kPlace) {
                row.top = first - 1 - (int64_t)at;
                row.number = served;
                a.placed[at_row] = served;
                a.r.held_out[at_row] = (int32_t)(served ? d.held + d.add : d.held);
            } else {
                row.top = first + (int64_t)at + d.blocks - 1;
                row.number = served ? (int32_t)d.blocks : 0;
                a.r.held_out[at_row] = served ? 0 : (int32_t)d.held;
            }
            if (kOne && kPlace && fill) {
                const int64_t tok = (int64_t)end - d.add;
                start[tid] = (int32_t)(tok < kFillHere ? tok : kFillHere);
                own[tid] = row;
            } else {
                a.row[at_row] = row;
            }
        }
    }
    __syncthreads();
    if (tid < R) {
        const int64_t by = (int64_t)moved[tid];
        if (kOne) a.p.free_out[tid] = (int32_t)(kPlace ? free0[tid] - by : free0[tid] + by);
        else if (moved[tid]) atomicMax(&a.moved[tid], moved[tid]);
    }
    if (kPlace && kOne && fill) {
        const int tokens = (int)((int64_t)carry < a.max_slots ? (int64_t)carry : a.max_slots);
        for (int t = tid; t < tokens; t += kLanes) {
            int lo = 0, hi = a.r.n_rows - 1;  // the last row that starts at or before t
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (start[mid] <= t) lo = mid;
                else hi = mid - 1;
            }
            a.slots[t] = slot_of(a, lo, own[lo], t, start[lo]);
        }
    }
}

__device__ __forceinline__ void write_free(const KvArgs& a, bool place) {
    if (a.chunks > 1 && blockIdx.x == 0 && blockIdx.y == 0)
        for (int q = threadIdx.x; q < a.p.n_replicas; q += blockDim.x)
            a.p.free_out[q] = (int32_t)(place ? a.free0[q] - (int64_t)a.moved[q] : a.free0[q] + (int64_t)a.moved[q]);
}

// Slots of kFillTokens tokens: row by row where few rows have them, otherwise each token looks for its row.  Most of a
// workgroup's time is the chain of its loads (the search, the rows, the blocks), so the chain is kept short: 4,096
// prompts, 4.2 million tokens, 15 us, where 34 MB of slots take 7 to write.
constexpr int kFillLanes = 256, kFillTokens = 2048, kFillRows = 8;
__global__ void __launch_bounds__(kFillLanes) place_fill_kernel(KvArgs a) {
    __shared__ int64_t start[kFillRows + 1];
    __shared__ KvRow rows[kFillRows];
    write_free(a, true);
    const int64_t all = a.tok_base[a.r.n_rows];
    const int64_t t0 = (int64_t)blockIdx.x * kFillTokens;
    // the last rows whose tokens start at or before the first token (lanes 0 to 31 of a wavefront) and the last one (32
    // to 63), by 32 probes a round: row lo does, row hi (or none) does not
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int64_t want = half ? t0 + kFillTokens - 1 : t0;
    int64_t lo = 0, hi = a.r.n_rows;
    while (__any(hi - lo > 1)) {
        const int64_t step = hi - lo > 1 ? ((hi - lo - 1) >> 5) + 1 : 1, probe = lo + step * ((lane & 31) + 1);
        const u64 past = __ballot(probe >= hi || a.tok_base[probe] > want);
        const int first = __ffs((unsigned)(past >> (32 * half))) - 1;
        const int64_t up = lo + step * (first + 1);
        lo += step * first;
        hi = up < hi ? up : hi;
    }
    const int64_t first = __shfl(lo, 0, 64), last = __shfl(lo, 32, 64);
    const int64_t n = all < a.max_slots ? all : a.max_slots;
    if (t0 >= n) return;
    const int64_t t1 = t0 + kFillTokens < n ? t0 + kFillTokens : n;
    if (last - first < kFillRows) {
        const int number = (int)(last - first) + 1;
        if ((int)threadIdx.x <= number) start[threadIdx.x] = a.tok_base[first + threadIdx.x];
        if ((int)threadIdx.x < number) rows[threadIdx.x] = a.row[first + threadIdx.x];
        __syncthreads();
        for (int k = 0; k < number; ++k) {
            const KvRow row = rows[k];
            const int64_t from = start[k] > t0 ? start[k] : t0, to = start[k + 1] < t1 ? start[k + 1] : t1;
#pragma unroll 8
            for (int64_t t = from + threadIdx.x; t < to; t += kFillLanes)
                a.slots[t] = slot_of(a, first + k, row, t, start[k]);
        }
        return;
    }
    for (int64_t t = t0 + threadIdx.x; t < t1; t += kFillLanes) {
        int64_t at = first, end = last;
        while (at < end) {
            const int64_t mid = (at + end + 1) / 2;
            if (a.tok_base[mid] <= t) at = mid;
            else end = mid - 1;
        }
        a.slots[t] = slot_of(a, at, a.row[at], t, a.tok_base[at]);
    }
}

// A wavefront copies kCopyBlocks blocks of one row at a time, the row's last block lowest.  8,192 rows: 5 us.
constexpr int kCopyLanes = 256, kCopyBlocks = 1024;
__global__ void __launch_bounds__(kCopyLanes) release_copy_kernel(KvArgs a) {
    write_free(a, false);
    for (int64_t i = (int64_t)blockIdx.x * (kCopyLanes / 64) + (threadIdx.x >> 6); i < a.r.n_rows;
         i += (int64_t)gridDim.x * (kCopyLanes / 64)) {
        const KvRow row = a.row[i];
        const int32_t* table = a.r.block_table + i * a.r.table_stride;
        for (int64_t c0 = (int64_t)blockIdx.y * kCopyBlocks; c0 < row.number; c0 += (int64_t)gridDim.y * kCopyBlocks) {
            const int64_t c1 = c0 + kCopyBlocks < row.number ? c0 + kCopyBlocks : row.number;
#pragma unroll 4
            for (int64_t c = c0 + (threadIdx.x & 63); c < c1; c += 64) a.p.free_list[row.top - c] = table[c];
        }
    }
}

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

struct KvScratch {
    size_t row, total, tokens, moved, free0, room, bytes;
    explicit KvScratch(int32_t n_rows) {
        row = 0;
        total = align256((size_t)n_rows * sizeof(KvRow));
        tokens = total + sizeof(u64) * kChunks * kKeys;
        moved = tokens + align256(sizeof(u64) * kChunks);
        free0 = moved + sizeof(u64) * kKeys;
        room = free0 + sizeof(int64_t) * kKeys;
        bytes = room + sizeof(int64_t) * kKeys;
    }
};

KvArgs kv_args(const hx_kv_pool& p, const hx_kv_rows& r, void* workspace) {
    const Chunks c(r.n_rows);
    const KvScratch w(r.n_rows);
    unsigned char* b = static_cast<unsigned char*>(workspace);
    KvArgs a{};
    a.p = p;
    a.r = r;
    a.chunk = c.rows;
    a.chunks = c.number;
    uint32_t l = 1;
    while ((1u << l) < (uint32_t)p.block_size) ++l;
    const uint64_t one = (uint64_t)1 << (31 + l);
    a.factor = p.block_size == 1 ? 0 : (uint32_t)((one + (uint32_t)p.block_size - 1) / (uint32_t)p.block_size);
    a.shift = l - 1;
    a.row = reinterpret_cast<KvRow*>(b + w.row);
    a.total = reinterpret_cast<u64*>(b + w.total);
    a.tokens = reinterpret_cast<u64*>(b + w.tokens);
    a.moved = reinterpret_cast<u64*>(b + w.moved);
    a.free0 = reinterpret_cast<int64_t*>(b + w.free0);
    a.room = reinterpret_cast<int64_t*>(b + w.room);
    return a;
}

}  // namespace

size_t route_workspace_bytes(int32_t, int32_t, int32_t max_pd, int32_t n_req) {
    const size_t ends = max_pd > kEdgesLds ? align256((size_t)max_pd * sizeof(u64)) : 0;
    const Chunks c(n_req);
    return ends + (c.number > 1 ? sizeof(uint32_t) * 2 * c.number * kKeys : 0) + 256;
}

hipError_t launch_route(const FlowNet& f, int32_t cand, const int32_t* kv_flow, const uint64_t* rnd, const hx_routes& o,
                        void* workspace, hipStream_t s) {
    const Chunks c(o.n_req);
    const bool lds = f.max_pd <= kEdgesLds;
    const size_t ends = lds ? 0 : align256((size_t)f.max_pd * sizeof(u64));
    const size_t dyn = lds ? (size_t)f.max_pd * sizeof(u64) : 0;
    const size_t one = dyn > sizeof(KeySums) ? dyn : sizeof(KeySums);
    unsigned char* b = static_cast<unsigned char*>(workspace);
    const RouteArgs a{f.max_p, f.max_d, f.max_pd, f.N, cand, o.n_req, c.rows, f.n_p, f.n_d, kv_flow, rnd, o,
                      reinterpret_cast<u64*>(b), reinterpret_cast<uint32_t*>(b + ends)};
    prof_mark(kKRoute, false, s);
    if (c.number == 1) {
        if (lds) hipLaunchKernelGGL(route_kernel<true>, dim3(1), dim3(kLanes), one, s, a);
        else hipLaunchKernelGGL(route_kernel<false>, dim3(1), dim3(kLanes), one, s, a);
    } else {
        if (!lds) hipLaunchKernelGGL(route_ends_kernel, dim3(1), dim3(kLanes), 0, s, a);
        if (lds) hipLaunchKernelGGL(route_edges_kernel<true>, dim3(c.number), dim3(kLanes), dyn, s, a);
        else hipLaunchKernelGGL(route_edges_kernel<false>, dim3(c.number), dim3(kLanes), 0, s, a);
        if (o.p_order || o.d_order) hipLaunchKernelGGL(route_lists_kernel, dim3(c.number, 2), dim3(kLanes), 0, s, a);
    }
    prof_mark(kKRoute, true, s);
    return hipGetLastError();
}

size_t kv_workspace_bytes(int32_t n_rows, int32_t) { return KvScratch(n_rows).bytes; }

hipError_t launch_place(const hx_kv_pool& p, const hx_kv_rows& r, const int32_t* n_new, int64_t* tok_base,
                        int64_t* slots, int64_t max_slots, uint8_t* placed, void* workspace, hipStream_t s) {
    KvArgs a = kv_args(p, r, workspace);
    a.n_new = n_new;
    a.tok_base = tok_base;
    a.slots = slots;
    a.max_slots = max_slots;
    a.placed = placed;
    prof_mark(kKPlace, false, s);
    const bool fill = a.chunks == 1 && max_slots <= kFillHere;
    if (a.chunks == 1) {
        hipLaunchKernelGGL((kv_rows_kernel<true, true>), dim3(1), dim3(kLanes), 0, s, a, (int)fill);
    } else {
        hipLaunchKernelGGL(kv_totals_kernel<true>, dim3(a.chunks), dim3(kLanes), 0, s, a);
        hipLaunchKernelGGL((kv_rows_kernel<true, false>), dim3(a.chunks), dim3(kLanes), 0, s, a, 0);
    }
    if (!fill) {
        static_assert(kMaxSlots / kFillTokens * kFillLanes < (int64_t)1 << 32, "a grid's lanes");
        const int64_t fills = (max_slots + kFillTokens - 1) / kFillTokens;
        hipLaunchKernelGGL(place_fill_kernel, dim3((unsigned)(fills < 1 ? 1 : fills)), dim3(kFillLanes), 0, s, a);
    }
    prof_mark(kKPlace, true, s);
    return hipGetLastError();
}

hipError_t launch_release(const hx_kv_pool& p, const hx_kv_rows& r, const uint8_t* done, void* workspace,
                          hipStream_t s) {
    KvArgs a = kv_args(p, r, workspace);
    a.done = done;
    prof_mark(kKRelease, false, s);
    if (a.chunks == 1) {
        hipLaunchKernelGGL((kv_rows_kernel<false, true>), dim3(1), dim3(kLanes), 0, s, a, 0);
    } else {
        hipLaunchKernelGGL(kv_totals_kernel<false>, dim3(a.chunks), dim3(kLanes), 0, s, a);
        hipLaunchKernelGGL((kv_rows_kernel<false, false>), dim3(a.chunks), dim3(kLanes), 0, s, a, 0);
    }
    const int64_t per = kCopyLanes / 64, x = (r.n_rows + per - 1) / per;
    const int64_t y = (r.max_blocks + (int64_t)kCopyBlocks - 1) / kCopyBlocks;
    const dim3 grid((unsigned)(x < 65536 ? x : 65536), (unsigned)(y < 64 ? y : 64));
    hipLaunchKernelGGL(release_copy_kernel, grid, dim3(kCopyLanes), 0, s, a);
    prof_mark(kKRelease, true, s);
    return hipGetLastError();
}

}  // namespace hx
