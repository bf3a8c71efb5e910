// A learned bias of attention for the relative position of its tokens, and the table's gradient.
//
// Of query i and key j, at positions of up to four axes, the bucket is the sum over the axes of map[axis][difference], the difference key - query held between -reach
// and reach; the bias of head h is table[bucket][h].  Tokens of different segments are -inf, rows of queries without a segment (padding) 0.  The
// gradient of table[bucket][h] is the sum of the incoming gradient over all pairs of that bucket.
#pragma once
#include "pcr_vec.h"

namespace pcr {

struct Places {                                                    // of queries or keys
    const void* position; const int32_t* segment;
    int64_t axis, batch, token, segment_batch, segment_token;      // strides
};
typedef uint16_t Places8 __attribute__((ext_vector_type(8)));     // of eight keys
struct Steps { uint32_t run, query, batch; };                      // of an item
struct BiasArgs {
    Places q, k;
    const int32_t* map; const void* table; void* values;           // values: the bias, or its incoming gradient
    int64_t value_batch, value_head, value_query;
    int64_t batch, heads, queries, keys, buckets, runs, items;     // runs: of a row; items: runs of all rows of all sequences
    int64_t step_batch, step_query, step_run;                      // a thread's step to its next item
    int axes, reach, wide, table_float;
    // gradient
    float* part; Places8* places; uint64_t* live;                  // part: [share][head][bucket]; direct: one share, [bucket][head]
    int64_t first_bucket, held_buckets;
    Steps near, far;                                               // from one item of a lane to the next; from the last of those that are under way together to the first of the next ones
    int waves, copies, direct;
};

// The clipped difference of two positions.
__device__ __forceinline__ int apart(int32_t key, int32_t query, int reach) { return min(max(__builtin_elementwise_sub_sat(key, query), -reach), reach); }
__device__ __forceinline__ int apart(int64_t key, int64_t query, int reach) {
    return (int)min(max(__builtin_elementwise_sub_sat(key, query), (int64_t)-reach), (int64_t)reach);
}

enum : uint32_t { kNoBias = 0, kNeverSeen = 1 };                   // behind the buckets: a pair without a bias (0), and one of different segments (-inf)

// An item: a run of V keys of a query.  A row's last run ends with the row, and so begins inside the run before it: every run is whole where a row has V keys at all.
struct Item { int64_t b, i, run; };
__device__ __forceinline__ Item item_at(const BiasArgs& A, int64_t t) {
    Item I;
    if (t >> 32 | A.runs >> 32) {                                  // (a division in 64 bits takes 130 instructions, in 32 bits 25)
        const int64_t row = t / A.runs;
        I.run = t - row * A.runs;
        I.b = row / A.queries;
        I.i = row - I.b * A.queries;
    } else {
        const uint32_t row = (uint32_t)t / (uint32_t)A.runs, b = row / (uint32_t)A.queries;
        I.run = (uint32_t)t - row * (uint32_t)A.runs;
        I.b = b;
        I.i = row - b * (uint32_t)A.queries;
    }
    return I;
}
__device__ __forceinline__ void step_on(Item& I, const BiasArgs& A) {
    I.run += A.step_run;
    if (I.run >= A.runs) { I.run -= A.runs; I.i++; }
    I.i += A.step_query;
    if (I.i >= A.queries) { I.i -= A.queries; I.b++; }
    I.b += A.step_batch;
}

template <int V> __device__ __forceinline__ int64_t first_key(const BiasArgs& A, const Item& I) { return min(I.run * V, max(A.keys - V, (int64_t)0)); }

// Positions (or segments) of an item's keys.  Keys behind the row's end (of rows of fewer than V): of no account.
template <typename P, int V> __device__ __forceinline__ void load_places(const P* from, int64_t stride, int here, P without, P (&at)[V]) {
    if (here == V && stride == 1) {
#pragma unroll
        for (int v = 0; v < V; v += 4) {
            const typename Run<P, 4>::Vec four = reinterpret_cast<const typename Run<P, 4>::Loose*>(from + v)->v;
#pragma unroll
            for (int u = 0; u < 4; u++) at[v + u] = four[u];
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; v++) at[v] = v < here ? from[v * stride] : without;
    }
}
// Adds what the axes of any type and stride make of an item's keys.
template <typename P, int V> __device__ __forceinline__ void sum_axes(const BiasArgs& A, const int32_t* map, const Item& I, int here, int32_t (&sum)[V]) {
    const int width = 2 * A.reach + 1;
    for (int a = 0; a < A.axes; a++) {
        const P query = ((const P*)A.q.position)[a * A.q.axis + I.b * A.q.batch + I.i * A.q.token];
        P at[V];
        load_places<P, V>((const P*)A.k.position + a * A.k.axis + I.b * A.k.batch + first_key<V>(A, I) * A.k.token, A.k.token, here, query, at);
        const int32_t* middle = map + a * width + A.reach;
#pragma unroll
        for (int v = 0; v < V; v++) sum[v] = (int32_t)((uint32_t)sum[v] + (uint32_t)middle[apart(at[v], query, A.reach)]);
    }
}
// The buckets of an item's keys, less `start`: `none` for one that is not below `limit`, `never` for one of another segment, all `none` for a query that is padding.  AXES: so many 32-bit
// positions whose keys, V at least, follow each other in memory, as their segments do; 0: any.
template <int V, int AXES> __device__ __forceinline__ void buckets_of(const BiasArgs& A, const int32_t* map, const Item& I, int here, uint32_t start, uint32_t limit, uint32_t none,
                                                                       uint32_t never, uint32_t (&bucket)[V]) {
    int32_t mine = 0, other[V], sum[V];
#pragma unroll
    for (int v = 0; v < V; v++) sum[v] = (int32_t)(0u - start);
    if constexpr (AXES > 0) {
        const int64_t key = first_key<V>(A, I);
        int32_t query[AXES], at[AXES][V];
#pragma unroll
        for (int a = 0; a < AXES; a++) {
            query[a] = ((const int32_t*)A.q.position)[a * A.q.axis + I.b * A.q.batch + I.i * A.q.token];
            load_places<int32_t, V>((const int32_t*)A.k.position + a * A.k.axis + I.b * A.k.batch + key, 1, V, 0, at[a]);
        }
        if (A.q.segment) {
            mine = A.q.segment[I.b * A.q.segment_batch + I.i * A.q.segment_token];
            load_places<int32_t, V>(A.k.segment + I.b * A.k.segment_batch + key, 1, V, 0, other);
        }
        const int width = 2 * A.reach + 1;
#pragma unroll
        for (int a = 0; a < AXES; a++) {
            const int32_t* middle = map + a * width + A.reach;
#pragma unroll
            for (int v = 0; v < V; v++) sum[v] = (int32_t)((uint32_t)sum[v] + (uint32_t)middle[apart(at[a][v], query[a], A.reach)]);
        }
    } else {
        if (A.wide) sum_axes<int64_t, V>(A, map, I, here, sum);
        else sum_axes<int32_t, V>(A, map, I, here, sum);
        if (A.q.segment) {
            mine = A.q.segment[I.b * A.q.segment_batch + I.i * A.q.segment_token];
            load_places<int32_t, V>(A.k.segment + I.b * A.k.segment_batch + first_key<V>(A, I) * A.k.segment_token, A.k.segment_token, here, mine, other);
        }
    }
#pragma unroll
    for (int v = 0; v < V; v++) bucket[v] = (uint32_t)sum[v] < limit ? (uint32_t)sum[v] : none;
    if (A.q.segment) {
        if (mine < 0) never = none;
#pragma unroll
        for (int v = 0; v < V; v++) bucket[v] = mine >= 0 && other[v] == mine ? bucket[v] : never;
    }
}

template <typename T> __device__ __forceinline__ T table_value(const BiasArgs& A, int64_t at) {
    return A.table_float ? (T)((const float*)A.table)[at] : ((const T*)A.table)[at];
}

// The bias.  Bound by its stores.  H: heads of a workgroup, whose values of a bucket lie side by side in LDS, so that a key costs one read for all of them and its bucket is found
// once; V keys of H heads are V reads and H stores of 16 bytes.  HELD: the map and the table of these heads are in LDS (else read where they are).  us: 16 sequences of 1024 packed
// tokens, 12 heads, 3969 buckets, half, 403 MB 88 (81 at 5.0 TB/s; 136 with the axes in a loop and divisions in 64 bits), 16 heads for one query each of 32 sequences of 4099 keys 5.2.
template <typename T, int H, bool HELD, int AXES> __global__ __launch_bounds__(1024) void k_bias(BiasArgs A) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int V = 16 / sizeof(T);
    typedef typename Run<T, H>::Vec Entry;
    Entry* table = (Entry*)lds;
    int32_t* map = (int32_t*)(lds + ((A.buckets + 2) * sizeof(Entry) + 15) / 16 * 16);
    const int64_t first_head = (int64_t)blockIdx.y * H;
    const int heads = (int)min((int64_t)H, A.heads - first_head);
    if (HELD) {
        T* flat = (T*)lds;
        const int count = (int)A.buckets * H;
        for (int e = threadIdx.x; e < count; e += blockDim.x) {
            const int b = e / H, h = e - b * H;
            flat[e] = h < heads ? table_value<T>(A, b * A.heads + first_head + h) : (T)0.f;
        }
        for (int e = threadIdx.x; e < 2 * H; e += blockDim.x) flat[count + e] = e < H ? (T)0.f : (T)(-__builtin_inff());
        const int places = A.axes * (2 * A.reach + 1);
        for (int e = threadIdx.x; e < places; e += blockDim.x) map[e] = A.map[e];
        __syncthreads();
    }
    int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    Item I = item_at(A, t);
    const int here = (int)min((int64_t)V, A.keys);
    for (; t < A.items; t += (int64_t)gridDim.x * blockDim.x, step_on(I, A)) {
        uint32_t bucket[V];
        const uint32_t count = (uint32_t)A.buckets;
        buckets_of<V, AXES>(A, HELD ? map : A.map, I, here, 0, count, count + kNoBias, count + kNeverSeen, bucket);
        T* out = (T*)A.values + I.b * A.value_batch + first_head * A.value_head + I.i * A.value_query + first_key<V>(A, I);
        if constexpr (HELD) {
            Entry entry[V];
#pragma unroll
            for (int v = 0; v < V; v++) entry[v] = table[bucket[v]];
#pragma unroll
            for (int h = 0; h < H; h++) {
                if (h >= heads) break;
                typename Run<T, V>::Vec row;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    if constexpr (H == 1) row[v] = entry[v];
                    else row[v] = entry[v][h];
                }
                if (here == V) reinterpret_cast<typename Run<T, V>::Loose*>(out)->v = row;
                else {
#pragma unroll
                    for (int v = 0; v < V; v++)
                        if (v < here) out[v] = row[v];
                }
                out += A.value_head;
            }
        } else {
            for (int h = 0; h < heads; h++) {
#pragma unroll
                for (int v = 0; v < V; v++)
                    if (v < here)
                        out[v] = bucket[v] < A.buckets ? table_value<T>(A, bucket[v] * A.heads + first_head + h) : (T)(bucket[v] == A.buckets + kNoBias ? 0.f : -__builtin_inff());
                out += A.value_head;
            }
        }
    }
}

// ---- the table's gradient ----
//
// First every pair's bucket is found once for all heads (k_bias_places), as 16 bits; then the values are added by a kernel that reads both side by side, share by
// share of the items (k_bias_bins), and the shares' sums are added in 64 bits (k_bias_sums).  Items are runs of eight keys here whatever the type.
// us (what reading the gradient takes at 5.0 TB/s): 4096 x 4096 pairs of 12 heads in 31 buckets, bfloat 116 (81): 16 + 97 + 5; four sequences of 1501 packed tokens, 12 heads, 3969 buckets
// 106 (43): 14 + 85 + 7.  With the buckets found by every workgroup for its own heads, in a tile that its wavefronts shared, these were 144 and 239.
constexpr int kRun = 8;                                            // keys of an item

__host__ __device__ __forceinline__ int bins_of(int64_t held, int copies) { return (int)held * copies; }

// places[item][key]: the bin of the pair, in the copy for the lane that will add it, or behind the bins one of 64 that nobody reads.  Buckets outside
// first_bucket .. first_bucket + held_buckets - 1 have none.  live: a bit for every item of 64 that has a pair.
template <bool HELD, int AXES> __global__ __launch_bounds__(256) void k_bias_places(BiasArgs A) {
    extern __shared__ __attribute__((aligned(16))) int32_t held_map[];
    if (HELD) {
        const int places = A.axes * (2 * A.reach + 1);
        for (int e = threadIdx.x; e < places; e += 256) held_map[e] = A.map[e];
        __syncthreads();
    }
    const int here = (int)min((int64_t)kRun, A.keys), lane = threadIdx.x & 63;
    const uint32_t nowhere = bins_of(A.held_buckets, A.copies) + lane, held = (uint32_t)A.held_buckets, copy = lane & (A.copies - 1);
    const int shift = 31 - __clz(A.copies);
    const int64_t end = (A.items + 63) / 64 * 64;
    int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    Item I = item_at(A, t);
    for (; t < end; t += (int64_t)gridDim.x * 256, step_on(I, A)) {
        uint32_t place[kRun], least = ~0u;
#pragma unroll
        for (int v = 0; v < kRun; v++) place[v] = nowhere;
        if (t < A.items) {
            uint32_t bucket[kRun];
            buckets_of<kRun, AXES>(A, HELD ? held_map : A.map, I, here, (uint32_t)A.first_bucket, held, ~0u, ~0u, bucket);
            const int again = (int)(I.run * kRun - first_key<kRun>(A, I));     // (keys of the run before)
            if (again > 0 || here < kRun) {
#pragma unroll
                for (int v = 0; v < kRun; v++)
                    if (v < again || v >= here) bucket[v] = ~0u;
            }
#pragma unroll
            for (int v = 0; v < kRun; v++) {
                place[v] = bucket[v] < held ? bucket[v] << shift | copy : nowhere;
                least = min(least, bucket[v]);
            }
        }
        Places8 packed;
#pragma unroll
        for (int v = 0; v < kRun; v++) packed[v] = (uint16_t)place[v];
        A.places[t] = packed;
        const uint64_t live = __ballot(least < held);
        if (lane == 0) A.live[t / 64] = live;
    }
}

// Where an item's values lie, stepped through with little arithmetic.
template <typename T> struct Place {
    const T* row;
    uint32_t b, i, run;
    __device__ __forceinline__ void begin(const BiasArgs& A, const T* values, int64_t t) {
        const Item I = item_at(A, t);
        b = (uint32_t)I.b; i = (uint32_t)I.i; run = (uint32_t)I.run;
        row = values + b * A.value_batch + i * A.value_query;
    }
    __device__ __forceinline__ void on(const BiasArgs& A, const T* values, const Steps& by) {
        run += by.run;
        const bool more = run >= (uint32_t)A.runs;
        if (more || by.query | by.batch) {
            if (more) { run -= (uint32_t)A.runs; i++; }
            i += by.query;
            b += by.batch;
            if (i >= (uint32_t)A.queries) { i -= (uint32_t)A.queries; b++; }
            row = values + b * A.value_batch + i * A.value_query;
        }
    }
    __device__ __forceinline__ const T* at(uint32_t last) const { return row + min(run * kRun, last); }      // last: where a row's last run begins
};
// A run of values as it lies in memory; 8 of 16 or 32 bits.
template <typename T> struct Eight {
    typename Run<T, 16 / sizeof(T)>::Vec part[sizeof(T) / 2];
    template <bool WHOLE> __device__ __forceinline__ void load(const T* p, int here) {
        constexpr int V = 16 / sizeof(T);
        if constexpr (WHOLE) {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(T) / 2); i++) part[i] = reinterpret_cast<const typename Run<T, V>::Loose*>(p + i * V)->v;
        } else {
#pragma unroll
            for (int v = 0; v < kRun; v++) part[v / V][v % V] = v < here ? p[v] : (T)0.f;
        }
    }
    __device__ __forceinline__ float at(int v) const { return (float)part[v / (16 / sizeof(T))][v % (16 / sizeof(T))]; }
};

// A wavefront has a share and a head, and bins for that in LDS, in 64 bits, which are its own: they are added to in the order of its instructions, and lanes
// of one instruction that meet in a bin in the order in which the LDS unit takes lanes of the same address: nothing else has a part in it and it has been the same at every call, but no
// document promises it.  (It shows only in sums that 64 bits do not hold exactly.)  Where there are few buckets
// there are several copies of the bins, for the lanes in turn, so that few meet.
// (LDS adds floats of 64 bits in 9 clocks a wavefront's instruction, those of 32 in 193: the long sequence took 1063 us with these.  Sums of up to 64 buckets as matrix products, each
// pair a row with a one at its bucket, took 94 to 99 % of this kernel's time with 8 and more heads and 120 to 200 % with fewer: both wait for memory.  Six or eight items under way
// took 1 to 9 % longer than four.)
constexpr int kBinItems = 4;                                       // items of a lane that are under way together
// WHOLE: rows have eight keys at least.
template <typename T, bool WHOLE> __global__ __launch_bounds__(512) void k_bias_bins(BiasArgs A) {
    extern __shared__ __attribute__((aligned(16))) double all_bins[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bins = bins_of(A.held_buckets, A.copies), copies = A.copies;
    double* mine = all_bins + wave * (bins + 64);
    const int64_t head = (int64_t)blockIdx.y * A.waves + wave;
    if (head >= A.heads) return;                                   // (wavefronts do not wait for each other)
    for (int e = lane; e < bins + 64; e += 64) mine[e] = 0.0;
    const T* values = (const T*)A.values + head * A.value_head;
    const int here = (int)min((int64_t)kRun, A.keys);
    const int64_t blocks = (A.items + 63) / 64, stride = (int64_t)gridDim.x * kBinItems;      // blocks of 64 items

    struct Stage { Places8 place[kBinItems]; Eight<T> value[kBinItems]; uint64_t live[kBinItems]; };
    typedef const __attribute__((address_space(4))) uint64_t* Scalars;         // (read by scalar loads: the vector loads under way are not waited for)
    const uint32_t last = (uint32_t)max(A.keys - kRun, (int64_t)0);
    Place<T> at;
    int64_t block = (int64_t)blockIdx.x * kBinItems;
    at.begin(A, values, block * 64 + lane);
    uint64_t live[kBinItems];
    auto look = [&]() {
#pragma unroll
        for (int u = 0; u < kBinItems; u++) live[u] = block + u < blocks ? ((Scalars)(uintptr_t)A.live)[block + u] : 0;
    };
    look();
    // The next items.  All lanes load, those of items without a pair what is at the beginning: the compiler lets no load pass another one that stands under a condition.
    auto fetch = [&](Stage& S) {
#pragma unroll
        for (int u = 0; u < kBinItems; u++) {
            S.live[u] = live[u];
            S.place[u] = A.places[min(block + u, blocks - 1) * 64 + lane];
            S.value[u].template load<WHOLE>(live[u] >> lane & 1 ? at.at(last) : values, here);
            at.on(A, values, A.near);
        }
        block += stride;
        at.on(A, values, A.far);
        look();
    };
    auto add = [&](const Stage& S) {
#pragma unroll
        for (int u = 0; u < kBinItems; u++)
            if (S.live[u]) {
#pragma unroll
                for (int v = 0; v < kRun; v++) unsafeAtomicAdd(&mine[S.place[u][v]], (double)S.value[u].at(v));
            }
    };
    Stage one, other;
    fetch(one);
    while (true) {
        if (block >= blocks) { add(one); break; }
        fetch(other);
        add(one);
        if (block >= blocks) { add(other); break; }
        fetch(one);
        add(other);
    }
    // The sums over the copies.
    float* part = A.direct ? A.part + head : A.part + ((int64_t)blockIdx.x * A.heads + head) * A.buckets;
    const int64_t step = A.direct ? A.heads : 1;
    const int side_by_side = 64 / copies;
    for (int b0 = lane / copies; b0 < A.held_buckets + lane / copies; b0 += 4 * side_by_side) {
        double sum[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int b = b0 + j * side_by_side;
            sum[j] = b < A.held_buckets ? mine[b * copies + (lane & (copies - 1))] : 0.0;
        }
        for (int d = 1; d < copies; d <<= 1)
#pragma unroll
            for (int j = 0; j < 4; j++) sum[j] += __shfl_xor(sum[j], d);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int64_t b = b0 + j * side_by_side;
            if ((lane & (copies - 1)) == 0 && b < A.held_buckets && A.first_bucket + b < A.buckets) part[(A.first_bucket + b) * step] = (float)sum[j];
        }
    }
}

// Sums of the shares' parts [share][head][bucket], in 64 bits and in a fixed order, into [bucket][head]: 64 bins to a workgroup, 16 threads to a bin.
struct BiasSums { const float* part; float* out; int64_t shares, heads, buckets, begin; };       // begin: workgroups of earlier launches
__global__ __launch_bounds__(1024) void k_bias_sums(BiasSums A) {
    __shared__ double joined[1024];
    const int64_t n = A.heads * A.buckets, e = (blockIdx.x + A.begin) * 64 + (threadIdx.x & 63);
    double sum = 0.0;
    if (e < n) {
#pragma unroll 8
        for (int64_t s = threadIdx.x >> 6; s < A.shares; s += 16) sum += (double)A.part[s * n + e];
    }
    joined[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 64 && e < n) {
#pragma unroll
        for (int q = 1; q < 16; q++) sum += joined[q * 64 + threadIdx.x];
        const int64_t h = e / A.buckets, b = e - h * A.buckets;
        A.out[b * A.heads + h] = (float)sum;
    }
}

}  // namespace pcr
