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
struct BiasArgs {
    Places q, k;
    const int32_t* map; const void* table; void* values;           // values: the bias, or its incoming gradient
    int64_t value_batch, value_head, value_query;
    int64_t batch, heads, queries, keys, buckets, runs, items;     // runs: of a row; items: runs of all rows of all sequences
    int64_t step_batch, step_query, step_run;                      // a thread's step to its next item
    int axes, reach, wide, table_float;
    // gradient
    float* part; int64_t share_items, held_buckets;  // part: [share][head][bucket]; direct: one share, [bucket][head]
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
    const int64_t row = t / A.runs;
    I.run = t - row * A.runs;
    I.b = row / A.queries;
    I.i = row - I.b * A.queries;
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

// The buckets of an item's keys; buckets + kNoBias where there is none, buckets + kNeverSeen across segments.  Keys behind the row's end (of rows of fewer than V): of no account.
template <typename P, int V> __device__ __forceinline__ void sum_axes(const BiasArgs& A, const int32_t* map, const Item& I, int here, int32_t (&sum)[V]) {
    const int width = 2 * A.reach + 1;
    for (int a = 0; a < A.axes; a++) {
        const P query = ((const P*)A.q.position)[a * A.q.axis + I.b * A.q.batch + I.i * A.q.token];
        const P* key = (const P*)A.k.position + a * A.k.axis + I.b * A.k.batch + first_key<V>(A, I) * A.k.token;
        P at[V];
        if (here == V && A.k.token == 1) {
#pragma unroll
            for (int v = 0; v < V; v += 4) {
                const typename Run<P, 4>::Vec four = reinterpret_cast<const typename Run<P, 4>::Loose*>(key + v)->v;
#pragma unroll
                for (int u = 0; u < 4; u++) at[v + u] = four[u];
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; v++) at[v] = v < here ? key[v * A.k.token] : query;
        }
#pragma unroll
        for (int v = 0; v < V; v++) sum[v] = (int32_t)((uint32_t)sum[v] + (uint32_t)map[a * width + A.reach + apart(at[v], query, A.reach)]);
    }
}
template <int V> __device__ __forceinline__ void buckets_of(const BiasArgs& A, const int32_t* map, const Item& I, int here, uint32_t (&bucket)[V]) {
    int32_t sum[V];
#pragma unroll
    for (int v = 0; v < V; v++) sum[v] = 0;
    if (A.wide) sum_axes<int64_t, V>(A, map, I, here, sum);
    else sum_axes<int32_t, V>(A, map, I, here, sum);
    const uint32_t count = (uint32_t)A.buckets;
#pragma unroll
    for (int v = 0; v < V; v++) bucket[v] = (uint32_t)sum[v] < count ? (uint32_t)sum[v] : count + kNoBias;
    if (A.q.segment) {
        const int32_t mine = A.q.segment[I.b * A.q.segment_batch + I.i * A.q.segment_token];
        const int32_t* key = A.k.segment + I.b * A.k.segment_batch + first_key<V>(A, I) * A.k.segment_token;
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int32_t other = v < here ? key[v * A.k.segment_token] : mine;
            if (mine < 0) bucket[v] = count + kNoBias;
            else if (other != mine) bucket[v] = count + kNeverSeen;
        }
    }
}

template <typename T> __device__ __forceinline__ T table_value(const BiasArgs& A, int64_t at) {
    return A.table_float ? (T)((const float*)A.table)[at] : ((const T*)A.table)[at];
}

// The bias.  H: heads of a workgroup, whose values of a bucket lie side by side in LDS, so that a key costs one read for all of them; HELD: the map and the table of these
// heads are in LDS (else read where they are).  V keys of H heads are V reads and H stores of 16 bytes.
template <typename T, int H, bool HELD> __global__ __launch_bounds__(1024) void k_bias(BiasArgs A) {
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
        buckets_of<V>(A, HELD ? map : A.map, I, here, bucket);
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

// The table's gradient.  A workgroup takes a share of the items and a head for each of its wavefronts, whose bins, in LDS and in 64 bits, are its own: they are added to in
// the order of its instructions, and lanes of one instruction that meet in a bin in the order in which the LDS unit takes lanes of the same address, which nothing else
// has a part in.  Where there are few buckets a wavefront has several copies of its bins, for the lanes in turn, so that few meet.
// (LDS adds floats of 64 bits in 9 clocks a wavefront's instruction, those of 32 in 193: a long sequence of 4096 tokens and 12 heads took 1063 us with these.)
// The items' buckets are made by all wavefronts, one item a thread, in a tile that all of them then go through; the next tile is made while the values of one are on
// their way.  Pairs without a bias go to bins that nobody reads, one for each lane, and runs of nothing else are not loaded.  HELD: the map is in LDS, too.
constexpr int kBackWaves = 8;
constexpr int64_t kNoItem = -1;
// Where a bucket's bins begin: neighbouring lanes' runs are eight keys apart, which would be every eighth bin; buckets' lowest bits are mixed with those of 32s.
__device__ __forceinline__ uint32_t bin_of(uint32_t bucket, int copies) { return (bucket ^ (bucket >> 5 & 7)) * copies; }

template <typename T> struct BackTile {                            // LDS, for one tile of 64 items a wavefront
    static constexpr int V = 16 / sizeof(T);
    typedef uint16_t Places __attribute__((ext_vector_type(V)));
    Places* place; int64_t* where;                                 // bins of an item's keys; where its values lie
    static __host__ __device__ int64_t bytes(int waves) { return (int64_t)waves * 64 * (2 * V + 8); }
    __device__ BackTile(char* at, int waves) {
        place = (Places*)at;
        where = (int64_t*)(place + waves * 64);
    }
};

template <typename T, bool HELD> __global__ __launch_bounds__(512) void k_bias_back(BiasArgs A) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef BackTile<T> Tile;
    constexpr int V = Tile::V;
    typedef typename Run<T, V>::Vec Values;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = A.waves, copies = A.copies;
    const int bins = (int)(A.held_buckets + 7) / 8 * 8 * copies;
    const int64_t tile_bytes = Tile::bytes(waves);
    double* all_bins = (double*)(lds + 2 * tile_bytes);
    int32_t* held_map = (int32_t*)(all_bins + waves * (bins + 64));
    double* mine = all_bins + wave * (bins + 64);
    for (int e = threadIdx.x; e < waves * (bins + 64); e += blockDim.x) all_bins[e] = 0.0;
    if (HELD) {
        const int places = A.axes * (2 * A.reach + 1);
        for (int e = threadIdx.x; e < places; e += blockDim.x) held_map[e] = A.map[e];
    }
    __syncthreads();

    const int64_t head = (int64_t)blockIdx.y * waves + wave, first_bucket = blockIdx.z * A.held_buckets;
    const T* values = (const T*)A.values + head * A.value_head;
    const int64_t from = (int64_t)blockIdx.x * A.share_items, to = min(from + A.share_items, A.items);
    const int here = (int)min((int64_t)V, A.keys);

    int64_t t = from + threadIdx.x;
    Item I = item_at(A, t);
    auto make = [&](const Tile& tile) {                            // of the items from t on, one a thread
        typename Tile::Places place;
#pragma unroll
        for (int v = 0; v < V; v++) place[v] = (uint16_t)(bins + lane);
        bool any = false;
        if (t < to) {
            uint32_t bucket[V];
            buckets_of<V>(A, HELD ? held_map : A.map, I, here, bucket);
            const int again = (int)(I.run * V - first_key<V>(A, I));       // (keys of the run before)
#pragma unroll
            for (int v = 0; v < V; v++) {
                const uint32_t b = bucket[v] - (uint32_t)first_bucket;
                if (v < here && v >= again && bucket[v] < A.buckets && b < A.held_buckets) {
                    place[v] = (uint16_t)(bin_of(b, copies) + (lane & (copies - 1)));
                    any = true;
                }
            }
        }
        tile.place[threadIdx.x] = place;
        tile.where[threadIdx.x] = any ? I.b * A.value_batch + I.i * A.value_query + first_key<V>(A, I) : kNoItem;
    };
    make(Tile(lds, waves));
    __syncthreads();
    for (int64_t t0 = from, k = 0; t0 < to; t0 += waves * 64, k ^= 1) {
        const Tile tile(lds + k * tile_bytes, waves);
        Values got[kBackWaves];
        uint32_t live = 0;
        if (head < A.heads) {
#pragma unroll
            for (int s = 0; s < kBackWaves; s++)
                if (s < waves) {
                    const int64_t at = tile.where[s * 64 + lane];
                    if (at != kNoItem) {
                        live |= 1u << s;
                        if (here == V) got[s] = reinterpret_cast<const typename Run<T, V>::Loose*>(values + at)->v;
                        else {
#pragma unroll
                            for (int v = 0; v < V; v++) got[s][v] = v < here ? values[at + v] : (T)0.f;
                        }
                    }
                }
        }
        t += waves * 64;
        step_on(I, A);
        if (t0 + waves * 64 < to) make(Tile(lds + (k ^ 1) * tile_bytes, waves));
        if (head < A.heads) {
#pragma unroll
            for (int s = 0; s < kBackWaves; s++)
                if (s < waves && live >> s & 1) {
                    const typename Tile::Places place = tile.place[s * 64 + lane];
#pragma unroll
                    for (int v = 0; v < V; v++) unsafeAtomicAdd(&mine[place[v]], (double)(float)got[s][v]);
                }
        }
        __syncthreads();
    }
    // A wavefront's sums over the copies of its bins.
    if (head < A.heads) {
        float* part = A.direct ? A.part + head : A.part + ((int64_t)blockIdx.x * A.heads + head) * A.buckets;
        const int64_t step = A.direct ? A.heads : 1;
        const int side_by_side = 64 / copies;
        for (int b0 = lane / copies; b0 < A.held_buckets + lane / copies; b0 += 4 * side_by_side) {
            double sum[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int b = b0 + j * side_by_side;
                sum[j] = b < A.held_buckets ? mine[bin_of(b, copies) + (lane & (copies - 1))] : 0.0;
            }
            for (int d = 1; d < copies; d <<= 1)
#pragma unroll
                for (int j = 0; j < 4; j++) sum[j] += __shfl_xor(sum[j], d);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int64_t b = b0 + j * side_by_side;
                if ((lane & (copies - 1)) == 0 && b < A.held_buckets && first_bucket + b < A.buckets) part[(first_bucket + b) * step] = (float)sum[j];
            }
        }
    }
}

// Sums of the shares' parts [share][head][bucket], in 64 bits and in a fixed order, into [bucket][head]: 64 bins to a workgroup, 16 threads to a bin.
struct BiasSums { const float* part; float* out; int64_t shares, heads, buckets; };
__global__ __launch_bounds__(1024) void k_bias_sums(BiasSums A) {
    __shared__ double joined[1024];
    const int64_t n = A.heads * A.buckets, e = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
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
