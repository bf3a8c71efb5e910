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
    float* part; int64_t share_items, first_bucket, held_buckets;  // part: [share][head][bucket]
    int waves, copies, steps_a_share;
};

// The clipped difference of two positions.
__device__ __forceinline__ int apart(int32_t key, int32_t query, int reach) { return min(max(__builtin_elementwise_sub_sat(key, query), -reach), reach); }
__device__ __forceinline__ int apart(int64_t key, int64_t query, int reach) {
    return (int)min(max(__builtin_elementwise_sub_sat(key, query), (int64_t)-reach), (int64_t)reach);
}

enum : uint32_t { kNoBias = 0, kNeverSeen = 1 };                   // behind the buckets: a pair without a bias (0), and one of different segments (-inf)

// An item: a run of V keys of a query.
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

// The buckets of an item's keys; buckets + kNoBias where there is none, buckets + kNeverSeen across segments.  Keys behind the row's end: of no account.
template <typename P, int V> __device__ __forceinline__ void sum_axes(const BiasArgs& A, const int32_t* map, const Item& I, int here, int32_t (&sum)[V]) {
    const int width = 2 * A.reach + 1;
    for (int a = 0; a < A.axes; a++) {
        const P query = ((const P*)A.q.position)[a * A.q.axis + I.b * A.q.batch + I.i * A.q.token];
        const P* key = (const P*)A.k.position + a * A.k.axis + I.b * A.k.batch + I.run * V * A.k.token;
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
        const int32_t* key = A.k.segment + I.b * A.k.segment_batch + I.run * V * A.k.segment_token;
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
    for (; t < A.items; t += (int64_t)gridDim.x * blockDim.x, step_on(I, A)) {
        const int here = (int)min((int64_t)V, A.keys - I.run * V);
        uint32_t bucket[V];
        buckets_of<V>(A, HELD ? map : A.map, I, here, bucket);
        T* out = (T*)A.values + I.b * A.value_batch + first_head * A.value_head + I.i * A.value_query + I.run * V;
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

// The table's gradient.  A workgroup takes a share of the items and a head for each of its wavefronts; a wavefront's bins, in LDS, are its own, so that they are added to
// in the order of its instructions.  HELD: the map is in LDS, too.  Where there are few buckets a wavefront has several copies of its bins, for the lanes in turn.  What is left are lanes of one instruction that meet
// in a bin, whose order nothing says: their ranks among each other are found once for all heads (a byte written for each lane's bin and read back tells whether there
// are any), and they add in as many instructions.
// The items' buckets are made by all wavefronts, one item a thread, in a tile that all of them then go through.
constexpr uint32_t kNowhere = 0xffff;
template <typename T, bool HELD> __global__ __launch_bounds__(512) void k_bias_back(BiasArgs A) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int V = 16 / sizeof(T);
    typedef uint16_t Places16 __attribute__((ext_vector_type(V)));
    typedef uint8_t Ranks8 __attribute__((ext_vector_type(V)));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = A.waves, copies = A.copies;
    const int bins = (int)A.held_buckets * copies;
    // LDS: tile of places and of ranks, most ranks of a wavefront's items, bins, tags, map
    Places16* tile = (Places16*)lds;
    Ranks8* ranks = (Ranks8*)(tile + waves * 64);
    int* most = (int*)(ranks + waves * 64);
    float* all_bins = (float*)(most + 8);
    uint8_t* all_tags = (uint8_t*)(all_bins + (int64_t)waves * bins);
    int32_t* held_map = (int32_t*)(all_tags + (copies < 64 ? (waves * bins + 15) / 16 * 16 : 0));
    float* mine = all_bins + wave * bins;
    uint8_t* tags = all_tags + wave * bins;
    for (int e = threadIdx.x; e < waves * bins; e += blockDim.x) all_bins[e] = 0.f;
    if (HELD) {
        const int places = A.axes * (2 * A.reach + 1);
        for (int e = threadIdx.x; e < places; e += blockDim.x) held_map[e] = A.map[e];
    }
    __syncthreads();

    const int64_t head = (int64_t)blockIdx.y * waves + wave;
    const T* values = (const T*)A.values + head * A.value_head;
    const int64_t from = (int64_t)blockIdx.x * A.share_items, to = min(from + A.share_items, A.items);
    const uint32_t copy = lane & (copies - 1);
    for (int64_t t0 = from; t0 < to; t0 += waves * 64) {
        // the tile
        {
            const int64_t t = t0 + threadIdx.x;
            Places16 place;
            Ranks8 rank;
#pragma unroll
            for (int v = 0; v < V; v++) { place[v] = kNowhere; rank[v] = 0; }
            if (t < to) {
                const Item I = item_at(A, t);
                const int here = (int)min((int64_t)V, A.keys - I.run * V);
                uint32_t bucket[V];
                buckets_of<V>(A, HELD ? held_map : A.map, I, here, bucket);
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const uint32_t b = bucket[v] - (uint32_t)A.first_bucket;
                    if (v < here && bucket[v] < A.buckets && b < A.held_buckets) {
                        const uint32_t at = b * copies + copy;
                        place[v] = (uint16_t)at;
                    }
                }
            }
            int highest = 0;
            if (copies < 64) {
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const uint32_t at = place[v];
                    bool met = false;
                    if (at != kNowhere) {
                        ((volatile uint8_t*)tags)[at] = (uint8_t)lane;
                        __builtin_amdgcn_wave_barrier();
                        met = ((volatile uint8_t*)tags)[at] != lane;
                    }
                    if (__ballot(met)) {
                        uint64_t same = __ballot(at != kNowhere);
                        for (int bit = 0; bit < 16; bit++) {
                            const uint64_t set = __ballot(at >> bit & 1);
                            same &= at >> bit & 1 ? set : ~set;
                        }
                        const int r = at != kNowhere ? __popcll(same & ((1ull << lane) - 1)) : 0;
                        rank[v] = (uint8_t)r;
                        highest = max(highest, r);
                    }
                }
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) highest = max(highest, __shfl_xor(highest, d));
                if (highest) ranks[threadIdx.x] = rank;
            }
            tile[threadIdx.x] = place;
            if (lane == 0) most[wave] = highest;
        }
        __syncthreads();
        if (head < A.heads) {
            for (int s = 0; s < waves; s++) {
                const int64_t t = t0 + s * 64 + lane;
                if (t < to) {
                    const Item I = item_at(A, t);
                    const int here = (int)min((int64_t)V, A.keys - I.run * V);
                    const T* from_row = values + I.b * A.value_batch + I.i * A.value_query + I.run * V;
                    float g[V];
                    if (here == V) load_run<T, V>(from_row, g);
                    else {
#pragma unroll
                        for (int v = 0; v < V; v++) g[v] = v < here ? (float)from_row[v] : 0.f;
                    }
                    const Places16 place = tile[s * 64 + lane];
                    const int highest = most[s];
                    if (highest == 0) {
#pragma unroll
                        for (int v = 0; v < V; v++)
                            if (place[v] != kNowhere) unsafeAtomicAdd(&mine[place[v]], g[v]);
                    } else {
                        const Ranks8 rank = ranks[s * 64 + lane];
#pragma unroll
                        for (int v = 0; v < V; v++)
                            for (int r = 0; r <= highest; r++)
                                if (place[v] != kNowhere && rank[v] == r) unsafeAtomicAdd(&mine[place[v]], g[v]);
                    }
                }
            }
        }
        __syncthreads();
    }
    // A wavefront's sums over the copies of its bins.
    if (head < A.heads) {
        float* part = A.part + ((int64_t)blockIdx.x * A.heads + head) * A.buckets + A.first_bucket;
        const int side_by_side = 64 / copies;
        for (int b0 = 0; b0 < A.held_buckets; b0 += side_by_side) {
            const int e = b0 * copies + lane;
            float sum = e < bins ? mine[e] : 0.f;
            for (int d = 1; d < copies; d <<= 1) sum += __shfl_xor(sum, d);
            const int b = b0 + lane / copies;
            if ((lane & (copies - 1)) == 0 && b < A.held_buckets && A.first_bucket + b < A.buckets) part[b] = sum;
        }
    }
}

// Sums of the shares' parts [share][head][bucket], in 64 bits and in their order, into [bucket][head].
struct BiasSums { const float* part; float* out; int64_t shares, heads, buckets; };
__global__ __launch_bounds__(256) void k_bias_sums(BiasSums A) {
    const int64_t n = A.heads * A.buckets;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
        double sum = 0.0;
#pragma unroll 8
        for (int64_t s = 0; s < A.shares; s++) sum += (double)A.part[s * n + e];
        const int64_t h = e / A.buckets, b = e - h * A.buckets;
        A.out[b * A.heads + h] = (float)sum;
    }
}

}  // namespace pcr
