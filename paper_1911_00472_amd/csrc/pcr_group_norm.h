// Group norm and its gradient in two passes.
//
// Larger pictures are gone through twice, chunk by chunk of their pixels: sums of every chunk, then what is written; what the second pass reads mostly comes out of the
// memory-side cache.  (More than 256 runs of channels, 2048 of 16 bits, three times: the sums hold one block of columns in registers, and go through several twice.  us: 8 of
// 112 x 112 x 2048 261, x 2304 368.)  Loads of four pixels are under way together, without conditions about them (behind which the compiler would wait for those before).
// Results are bound by memory; sums by what follows each other in a thread, four loads, a wait for them, the running means.  us: 64 pictures of 112 x 112 x 64, bfloat, sums 32
// (103 MB, 3.2 TB/s; 26 where x is in the cache), result 39 (206 MB, 5.3 TB/s); gradient of 64 of 56 x 56 x 256 sums 57 (206 MB, 3.6 TB/s), result 55 (308 MB, 5.6 TB/s), sums of the
// weights' gradients 5.
#pragma once
#include "pcr_norm.h"

namespace pcr {

// A block of columns: runs of V channels, as many as there are threads; `lanes` threads to a column take the pixels in turn.
struct Columns { int count, lanes, lane, column; bool works; };
__device__ __forceinline__ Columns columns_of(int from, int all) {
    Columns C;
    C.count = min(all - from, kNormThreads);
    C.lanes = kNormThreads / C.count;
    C.lane = threadIdx.x / C.count;
    C.column = threadIdx.x - C.lane * C.count;
    C.works = C.lane < C.lanes;
    return C;
}
struct Chunk { int64_t image, first, end; };
__device__ __forceinline__ Chunk chunk_of(const NormArgs& A, int64_t at) {
    Chunk K;
    K.image = at / A.chunks;
    K.first = (at - K.image * A.chunks) * A.chunk;
    K.end = min(K.first + A.chunk, A.pixels);
    return K;
}
// f(pixel) for a lane's pixels of a chunk, kNormTogether of them at a time as long as all lanes have that many: f4(pixels' first), the others `lanes` apart.
template <typename F4, typename F> __device__ __forceinline__ void through(const Chunk& K, const Columns& C, F4 f4, F f) {
    int64_t p = K.first + C.lane;
    const int64_t whole = (K.end - K.first) / (kNormTogether * C.lanes);
    for (int64_t n = 0; n < whole; n++, p += kNormTogether * C.lanes) f4(p);
    for (; p < K.end; p += C.lanes) f(p);
}

// Mean and sum of squares around it of every group over a chunk of pixels.  Running means of equal values are exact; their sum over lanes and channels is in 64 bits, so that the mean is, too.
inline size_t norm_sums_lds(int run, int groups) { return (size_t)kNormThreads * run * 8 + (size_t)groups * 12; }
template <typename T, int V> __global__ __launch_bounds__(256) void k_norm_sums(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    double* sums = (double*)shared;                                // [lane][channel of the block]
    float* values = shared;                                        // [lane][channel of the block]: of squares
    double* whole = sums + kNormThreads * V;                       // [group]
    float* total = (float*)whole;                                  // [group]: of squares
    float* mean = (float*)(whole + A.groups);
    const Chunk K = chunk_of(A, blockIdx.x + A.begin);
    const T* x = (const T*)A.x + K.image * A.x_image;
    const int all = A.channels / V;
    for (int g = threadIdx.x; g < A.groups; g += kNormThreads) whole[g] = 0.0;
    // One block of columns holds its means and squares in registers; of more of them each is gone through twice.
    const int blocks = (all + kNormThreads - 1) / kNormThreads;
    float m[V], q[V];
    int n = 0;
    for (int phase = 0; phase < 2; phase++) {
        for (int k = 0; k < blocks; k++) {
            const Columns C = columns_of(k * kNormThreads, all);
            const int c = (k * kNormThreads + C.column) * V, first = k * kNormThreads * V, width = C.count * V;
            const bool again = phase == 1 && blocks == 1;
            if (!again) {
#pragma unroll
                for (int i = 0; i < V; i++) m[i] = q[i] = 0.f;
                n = 0;
            }
            if (C.works && !again)
                through(K, C, [&](int64_t p) {
                    float a[kNormTogether][V];
#pragma unroll
                    for (int j = 0; j < kNormTogether; j++) load_run<T, V>(x + (p + j * C.lanes) * A.x_pixel + c, a[j]);
                    const float part = (float)kNormTogether / (float)(n + kNormTogether), by = n * part;
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float s = ((a[0][i] + a[1][i]) + (a[2][i] + a[3][i])) * 0.25f;
                        float t = 0.f;
#pragma unroll
                        for (int j = 0; j < kNormTogether; j++) t = __builtin_fmaf(a[j][i] - s, a[j][i] - s, t);
                        const float d = s - m[i];
                        m[i] = __builtin_fmaf(d, part, m[i]);
                        q[i] += __builtin_fmaf(d * d, by, t);
                    }
                    n += kNormTogether;
                }, [&](int64_t p) {
                    float a[V];
                    load_run<T, V>(x + p * A.x_pixel + c, a);
                    const float part = 1.f / (float)(n + 1), by = n * part;
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float d = a[i] - m[i];
                        m[i] = __builtin_fmaf(d, part, m[i]);
                        q[i] = __builtin_fmaf(d * d, by, q[i]);
                    }
                    n++;
                });
            const int g0 = first / A.each, g1 = min((first + width + A.each - 1) / A.each, A.groups);
            if (C.works) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const int at = C.lane * width + C.column * V + i;
                    if (phase == 0) sums[at] = (double)m[i] * n;
                    else {
                        const float d = m[i] - mean[(c + i) / A.each];
                        values[at] = __builtin_fmaf(d * d, (float)n, q[i]);
                    }
                }
            }
            __syncthreads();
            if (phase == 0) group_totals(sums, whole, C.lanes, width, first, A.each, g0, g1, (int)threadIdx.x, kNormThreads);
            else group_totals(values, total, C.lanes, width, first, A.each, g0, g1, (int)threadIdx.x, kNormThreads);
            __syncthreads();
        }
        const double count = (double)(K.end - K.first) * A.each;
        float* part = A.part + ((blockIdx.x + A.begin) * A.groups) * 2 + phase;
        for (int g = threadIdx.x; g < A.groups; g += kNormThreads) {
            if (phase == 0) mean[g] = (float)(whole[g] / count);
            part[2 * g] = phase == 0 ? mean[g] : total[g];
        }
        __syncthreads();
        if (phase == 0) {
            for (int g = threadIdx.x; g < A.groups; g += kNormThreads) total[g] = 0.f;
            __syncthreads();
        }
    }
}

// Mean and r of a group from its chunks', by a team of threads.
__device__ __forceinline__ float2 joined_chunks(const NormArgs& A, int64_t image, int64_t g, int member, int team) {
    const float2* part = (const float2*)A.part + image * A.chunks * A.groups + g;
    double mean = 0.0, squares = 0.0;
    for (int k = member; k < A.chunks; k += team) mean += (double)part[(int64_t)k * A.groups].x * (double)min(A.chunk, A.pixels - k * A.chunk);
    for (int d = 1; d < team; d <<= 1) mean += __shfl_xor(mean, d);
    mean /= (double)A.pixels;
    for (int k = member; k < A.chunks; k += team) {
        const float2 of = part[(int64_t)k * A.groups];
        const double d = (double)of.x - mean;
        squares += (double)of.y + d * d * ((double)min(A.chunk, A.pixels - k * A.chunk) * A.each);
    }
    for (int d = 1; d < team; d <<= 1) squares += __shfl_xor(squares, d);
    return make_float2((float)mean, (float)(1.0 / sqrt(squares / ((double)A.pixels * A.each) + (double)A.eps)));
}
// Sums of a chunk's two sums of a group, over the chunks and by the number of values, by a team of threads.
__device__ __forceinline__ float2 joined_sums(const NormArgs& A, int64_t image, int64_t g, int member, int team) {
    const float2* part = (const float2*)A.part + image * A.chunks * A.groups + g;
    double a = 0.0, b = 0.0;
    for (int k = member; k < A.chunks; k += team) {
        const float2 of = part[(int64_t)k * A.groups];
        a += (double)of.x;
        b += (double)of.y;
    }
    for (int d = 1; d < team; d <<= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    const double count = (double)A.pixels * A.each;
    return make_float2((float)(a / count), (float)(b / count));
}
__device__ __forceinline__ int team_of(int groups) {               // threads of 256 that a group has
    int team = 64;
    while (team > 1 && team * groups > kNormThreads) team >>= 1;
    return team;
}
// Into held[group], by the whole workgroup.
template <bool BACK> __device__ __forceinline__ void join_chunks(const NormArgs& A, int64_t image, float2* held) {
    const int team = team_of(A.groups), member = threadIdx.x & (team - 1);
    for (int g0 = 0; g0 < A.groups; g0 += kNormThreads / team) {
        const int g = g0 + threadIdx.x / team, at = min(g, A.groups - 1);
        const float2 of = BACK ? joined_sums(A, image, at, member, team) : joined_chunks(A, image, at, member, team);
        if (g < A.groups && member == 0) held[g] = of;
    }
}

// Of pictures of many chunks, a wavefront to a group: their statistics, or (BACK) their sums in the place of the first chunk's.
template <bool BACK> __global__ __launch_bounds__(256) void k_norm_join(NormArgs A) {
    const int64_t at = (blockIdx.x + A.begin) * 4 + threadIdx.x / 64, group = min(at, A.images * A.groups - 1), image = group / A.groups, g = group - image * A.groups;
    const float2 of = BACK ? joined_sums(A, image, g, threadIdx.x & 63, 64) : joined_chunks(A, image, g, threadIdx.x & 63, 64);
    if ((threadIdx.x & 63) == 0 && at == group) ((float2*)A.stats)[at] = of;
}

template <typename T, int V, bool ONE> __global__ __launch_bounds__(256) void k_norm_apply(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float2 held[];  // [group]
    const Chunk K = chunk_of(A, blockIdx.x + A.begin);
    float2* stats = (float2*)A.stats + K.image * A.groups;
    if (A.chunks <= kMergedChunks) {
        join_chunks<false>(A, K.image, held);
        __syncthreads();
        if (K.first == 0)
            for (int g = threadIdx.x; g < A.groups; g += kNormThreads) stats[g] = held[g];
    } else {
        for (int g = threadIdx.x; g < A.groups; g += kNormThreads) held[g] = stats[g];
        __syncthreads();
    }
    const T* x = (const T*)A.x + K.image * A.x_image;
    T* out = (T*)A.out + K.image * A.out_image;
    const int all = A.channels / V;
    for (int k = 0; k < all; k += kNormThreads) {
        const Columns C = columns_of(k, all);
        if (!C.works) continue;
        const int c = (k + C.column) * V;
        constexpr int N = ONE ? 1 : V;
        float w[V], b[V], m[N];
        load_parameters<T, V>(A, A.weight, c, 1.f, w);
        load_parameters<T, V>(A, A.bias, c, 0.f, b);
#pragma unroll
        for (int i = 0; i < V; i++) {
            const float2 of = held[(ONE ? c : c + i) / A.each];
            m[ONE ? 0 : i] = of.x;
            w[i] *= of.y;
        }
        with_kind(A.activation, [&](auto kind) {
            auto one = [&](int64_t p, float (&a)[V]) {
#pragma unroll
                for (int i = 0; i < V; i++) a[i] = __builtin_fmaf(a[i] - m[ONE ? 0 : i], w[i], b[i]);
                activate<T, decltype(kind)::value>(a);
                store_run<T, V>(out + p * A.out_pixel + c, a);
            };
            through(K, C, [&](int64_t p) {
                Held<T, V> a[kNormTogether];
#pragma unroll
                for (int j = 0; j < kNormTogether; j++) a[j].v = reinterpret_cast<const typename Run<T, V>::Loose*>(x + (p + j * C.lanes) * A.x_pixel + c)->v;
#pragma unroll
                for (int j = 0; j < kNormTogether; j++) {
                    float v[V];
                    take(a[j], v);
                    one(p + j * C.lanes, v);
                    one_after_another();
                }
            }, [&](int64_t p) {
                float a[V];
                load_run<T, V>(x + p * A.x_pixel + c, a);
                one(p, a);
            });
        });
    }
}

// Of every chunk: sums of h u and h by channels, and of h w and h w u by groups.
template <typename T, int V, bool ONE> __global__ __launch_bounds__(256) void k_norm_back_sums(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    float* values = shared;                                        // [lane][channel of the block]
    float* total = shared + kNormThreads * V;                      // [2][group]
    float* channel = total + 2 * A.groups;                         // [2][channel of the block]
    const Chunk K = chunk_of(A, blockIdx.x + A.begin);
    const T* x = (const T*)A.x + K.image * A.x_image;
    const T* grad = (const T*)A.grad + K.image * A.grad_image;
    const int all = A.channels / V;
    for (int g = threadIdx.x; g < 2 * A.groups; g += kNormThreads) total[g] = 0.f;
    for (int k = 0; k < all; k += kNormThreads) {
        const Columns C = columns_of(k, all);
        const int c = (k + C.column) * V, first = k * V, width = C.count * V;
        float s[2][V];                                             // of h u, of h
#pragma unroll
        for (int i = 0; i < V; i++) s[0][i] = s[1][i] = 0.f;
        for (int e = threadIdx.x; e < 2 * width; e += kNormThreads) channel[e] = 0.f;
        constexpr int N = ONE ? 1 : V;
        float w[V], b[V], m[N], r[N];
        if (C.works) {
            load_parameters<T, V>(A, A.weight, c, 1.f, w);
            load_parameters<T, V>(A, A.bias, c, 0.f, b);
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float2 of = ((const float2*)A.stats)[K.image * A.groups + (c + i) / A.each];
                m[i] = of.x;
                r[i] = of.y;
            }
            with_kind(A.activation, [&](auto kind) {
                auto one = [&](float (&a)[V], float (&h)[V]) {
                    slopes<T, decltype(kind)::value, ONE>(a, h, m, r, w, b);
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        s[0][i] = __builtin_fmaf(h[i], a[i], s[0][i]);
                        s[1][i] += h[i];
                    }
                };
                through(K, C, [&](int64_t p) {
                    Held<T, V> a[kNormTogether], h[kNormTogether];
#pragma unroll
                    for (int j = 0; j < kNormTogether; j++) {
                        a[j].v = reinterpret_cast<const typename Run<T, V>::Loose*>(x + (p + j * C.lanes) * A.x_pixel + c)->v;
                        h[j].v = reinterpret_cast<const typename Run<T, V>::Loose*>(grad + (p + j * C.lanes) * A.grad_pixel + c)->v;
                    }
#pragma unroll
                    for (int j = 0; j < kNormTogether; j++) {
                        float u[V], g[V];
                        take(a[j], u);
                        take(h[j], g);
                        one(u, g);
                        one_after_another();
                    }
                }, [&](int64_t p) {
                    float a[V], h[V];
                    load_run<T, V>(x + p * A.x_pixel + c, a);
                    load_run<T, V>(grad + p * A.grad_pixel + c, h);
                    one(a, h);
                });
            });
        }
        const int g0 = first / A.each, g1 = min((first + width + A.each - 1) / A.each, A.groups);
#pragma unroll
        for (int z = 0; z < 2; z++) {
            if (C.works) {
#pragma unroll
                for (int i = 0; i < V; i++) values[C.lane * width + C.column * V + i] = s[z][i];
            }
            __syncthreads();
            group_totals(values, channel + z * width, C.lanes, width, 0, 1, 0, width, (int)threadIdx.x, kNormThreads);
            __syncthreads();
        }
        // The groups' from their channels'.
        float2* sums = (float2*)A.sums + (blockIdx.x + A.begin) * A.channels + first;
        for (int e = threadIdx.x; e < width; e += kNormThreads) {
            sums[e] = make_float2(channel[e], channel[width + e]);
            float by[1];
            load_parameters<T, 1>(A, A.weight, first + e, 1.f, by);
            channel[e] *= by[0];
            channel[width + e] *= by[0];
        }
        __syncthreads();
        group_totals(channel + width, total, 1, width, first, A.each, g0, g1, (int)threadIdx.x, kNormThreads);
        group_totals(channel, total + A.groups, 1, width, first, A.each, g0, g1, (int)threadIdx.x, kNormThreads);
        __syncthreads();
    }
    float2* part = (float2*)A.part + (blockIdx.x + A.begin) * A.groups;
    for (int g = threadIdx.x; g < A.groups; g += kNormThreads) part[g] = make_float2(total[g], total[A.groups + g]);
}

template <typename T, int V, bool ONE> __global__ __launch_bounds__(256) void k_norm_back_apply(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float2 held[];  // [group]
    const Chunk K = chunk_of(A, blockIdx.x + A.begin);
    if (A.chunks <= kMergedChunks) join_chunks<true>(A, K.image, held);
    else
        for (int g = threadIdx.x; g < A.groups; g += kNormThreads) held[g] = ((const float2*)A.joined)[K.image * A.groups + g];
    __syncthreads();
    const T* x = (const T*)A.x + K.image * A.x_image;
    const T* grad = (const T*)A.grad + K.image * A.grad_image;
    T* out = (T*)A.out + K.image * A.out_image;
    const int all = A.channels / V;
    for (int k = 0; k < all; k += kNormThreads) {
        const Columns C = columns_of(k, all);
        if (!C.works) continue;
        const int c = (k + C.column) * V;
        constexpr int N = ONE ? 1 : V;
        float w[V], b[V], m[N], r[N], s[N], t[N];
        load_parameters<T, V>(A, A.weight, c, 1.f, w);
        load_parameters<T, V>(A, A.bias, c, 0.f, b);
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int g = (c + i) / A.each;
            const float2 of = ((const float2*)A.stats)[K.image * A.groups + g];
            m[i] = of.x;
            r[i] = of.y;
            s[i] = held[g].x;
            t[i] = held[g].y;
        }
        with_kind(A.activation, [&](auto kind) {
            auto one = [&](int64_t p, float (&a)[V], float (&h)[V]) {
                slopes<T, decltype(kind)::value, ONE>(a, h, m, r, w, b);
#pragma unroll
                for (int i = 0; i < V; i++) a[i] = r[ONE ? 0 : i] * (__builtin_fmaf(h[i], w[i], -s[ONE ? 0 : i]) - a[i] * t[ONE ? 0 : i]);
                store_run<T, V>(out + p * A.out_pixel + c, a);
            };
            through(K, C, [&](int64_t p) {
                Held<T, V> a[kNormTogether], h[kNormTogether];
#pragma unroll
                for (int j = 0; j < kNormTogether; j++) {
                    a[j].v = reinterpret_cast<const typename Run<T, V>::Loose*>(x + (p + j * C.lanes) * A.x_pixel + c)->v;
                    h[j].v = reinterpret_cast<const typename Run<T, V>::Loose*>(grad + (p + j * C.lanes) * A.grad_pixel + c)->v;
                }
#pragma unroll
                for (int j = 0; j < kNormTogether; j++) {
                    float u[V], g[V];
                    take(a[j], u);
                    take(h[j], g);
                    one(p + j * C.lanes, u, g);
                    one_after_another();
                }
            }, [&](int64_t p) {
                float a[V], h[V];
                load_run<T, V>(x + p * A.x_pixel + c, a);
                load_run<T, V>(grad + p * A.grad_pixel + c, h);
                one(p, a, h);
            });
        });
    }
}

// Gradients of weight and bias: sums [image and chunk][channel][2] over their first axis, 16 values of a row to a workgroup, 64 threads to a value, in a fixed order.
struct NormWeightSums { const float* sums; float* weight_grad; float* bias_grad; int64_t parts; int channels; };
__global__ __launch_bounds__(1024) void k_norm_weight_sums(NormWeightSums A) {
    __shared__ double joined[1024];
    const int column = threadIdx.x & 15, share = threadIdx.x >> 4, e = blockIdx.x * 16 + column;
    double sum = 0.0;
    if (e < 2 * A.channels) {
#pragma unroll 8
        for (int64_t p = share; p < A.parts; p += 64) sum += (double)A.sums[p * 2 * A.channels + e];
    }
    joined[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 256) {
        sum = (sum + joined[threadIdx.x + 256]) + (joined[threadIdx.x + 512] + joined[threadIdx.x + 768]);
        joined[threadIdx.x] = sum;
    }
    __syncthreads();
    if (share == 0 && e < 2 * A.channels) {
#pragma unroll
        for (int q = 1; q < 16; q++) sum += joined[q * 16 + column];
        float* to = e & 1 ? A.bias_grad : A.weight_grad;
        if (to) to[e >> 1] = (float)sum;
    }
}

}  // namespace pcr
