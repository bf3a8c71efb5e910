// Group norm with an activation, channels last, and its gradients.
//
// Over the pixels of a picture and the channels of a group:  m = mean x, r = (mean (x - m)^2 + eps)^-1/2, u = (x - m) r, z = u w + b, y = act(z).
// With the incoming gradient g and h = g act'(z):  dw = sum h u and db = sum h over pictures and pixels,  dx = r (h w - mean(h w) - u mean(h w u)).
#pragma once
#include "pcr_vec.h"

namespace pcr {

enum { kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3 };

struct NormArgs {
    const void* x; const void* grad; const void* weight; const void* bias; void* out;
    float* stats;                                                  // [image][group][2]: m, r
    float* part;                                                   // [image][chunk][group][2]: mean and sum of squares around it, or sums of h w and h w u
    float* sums;                                                   // [image][chunk][channel][2]: sums of h u and h (one pass: of a workgroup's pictures)
    float* joined;                                                 // [image][group][2]: the chunks' sums of h w and h w u, by the number of values
    int64_t images, pixels, x_image, x_pixel, grad_image, grad_pixel, out_image, out_pixel;
    int64_t chunk;                                                 // pixels of a workgroup
    int64_t begin;                                                 // workgroups of earlier launches
    int chunks, channels, groups, each, activation, weight_float;  // each: channels of a group
    int block, blocks, pack, turns;                                // one pass: channels of a workgroup, workgroups of a picture; pictures of a workgroup side by side (its threads divided
                                                                   // among them), and one after another
    float eps;
};

// What runs become is computed one after another: side by side their intermediate values would take the registers of whole wavefronts (168 and spills for 90 in the gradient's sums).
__device__ __forceinline__ void one_after_another() { __builtin_amdgcn_sched_barrier(0); }

// exp(-v), and 1 / v to a unit or two in the last place: a division has ten instructions.
__device__ __forceinline__ float exp_of_minus(float v) { return __builtin_amdgcn_exp2f(v * -1.4426950408889634f); }
__device__ __forceinline__ float inverse(float v) { return __builtin_amdgcn_rcpf(v); }
// The normal distribution at z, and exp(-z^2 / 2), by Abramowitz and Stegun's 7.1.26 (Handbook of Mathematical Functions, 1964): with t = 1 / (1 + 0.3275911 |z| / sqrt 2)
// the upper tail is half of a polynomial of t times that exponential, 7.5e-8 off at most.
__device__ __forceinline__ float normal_of(float z, float& bell) {
    const float far = __builtin_fabsf(z), t = inverse(__builtin_fmaf(0.23164188770f, far, 1.f));
    bell = exp_of_minus(0.5f * z * z);
    const float tail = t * __builtin_fmaf(t, __builtin_fmaf(t, __builtin_fmaf(t, __builtin_fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f) * bell;
    return z < 0.f ? tail : 1.f - tail;
}
template <int KIND> __device__ __forceinline__ float activated(float z) {
    if (KIND == kActRelu) return z <= 0.f ? 0.f : z;
    if (KIND == kActSilu) return z * inverse(1.f + exp_of_minus(z));
    if (KIND == kActGelu) {
        float bell;
        return z * normal_of(z, bell);
    }
    return z;
}
template <int KIND, int V> __device__ __forceinline__ void activate(float (&z)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) z[i] = activated<KIND>(z[i]);
}
// f with the activation as a constant: asked once for a loop, not in it, where the ways that it might go take registers side by side.
template <int K> struct Kind { static constexpr int value = K; };
template <typename F> __device__ __forceinline__ void with_kind(int kind, F f) {
    if (kind == kActSilu) f(Kind<kActSilu>());
    else if (kind == kActRelu) f(Kind<kActRelu>());
    else if (kind == kActGelu) f(Kind<kActGelu>());
    else f(Kind<kActNone>());
}
// (x - m) r w + b where that is near 0, with the roundings of difference and products added: what the sum of two floats for each leaves out is 2^-45 of b.
__device__ __forceinline__ float sum_near_0(float x, float m, float r, float w, float b) {
#pragma clang fp contract(off)
    const float d = x - m, of_m = x - d, d_low = (x - (d + of_m)) + (of_m - m);         // x - m = d + d_low
    const float q = r * w, q_low = __builtin_fmaf(r, w, -q), p = d * q, p_low = __builtin_fmaf(d, q, -p);
    return (p + b) + (p_low + __builtin_fmaf(d, q_low, d_low * q));
}
// x becomes u = (x - m) r, and g becomes g act'(u w + b).  On which side of 0 a rectified z lies is asked more exactly where 32 bits might not tell.  (ONE: the run's channels are of one group.)
template <int KIND, bool ONE, int V, int N> __device__ __forceinline__ void slopes(float (&x)[V], float (&g)[V], const float (&m)[N], const float (&r)[N], const float (&w)[V], const float (&b)[V]) {
    bool near = false;
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int j = ONE ? 0 : i;
        const float u = (x[i] - m[j]) * r[j], z = __builtin_fmaf(u, w[i], b[i]);
        if (KIND == kActRelu) near = near || __builtin_fabsf(z) <= 9.5367431640625e-7f * __builtin_fabsf(b[i]);      // 2^-20
        if (KIND == kActSilu) {
            const float s = inverse(1.f + exp_of_minus(z));
            g[i] *= s * __builtin_fmaf(z, 1.f - s, 1.f);
        }
        if (KIND == kActGelu) {
            float bell;
            const float under = normal_of(z, bell);
            g[i] *= __builtin_fmaf(z * 0.39894228040143268f, bell, under);
        }
        if (KIND != kActRelu) x[i] = u;
    }
    if (KIND == kActRelu) {
        if (__builtin_expect(near, 0)) {
#pragma unroll
            for (int i = 0; i < V; i++) g[i] = sum_near_0(x[i], m[ONE ? 0 : i], r[ONE ? 0 : i], w[i], b[i]) <= 0.f ? g[i] * 0.f : g[i];
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int j = ONE ? 0 : i;
            x[i] = (x[i] - m[j]) * r[j];
            if (!near) g[i] = __builtin_fmaf(x[i], w[i], b[i]) <= 0.f ? g[i] * 0.f : g[i];
        }
    }
}

// Sums over a workgroup's lanes of pixels (values[lane][unit], `units` of them from `first` on) and over the `each` units of a group, added to total[group].
// A group's team of threads adds in a fixed order, then their sums are joined; all of `threads` threads, a power of two of them, are needed.
__device__ __forceinline__ void group_totals(const float* values, float* total, int lanes, int units, int first, int each, int groups_from, int groups_to, int thread, int threads) {
    const int n = groups_to - groups_from;
    int team = 64;
    while (team > 1 && team * n > threads) team >>= 1;
    for (int g0 = 0; g0 < n; g0 += threads / team) {
        const int g = g0 + thread / team, member = thread & (team - 1);
        float sum = 0.f;
        if (g < n) {
            const int c0 = max((groups_from + g) * each - first, 0), c1 = min((groups_from + g + 1) * each - first, units), width = c1 - c0;
            if (width == units) {                                  // (one group: everything)
#pragma unroll 4
                for (int e = member; e < lanes * width; e += team) sum += values[e];
            } else if (width == 1) {
#pragma unroll 4
                for (int lane = member; lane < lanes; lane += team) sum += values[lane * units + c0];
            } else {
                int lane = member / width, c = member - lane * width;
                const int down = team / width, across_ = team - down * width;
                for (int e = member; e < lanes * width; e += team) {
                    sum += values[lane * units + c0 + c];
                    lane += down;
                    c += across_;
                    if (c >= width) { c -= width; lane++; }
                }
            }
        }
        for (int d = 1; d < team; d <<= 1) sum += __shfl_xor(sum, d);
        if (g < n && member == 0) total[groups_from + g] += sum;
    }
}

template <typename T, int V> __device__ __forceinline__ void load_parameters(const NormArgs& A, const void* p, int at, float without, float (&x)[V]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < V; i++) x[i] = without;
    } else if (A.weight_float) load_run<float, V>((const float*)p + at, x);
    else load_run<T, V>((const T*)p + at, x);
}

// ---- in one pass ----
//
// Where the pixels of a picture with a few groups' channels fit into the registers of a workgroup, it reads them once: the mean, then the squares around it, are
// summed from registers, and what is written is made from them.  A thread has a run of V channels of every few pixels; block: channels of a workgroup, whole groups and whole
// runs.  us: 64 pictures of 14 x 14 x 256, bfloat 8.3 (2.6 at 5.0 TB/s), the gradient 15 (3.9), one of 14 x 14 x 64 5.7: the launch, and loads, sums and stores of a workgroup, which
// follow each other, bound it.  The workgroups of a picture run on one die (blockIdx modulo 8 goes round the dies), where they find in its cache what lies beside their own channels in a line.
struct Slab {
    int64_t image, row;                                            // the first of the thread's pictures; where its workgroup's sums go
    int first, channels, columns, lanes, lane, column;             // of the workgroup's channels; runs of a pixel; threads to a run, the thread's place
    int slot, thread, threads;                                     // of the workgroup's pictures; of the picture's threads
    bool works;
};
__device__ __forceinline__ Slab slab_of(const NormArgs& A, int V) {
    Slab S;
    const int64_t at = blockIdx.x + A.begin;
    const int dies = A.images % 8 || A.blocks == 1 ? 1 : 8;
    const int64_t row = at / dies, turn = row / A.blocks;
    S.threads = (int)blockDim.x / A.pack;
    S.slot = threadIdx.x / S.threads;
    S.thread = threadIdx.x & (S.threads - 1);
    S.row = turn * dies + at % dies;
    S.image = S.row * A.pack * A.turns + S.slot;
    S.first = (int)(row - turn * A.blocks) * A.block;
    S.channels = min(A.block, A.channels - S.first);
    S.columns = S.channels / V;
    S.lanes = S.threads / S.columns;
    S.lane = S.thread / S.columns;
    S.column = S.thread - S.lane * S.columns;
    S.works = S.lane < S.lanes;
    return S;
}
// ONE: the channels of a run are of one group.
template <int V, bool ONE> __device__ __forceinline__ int value_units(int channels) { return ONE ? channels / V : channels; }
template <int V, bool ONE> __device__ __forceinline__ void put_values(float* values, const Slab& S, const float (&x)[V]) {
    if (!S.works) return;
    if constexpr (ONE) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) sum += x[i];
        values[S.lane * S.columns + S.column] = sum;
    } else {
#pragma unroll
        for (int i = 0; i < V; i++) values[(S.lane * S.columns + S.column) * V + i] = x[i];
    }
}

template <typename T, int V> struct Held { typename Run<T, V>::Vec v; };
template <typename T, int V> __device__ __forceinline__ void take(const Held<T, V>& from, float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) {
        if constexpr (V == 1) x[i] = (float)from.v;
        else x[i] = (float)from.v[i];
    }
}
template <typename T, int V, int K> __device__ __forceinline__ void hold(Held<T, V> (&h)[K], const T* from, int64_t pixel, const Slab& S, int pixels) {
#pragma unroll
    for (int k = 0; k < K; k++)
        if (k * S.lanes < pixels) h[k].v = reinterpret_cast<const typename Run<T, V>::Loose*>(from + (int64_t)min(S.lane + k * S.lanes, pixels - 1) * pixel)->v;
}

// MANY: a workgroup has several pictures, A.pack side by side and A.turns after one another.
template <typename T, int V, int K, int THREADS, bool ONE, bool MANY> __global__ __launch_bounds__(THREADS) void k_norm_held(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const Slab S = slab_of(A, V);
    const int groups = S.channels / A.each;
    float* values = shared + S.slot * S.threads * (ONE ? 1 : V);   // [lane][unit]
    float* total = shared + THREADS * (ONE ? 1 : V) + S.slot * 3 * groups;     // [group of the block]: sums; then means; then r
    const int pixels = (int)A.pixels, c = S.first + S.column * V, unit_groups = ONE ? A.each / V : A.each;
    constexpr bool EARLY = THREADS == 256;                         // (workgroups of 512 threads have registers for the parameters when the sums are made)
    float w[V], b[V];
    auto parameters = [&]() {
        load_parameters<T, V>(A, A.weight, S.works ? c : S.first, 1.f, w);
        load_parameters<T, V>(A, A.bias, S.works ? c : S.first, 0.f, b);
    };
    const int units = value_units<V, ONE>(S.channels);
    const float inv = 1.f / ((float)pixels * A.each);
    for (int turn = 0;; turn++) {
        const int64_t image = S.image + turn * A.pack;
        const bool last = !MANY || turn + 1 == A.turns, there = image < A.images;
        Held<T, V> x[K];
        hold<T, V, K>(x, (const T*)A.x + min(image, A.images - 1) * A.x_image + (S.works ? c : S.first), A.x_pixel, S, pixels);
        if (EARLY && turn == 0) parameters();
        for (int g = S.thread; g < 3 * groups; g += S.threads) total[g] = 0.f;
        float sum[V];
#pragma unroll
        for (int i = 0; i < V; i++) sum[i] = 0.f;
#pragma unroll
        for (int k = 0; k < K; k++)
            if (k * S.lanes < pixels) {
                float a[V];
                take(x[k], a);
                if (S.lane + k * S.lanes < pixels) {
#pragma unroll
                    for (int i = 0; i < V; i++) sum[i] += a[i];
                }
            }
        put_values<V, ONE>(values, S, sum);
        __syncthreads();
        group_totals(values, total, S.lanes, units, 0, unit_groups, 0, groups, S.thread, S.threads);
        __syncthreads();
        float m[ONE ? 1 : V];
#pragma unroll
        for (int i = 0; i < (ONE ? 1 : V); i++) m[i] = S.works ? total[(S.column * V + i) / A.each] * inv : 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) sum[i] = 0.f;
#pragma unroll
        for (int k = 0; k < K; k++)
            if (k * S.lanes < pixels) {
                float a[V];
                take(x[k], a);
                if (S.lane + k * S.lanes < pixels) {
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float d = a[i] - m[ONE ? 0 : i];
                        sum[i] = __builtin_fmaf(d, d, sum[i]);
                    }
                }
            }
        put_values<V, ONE>(values, S, sum);
        __syncthreads();
        group_totals(values, total + groups, S.lanes, units, 0, unit_groups, 0, groups, S.thread, S.threads);
        __syncthreads();
        for (int g = S.thread; g < groups; g += S.threads) {
            const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(total[groups + g], inv, A.eps));
            total[2 * groups + g] = r;
            float2* to = (float2*)A.stats + image * A.groups + S.first / A.each + g;
            if (there) *to = make_float2(total[g] * inv, r);
        }
        __syncthreads();
        if (S.works && there) {
            float by[V];
            if (!EARLY) parameters();
#pragma unroll
            for (int i = 0; i < V; i++) by[i] = w[i] * total[2 * groups + (S.column * V + i) / A.each];
            T* out = (T*)A.out + image * A.out_image + c;
            with_kind(A.activation, [&](auto kind) {
#pragma unroll
                for (int k = 0; k < K; k++) {
                    const int p = S.lane + k * S.lanes;
                    if (p < pixels) {
                        float a[V];
                        take(x[k], a);
#pragma unroll
                        for (int i = 0; i < V; i++) a[i] = __builtin_fmaf(a[i] - m[ONE ? 0 : i], by[i], b[i]);
                        activate<decltype(kind)::value>(a);
                        store_run<T, V>(out + (int64_t)p * A.out_pixel, a);
                    }
                    one_after_another();
                }
            });
        }
        if (last) break;
        __syncthreads();
    }
}

// The gradient.  What a thread has summed over its pictures, by channels, is summed over the workgroup at the end.
template <typename T, int V, int K, int THREADS, bool ONE, bool MANY> __global__ __launch_bounds__(THREADS) void k_norm_back_held(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const Slab S = slab_of(A, V);
    const int groups = S.channels / A.each, pixels = (int)A.pixels, c = S.first + S.column * V, unit_groups = ONE ? A.each / V : A.each;
    const int units = value_units<V, ONE>(S.channels), half = S.threads * (ONE ? 1 : V);
    float* values = shared + S.slot * 2 * half;                    // [2][lane][unit]; at the end [lane of all pictures][channel]
    float* total = shared + 2 * THREADS * (ONE ? 1 : V) + S.slot * 2 * groups;             // [2][group]
    float w[V], b[V], sums[2][V];                                  // sums: of h u and h
    load_parameters<T, V>(A, A.weight, S.works ? c : S.first, 1.f, w);
    load_parameters<T, V>(A, A.bias, S.works ? c : S.first, 0.f, b);
#pragma unroll
    for (int i = 0; i < V; i++) sums[0][i] = sums[1][i] = 0.f;
    const float inv = 1.f / ((float)pixels * A.each);
    for (int turn = 0;; turn++) {
        const int64_t image = S.image + turn * A.pack, at = min(image, A.images - 1);
        const bool last = !MANY || turn + 1 == A.turns, there = image < A.images;
        Held<T, V> x[K], h[K];
        hold<T, V, K>(x, (const T*)A.x + at * A.x_image + (S.works ? c : S.first), A.x_pixel, S, pixels);
        hold<T, V, K>(h, (const T*)A.grad + at * A.grad_image + (S.works ? c : S.first), A.grad_pixel, S, pixels);
        for (int e = S.thread; e < 2 * groups; e += S.threads) total[e] = 0.f;
        float m[ONE ? 1 : V], r[ONE ? 1 : V], s[2][V];
#pragma unroll
        for (int i = 0; i < (ONE ? 1 : V); i++) {
            const float2 of = ((const float2*)A.stats)[at * A.groups + ((S.works ? c : S.first) + i) / A.each];
            m[i] = of.x;
            r[i] = of.y;
        }
#pragma unroll
        for (int i = 0; i < V; i++) s[0][i] = s[1][i] = 0.f;
        with_kind(A.activation, [&](auto kind) {
#pragma unroll
            for (int k = 0; k < K; k++)
                if (k * S.lanes < pixels) {
                    float a[V], g[V];
                    take(x[k], a);
                    take(h[k], g);
                    slopes<decltype(kind)::value, ONE>(a, g, m, r, w, b);
                    if (S.lane + k * S.lanes < pixels) {
#pragma unroll
                        for (int i = 0; i < V; i++) {
                            s[0][i] = __builtin_fmaf(g[i], a[i], s[0][i]);
                            s[1][i] += g[i];
                        }
                    }
                    one_after_another();
                }
        });
        // The groups'.
#pragma unroll
        for (int z = 0; z < 2; z++) {
            float weighted[V];
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (there) sums[z][i] += s[z][i];
                weighted[i] = s[z][i] * w[i];
            }
            put_values<V, ONE>(values + z * half, S, weighted);
        }
        __syncthreads();
        group_totals(values, total, S.lanes, units, 0, unit_groups, 0, groups, S.thread, S.threads);
        group_totals(values + half, total + groups, S.lanes, units, 0, unit_groups, 0, groups, S.thread, S.threads);
        __syncthreads();
        if (S.works && there) {
            float su[ONE ? 1 : V], sh[ONE ? 1 : V];
#pragma unroll
            for (int i = 0; i < (ONE ? 1 : V); i++) {
                const int g = (S.column * V + i) / A.each;
                su[i] = total[g] * inv;
                sh[i] = total[groups + g] * inv;
            }
            T* out = (T*)A.out + image * A.out_image + c;
            with_kind(A.activation, [&](auto kind) {
#pragma unroll
                for (int k = 0; k < K; k++) {
                    const int p = S.lane + k * S.lanes;
                    if (p < pixels) {
                        float a[V], g[V];
                        take(x[k], a);
                        take(h[k], g);
                        slopes<decltype(kind)::value, ONE>(a, g, m, r, w, b);
#pragma unroll
                        for (int i = 0; i < V; i++) {
                            const int j = ONE ? 0 : i;
                            a[i] = r[j] * (__builtin_fmaf(g[i], w[i], -sh[j]) - a[i] * su[j]);
                        }
                        store_run<T, V>(out + (int64_t)p * A.out_pixel, a);
                    }
                    one_after_another();
                }
            });
        }
        if (last) break;
        __syncthreads();
    }
    // The channels'.
    float* channel = shared + THREADS * V;                         // [channel]
    float2* to = (float2*)A.sums + S.row * A.channels + S.first;
    for (int z = 0; z < 2; z++) {
        __syncthreads();
        if (S.works) {
#pragma unroll
            for (int i = 0; i < V; i++) shared[((S.slot * S.lanes + S.lane) * S.columns + S.column) * V + i] = z ? sums[1][i] : sums[0][i];
        }
        for (int e = threadIdx.x; e < S.channels; e += THREADS) channel[e] = 0.f;
        __syncthreads();
        group_totals(shared, channel, (MANY ? A.pack : 1) * S.lanes, S.channels, 0, 1, 0, S.channels, (int)threadIdx.x, THREADS);
        __syncthreads();
        for (int e = threadIdx.x; e < S.channels; e += THREADS) (z ? to[e].y : to[e].x) = channel[e];
    }
}

// ---- in two passes ----
//
// Larger pictures are gone through twice, chunk by chunk of their pixels: sums of every chunk, then what is written; what the second pass reads mostly comes out of the
// memory-side cache.  Loads of four pixels are under way together, without conditions about them (behind which the compiler would wait for those before).
// Bound by memory.  us: 64 pictures of 112 x 112 x 64, bfloat, sums 32 (103 MB, 3.2 TB/s; 26 where x is in the cache), result 39 (206 MB, 5.3 TB/s); gradient of 64 of 56 x 56 x 256 sums 57
// (206 MB, 3.6 TB/s), result 55 (308 MB, 5.6 TB/s), sums of the weights' gradients 5.
constexpr int kNormThreads = 256;
constexpr int kNormTogether = 4;
constexpr int kMergedChunks = 64;                                  // so many of a picture's chunks are joined by every workgroup that needs them

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

// Mean and sum of squares around it of every group over a chunk of pixels.
template <typename T, int V> __global__ __launch_bounds__(256) void k_norm_sums(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    float* values = shared;                                        // [lane][channel of the block]
    float* total = shared + kNormThreads * V;                      // [group]
    float* mean = total + A.groups;
    const Chunk K = chunk_of(A, blockIdx.x + A.begin);
    const T* x = (const T*)A.x + K.image * A.x_image;
    const int all = A.channels / V;
    for (int g = threadIdx.x; g < A.groups; g += kNormThreads) total[g] = 0.f;
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
                    float v;
                    if (phase == 0) v = m[i] * n;
                    else {
                        const float d = m[i] - mean[(c + i) / A.each];
                        v = __builtin_fmaf(d * d, (float)n, q[i]);
                    }
                    values[C.lane * width + C.column * V + i] = v;
                }
            }
            __syncthreads();
            group_totals(values, total, C.lanes, width, first, A.each, g0, g1, (int)threadIdx.x, kNormThreads);
            __syncthreads();
        }
        const float count = (float)(K.end - K.first) * A.each;
        float* part = A.part + ((blockIdx.x + A.begin) * A.groups) * 2 + phase;
        for (int g = threadIdx.x; g < A.groups; g += kNormThreads) {
            if (phase == 0) mean[g] = total[g] / count;
            part[2 * g] = phase == 0 ? mean[g] : total[g];
            total[g] = 0.f;
        }
        __syncthreads();
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
                activate<decltype(kind)::value>(a);
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
                    slopes<decltype(kind)::value, ONE>(a, h, m, r, w, b);
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
                slopes<decltype(kind)::value, ONE>(a, h, m, r, w, b);
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
