// Group norm and its gradient in one pass, from registers.
#pragma once
#include <algorithm>

#include "pcr_norm.h"

namespace pcr {

// Where the pixels of a picture with a few groups' channels fit into the registers of a workgroup, it reads them once: the mean, then the squares around it, are
// summed from registers, and what is written is made from them.  A thread has a run of V channels of every few pixels; block: channels of a workgroup, whole groups and whole
// runs.  us: 64 pictures of 14 x 14 x 256, bfloat 8.6 (2.6 at 5.0 TB/s), the gradient 16 (3.9), one of 14 x 14 x 64 6.0: the launch, and loads, sums and stores of a workgroup, which
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
template <typename T, int V, int K> __device__ __forceinline__ void hold(Held<T, V> (&h)[K], const T* from, int64_t pixel, const Slab& S, int pixels) {
#pragma unroll
    for (int k = 0; k < K; k++)
        if (k * S.lanes < pixels) h[k].v = reinterpret_cast<const typename Run<T, V>::Loose*>(from + (int64_t)min(S.lane + k * S.lanes, pixels - 1) * pixel)->v;
}

// MANY: a workgroup has several pictures, A.pack side by side and A.turns after one another.  Workgroups of 512 threads have 128 registers, so that two fit a compute unit, where that takes no
// scratch memory (32 pictures of 56 x 56 x 256 41 us with one, 33 with two).
template <typename T, int V, int K, int THREADS, bool ONE, bool MANY> __global__ __launch_bounds__(THREADS, THREADS == 512 && ONE ? 4 : 1) void k_norm_held(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const Slab S = slab_of(A, V);
    const int groups = S.channels / A.each;
    // A sum of the values in 32 bits would leave the mean off by some roundings of it, which 1 / sqrt(eps) makes seen where they are equal or close to each other (a picture of 900.1 gave 0.02
    // for 0).  A thread sums what its values are off its first one (of each channel, where its run has several groups), and these sums are added in 64 bits.  FIRST: what is summed is
    // off the group's first value, which is a load more, in 32 bits (for tens of thousands of small pictures 64 bits took 9 and 15 % longer, for others 1 to 5 % longer than sums of the values in 32).
    constexpr bool FIRST = ONE && MANY;
    typedef typename std::conditional<FIRST, float, double>::type Sum;
    float* values = shared + S.slot * S.threads * (ONE ? 2 : 2 * V);           // [lane][unit]
    float* squares = shared + THREADS * (ONE ? 2 : 2 * V) + S.slot * 4 * groups;           // [group of the block]; then r
    float* origin = squares + groups;                              // [group of the block]: its first value, of which the sums leave it out
    Sum* total = (Sum*)(squares + 2 * groups);                     // [group of the block]
    const int pixels = (int)A.pixels, c = S.first + S.column * V, unit_groups = ONE ? A.each / V : A.each;
    constexpr bool EARLY = THREADS == 256;                         // (workgroups of 512 threads have registers for the parameters when the sums are made)
    float w[V], b[V];
    auto parameters = [&]() {
        load_parameters<T, V>(A, A.weight, S.works ? c : S.first, 1.f, w);
        load_parameters<T, V>(A, A.bias, S.works ? c : S.first, 0.f, b);
    };
    const int units = value_units<V, ONE>(S.channels);
    const float inv = 1.f / ((float)pixels * A.each);
    const double exact_inv = 1.0 / ((double)pixels * A.each);
    auto mean_of = [&](int g) { return FIRST ? __builtin_fmaf((float)total[g], inv, origin[g]) : (float)((double)total[g] * exact_inv); };
    for (int turn = 0;; turn++) {
        const int64_t image = S.image + turn * A.pack;
        const bool last = !MANY || turn + 1 == A.turns, there = image < A.images;
        Held<T, V> x[K];
        hold<T, V, K>(x, (const T*)A.x + min(image, A.images - 1) * A.x_image + (S.works ? c : S.first), A.x_pixel, S, pixels);
        float from[ONE ? 1 : V], sum[V];
        const int of = S.column * V / A.each;                      // the run's group, its first
        if (FIRST) from[0] = (float)((const T*)A.x)[min(image, A.images - 1) * A.x_image + S.first + (S.works ? of * A.each : 0)];
        if (EARLY && turn == 0) parameters();
        for (int g = S.thread; g < groups; g += S.threads) {
            total[g] = 0;
            squares[g] = 0.f;
        }
        if (FIRST) {
            if (S.works && S.lane == 0 && S.column * V == of * A.each) origin[of] = from[0];
        } else {
            float a[V];
            take(x[0], a);
#pragma unroll
            for (int i = 0; i < (ONE ? 1 : V); i++) from[i] = a[i];
        }
        int mine = 0;
#pragma unroll
        for (int i = 0; i < V; i++) sum[i] = 0.f;
#pragma unroll
        for (int k = 0; k < K; k++)
            if (k * S.lanes < pixels) {
                float a[V];
                take(x[k], a);
                if (S.lane + k * S.lanes < pixels) {
                    mine = k + 1;
#pragma unroll
                    for (int i = 0; i < V; i++) sum[i] += a[i] - from[ONE ? 0 : i];
                }
            }
        if constexpr (FIRST) put_values<V, ONE>(values, S, sum);
        else if (S.works) {
            double* to = (double*)values + (S.lane * S.columns + S.column) * (ONE ? 1 : V);
            if constexpr (ONE) {
#pragma unroll
                for (int i = 1; i < V; i++) sum[0] += sum[i];
                to[0] = __builtin_fma((double)from[0], (double)(mine * V), (double)sum[0]);
            } else {
#pragma unroll
                for (int i = 0; i < V; i++) to[i] = __builtin_fma((double)from[i], (double)mine, (double)sum[i]);
            }
        }
        __syncthreads();
        group_totals((const Sum*)values, total, S.lanes, units, 0, unit_groups, 0, groups, S.thread, S.threads);
        __syncthreads();
        float m[ONE ? 1 : V];
#pragma unroll
        for (int i = 0; i < (ONE ? 1 : V); i++) m[i] = S.works ? mean_of((S.column * V + i) / A.each) : 0.f;
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
        group_totals(values, squares, S.lanes, units, 0, unit_groups, 0, groups, S.thread, S.threads);
        __syncthreads();
        for (int g = S.thread; g < groups; g += S.threads) {
            const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(squares[g], inv, A.eps));
            squares[g] = r;
            float2* to = (float2*)A.stats + image * A.groups + S.first / A.each + g;
            if (there) *to = make_float2(mean_of(g), r);
        }
        __syncthreads();
        if (S.works && there) {
            float by[V];
            if (!EARLY) parameters();
#pragma unroll
            for (int i = 0; i < V; i++) by[i] = w[i] * squares[(S.column * V + i) / A.each];
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
                        activate<T, decltype(kind)::value>(a);
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
                    slopes<T, decltype(kind)::value, ONE>(a, g, m, r, w, b);
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
                        slopes<T, decltype(kind)::value, ONE>(a, g, m, r, w, b);
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

// One pass of either kind.  (A kernel whose threads would not hold the picture, or that is not the one of the plan, is not launched.)
template <bool BACK> bool run_held(const pcr_group_norm* N, const NormPlan& P, NormArgs A, hipStream_t s) {
    bool ok = true;
    const bool one = A.each % P.run == 0;
    with_run(N->dtype, P.run, [&](auto t, auto v) {
        typedef decltype(t) T;
        constexpr int V = decltype(v)::value;
        auto launch = [&](auto k, auto threads, auto in_one, auto of_many) {
            constexpr int K = decltype(k)::value, THREADS = decltype(threads)::value;
            constexpr bool ONE = decltype(in_one)::value, MANY = decltype(of_many)::value;
            ok = ok && P.held == K && P.threads == THREADS && P.many == MANY && P.holds(N->pixels);
            if (!ok) return;
            const size_t lds = P.lds(A.each, BACK);
            in_ranges(P.rows * A.blocks, THREADS, [&](int64_t begin, unsigned workgroups) {
                A.begin = begin;
                if constexpr (BACK) {
                    ok = ok && allow_lds(k_norm_back_held<T, V, K, THREADS, ONE, MANY>, lds);
                    if (ok) hipLaunchKernelGGL((k_norm_back_held<T, V, K, THREADS, ONE, MANY>), dim3(workgroups), dim3(THREADS), lds, s, A);
                } else {
                    ok = ok && allow_lds(k_norm_held<T, V, K, THREADS, ONE, MANY>, lds);
                    if (ok) hipLaunchKernelGGL((k_norm_held<T, V, K, THREADS, ONE, MANY>), dim3(workgroups), dim3(THREADS), lds, s, A);
                }
            });
        };
        auto by_one = [&](auto k, auto threads, auto of_many) {
            if (one) launch(k, threads, std::true_type(), of_many);
            else if constexpr (V > 1) launch(k, threads, std::false_type(), of_many);
        };
        constexpr bool WHOLE = V * sizeof(T) == 16;
        if (P.many) by_one(Int<WHOLE ? 1 : 3>(), Int<256>(), std::true_type());
        else if (P.threads == 256) by_one(Int<WHOLE ? 4 : 8>(), Int<256>(), std::false_type());
        else if constexpr (WHOLE) {
            if (P.held <= 8) by_one(Int<8>(), Int<512>(), std::false_type());
            else if constexpr (!BACK) by_one(Int<16>(), Int<512>(), std::false_type());
        }
    });
    return ok;
}

}  // namespace pcr
