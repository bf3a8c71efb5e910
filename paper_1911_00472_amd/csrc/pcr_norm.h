// Group norm with an activation, channels last, and its gradients.
//
// Over the pixels of a picture and the channels of a group:  m = mean x, r = (mean (x - m)^2 + eps)^-1/2, u = (x - m) r, z = u w + b, y = act(z).
// With the incoming gradient g and h = g act'(z):  dw = sum h u and db = sum h over pictures and pixels,  dx = r (h w - mean(h w) - u mean(h w u)).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/pcr.h"
#include "pcr_host.h"
#include "pcr_norm_plan.h"
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

// T: the type of values and results.  Those of 16 bits, which round to 2^-9 and 2^-12 of themselves, take the shorter forms (so do the gradients of weight and bias beside them, which are of 32 bits: sums
// of gradients that were rounded to 16).
template <typename T> constexpr bool kFull = sizeof(T) == 4;
// exp(-v), and 1 / v to a unit or two in the last place: a division has ten instructions.  The exponential's argument is rounded, which leaves |v| 2^-24 of it; in 32 bits that is made good (of v
// between -104 and 104, where it is infinite and 0).  In place of the library's exponential, error function and division, with which 32 of 56 x 56 x 128 in 32 bits took 27 us (SiLU) and 36 (GELU): 23 and 28.
template <typename T> __device__ __forceinline__ float exp_of_minus(float v) {
    if constexpr (!kFull<T>) return __builtin_amdgcn_exp2f(v * -1.4426950408889634f);
    const float at = __builtin_amdgcn_fmed3f(v, -104.f, 104.f), h = at * -1.4426950408889634f;
    const float low = __builtin_fmaf(at, -1.9259629891e-8f, __builtin_fmaf(at, -1.4426950408889634f, -h));               // (of log2 e, what its float leaves out)
    return __builtin_amdgcn_exp2f(h) * __builtin_fmaf(low, 0.69314718055994531f, 1.f);
}
__device__ __forceinline__ float inverse(float v) { return __builtin_amdgcn_rcpf(v); }
// The normal distribution at z, and exp(-z^2 / 2).  With u = (1 - 0.4 |z|) / (1 + 0.4 |z|) the upper tail is that exponential times a polynomial of u, fitted to the least relative error over
// |z| < 13.5 (6.9e-8; behind it both are 0 in 32 bits).  With its roundings the distribution is 6e-8 off at most, as one plus the error function is, and below -2 nearer by far.
// 16 bits: Abramowitz and Stegun's 7.1.26 (Handbook of Mathematical Functions, 1964): with t = 1 / (1 + 0.3275911 |z| / sqrt 2) the tail is half of a polynomial of t times the exponential,
// 7.5e-8 off at most, 1.5e-7 with its roundings.
template <typename T> __device__ __forceinline__ float normal_of(float z, float& bell) {
    const float far = __builtin_fabsf(z);
    bell = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    float tail;
    if constexpr (kFull<T>) {
        const float x = __builtin_fminf(far, 64.f), u = __builtin_fmaf(x * -0.8f, inverse(__builtin_fmaf(0.4f, x, 1.f)), 1.f);
        constexpr float of[] = {1.413313448e-01f, 2.280697972e-01f, 1.131352410e-01f, 2.454813756e-02f, -5.118664354e-03f, -2.942227526e-03f, 8.019402740e-04f, 3.306535073e-04f, -1.562505349e-04f};
        tail = of[8];
#pragma unroll
        for (int i = 7; i >= 0; i--) tail = __builtin_fmaf(tail, u, of[i]);
        tail *= bell;
    } else {
        const float t = inverse(__builtin_fmaf(0.23164188770f, far, 1.f));
        tail = t * __builtin_fmaf(t, __builtin_fmaf(t, __builtin_fmaf(t, __builtin_fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f) * bell;
    }
    return z < 0.f ? tail : 1.f - tail;
}
template <typename T, int KIND> __device__ __forceinline__ float activated(float z) {
    if (KIND == kActRelu) return z <= 0.f ? 0.f : z;
    if (KIND == kActSilu) return z * inverse(1.f + exp_of_minus<T>(z));
    if (KIND == kActGelu) {
        float bell;
        return z * normal_of<T>(z, bell);
    }
    return z;
}
template <typename T, int KIND, int V> __device__ __forceinline__ void activate(float (&z)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) z[i] = activated<T, KIND>(z[i]);
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
template <typename T, int KIND, bool ONE, int V, int N> __device__ __forceinline__ void slopes(float (&x)[V], float (&g)[V], const float (&m)[N], const float (&r)[N], const float (&w)[V], const float (&b)[V]) {
    bool near = false;
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int j = ONE ? 0 : i;
        const float u = (x[i] - m[j]) * r[j], z = __builtin_fmaf(u, w[i], b[i]);
        if (KIND == kActRelu) near = near || __builtin_fabsf(z) <= 9.5367431640625e-7f * __builtin_fabsf(b[i]);      // 2^-20
        if (KIND == kActSilu) {
            const float s = inverse(1.f + exp_of_minus<T>(z));
            g[i] *= s * __builtin_fmaf(z, 1.f - s, 1.f);
        }
        if (KIND == kActGelu) {
            float bell;
            const float under = normal_of<T>(z, bell);
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
// A group's team of threads adds in a fixed order, then their sums are joined; all of `threads` threads, a power of two of them, are needed.  S: float or double.
template <typename S> __device__ __forceinline__ void group_totals(const S* values, S* total, int lanes, int units, int first, int each, int groups_from, int groups_to, int thread, int threads) {
    const int n = groups_to - groups_from;
    int team = 64;
    while (team > 1 && team * n > threads) team >>= 1;
    for (int g0 = 0; g0 < n; g0 += threads / team) {
        const int g = g0 + thread / team, member = thread & (team - 1);
        S sum = 0;
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

// Runs as they lie in memory.
template <typename T, int V> struct Held { typename Run<T, V>::Vec v; };
template <typename T, int V> __device__ __forceinline__ void take(const Held<T, V>& from, float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) {
        if constexpr (V == 1) x[i] = (float)from.v;
        else x[i] = (float)from.v[i];
    }
}

// ---- launches ----

template <int N> using Int = std::integral_constant<int, N>;

// Lets a kernel have more LDS than is common.
template <typename K> bool allow_lds(K kernel, size_t bytes) {
    return bytes <= 65536 || hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess;
}

template <typename F> void with_run(int dtype, int run, F f) {
    with_type(dtype, [&](auto t) {
        if (run == 8) { if constexpr (sizeof(t) == 2) f(t, Int<8>()); }
        else if (run == 4) { if constexpr (sizeof(t) == 4) f(t, Int<4>()); }
        else if (run == 2) f(t, Int<2>());
        else f(t, Int<1>());
    });
}

// The kernels of one pass are compiled beside each other; false: a kernel cannot have its LDS.
__attribute__((visibility("hidden"))) bool run_norm_held(const pcr_group_norm* N, const NormPlan& P, NormArgs A, hipStream_t s);
__attribute__((visibility("hidden"))) bool run_norm_back_held(const pcr_group_norm* N, const NormPlan& P, NormArgs A, hipStream_t s);

}  // namespace pcr
