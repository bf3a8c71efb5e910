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
    float* sums;                                                   // [image][chunk][channel][2]: sums of h u and h
    int64_t images, pixels, x_image, x_pixel, grad_image, grad_pixel, out_image, out_pixel;
    int64_t chunk;                                                 // pixels of a workgroup
    int chunks, channels, groups, each, activation, weight_float;  // each: channels of a group
    float eps;
};

__device__ __forceinline__ float activated(float z, int kind) {
    if (kind == kActRelu) return z <= 0.f ? 0.f : z;
    if (kind == kActSilu) return z / (1.f + __expf(-z));
    if (kind == kActGelu) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    return z;
}
// act'(z) of z = u w + b, u = (x - m) r.  On which side of 0 a rectified z lies is asked in 64 bits where 32 might not tell.
__device__ __forceinline__ float slope(float z, int kind, float x, float m, float r, float w, float b) {
    if (kind == kActRelu) {
        if (__builtin_expect(fabsf(z) <= 9.5367431640625e-7f * fabsf(b), 0)) return ((double)x - m) * r * w + b <= 0.0 ? 0.f : 1.f;      // 2^-20
        return z <= 0.f ? 0.f : 1.f;
    }
    if (kind == kActSilu) {
        const float s = 1.f / (1.f + __expf(-z));
        return s * __builtin_fmaf(z, 1.f - s, 1.f);
    }
    if (kind == kActGelu) return __builtin_fmaf(z * 0.39894228040143268f, __expf(-0.5f * z * z), 0.5f * (1.f + erff(z * 0.70710678118654752f)));
    return 1.f;
}

// Sums over a workgroup's lanes of pixels (values[lane][channel], `channels` of them from `first` on) and over the channels of a group: into total[group].
// 256 threads; every thread of a group's team adds in a fixed order, then the team's.
__device__ __forceinline__ void group_totals(const float* values, float* total, int lanes, int channels, int first, int each, int groups_from, int groups_to) {
    const int n = groups_to - groups_from;
    int team = 64;
    while (team > 1 && team * n > 256) team >>= 1;
    for (int g0 = 0; g0 < n; g0 += 256 / team) {
        const int g = g0 + threadIdx.x / team, member = threadIdx.x & (team - 1);
        float sum = 0.f;
        if (g < n) {
            const int c0 = max((groups_from + g) * each - first, 0), c1 = min((groups_from + g + 1) * each - first, channels), width = c1 - c0;
            for (int e = member; e < lanes * width; e += team) {
                const int lane = e / width;
                sum += values[lane * channels + c0 + (e - lane * width)];
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

constexpr int kNormThreads = 256;

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

// Mean and sum of squares around it of every group over a chunk of pixels.
template <typename T, int V> __global__ __launch_bounds__(256) void k_norm_sums(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    float* values = shared;                                        // [lane][channel of the block]
    float* total = shared + kNormThreads * V;                      // [group]
    float* mean = total + A.groups;
    const int64_t image = blockIdx.x / A.chunks, p0 = (blockIdx.x - image * A.chunks) * A.chunk, p1 = min(p0 + A.chunk, A.pixels);
    const T* x = (const T*)A.x + image * A.x_image;
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
                for (int64_t p = p0 + C.lane; p < p1; p += 4 * C.lanes) {
                    float a[4][V];
                    const int here = (int)min((int64_t)4, (p1 - p + C.lanes - 1) / C.lanes);
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        if (j < here) load_run<T, V>(x + (p + j * C.lanes) * A.x_pixel + c, a[j]);
                    const float inv = here == 4 ? 0.25f : 1.f / here, part = (float)here / (float)(n + here);
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        float s = 0.f, t = 0.f;
#pragma unroll
                        for (int j = 0; j < 4; j++) if (j < here) s += a[j][i];
                        s *= inv;
#pragma unroll
                        for (int j = 0; j < 4; j++) if (j < here) t = __builtin_fmaf(a[j][i] - s, a[j][i] - s, t);
                        const float d = s - m[i];
                        m[i] = __builtin_fmaf(d, part, m[i]);
                        q[i] += __builtin_fmaf(d * d, n * part, t);
                    }
                    n += here;
                }
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
            group_totals(values, total, C.lanes, width, first, A.each, g0, g1);
            __syncthreads();
        }
        const float count = (float)(p1 - p0) * A.each;
        float* part = A.part + ((int64_t)blockIdx.x * A.groups) * 2 + phase;
        for (int g = threadIdx.x; g < A.groups; g += kNormThreads) {
            if (phase == 0) mean[g] = total[g] / count;
            part[2 * g] = phase == 0 ? mean[g] : total[g];
            total[g] = 0.f;
        }
        __syncthreads();
    }
}

// The statistics of every picture's groups from its chunks': one thread a group.
__global__ __launch_bounds__(64) void k_norm_stats(NormArgs A) {
    const int64_t at = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (at >= A.images * A.groups) return;
    const int64_t image = at / A.groups, g = at - image * A.groups;
    const float* part = A.part + (image * A.chunks * A.groups + g) * 2;
    double mean = 0.0, squares = 0.0;
    for (int k = 0; k < A.chunks; k++) mean += (double)part[(int64_t)k * A.groups * 2] * (double)(min(A.chunk, A.pixels - k * A.chunk));
    mean /= (double)A.pixels;
    for (int k = 0; k < A.chunks; k++) {
        const double d = (double)part[(int64_t)k * A.groups * 2] - mean;
        squares += (double)part[(int64_t)k * A.groups * 2 + 1] + d * d * (double)(min(A.chunk, A.pixels - k * A.chunk)) * A.each;
    }
    A.stats[2 * at] = (float)mean;
    A.stats[2 * at + 1] = (float)(1.0 / sqrt(squares / ((double)A.pixels * A.each) + (double)A.eps));
}

template <typename T, int V> __global__ __launch_bounds__(256) void k_norm_apply(NormArgs A) {
    const int64_t image = blockIdx.x / A.chunks, p0 = (blockIdx.x - image * A.chunks) * A.chunk, p1 = min(p0 + A.chunk, A.pixels);
    const T* x = (const T*)A.x + image * A.x_image;
    T* out = (T*)A.out + image * A.out_image;
    const int all = A.channels / V;
    for (int k = 0; k < all; k += kNormThreads) {
        const Columns C = columns_of(k, all);
        if (!C.works) continue;
        const int c = (k + C.column) * V;
        float w[V], b[V], m[V], r[V];
        load_parameters<T, V>(A, A.weight, c, 1.f, w);
        load_parameters<T, V>(A, A.bias, c, 0.f, b);
#pragma unroll
        for (int i = 0; i < V; i++) {
            const float* s = A.stats + (image * A.groups + (c + i) / A.each) * 2;
            m[i] = s[0];
            r[i] = s[1];
        }
        for (int64_t p = p0 + C.lane; p < p1; p += C.lanes) {
            float a[V];
            load_run<T, V>(x + p * A.x_pixel + c, a);
#pragma unroll
            for (int i = 0; i < V; i++) a[i] = activated(__builtin_fmaf((a[i] - m[i]) * r[i], w[i], b[i]), A.activation);
            store_run<T, V>(out + p * A.out_pixel + c, a);
        }
    }
}

// Of every chunk: sums of h u and h by channels, and of h w and h w u by groups.
template <typename T, int V> __global__ __launch_bounds__(256) void k_norm_back_sums(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    float* values = shared;
    float* total = shared + kNormThreads * V;
    const int64_t image = blockIdx.x / A.chunks, p0 = (blockIdx.x - image * A.chunks) * A.chunk, p1 = min(p0 + A.chunk, A.pixels);
    const T* x = (const T*)A.x + image * A.x_image;
    const T* grad = (const T*)A.grad + image * A.grad_image;
    const int all = A.channels / V;
    for (int g = threadIdx.x; g < 2 * A.groups; g += kNormThreads) total[g] = 0.f;
    for (int k = 0; k < all; k += kNormThreads) {
        const Columns C = columns_of(k, all);
        const int c = (k + C.column) * V, first = k * V, width = C.count * V;
        float s[2][V];                                             // of h u, of h
#pragma unroll
        for (int i = 0; i < V; i++) s[0][i] = s[1][i] = 0.f;
        float w[V], b[V], m[V], r[V];
        if (C.works) {
            load_parameters<T, V>(A, A.weight, c, 1.f, w);
            load_parameters<T, V>(A, A.bias, c, 0.f, b);
#pragma unroll
            for (int i = 0; i < V; i++) {
                const float* t = A.stats + (image * A.groups + (c + i) / A.each) * 2;
                m[i] = t[0];
                r[i] = t[1];
            }
            for (int64_t p = p0 + C.lane; p < p1; p += C.lanes) {
                float a[V], h[V];
                load_run<T, V>(x + p * A.x_pixel + c, a);
                load_run<T, V>(grad + p * A.grad_pixel + c, h);
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float u = (a[i] - m[i]) * r[i];
                    h[i] *= slope(__builtin_fmaf(u, w[i], b[i]), A.activation, a[i], m[i], r[i], w[i], b[i]);
                    s[0][i] = __builtin_fmaf(h[i], u, s[0][i]);
                    s[1][i] += h[i];
                }
            }
        }
        const int g0 = first / A.each, g1 = min((first + width + A.each - 1) / A.each, A.groups);
#pragma unroll
        for (int z = 0; z < 2; z++) {
            if (C.works) {
#pragma unroll
                for (int i = 0; i < V; i++) values[C.lane * width + C.column * V + i] = s[z][i];
            }
            __syncthreads();
            for (int e = threadIdx.x; e < width; e += kNormThreads) {
                float sum = 0.f;
                for (int l = 0; l < C.lanes; l++) sum += values[l * width + e];
                A.sums[((int64_t)blockIdx.x * A.channels + first + e) * 2 + z] = sum;
            }
            __syncthreads();
            if (C.works) {
#pragma unroll
                for (int i = 0; i < V; i++) values[C.lane * width + C.column * V + i] = s[z][i] * w[i];
            }
            __syncthreads();
            group_totals(values, total + (1 - z) * A.groups, C.lanes, width, first, A.each, g0, g1);      // (h w first)
            __syncthreads();
        }
    }
    for (int g = threadIdx.x; g < A.groups; g += kNormThreads) {
        float* part = A.part + ((int64_t)blockIdx.x * A.groups + g) * 2;
        part[0] = total[g];
        part[1] = total[A.groups + g];
    }
}

template <typename T, int V> __global__ __launch_bounds__(256) void k_norm_back_apply(NormArgs A) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const int64_t image = blockIdx.x / A.chunks, p0 = (blockIdx.x - image * A.chunks) * A.chunk, p1 = min(p0 + A.chunk, A.pixels);
    const double count = (double)A.pixels * A.each;
    for (int g = threadIdx.x; g < 2 * A.groups; g += kNormThreads) {
        double sum = 0.0;
        const float* part = A.part + image * A.chunks * A.groups * 2 + g;
        for (int k = 0; k < A.chunks; k++) sum += (double)part[(int64_t)k * A.groups * 2];
        shared[g] = (float)(sum / count);
    }
    __syncthreads();
    const T* x = (const T*)A.x + image * A.x_image;
    const T* grad = (const T*)A.grad + image * A.grad_image;
    T* out = (T*)A.out + image * A.out_image;
    const int all = A.channels / V;
    for (int k = 0; k < all; k += kNormThreads) {
        const Columns C = columns_of(k, all);
        if (!C.works) continue;
        const int c = (k + C.column) * V;
        float w[V], b[V], m[V], r[V], s[V], t[V];
        load_parameters<T, V>(A, A.weight, c, 1.f, w);
        load_parameters<T, V>(A, A.bias, c, 0.f, b);
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int g = (c + i) / A.each;
            const float* q = A.stats + (image * A.groups + g) * 2;
            m[i] = q[0];
            r[i] = q[1];
            s[i] = shared[2 * g];
            t[i] = shared[2 * g + 1];
        }
        for (int64_t p = p0 + C.lane; p < p1; p += C.lanes) {
            float a[V], h[V];
            load_run<T, V>(x + p * A.x_pixel + c, a);
            load_run<T, V>(grad + p * A.grad_pixel + c, h);
#pragma unroll
            for (int i = 0; i < V; i++) {
                const float u = (a[i] - m[i]) * r[i];
                h[i] *= slope(__builtin_fmaf(u, w[i], b[i]), A.activation, a[i], m[i], r[i], w[i], b[i]);
                a[i] = r[i] * (__builtin_fmaf(h[i], w[i], -s[i]) - u * t[i]);
            }
            store_run<T, V>(out + p * A.out_pixel + c, a);
        }
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
