// Positions of several axes turned into the heads of queries and keys, alone or behind a norm of every head, and the gradients.
//
// With pair (x, y) of a head at angle a = position[axis] * frequency:   x' = x cos a - y sin a,   y' = x sin a + y cos a;
// its gradient is the same with -a.  Behind a norm u = x r w, r = (mean x^2 + eps)^-1/2; with h the incoming gradient turned back,
//   dw = sum over tokens and heads of h x r,      dx = r (h w - x r^2 mean(h w x)).
//
// The angle is the 32-bit product of the position and the frequency, each a 32-bit float: what a program gets that multiplies a table of frequencies by
// positions as tensors, and what weights were trained with, 2^-24 of itself off (0.002 radians at position 32768 in the fastest pair).  From there on
// nothing is lost: the float becomes a fraction of a turn in 64-bit fixed point, whose upper 32 bits go to sine and cosine of a half-turn's multiple.
//
// Bound by memory: every element is read once and written once.  A workgroup takes a few tokens: its lanes make the tokens' sines and cosines once,
// in LDS, for all heads of both sides; then a row (a head of a token) goes to a group of lanes, a lane holding one slot: a run of pairs, that is
// two runs of elements of up to 16 bytes, so that pairs meet in a lane whichever way they lie.  The sums of a norm go round the group.
#pragma once
#include "pcr_vec.h"

namespace pcr {

struct HeadSide {
    const void* in; const void* grad; void* out; const void* weight; float* part;    // part: [workgroup][dim] sums of the weight's gradient
    int64_t in_b, in_t, in_h, out_b, out_t, out_h, grad_b, grad_t, grad_h;
    int heads;
};
struct AxesArgs {
    HeadSide side[2];
    const void* position; const float* frequency; const int32_t* axis;
    int64_t pos_a, pos_b, pos_t, batch_tokens, chunks;
    int64_t tokens;
    int wide, axes, dim, pairs, inverse, weight_float;
    int slots, per_wave;                                       // slots of a row; rows of a wavefront (64 / slots, at least 1)
    int chunk;                                                 // tokens of a workgroup at a time
    float eps;
};

enum { kRotate = 0, kNorm = 1, kNormBack = 2 };
constexpr int kAxesTable = 2048;                               // pairs of sine and cosine that a workgroup keeps (16 KB)

// f radians as a fraction of a turn, in 64 bits behind the point: f's 24 bits times 1 / (2 pi) to 128 bits, moved by f's exponent and cut.
// (What is infinite or NaN gives some angle.)
__device__ __forceinline__ uint64_t turns_of(float f) {
    const uint32_t bits = __float_as_uint(f), e = bits >> 23 & 255;
    const uint64_t m = (bits & 0x7fffff) | (e ? 0x800000 : 0);
    const unsigned __int128 low = (unsigned __int128)m * 0x7f09d5f47d4d3770ull;
    const unsigned __int128 high = (unsigned __int128)m * 0x28be60db9391054aull + (uint64_t)(low >> 64);      // m / (2 pi) = high 2^-64 + its 64 bits behind
    const int down = 214 - (int)(e ? e : 1);                   // 2^(e - 150) of the float, 2^-128 of the product, 2^64 of the result
    uint64_t v;
    if (down >= 64) v = down < 192 ? (uint64_t)(high >> (down - 64)) : 0;
    else if (down > 0) v = (uint64_t)(high << (64 - down)) | (uint64_t)low >> down;
    else v = (uint64_t)low << -down;
    return bits >> 31 ? 0 - v : v;
}

// A token: its sequence and its place there.  The token `more` places on, of sequences of `tokens`, which may be several on.
struct Place {
    int64_t b; uint32_t t;
    __device__ __forceinline__ Place of(int more, int64_t tokens) const {
        const uint32_t n = (uint32_t)tokens, at = t + (uint32_t)more;
        if (at < n) return {b, at};
        return {b + at / n, at % n};
    }
};

__device__ __forceinline__ void turn_of(const AxesArgs& A, Place place, int pair, float& c, float& s) {
    const int a = min(max(A.axis[pair], 0), A.axes - 1);
    const int64_t at = a * A.pos_a + place.b * A.pos_b + place.t * A.pos_t;
    const int64_t pos = A.wide ? ((const int64_t*)A.position)[at] : (int64_t)((const int32_t*)A.position)[at];
    const int32_t phase = (int32_t)(turns_of((float)pos * A.frequency[pair]) >> 32);
    sincospif((float)phase * 4.656612873077392578125e-10f, &s, &c);              // 2^-31: in halves of a turn
    if (A.inverse) s = -s;
}

// Sum over a row's group of lanes (`slots` neighbouring ones from `head` on), the same in all of them; `width`: a power of two that is not below it.
__device__ __forceinline__ float group_sum(float v, int head, int member, int slots, int width) {
    for (int d = width >> 1; d; d >>= 1) {
        const float o = __shfl(v, head + member + d);
        if (member + d < slots) v += o;
    }
    return __shfl(v, head);
}

template <typename T, int N> __device__ __forceinline__ void load_weight(const AxesArgs& A, const void* w, int at, float (&x)[N]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = 1.f;
    } else if (A.weight_float) load_run<float, N>((const float*)w + at, x);
    else load_run<T, N>((const T*)w + at, x);
}

// T: elements; N: elements of a run; ADJ: a pair's elements are neighbours (a slot is two runs behind each other) or half the rotated part apart;
// K: slots of a lane (more than one where a row has more than 64).
template <typename T, int N, bool ADJ, int MODE, int K>
__global__ __launch_bounds__(256) void k_axes(AxesArgs A) {
    __shared__ float2 table[kAxesTable];
    __shared__ float joined[MODE == kNormBack ? 4 * 512 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slots = A.slots, width_slots = K > 1 ? 64 : slots;
    const int head = K > 1 ? 0 : lane / width_slots * width_slots, member = lane - head;
    const bool works = K > 1 || lane / width_slots < A.per_wave;
    int width = 1;
    while (width < width_slots) width <<= 1;
    const int R = 2 * A.pairs;

    int first[K], second[K];                                   // where the lane's runs begin; dim: there is none
#pragma unroll
    for (int j = 0; j < K; j++) {
        const int s = member + 64 * j;
        if (ADJ) { first[j] = 2 * N * s; second[j] = first[j] + N; }
        else if (s * N < A.pairs) { first[j] = s * N; second[j] = A.pairs + s * N; }
        else { first[j] = R + 2 * (s * N - A.pairs); second[j] = first[j] + N; }
        if (s >= slots || first[j] >= A.dim) first[j] = A.dim;
        if (s >= slots || second[j] >= A.dim) second[j] = A.dim;
    }
    float dw[2][K][2 * N];
    if (MODE == kNormBack) {
#pragma unroll
        for (int e = 0; e < 2 * K * 2 * N; e++) (&dw[0][0][0])[e] = 0.f;
    }

    for (int64_t chunk = blockIdx.x; chunk < A.chunks; chunk += gridDim.x) {
        const int64_t t0 = chunk * A.chunk;
        const Place base = {t0 / A.tokens, (uint32_t)(t0 % A.tokens)};
        const int here = (int)min((int64_t)A.chunk, A.batch_tokens - t0);
        for (int e = threadIdx.x; e < here * A.pairs; e += 256) {
            float c, s;
            turn_of(A, base.of(e / A.pairs, A.tokens), e % A.pairs, c, s);
            table[e] = make_float2(c, s);
        }
        __syncthreads();
#pragma unroll
        for (int z = 0; z < 2; z++) {
            const HeadSide& S = A.side[z];
            float w[K][2 * N];
            if (MODE != kRotate && works && S.heads) {
#pragma unroll
                for (int j = 0; j < K; j++) {
                    float x[N];
                    if (first[j] < A.dim) { load_weight<T, N>(A, S.weight, first[j], x); for (int i = 0; i < N; i++) w[j][i] = x[i]; }
                    if (second[j] < A.dim) { load_weight<T, N>(A, S.weight, second[j], x); for (int i = 0; i < N; i++) w[j][N + i] = x[i]; }
                }
            }
            const int rows = here * S.heads;
            for (int r0 = wave * A.per_wave; r0 < rows; r0 += 4 * A.per_wave) {
                const int r = r0 + (K > 1 ? 0 : lane / width_slots);
                const bool on = works && r < rows;
                const int tl = on ? r / S.heads : 0, h = on ? r - tl * S.heads : 0;
                const Place at = base.of(tl, A.tokens);
                const int64_t b = at.b, t = at.t;
                const T* in = (const T*)S.in + b * S.in_b + t * S.in_t + h * S.in_h;
                const T* gin = (const T*)S.grad + b * S.grad_b + t * S.grad_t + h * S.grad_h;
                T* out = (T*)S.out + b * S.out_b + t * S.out_t + h * S.out_h;
                float x[K][2 * N], g[K][2 * N];
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < K; j++) {
#pragma unroll
                    for (int half = 0; half < 2; half++) {
                        const int at = half ? second[j] : first[j];
                        float v[N] = {};
                        if (on && at < A.dim) load_run<T, N>(in + at, v);
#pragma unroll
                        for (int i = 0; i < N; i++) x[j][half * N + i] = v[i];
                        if (MODE == kNormBack) {
                            float u[N] = {};
                            if (on && at < A.dim) load_run<T, N>(gin + at, u);
#pragma unroll
                            for (int i = 0; i < N; i++) g[j][half * N + i] = u[i];
                        }
                    }
                }
                float rms = 1.f;
                if (MODE != kRotate) {
#pragma unroll
                    for (int j = 0; j < K; j++)
#pragma unroll
                        for (int i = 0; i < 2 * N; i++) sum = __builtin_fmaf(x[j][i], x[j][i], sum);
                    sum = group_sum(sum, head, member, width_slots, width);
                    rms = 1.f / __builtin_sqrtf(sum / (float)A.dim + A.eps);
                }
                if (MODE == kNorm) {
#pragma unroll
                    for (int j = 0; j < K; j++)
#pragma unroll
                        for (int i = 0; i < 2 * N; i++) x[j][i] = x[j][i] * rms * w[j][i];
                }
                float (&y)[K][2 * N] = MODE == kNormBack ? g : x;   // what is turned
#pragma unroll
                for (int j = 0; j < K; j++)
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        const int p = (member + 64 * j) * N + i, ia = ADJ ? 2 * i : i, ib = ADJ ? 2 * i + 1 : N + i;
                        if (p < A.pairs) {
                            const float2 cs = table[tl * A.pairs + p];
                            const float u = y[j][ia], v = y[j][ib];
                            y[j][ia] = __builtin_fmaf(u, cs.x, -(v * cs.y));
                            y[j][ib] = __builtin_fmaf(u, cs.y, v * cs.x);
                        }
                    }
                if (MODE == kNormBack) {
                    float dot = 0.f;
#pragma unroll
                    for (int j = 0; j < K; j++)
#pragma unroll
                        for (int i = 0; i < 2 * N; i++) {
                            if (on) dw[z][j][i] = __builtin_fmaf(g[j][i], x[j][i] * rms, dw[z][j][i]);
                            const int at = i < N ? first[j] : second[j];
                            g[j][i] = at < A.dim ? g[j][i] * w[j][i] : 0.f;
                            dot = __builtin_fmaf(g[j][i], x[j][i], dot);
                        }
                    dot = group_sum(dot, head, member, width_slots, width);
                    const float back = dot / (float)A.dim * rms * rms;
#pragma unroll
                    for (int j = 0; j < K; j++)
#pragma unroll
                        for (int i = 0; i < 2 * N; i++) x[j][i] = rms * (g[j][i] - x[j][i] * back);
                }
#pragma unroll
                for (int j = 0; j < K; j++)
#pragma unroll
                    for (int half = 0; half < 2; half++) {
                        const int at = half ? second[j] : first[j];
                        float v[N];
#pragma unroll
                        for (int i = 0; i < N; i++) v[i] = x[j][half * N + i];
                        if (on && at < A.dim) store_run<T, N>(out + at, v);
                    }
            }
        }
        __syncthreads();                                       // the table is made anew
    }

    // The weights' gradients: a lane's sums over its rows, then over the groups of a wavefront and the wavefronts in their order.
    if (MODE == kNormBack) {
#pragma unroll
        for (int z = 0; z < 2; z++) {
            float* part = A.side[z].part;
            if (!part) continue;                               // (the same for all)
#pragma unroll
            for (int j = 0; j < K; j++)
#pragma unroll
                for (int i = 0; i < 2 * N; i++) {
                    float v = works ? dw[z][j][i] : 0.f;
                    if (K == 1) {
                        float all = 0.f;
                        for (int q = 0; q < A.per_wave; q++) all += __shfl(v, q * width_slots + member);
                        v = all;
                    }
                    const int at = i < N ? first[j] : second[j];
                    if (head == 0 && at < A.dim) joined[wave * 512 + at + (i < N ? i : i - N)] = v;
                }
            __syncthreads();
            for (int e = threadIdx.x; e < A.dim; e += 256)
                part[(int64_t)blockIdx.x * A.dim + e] = ((joined[e] + joined[512 + e]) + joined[1024 + e]) + joined[1536 + e];
            __syncthreads();
        }
    }
}

// Sums [parts][dim] over the parts: a workgroup takes 16 columns of one side, 16 threads to a column, in a fixed order.
struct WeightSums { const float* part[2]; float* out[2]; int parts, dim; };
__global__ __launch_bounds__(256) void k_weight_sums(WeightSums A) {
    __shared__ float joined[256];
    const int column = threadIdx.x & 15, share = threadIdx.x >> 4, z = blockIdx.y, e = blockIdx.x * 16 + column;
    if (!A.out[z]) return;
    float sum = 0.f;
    if (e < A.dim)
        for (int p = share; p < A.parts; p += 16) sum += A.part[z][(int64_t)p * A.dim + e];
    joined[threadIdx.x] = sum;
    __syncthreads();
    if (share == 0 && e < A.dim) {
        for (int q = 1; q < 16; q++) sum += joined[q * 16 + column];
        A.out[z][e] = sum;
    }
}

}  // namespace pcr
