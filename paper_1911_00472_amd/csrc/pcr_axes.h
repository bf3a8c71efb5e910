// Positions of several axes turned into the heads of queries and keys, alone or behind a norm of every head, and the gradients.
//
// With pair (x, y) of a head at angle a = position[axis] * frequency:   x' = x cos a - y sin a,   y' = x sin a + y cos a;
// its gradient is the same with -a.  Behind a norm u = x r w, r = (mean x^2 + eps)^-1/2; with h the incoming gradient turned back,
//   dw = sum over tokens and heads of h x r,      dx = r (h w - x r^2 mean(h w x)).
//
// The angle is the 32-bit product of the position and the frequency, each a 32-bit float: what a program gets that multiplies a table of frequencies by
// positions as tensors, and what weights were trained with, 2^-24 of itself off (0.002 radians at position 32768 in the fastest pair).  From there on
// nothing is lost: the float is reduced to an eighth of a turn with a constant of 48 bits, or, from 2^20 on, in 64-bit fixed point.  (Fixed point for all
// of them and the compiler's sine and cosine took 511 us for 2 million tokens of one head of queries and keys, which share an angle between two rows;
// double precision and that 386, this 367, and 307 with what was gained elsewhere.)
//
// Bound by memory: every element is read once and written once.  A workgroup takes a few tokens: its lanes make the tokens' sines and cosines once,
// in LDS, for all heads of both sides; then a row (a head of a token) goes to a group of lanes, a lane holding one slot: a run of pairs, that is
// two runs of elements of up to 16 bytes, so that pairs meet in a lane whichever way they lie.  The sums of a norm go round the group.  The next row is loaded
// while one is worked on; a lane steps from row to row by adding (with a division a row, and 64-bit strides, there were 21 instructions an element, and 10 now).
// us (what the bytes take at the 5.0 TB/s of a large copy, which kernels that read more than they write can pass): inverse rotation of 65536 tokens of 40 heads
// of 128, bfloat 241 (269); rotation of 49999 tokens of 32 heads of 72 in neighbouring pairs, half 92 (92); norm and rotation of 8204 tokens of 16 heads of 96 in 32
// bits 19 (20); gradient of norm and rotation of 32768 tokens of 40 heads of 128, bfloat 209 + 5 for the sums (201).  One head of queries and keys alone is slower
// than a copy: 321 (262) for 2 million tokens of 80 and three axes, its gradient behind a norm 739 (393); there is an angle to make for every two rows.
#pragma once
#include "pcr_vec.h"

namespace pcr {

struct HeadSide {
    const void* in; const void* grad; void* out; const void* weight; float* part;    // part: [workgroup][dim] sums of the weight's gradient
    int64_t in_b, in_t, in_h, out_b, out_t, out_h, grad_b, grad_t, grad_h;
    int heads, step_tokens, step_heads;                        // a wavefront's step to its next rows, as tokens and heads
    uint32_t by_heads;                                         // 2^32 / heads, rounded up
};
struct AxesArgs {
    HeadSide side[2];
    const void* position; const float* frequency; const int32_t* axis;
    int64_t pos_a, pos_b, pos_t, tokens, shares, chunks;       // shares: chunks of a sequence
    int wide, axes, dim, pairs, inverse, weight_float;
    int apart;                                                 // the sides have workgroups of their own (blockIdx.y)
    int far;                                                   // a stride of tokens or heads is outside 32 bits
    int slots, per_wave;                                       // slots of a row; rows of a wavefront (64 / slots, at least 1)
    int chunk, table_tokens;                                   // tokens of a workgroup at a time; tokens whose angles it makes at a time (256 / pairs)
    float eps, inv_dim;
};

enum { kRotate = 0, kNorm = 1, kNormBack = 2 };
constexpr int kAxesTable = 4096;                               // pairs of sine and cosine that a workgroup keeps at most (32 KB)

// f radians (a number) as a fraction of a turn, in 64 bits behind the point: f's 24 bits times 1 / (2 pi) to 128 bits (from 2^87 on
// to the 64 of them that are behind the point once moved, of 192), moved by f's exponent and cut.
__device__ __forceinline__ uint64_t turns_of(float f) {
    const uint32_t bits = __float_as_uint(f), e = bits >> 23 & 255;
    const uint64_t m = (bits & 0x7fffff) | (e ? 0x800000 : 0);
    const unsigned __int128 low = (unsigned __int128)m * 0x7f09d5f47d4d3770ull;
    const unsigned __int128 high = (unsigned __int128)m * 0x28be60db9391054aull + (uint64_t)(low >> 64);      // m / (2 pi) = high 2^-64 + its 64 bits behind
    const int down = 214 - (int)(e ? e : 1);                   // 2^(e - 150) of the float, 2^-128 of the product, 2^64 of the result
    uint64_t v;
    if (down >= 64) v = down < 192 ? (uint64_t)(high >> (down - 64)) : 0;
    else if (down > 0) v = (uint64_t)(high << (64 - down)) | (uint64_t)low >> down;
    else v = m * (0x7f09d5f47d4d3770ull << -down | 0x36d8a5664f10e410ull >> 1 >> (63 + down));
    return bits >> 31 ? 0 - v : v;
}

// Cosine and sine of an angle, the sine's sign turned over for an inverse.  The angle becomes quarter turns and r, the rest as half-turns (-1/4 .. 1/4, and up
// to 0.28 near 2^20 radians, where the product that is rounded to quarters is off itself): the constant 1 / (2 pi) in two floats (2^-48 of it is missing, 2^-30
// turns at 2^20 radians), the products in fused operations, the rest off by 2^-27 turns; sin(pi r) / r and (cos(pi r) - 1) / r^2 are polynomials of third
// degree in r^2, fitted to least maximal error over -1/4 .. 1/4.  With their coefficients as the floats that they are the sine is off by 2.6e-8 and the cosine by
// 7e-9 there, by 7.3e-8 and 1.2e-8 at 0.28; in all 1.7e-7 at most over seven million angles below 2^20 (2^-22 is 2.4e-7).
__device__ __forceinline__ float2 turn_of(float angle, int inverse) {
    float rest, quarters;
    if (__builtin_expect(__builtin_fabsf(angle) < 1048576.f, 1)) {
        quarters = __builtin_rintf(angle * 0.63661974668502807617f);
        rest = __builtin_fmaf(angle, 6.4206382432985265e-9f, __builtin_fmaf(angle, 0.15915493667125701904f, -0.25f * quarters));
    } else {
        const uint64_t turns = turns_of(angle);
        quarters = (float)(uint32_t)((turns + (1ull << 61)) >> 62);
        rest = __builtin_fmaf((float)((int64_t)(turns - ((uint64_t)(uint32_t)quarters << 62)) >> 32), 2.3283064365386962891e-10f, angle - angle);      // 2^-32; NaN of what is no number
    }
    const float r = rest + rest, u = r * r;
    const float sine = r * __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(-0.5876994729042053f, u, 2.5496182441711426f), u, -5.167703151702881f), u, 3.141592502593994f);
    const float cosine = __builtin_fmaf(u, __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(0.2313908338546753f, u, -1.3350543975830078f), u, 4.0587077140808105f), u, -4.934802055358887f), 1.f);
    const uint32_t q = (uint32_t)(int32_t)quarters;
    const uint32_t s = __float_as_uint(q & 1 ? cosine : sine) ^ ((q & 2) << 30) ^ (inverse ? 0x80000000u : 0);
    const uint32_t c = __float_as_uint(q & 1 ? sine : cosine) ^ (((q + 1) & 2) << 30);
    return make_float2(__uint_as_float(c), __uint_as_float(s));
}

// Sum over a row's group of lanes (`slots` neighbouring ones from `head` on), the same bits in all of them.
__device__ __forceinline__ float group_sum(float v, int head, int member, int slots) {
    if ((slots & (slots - 1)) == 0) {                          // (the same for all lanes, as what follows)
        if (slots > 1) v += across<kNeighbour>(v);
        if (slots > 2) v += across<kPairOfFour>(v);
        if (slots > 4) v += across<kFourOfEight>(v);
        if (slots > 8) v += across<kEightOfSixteen>(v);
        if (slots > 16) v += __shfl_xor(v, 16);
        if (slots > 32) v += __shfl_xor(v, 32);
        return v;
    }
    int width = 1;
    while (width < slots) width <<= 1;
    for (int d = width >> 1; d; d >>= 1) {
        const float o = __shfl(v, head + member + d);
        if (member + d < slots) v += o;
    }
    return __shfl(v, head);
}

// v^-1/2, also of numbers that the instruction takes for 0.
__device__ __forceinline__ float inverse_root(float v) {
    const int up = v < 1.1754943508222875e-38f ? 32 : 0;       // 2^-126
    return __builtin_amdgcn_ldexpf(__builtin_amdgcn_rsqf(__builtin_amdgcn_ldexpf(v, up + up)), up);
}

template <typename T, int N> __device__ __forceinline__ void load_weight(const AxesArgs& A, const void* w, int at, float (&x)[N]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = 1.f;
    } else if (A.weight_float) load_run<float, N>((const float*)w + at, x);
    else load_run<T, N>((const T*)w + at, x);
}

// A lane's slot of a row as it lies in memory: two runs, which are one in memory where a pair's elements are neighbours.
template <typename T, int N, bool ADJ> struct Slot {
    typename Run<T, N>::Vec run[2];
    static constexpr bool kOne = ADJ && 2 * N * sizeof(T) <= 16;
    __device__ __forceinline__ void load(const T* row, int first, int second, int dim) {
        if constexpr (kOne && N > 1) {                         // (there always is a second run then)
            if (first < dim) {
                const typename Run<T, 2 * N>::Vec v = reinterpret_cast<const typename Run<T, 2 * N>::Loose*>(row + first)->v;
#pragma unroll
                for (int i = 0; i < N; i++) { run[0][i] = v[i]; run[1][i] = v[N + i]; }
            }
        } else {
            if (first < dim) run[0] = reinterpret_cast<const typename Run<T, N>::Loose*>(row + first)->v;
            if (second < dim) run[1] = reinterpret_cast<const typename Run<T, N>::Loose*>(row + second)->v;
        }
    }
    __device__ __forceinline__ void clear() { run[0] = run[1] = {}; }
    __device__ __forceinline__ void take(float (&x)[2 * N]) const {
#pragma unroll
        for (int i = 0; i < N; i++) {
            if constexpr (N == 1) { x[0] = (float)run[0]; x[1] = (float)run[1]; }
            else { x[i] = (float)run[0][i]; x[N + i] = (float)run[1][i]; }
        }
    }
    static __device__ __forceinline__ void store(T* row, int first, int second, int dim, const float (&x)[2 * N]) {
        if constexpr (kOne && N > 1) {
            if (first < dim) store_run<T, 2 * N>(row + first, x);
        } else {
            float v[N], u[N];
#pragma unroll
            for (int i = 0; i < N; i++) { v[i] = x[i]; u[i] = x[N + i]; }
            if (first < dim) store_run<T, N>(row + first, v);
            if (second < dim) store_run<T, N>(row + second, u);
        }
    }
};

__device__ __forceinline__ int64_t row_offset(int tl, int h, int64_t per_token, int64_t per_head, int far) {
    if (far) return tl * per_token + h * per_head;
    return (int64_t)tl * (int32_t)per_token + (int64_t)h * (int32_t)per_head;
}

// Turns the pairs of a lane's slots by the row's sines and cosines.
template <int N, bool ADJ, int K> __device__ __forceinline__ void turn(float (&y)[K][2 * N], const float2* turns, const AxesArgs& A, int member, bool on) {
#pragma unroll
    for (int j = 0; j < K; j++) {
        const int p = (member + 64 * j) * N;
        if (on && p < A.pairs) {
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int ia = ADJ ? 2 * i : i, ib = ADJ ? 2 * i + 1 : N + i;
                const float2 cs = turns[p + i];
                const float u = y[j][ia], v = y[j][ib];
                y[j][ia] = __builtin_fmaf(u, cs.x, -(v * cs.y));
                y[j][ib] = __builtin_fmaf(u, cs.y, v * cs.x);
            }
        }
    }
}

// T: elements; N: elements of a run; ADJ: a pair's elements are neighbours (a slot is two runs behind each other) or half the rotated part apart;
// K: slots of a lane (more than one where a row has more than 64).  Every slot is turned whole or not at all.
template <typename T, int N, bool ADJ, int MODE, int K>
__global__ __launch_bounds__(256) void k_axes(AxesArgs A) {
    extern __shared__ __attribute__((aligned(16))) float2 table[];
    __shared__ float joined[MODE == kNormBack ? 4 * 512 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, dim = A.dim;
    const int group = K > 1 ? 64 : A.slots, place = lane / group, head = place * group, member = lane - head;
    const bool works = place < A.per_wave;
    const int R = 2 * A.pairs;

    int first[K], second[K];                                   // where the lane's runs begin; dim: there is none
#pragma unroll
    for (int j = 0; j < K; j++) {
        const int s = member + 64 * j;
        if (ADJ) { first[j] = 2 * N * s; second[j] = first[j] + N; }
        else if (s * N < A.pairs) { first[j] = s * N; second[j] = A.pairs + s * N; }
        else { first[j] = R + 2 * (s * N - A.pairs); second[j] = first[j] + N; }
        if (s >= A.slots || first[j] >= dim) first[j] = dim;
        if (s >= A.slots || second[j] >= dim) second[j] = dim;
    }
    int mine = A.pairs, mine_token = 0;
    float frequency = 0.f;
    int64_t mine_position = 0;
    if (A.pairs) {
        mine_token = threadIdx.x / A.pairs;
        if (mine_token < A.table_tokens) {
            mine = threadIdx.x - mine_token * A.pairs;
            frequency = A.frequency[mine];
            mine_position = min(max(A.axis[mine], 0), A.axes - 1) * A.pos_a;
        }
    }

    // Few tokens: a workgroup takes one side.  A gradient takes one side after the other, so that the sums of one weight's gradient are held at a time.
    const int from = A.apart ? blockIdx.y : 0, to = A.apart ? from + 1 : 2;
#pragma unroll 1
    for (int side = from; side < (MODE == kNormBack ? to : from + 1); side++) {
        float dw[K][2 * N];
        if (MODE == kNormBack) {
            if (!A.side[side].heads && !A.side[side].part) continue;
#pragma unroll
            for (int j = 0; j < K; j++)
#pragma unroll
                for (int i = 0; i < 2 * N; i++) dw[j][i] = 0.f;
        }
        for (int64_t chunk = blockIdx.x; chunk < A.chunks; chunk += gridDim.x) {
            const int64_t b = A.shares == A.chunks ? 0 : chunk / A.shares, t0 = (chunk - b * A.shares) * A.chunk;
            const int here = (int)min((int64_t)A.chunk, A.tokens - t0);
            float w[K][2 * N];
            Slot<T, N, ADJ> X[K], G[K];
            int rows, r, tl, h;
            auto fetch = [&](const HeadSide& S) {
                if (works && r < rows) {
                    const T* row = (const T*)S.in + b * S.in_b + t0 * S.in_t + row_offset(tl, h, S.in_t, S.in_h, A.far);
                    const T* grow = (const T*)S.grad + b * S.grad_b + t0 * S.grad_t + row_offset(tl, h, S.grad_t, S.grad_h, A.far);
#pragma unroll
                    for (int j = 0; j < K; j++) {
                        X[j].load(row, first[j], second[j], dim);
                        if (MODE == kNormBack) G[j].load(grow, first[j], second[j], dim);
                    }
                }
            };
            // A side's weights and its first rows.  A wavefront's rows are per_wave ones side by side, then those 4 per_wave further on.
            auto begin = [&](const HeadSide& S) {
                rows = here * S.heads;
                r = wave * A.per_wave + place;
                tl = S.heads == 1 ? r : (int)__umulhi((uint32_t)r, S.by_heads);
                h = r - tl * S.heads;
#pragma unroll
                for (int j = 0; j < K; j++) { X[j].clear(); G[j].clear(); }
                fetch(S);
                if (MODE != kRotate && S.heads) {
#pragma unroll
                    for (int j = 0; j < K; j++) {
                        float x[N], y[N];
#pragma unroll
                        for (int i = 0; i < N; i++) x[i] = y[i] = 0.f;
                        if (first[j] < dim) load_weight<T, N>(A, S.weight, first[j], x);
                        if (second[j] < dim) load_weight<T, N>(A, S.weight, second[j], y);
#pragma unroll
                        for (int i = 0; i < N; i++) { w[j][i] = x[i]; w[j][N + i] = y[i]; }
                    }
                }
            };
            begin(A.side[side]);
            if (mine < A.pairs)                                    // a thread makes one pair's angles, of every few tokens
                for (int t = mine_token; t < here; t += A.table_tokens) {
                    const int64_t at = mine_position + b * A.pos_b + (t0 + t) * A.pos_t;
                    const float position = A.wide ? (float)((const int64_t*)A.position)[at] : (float)((const int32_t*)A.position)[at];
                    table[t * A.pairs + mine] = turn_of(position * frequency, A.inverse);
                }
            __syncthreads();
#pragma unroll 1
            for (int z = side; z < (MODE == kNormBack ? side + 1 : to); z++) {
                const HeadSide& S = A.side[z];
                if (z != side) begin(S);
                T* out = (T*)S.out + b * S.out_b + t0 * S.out_t;
                for (int r0 = wave * A.per_wave; r0 < rows; r0 += 4 * A.per_wave) {
                    const bool on = works && r < rows;
                    const float2* turns = table + tl * A.pairs;
                    T* orow = out + row_offset(tl, h, S.out_t, S.out_h, A.far);
                    float x[K][2 * N], g[K][2 * N];
#pragma unroll
                    for (int j = 0; j < K; j++) {
                        X[j].take(x[j]);
                        if (MODE == kNormBack) G[j].take(g[j]);
                    }
                    r += 4 * A.per_wave;
                    tl += S.step_tokens;
                    h += S.step_heads;
                    if (h >= S.heads) { h -= S.heads; tl++; }
                    fetch(S);                                      // (the next row is loaded before this one is done)
                    if (MODE != kRotate) {
                        float sum = 0.f;
#pragma unroll
                        for (int j = 0; j < K; j++)
#pragma unroll
                            for (int i = 0; i < 2 * N; i++) sum = __builtin_fmaf(x[j][i], x[j][i], sum);
                        sum = group_sum(sum, head, member, group);
                        const float rms = inverse_root(__builtin_fmaf(sum, A.inv_dim, A.eps));
#pragma unroll
                        for (int j = 0; j < K; j++)
#pragma unroll
                            for (int i = 0; i < 2 * N; i++) {
                                x[j][i] *= rms;
                                if (MODE == kNorm) x[j][i] *= w[j][i];
                            }
                        if (MODE == kNormBack) {
                            turn<N, ADJ, K>(g, turns, A, member, on);
                            float dot = 0.f;
#pragma unroll
                            for (int j = 0; j < K; j++)
#pragma unroll
                                for (int i = 0; i < 2 * N; i++) {
                                    if (on) dw[j][i] = __builtin_fmaf(g[j][i], x[j][i], dw[j][i]);
                                    g[j][i] *= w[j][i];
                                    dot = __builtin_fmaf(g[j][i], x[j][i], dot);
                                }
                            dot = group_sum(dot, head, member, group) * A.inv_dim;
#pragma unroll
                            for (int j = 0; j < K; j++)
#pragma unroll
                                for (int i = 0; i < 2 * N; i++) x[j][i] = rms * __builtin_fmaf(-x[j][i], dot, g[j][i]);
                        }
                    }
                    if (MODE != kNormBack) turn<N, ADJ, K>(x, turns, A, member, on);
                    if (on) {
#pragma unroll
                        for (int j = 0; j < K; j++) Slot<T, N, ADJ>::store(orow, first[j], second[j], dim, x[j]);
                    }
                }
            }
            __syncthreads();                                       // the table is made anew
        }

        // The weight's gradient: a lane's sums over its rows, then over the groups of a wavefront and the wavefronts in their order.
        if (MODE == kNormBack && A.side[side].part) {              // (the same for all)
            float* part = A.side[side].part;
#pragma unroll
            for (int j = 0; j < K; j++)
#pragma unroll
                for (int i = 0; i < 2 * N; i++) {
                    float v = works ? dw[j][i] : 0.f;
                    if (K == 1 && (group & (group - 1)) == 0) {
                        for (int d = group; d < 64; d <<= 1) v += __shfl_xor(v, d);
                    } else if (K == 1) {
                        float all = 0.f;
                        for (int q = 0; q < A.per_wave; q++) all += __shfl(v, q * group + member);
                        v = all;
                    }
                    const int at = i < N ? first[j] : second[j];
                    if (place == 0 && at < dim) joined[wave * 512 + at + (i < N ? i : i - N)] = v;
                }
            __syncthreads();
            for (int e = threadIdx.x; e < dim; e += 256)
                part[(int64_t)blockIdx.x * dim + e] = ((joined[e] + joined[512 + e]) + joined[1024 + e]) + joined[1536 + e];
            __syncthreads();
        }
    }
}

// Sums [parts][dim] over the parts: a workgroup takes 16 columns of one side, 64 threads to a column, in a fixed order.
struct WeightSums { const float* part[2]; float* out[2]; int parts, dim; };
__global__ __launch_bounds__(1024) void k_weight_sums(WeightSums A) {
    __shared__ float joined[1024];
    const int column = threadIdx.x & 15, share = threadIdx.x >> 4, z = blockIdx.y, e = blockIdx.x * 16 + column;
    if (!A.out[z]) return;
    float sum = 0.f;
    if (e < A.dim) {
#pragma unroll 8
        for (int p = share; p < A.parts; p += 64) sum += A.part[z][(int64_t)p * A.dim + e];
    }
    joined[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 256) {
        sum = (sum + joined[threadIdx.x + 256]) + (joined[threadIdx.x + 512] + joined[threadIdx.x + 768]);
        joined[threadIdx.x] = sum;
    }
    __syncthreads();
    if (share == 0 && e < A.dim) {
#pragma unroll
        for (int q = 1; q < 16; q++) sum += joined[q * 16 + column];
        A.out[z][e] = sum;
    }
}

}  // namespace pcr
