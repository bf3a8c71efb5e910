// The loss of a student's logits against a teacher's top logits, with the loss of labels beside it, and its gradient.
//
// A row: logits z over V classes, kept teacher logits t_k at classes i_k, temperature T; p = softmax of t / T over the entries that count.
//   L = logsumexp(z / T), L1 = logsumexp z;   loss = a T^2 sum p_k (log p_k - z_{i_k} / T + L) + b (L1 - z_label)
//   dz_v = g (a T P exp(z_v / T - L) + b exp(z_v - L1))  +  sum over entries at v of their delta,   P = 1 (0: no entry counts),
// with delta = -g a T p_k for a kept logit and -g b for the label: the dense part is written first and the few classes with a delta again
// behind it, every one with the deltas of all entries at its class, in their order.
//
// Sums over a row are made in 32 bits relative to its maximum.  Bound by memory: a row is read once for the loss, and read and written once for loss and
// gradient: a team of threads holds it in its registers, packed as it came, and makes its exponentials where they are used (k_distill_rows).  Rows too
// long for that are read with a running maximum and again for the gradient (k_distill), a few long ones in shares (k_distill_part, k_distill_join).
// us (what the bytes take at the 5.0 TB/s of a large copy): loss and gradient of 4096 rows of 50001 bfloat logits with labels, T = 2: 166 (164), read twice 323; of
// 2048 of 131071: 261 (215), 243 with T = 1; of 4096 of 32000: 106 (105); of 8192 of 10000: 73 (66); loss of 8192 rows of 50001: 182 (164), with a running maximum
// 262; gradient from saved sums of 4096 rows of 131072 half-precision logits: 423 (430).  Short rows are bound by the trips to memory of a wavefront that
// follow each other: 16384 rows of 300 classes with 10 entries take 13 for the loss (2), 16 for the gradient (4), 18 for both (4).
#pragma once
#include <type_traits>

#include "pcr_vec.h"

namespace pcr {

struct DistillArgs {
    const void* logits; const void* top_index; const void* top_logits; const int64_t* labels;
    const float* sums_in; const float* row_grad;              // backward: saved sums; step: row_grad holds the rows' weights
    float* loss; float* sums; void* out; float* part;
    int64_t row_stride, out_stride, rows, V;
    int64_t first;                                             // workgroups of launches before this one
    int64_t chunk; int chunks;                                 // classes of a workgroup's share of a row, shares of a row
    int K, top_dtype, wide, two;
    float T, inv_T, a, b;
};

constexpr float kLog2e = 1.4426950408889634074f;
enum { kLoss = 0, kGrad = 1, kStep = 2 };

template <int TEAM> __device__ __forceinline__ void team_sync() {
    if (TEAM > 64) __syncthreads();
    else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}
// Maximum and sum over a team, the same bits in all of it.  `lds`: a float for every wavefront of the team.
template <int TEAM, bool MAX> __device__ __forceinline__ float team_join(float v, float* lds) {
    v = wave_join<MAX>(v);
    if (TEAM == 64) return v;
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < TEAM / 64; w++) v = MAX ? fmaxf(v, lds[w]) : v + lds[w];
    return v;
}

__device__ __forceinline__ float top_logit(const DistillArgs& A, int64_t at) {
    if (A.top_dtype == 0) return ((const float*)A.top_logits)[at];
    if (A.top_dtype == 1) return (float)((const _Float16*)A.top_logits)[at];
    return (float)((const __bf16*)A.top_logits)[at];
}
// The class of an entry, -1 if it does not count.
__device__ __forceinline__ int64_t top_class(const DistillArgs& A, int64_t at) {
    const int64_t v = A.wide ? ((const int64_t*)A.top_index)[at] : (int64_t)((const int32_t*)A.top_index)[at];
    return v >= 0 && v < A.V ? v : -1;
}

// The kept entries of a row in LDS: class (-1: it does not count), the teacher's logit and later what the entry adds to its class's gradient, the
// student's logit.  (Differences are taken before they are divided by T: a mask's value over a T below 1 is infinite.)  `seen` and `several`: a bit for every class (for every 65536th, of more classes) that an entry, or several, have; only the latter look for
// each other.  (Every entry looking at every other took 143 us for 11145 rows of 344 classes with 256 entries.)
constexpr int64_t kEntryBits = 65536;
__host__ __device__ inline int entry_words(int64_t classes) { return (int)((classes < kEntryBits ? classes : kEntryBits) + 31) / 32; }
__host__ __device__ inline int entry_floats(int K, int64_t classes) { return 1 + 3 * K + 2 * entry_words(classes); }
struct Entries {
    int* labelled; int* at; float* delta; float* logit; uint32_t* seen; uint32_t* several;
    int words;
    __device__ __forceinline__ Entries(float* lds, int K, int64_t classes) {
        labelled = (int*)lds; at = labelled + 1; delta = lds + 1 + K; logit = delta + K;
        words = entry_words(classes);
        seen = (uint32_t*)(logit + K); several = seen + words;
    }
    template <int TEAM> __device__ __forceinline__ void clear(int tid) {
        for (int i = tid; i < 2 * words; i += TEAM) seen[i] = 0;
        if (tid == 0) *labelled = 0;
    }
    // Before a barrier of the team: class v (counted from the first one that the team writes) has this entry.
    __device__ __forceinline__ void mark(uint32_t v) {
        const uint32_t bit = v % (uint32_t)kEntryBits, mask = 1u << bit % 32;
        if (atomicOr(&seen[bit / 32], mask) & mask) atomicOr(&several[bit / 32], mask);
    }
    // Behind it: what all entries at the class of entry e add, if several are ...
    __device__ __forceinline__ float sum(int e, uint32_t v, int K) const {
        const uint32_t bit = v % (uint32_t)kEntryBits;
        return several[bit / 32] >> bit % 32 & 1 ? sum_of_all(e, K) : delta[e];
    }
    // ... and where no class is marked.
    __device__ __forceinline__ float sum_of_all(int e, int K) const {
        const int mine = at[e];
        float all = 0.f;
        for (int k = 0; k < K; k++) {
            const int v = at[k];
            const float d = delta[k];
            all += v == mine ? d : 0.f;
        }
        return all;
    }
};
// Reads a row's entries and returns the largest of the thread's logits.  A wavefront reads four of a lane's at a time; larger teams one, as their threads
// have one mostly and registers are short (with four 4096 rows of 50001 took 261 us, for 136 registers; 175).
template <typename T, int TEAM> __device__ __forceinline__ float load_entries(const DistillArgs& A, int64_t n, const T* z, const Entries& E, int tid) {
    constexpr int B = TEAM > 64 ? 1 : 4;
    float most = -INFINITY;
    for (int k0 = tid; k0 < A.K; k0 += B * TEAM) {
        int64_t v[B];
        float t[B], x[B];
#pragma unroll
        for (int j = 0; j < B; j++) {
            const int k = k0 + j * TEAM;
            v[j] = k < A.K && A.a != 0.f ? top_class(A, n * A.K + k) : -1;
            t[j] = k < A.K ? top_logit(A, n * A.K + k) : -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < B; j++) {
            if (v[j] < 0 || t[j] == -INFINITY) { v[j] = -1; t[j] = -INFINITY; }
            x[j] = v[j] >= 0 ? (float)z[v[j]] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < B; j++) {
            const int k = k0 + j * TEAM;
            if (k >= A.K) break;
            E.at[k] = (int)v[j];
            E.delta[k] = t[j];
            E.logit[k] = x[j];
            most = fmaxf(most, t[j] == t[j] ? t[j] : INFINITY);    // (of a NaN all that follows is one)
        }
    }
    return most;
}

// exp((x - m) / T) and exp(x - m) of a run, added to s and s1, with m raised first where the run holds more.
struct RowSums { float m, s, s1; };
template <int N, bool TWO> __device__ __forceinline__ void add_run(RowSums& R, const float (&x)[N], float c) {
    float most = x[0];
#pragma unroll
    for (int i = 1; i < N; i++) most = fmaxf(most, x[i]);
    if (most > R.m) {
        R.s *= __builtin_amdgcn_exp2f((R.m - most) * c);
        if (TWO) R.s1 *= __builtin_amdgcn_exp2f((R.m - most) * kLog2e);
        R.m = most;
    }
    const float m = R.m == -INFINITY ? 0.f : R.m;
#pragma unroll
    for (int i = 0; i < N; i++) {
        R.s += __builtin_amdgcn_exp2f((x[i] - m) * c);
        if (TWO) R.s1 += __builtin_amdgcn_exp2f((x[i] - m) * kLog2e);
    }
}

// Sums over z[0 .. count) by a team: elements in front of the first 16-byte boundary, whole runs (U of a thread's loaded together), the rest.
template <typename T, int TEAM, bool TWO, int U = 4> __device__ __forceinline__ RowSums row_sums(const T* z, int64_t count, float c, int tid) {
    constexpr int N = 16 / sizeof(T);
    RowSums R = {-INFINITY, 0.f, 0.f};
    const int64_t lead = min(count, (int64_t)((-(uintptr_t)z & 15) / sizeof(T)));
    const int64_t runs = (count - lead) / N, tail = lead + runs * N;
    if (tid < lead) { float x[1]; load_run<T, 1>(z + tid, x); add_run<1, TWO>(R, x, c); }
    if (tail + tid < count) { float x[1]; load_run<T, 1>(z + tail + tid, x); add_run<1, TWO>(R, x, c); }
    int64_t r = tid;
    for (; r + (U - 1) * TEAM < runs; r += U * TEAM) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; u++) load_run<T, N>(z + lead + (r + u * TEAM) * N, x[u]);
#pragma unroll
        for (int u = 0; u < U; u++) add_run<N, TWO>(R, x[u], c);
    }
    for (; r < runs; r += TEAM) {
        float x[N];
        load_run<T, N>(z + lead + r * N, x);
        add_run<N, TWO>(R, x, c);
    }
    return R;
}

__device__ __forceinline__ float scaled(float s, float m, float most, float c) { return m == -INFINITY ? 0.f : s * __builtin_amdgcn_exp2f((m - most) * c); }

// The dense part of the gradient of one element: against saved sums, or against the row's maximum (ca and cb are then divided by the sums).
template <bool TWO> struct BySaved {
    float inv_T, L, L1, ca, cb;
    __device__ __forceinline__ float operator()(float x) const {
        float v = ca * __builtin_amdgcn_exp2f(__builtin_fmaf(x, inv_T, -L) * kLog2e);
        if (TWO) v = __builtin_fmaf(cb, __builtin_amdgcn_exp2f((x - L1) * kLog2e), v);
        return v;
    }
};
template <bool TWO> struct ByMaximum {
    float c, m, ca, cb;
    __device__ __forceinline__ float operator()(float x) const {
        const float v = ca * __builtin_amdgcn_exp2f((x - m) * c);
        return TWO ? __builtin_fmaf(cb, __builtin_amdgcn_exp2f((x - m) * kLog2e), v) : v;
    }
};
template <typename T, int TEAM, int U = 4, typename D> __device__ __forceinline__ void write_dense(const T* z, T* out, int64_t count, const D& dense, int tid) {
    constexpr int N = 16 / sizeof(T);
    const int64_t lead = min(count, (int64_t)((-(uintptr_t)out & 15) / sizeof(T)));
    const int64_t runs = (count - lead) / N, tail = lead + runs * N;
    if (tid < lead) { float x[1]; load_run<T, 1>(z + tid, x); x[0] = dense(x[0]); store_run<T, 1>(out + tid, x); }
    if (tail + tid < count) { float x[1]; load_run<T, 1>(z + tail + tid, x); x[0] = dense(x[0]); store_run<T, 1>(out + tail + tid, x); }
    int64_t r = tid;
    for (; r + (U - 1) * TEAM < runs; r += U * TEAM) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; u++) load_run<T, N>(z + lead + (r + u * TEAM) * N, x[u]);
#pragma unroll
        for (int u = 0; u < U; u++) {
#pragma unroll
            for (int i = 0; i < N; i++) x[u][i] = dense(x[u][i]);
            store_run<T, N>(out + lead + (r + u * TEAM) * N, x[u]);
        }
    }
    for (; r < runs; r += TEAM) {
        float x[N];
        load_run<T, N>(z + lead + r * N, x);
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = dense(x[i]);
        store_run<T, N>(out + lead + r * N, x);
    }
}
template <typename T, int TEAM> __device__ __forceinline__ void write_zeros(T* out, int64_t count, int tid) {
    constexpr int N = 16 / sizeof(T);
    const int64_t lead = min(count, (int64_t)((-(uintptr_t)out & 15) / sizeof(T)));
    const int64_t runs = (count - lead) / N, tail = lead + runs * N;
    const float one[1] = {0.f}, none[N] = {};
    if (tid < lead) store_run<T, 1>(out + tid, one);
    if (tail + tid < count) store_run<T, 1>(out + tail + tid, one);
    for (int64_t r = tid; r < runs; r += TEAM) store_run<T, N>(out + lead + r * N, none);
}

// Saved sums that are too far from 0: from 128 on the two roundings in one come to more than 2^-17, and every element of the gradient is off by that part of
// itself; where a float holds nothing of the sum's logarithm beside the maximum, x / T less it is a rounding error of any size.  The maximum and the sums of
// such a row are made anew (write_anew).
__device__ __forceinline__ bool saved_too_far(float L) { return !(__builtin_fabsf(L) < 128.f); }
// Such a row's gradient, by one team: the row is read before any of it is written, which may be in its place.  The entries hold what they add.
template <typename T, int TEAM, bool TWO>
__device__ __forceinline__ void write_anew(const DistillArgs& A, const T* z, T* out, const Entries& E, float ca, float cb, int64_t label, float zl, float* join, int tid) {
    const float c = A.inv_T * kLog2e;
    const RowSums R = row_sums<T, TEAM, TWO, 1>(z, A.V, c, tid);           // (one run at a time: the kernel keeps its registers)
    const float m = team_join<TEAM, true>(R.m, join);
    const float s = team_join<TEAM, false>(scaled(R.s, R.m, m, c), join);
    const float s1 = TWO ? team_join<TEAM, false>(scaled(R.s1, R.m, m, kLog2e), join) : s;
    const ByMaximum<TWO> dense = {c, m, TWO ? ca / s : (ca + cb) / s, cb / s1};
    write_dense<T, TEAM, 1>(z, out, A.V, dense, tid);
    team_sync<TEAM>();
    for (int e = tid; e < A.K; e += TEAM) {
        const int64_t v = E.at[e];
        if (v >= 0) out[v] = (T)(dense(E.logit[e]) + (E.sum_of_all(e, A.K) - (v == label ? cb : 0.f)));
    }
    if (tid == 0 && label >= 0 && label < A.V && !*E.labelled) out[label] = (T)(dense(zl) - cb);
}

// A workgroup of TEAM threads takes a row, or one of the shares of a row (gradient alone).  MODE: the loss and the sums, the gradient from saved sums, or both.
template <typename T, int TEAM, bool TWO, int MODE>
__global__ __launch_bounds__(TEAM) void k_distill(DistillArgs A) {
    extern __shared__ float lds[];                             // joins [16], entries
    const int tid = threadIdx.x;
    const int64_t unit = A.first + blockIdx.x, n = unit / A.chunks;
    const int share = (int)(unit - n * A.chunks);
    const int64_t v0 = share * A.chunk, count = min(A.chunk, A.V - v0);
    float* join = lds;
    Entries E(join + 16, A.K, A.chunk);
    const T* z = (const T*)A.logits + n * A.row_stride;
    T* out = MODE == kLoss ? nullptr : (T*)A.out + n * A.out_stride + v0;
    const float g = MODE == kLoss ? 1.f : A.row_grad[n];

    if (MODE != kLoss && g == 0.f) {
        write_zeros<T, TEAM>(out, count, tid);
        if (MODE == kStep && tid == 0) A.loss[n] = 0.f;
        return;
    }
    if (MODE != kLoss) E.clear<TEAM>(tid);
    // entries: softmax of the teacher's logits over those that count
    float most = load_entries<T, TEAM>(A, n, z, E, tid);
    const int64_t label = A.labels && A.b != 0.f ? A.labels[n] : -1;
    const bool labelled = label >= 0 && label < A.V;
    const float zl = labelled ? (float)z[label] : 0.f;
    most = team_join<TEAM, true>(most, join);
    const float c = A.inv_T * kLog2e;
    float total = 0.f;
    for (int k = tid; k < A.K; k += TEAM) if (E.at[k] >= 0) total += __builtin_amdgcn_exp2f((E.delta[k] - most) * c);
    total = team_join<TEAM, false>(total, join);
    const bool kept = most != -INFINITY;

    if (MODE != kLoss && !kept && !labelled) {
        write_zeros<T, TEAM>(out, count, tid);
        if (MODE == kStep && tid == 0) A.loss[n] = 0.f;
        return;
    }
    // What the dense part is taken against: the saved sums, or (exact also where the logarithm is lost beside it) the maximum and the sums' reciprocals.
    float m = 0.f, s = 1.f, s1 = 1.f, saved = 0.f, saved1 = 0.f;
    if (MODE == kGrad) {
        saved = A.sums_in[2 * n]; saved1 = A.sums_in[2 * n + 1];
    } else {
        RowSums R = row_sums<T, TEAM, TWO>(z, A.V, c, tid);
        m = team_join<TEAM, true>(R.m, join);
        s = team_join<TEAM, false>(scaled(R.s, R.m, m, c), join);
        s1 = TWO ? team_join<TEAM, false>(scaled(R.s1, R.m, m, kLog2e), join) : s;
    }
    if (MODE != kGrad) {
        const float log_s = logf(s), log_s1 = TWO ? logf(s1) : log_s;
        float sum = 0.f;
        for (int k = tid; k < A.K; k += TEAM)
            if (E.at[k] >= 0) {
                const float t = (E.delta[k] - most) * A.inv_T, e = __builtin_amdgcn_exp2f((E.delta[k] - most) * c);
                if (e > 0.f || t != t) sum += e * ((t - logf(total)) - ((E.logit[k] - m) * A.inv_T - log_s));
            }
        sum = team_join<TEAM, false>(sum, join);
        if (tid == 0) {
            float loss = kept ? A.a * A.T * A.T * (sum / total) : 0.f;
            if (labelled) loss += A.b * (log_s1 - (zl - m));
            A.loss[n] = g * loss;
            if (MODE == kLoss) { A.sums[2 * n] = m * A.inv_T + log_s; A.sums[2 * n + 1] = A.two ? m + log_s1 : 0.f; }
        }
    }
    if (MODE == kLoss) return;
    team_sync<TEAM>();                                         // (the bits are cleared)
    for (int k = tid; k < A.K; k += TEAM) {
        const int64_t v = E.at[k];
        E.delta[k] = v >= 0 ? -g * A.a * A.T * (__builtin_amdgcn_exp2f((E.delta[k] - most) * c) / total) : 0.f;
        if (v >= v0 && v < v0 + count) E.mark((uint32_t)(v - v0));
        if (labelled && v == label) *E.labelled = 1;
    }
    const float ca = kept ? g * A.a * A.T : 0.f, cb = labelled ? g * A.b : 0.f;
    if (MODE == kGrad && (saved_too_far(saved) || (TWO && saved_too_far(saved1)))) {
        if (share == 0) write_anew<T, TEAM, TWO>(A, z, out, E, ca, cb, labelled ? label : -1, zl, join, tid);
        return;
    }
    typename std::conditional<MODE == kGrad, BySaved<TWO>, ByMaximum<TWO>>::type dense;
    if constexpr (MODE == kGrad) dense = {A.inv_T, saved, saved1, ca, cb};
    else dense = {c, m, ca / s, cb / s1};
    if (!TWO) dense.ca += dense.cb;
    write_dense<T, TEAM>(z + v0, out, count, dense, tid);
    team_sync<TEAM>();                                         // the dense part is written, the entries are marked
    for (int e = tid; e < A.K; e += TEAM) {
        const int64_t v = E.at[e];
        if (v < v0 || v >= v0 + count) continue;
        const float x[1] = {dense(E.logit[e]) + (E.sum(e, (uint32_t)(v - v0), A.K) - (v == label ? g * A.b : 0.f))};
        store_run<T, 1>(out + (v - v0), x);
    }
    if (tid == 0 && labelled && !*E.labelled && label >= v0 && label < v0 + count) {
        const float x[1] = {dense(zl) - g * A.b};
        store_run<T, 1>(out + (label - v0), x);
    }
}

// Several values at a time, with one barrier: `lds` holds C floats for every wavefront of the team and is used by no other join.
template <int TEAM, int C, bool MAX> __device__ __forceinline__ void team_join_all(float (&v)[C], float* lds) {
    constexpr int W = TEAM / 64;
#pragma unroll
    for (int i = 0; i < C; i++) v[i] = wave_join<MAX>(v[i]);
    if (W == 1) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < C; i++) lds[wave * C + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < C; i++) {
        float x = lds[lane % W * C + i];
        if (W > 1) x = both<MAX>(x, across<kNeighbour>(x));
        if (W > 2) x = both<MAX>(x, across<kPairOfFour>(x));
        if (W > 4) x = both<MAX>(x, across<kFourOfEight>(x));
        if (W > 8) x = both<MAX>(x, across<kEightOfSixteen>(x));
        v[i] = x;
    }
}

// exp((x - m) / T) and, where BY is not kOneSum, exp(x - m): by an exponential of its own, or as the second or fourth power of the first (T = 2, 4), which is
// twice or four times as far off, 2^-21 of itself.  (2048 rows of 131071 logits with labels: 261 us with T = 2, 278 with T = 4, 300 with T = 3; 8192 of 10000: 73, 74, 77.)
enum { kOneSum = 1, kTwoSums = 0, kSquare = 2, kFourth = 4 };
template <int BY> __device__ __forceinline__ void exps(float x, float m, float c, float T, float& e, float& e1) {
    const float y = (x - m) * c;
    e = __builtin_amdgcn_exp2f(y);
    if (BY == kTwoSums) e1 = __builtin_amdgcn_exp2f(y * T);
    if (BY == kSquare) e1 = e * e;
    if (BY == kFourth) e1 = (e * e) * (e * e);
}

// A run's elements, in a way that keeps the compiler from carrying what it made of them before (32 bits an element, their exponentials: twice to four times
// the registers) to this use.
template <typename T, typename V, int N> __device__ __forceinline__ void take_again(V& raw, float (&x)[N]) {
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    Words w = __builtin_bit_cast(Words, raw);
    asm volatile("" : "+v"(w));
    raw = __builtin_bit_cast(V, w);
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = (float)raw[i];
}

// Loss (MODE kLoss), loss and gradient (kStep) or the gradient from saved sums (kGrad) of rows that a team of TEAM threads holds in its registers, R runs of 16
// bytes a thread: read once, written once.
template <typename T, int TEAM, int R, int BY, int MODE>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_distill_rows(DistillArgs A) {
    extern __shared__ float lds[];                             // a team's: joins [6 a wavefront], entries
    constexpr int N = 16 / sizeof(T), W = TEAM / 64;
    typedef typename Run<T, N>::Vec Vec;
    const int tid = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const int64_t n = (A.first + blockIdx.x) * (TEAM < 256 ? 256 / TEAM : 1) + team;
    if (n >= A.rows) return;                                   // (a whole wavefront, or nobody of a workgroup that shares a row)
    float* join = lds + team * (6 * W + entry_floats(A.K, A.V));
    Entries E(join + 6 * W, A.K, A.V);
    const T* z = (const T*)A.logits + n * A.row_stride;
    constexpr bool WRITES = MODE != kLoss, SUMS = MODE != kGrad;
    T* out = WRITES ? (T*)A.out + n * A.out_stride : nullptr;
    const float g = WRITES ? A.row_grad[n] : 1.f, c = A.inv_T * kLog2e;
    auto left_out = [&]() {
        write_zeros<T, TEAM>(out, A.V, tid);
        if (SUMS && tid == 0) A.loss[n] = 0.f;
    };
    // A wavefront asks for its row before it knows whether it counts (a trip to memory less, of three); larger teams leave the row's bytes where they are.
    if (TEAM > 64 && WRITES && g == 0.f) return left_out();
    const int64_t label = A.labels && A.b != 0.f ? A.labels[n] : -1;
    const float saved = SUMS ? 0.f : A.sums_in[2 * n], saved1 = SUMS ? 0.f : A.sums_in[2 * n + 1];
    const int V = (int)A.V, lead = min(V, (int)((-(uintptr_t)z & 15) / sizeof(T))), runs = (V - lead) / N, tail = lead + runs * N;
    if (WRITES) E.clear<TEAM>(tid);
    Vec raw[R];
    Vec least;
#pragma unroll
    for (int i = 0; i < N; i++) least[i] = (T)-INFINITY;
    const T* body = z + lead;
#pragma unroll
    for (int u = 0; u < R; u++) raw[u] = tid + u * TEAM < runs ? reinterpret_cast<const Vec*>(body)[tid + u * TEAM] : least;
    const int edge = tid < lead ? tid : tail + tid - lead;     // the elements in front of and behind the runs: one of some threads
    const bool edged = edge < V;
    const float x_edge = edged ? (float)z[edge] : -INFINITY;
    if (TEAM == 64 && WRITES && g == 0.f) return left_out();

    float most[2] = {x_edge, load_entries<T, TEAM>(A, n, z, E, tid)};            // of the logits, of the kept teacher's logits
    const bool labelled = label >= 0 && label < A.V;
    const float zl = labelled ? (float)z[label] : 0.f;
    if (SUMS) {
#pragma unroll
        for (int u = 0; u < R; u++)
#pragma unroll
            for (int i = 0; i < N; i++) most[0] = fmaxf(most[0], (float)raw[u][i]);
    }
    team_join_all<TEAM, 2, true>(most, join);
    const float m = most[0];
    const bool kept = most[1] != -INFINITY;
    if (WRITES && !kept && !labelled) return left_out();
    float sum[3] = {0.f, 0.f, 0.f};                            // of exp((z - m) / T), of exp(z - m), of the teacher's
    auto add = [&](float x) {
        float e, e1 = 0.f;
        exps<BY>(x, m, c, A.T, e, e1);
        sum[0] += e;
        sum[1] += e1;
    };
    if (SUMS) {
#pragma unroll
        for (int u = 0; u < R; u++) {
            if (u * TEAM < runs) {                             // (the same for the team)
                float x[N];
                take_again<T>(raw[u], x);
#pragma unroll
                for (int i = 0; i < N; i++) add(x[i]);
            }
        }
        if (edged) add(x_edge);
    }
    for (int k = tid; k < A.K; k += TEAM) if (E.at[k] >= 0) sum[2] += __builtin_amdgcn_exp2f((E.delta[k] - most[1]) * c);
    team_join_all<TEAM, 3, false>(sum, join + 2 * W);
    if (BY == kOneSum) sum[1] = sum[0];
    const float total = sum[2], log_s = logf(sum[0]), log_s1 = logf(sum[1]), log_total = logf(total);
    const float unit = -g * A.a * A.T;
    const float ca = kept ? (SUMS ? -unit / sum[0] : -unit) : 0.f, cb = labelled ? (SUMS ? g * A.b / sum[1] : g * A.b) : 0.f;

    // entries: their share of the loss, and what each adds to the dense part of its class
    auto finish = [&](float entries) {                         // the row's loss, from the sum of the entries' shares
        float all = kept ? A.a * A.T * A.T * (entries / total) : 0.f;
        if (labelled) all += A.b * (log_s1 - (zl - m));
        A.loss[n] = g * all;
    };
    float loss[1] = {0.f};
    if (WRITES) team_sync<TEAM>();                             // (the bits are cleared)
    for (int k = tid; k < A.K; k += TEAM) {
        const int v = E.at[k];
        float d = 0.f;
        if (v >= 0) {
            const float t = (E.delta[k] - most[1]) * A.inv_T, e = __builtin_amdgcn_exp2f((E.delta[k] - most[1]) * c);
            if (SUMS && (e > 0.f || t != t)) loss[0] += e * ((t - log_total) - ((E.logit[k] - m) * A.inv_T - log_s));
            d = unit * (e / total);
            if (WRITES) E.mark((uint32_t)v);
            if (WRITES && labelled && v == label) *E.labelled = 1;
        }
        E.delta[k] = d;
    }
    if (MODE == kLoss) {
        team_join_all<TEAM, 1, false>(loss, join + 5 * W);
        if (tid == 0) {
            finish(loss[0]);
            A.sums[2 * n] = m * A.inv_T + log_s;
            A.sums[2 * n + 1] = A.two ? m + log_s1 : 0.f;
        }
        return;
    }
    constexpr bool TWO = BY != kOneSum;
    if (!SUMS && (saved_too_far(saved) || (TWO && saved_too_far(saved1))))
        return write_anew<T, TEAM, TWO>(A, z, out, E, ca, cb, labelled ? label : -1, zl, join, tid);
    const BySaved<TWO> by_saved = {A.inv_T, saved, saved1, TWO ? ca : ca + cb, cb};
    auto dense = [&](float x) {
        if (!SUMS) return by_saved(x);
        float e, e1 = 0.f;
        exps<BY>(x, m, c, A.T, e, e1);
        if (BY == kOneSum) return (ca + cb) * e;
        if (BY == kSquare) return e * __builtin_fmaf(cb, e, ca);
        return __builtin_fmaf(cb, e1, ca * e);
    };
    T* to = out + lead;
#pragma unroll
    for (int u = 0; u < R; u++)
        if (tid + u * TEAM < runs) {
            float x[N];
            take_again<T>(raw[u], x);
#pragma unroll
            for (int i = 0; i < N; i++) x[i] = dense(x[i]);
            store_run<T, N>(to + (tid + u * TEAM) * N, x);
        }
    if (edged) out[edge] = (T)dense(x_edge);
    team_join_all<TEAM, 1, false>(loss, join + 5 * W);         // (the dense part and the entries are behind this barrier, too)
    team_sync<TEAM>();
    if (SUMS && tid == 0) finish(loss[0]);
    for (int e = tid; e < A.K; e += TEAM) {
        const int v = E.at[e];
        if (v >= 0) out[v] = (T)(dense(E.logit[e]) + (E.sum(e, (uint32_t)v, A.K) - (v == label ? g * A.b : 0.f)));
    }
    if (tid == 0 && labelled && !*E.labelled) out[label] = (T)(dense(zl) - g * A.b);
}

// Few rows: shares of a row are summed by workgroups of their own and joined by k_distill_join, a wavefront to a row.
template <typename T, bool TWO>
__global__ __launch_bounds__(256) void k_distill_part(DistillArgs A) {
    __shared__ float join[16];
    const int64_t n = blockIdx.x / A.chunks;
    const int share = (int)(blockIdx.x - n * A.chunks);
    const int64_t v0 = share * A.chunk, count = min(A.chunk, A.V - v0);
    const float c = A.inv_T * kLog2e;
    RowSums R = row_sums<T, 256, TWO>((const T*)A.logits + n * A.row_stride + v0, count, c, threadIdx.x);
    const float m = team_join<256, true>(R.m, join);
    const float s = team_join<256, false>(scaled(R.s, R.m, m, c), join);
    const float s1 = TWO ? team_join<256, false>(scaled(R.s1, R.m, m, kLog2e), join) : 0.f;
    if (threadIdx.x == 0) {
        float* p = A.part + 3 * (int64_t)blockIdx.x;
        p[0] = m; p[1] = s; p[2] = s1;
    }
}

template <typename T, bool TWO>
__global__ __launch_bounds__(64) void k_distill_join(DistillArgs A) {
    const int64_t n = blockIdx.x;
    const int lane = threadIdx.x;
    const float c = A.inv_T * kLog2e;
    const T* z = (const T*)A.logits + n * A.row_stride;
    float m = -INFINITY, s = 0.f, s1 = 0.f;
    for (int j = lane; j < A.chunks; j += 64) m = fmaxf(m, A.part[3 * (n * A.chunks + j)]);
    m = team_join<64, true>(m, nullptr);
    for (int j = lane; j < A.chunks; j += 64) {
        const float* p = A.part + 3 * (n * A.chunks + j);
        s += scaled(p[1], p[0], m, c);
        if (TWO) s1 += scaled(p[2], p[0], m, kLog2e);
    }
    s = team_join<64, false>(s, nullptr);
    const float log_s = logf(s), log_s1 = TWO ? logf(team_join<64, false>(s1, nullptr)) : log_s;
    float most = -INFINITY, total = 0.f, sum = 0.f;
    for (int k = lane; k < A.K; k += 64) {
        const int64_t v = A.a != 0.f ? top_class(A, n * A.K + k) : -1;
        const float t = v >= 0 ? top_logit(A, n * A.K + k) : -INFINITY;
        most = fmaxf(most, t == t ? t : INFINITY);             // (of a NaN all that follows is one)
    }
    most = team_join<64, true>(most, nullptr);
    for (int k = lane; k < A.K; k += 64) {
        const int64_t v = A.a != 0.f ? top_class(A, n * A.K + k) : -1;
        const float d = v >= 0 ? top_logit(A, n * A.K + k) - most : -INFINITY, t = d * A.inv_T;
        if (v < 0 || d == -INFINITY) continue;
        const float e = __builtin_amdgcn_exp2f(d * c);
        total += e;
        if (e > 0.f || t != t) sum += e * (t - (((float)z[v] - m) * A.inv_T - log_s));
    }
    total = team_join<64, false>(total, nullptr);
    sum = team_join<64, false>(sum, nullptr);
    if (lane == 0) {
        const int64_t label = A.labels && A.b != 0.f ? A.labels[n] : -1;
        float loss = most != -INFINITY ? A.a * A.T * A.T * (sum / total - logf(total)) : 0.f;
        if (label >= 0 && label < A.V) loss += A.b * (log_s1 - ((float)z[label] - m));
        const float g = A.row_grad ? A.row_grad[n] : 1.f;
        A.loss[n] = g == 0.f ? 0.f : g * loss;
        A.sums[2 * n] = m * A.inv_T + log_s; A.sums[2 * n + 1] = A.two ? m + log_s1 : 0.f;
    }
}

}  // namespace pcr
