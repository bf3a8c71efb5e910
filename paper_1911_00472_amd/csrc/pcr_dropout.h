// Dropout with random numbers from counters, onto a residual: out = residual + (kept ? x / (1 - p) : 0).
//
// Element e of the rows (in the order of their indexes, wherever they lie) takes word e mod 4 of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as
// 1, 2, 3, 2011) for the key `seed` and the counter (e / 4, call, step), and is dropped where that word is below p 2^32.  So nothing has to be stored for
// the gradient, which is the same with the incoming gradient as x, and the key and the step are read on the device: a captured graph whose step is counted up in it
// drops other elements at every replay.
#pragma once
#include "pcr_vec.h"

namespace pcr {

struct DropArgs {
    const void* x; const void* residual; void* out; const int64_t* seed; int64_t* used;
    int64_t count, dim, x_row, residual_row, out_row, begin;       // count: rows * dim; begin: runs of earlier launches
    uint64_t by_dim;                                               // 2^64 / dim, rounded up; 0: divide
    uint32_t below, call;                                          // dropped below this word
    float scale;
};

__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int round = 0; round < 10; round++) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

constexpr int kDropRun = 8;                                        // elements of a thread: two counters

// Bound by memory: ten rounds are 40 products of 32 bits for four elements, which the loads of other wavefronts hide (268 MB 88.2 us with them, 88.4 without).  A thread's loads are under way
// while it makes its words.  us: 33.5 million elements of bfloat onto 32 bits 55 (336 MB, 6.1 TB/s), the gradient of 24.6 million of half 18 (98 MB, 5.4 TB/s).
// T: of x; U: of the residual and the result; FLAT: rows lie behind each other in all three.
template <typename T, typename U, bool FLAT> __global__ __launch_bounds__(256) void k_dropout(DropArgs A) {
    const int64_t run = A.begin + (int64_t)blockIdx.x * 256 + threadIdx.x, e = run * kDropRun;
    const uint64_t key = (uint64_t)A.seed[0], step = (uint64_t)A.seed[1];
    if (A.used && run == 0) {
        A.used[0] = (int64_t)key;
        A.used[1] = (int64_t)step;
    }
    if (e >= A.count) return;
    const int here = (int)min((int64_t)kDropRun, A.count - e);
    int64_t row = 0, column = e;
    if (!FLAT) {
        row = A.by_dim ? (int64_t)__umul64hi((uint64_t)e, A.by_dim) : e / A.dim;
        column = e - row * A.dim;
    }
    const T* x = (const T*)A.x + row * A.x_row + column;
    const U* residual = A.residual ? (const U*)A.residual + row * A.residual_row + column : nullptr;
    U* out = (U*)A.out + row * A.out_row + column;
    const bool whole = here == kDropRun && (FLAT || column + kDropRun <= A.dim);
    float v[kDropRun], r[kDropRun];
    if (whole) {
        load_run<T, kDropRun>(x, v);
        if (residual) load_run<U, kDropRun>(residual, r);
    }
    uint32_t word[kDropRun];
#pragma unroll
    for (int half = 0; half < 2; half++) {
        const uint64_t at = (uint64_t)run * 2 + half;
        const uint4 w = philox(make_uint4((uint32_t)at, (uint32_t)(at >> 32) | A.call << 16, (uint32_t)step, (uint32_t)(step >> 32)), (uint32_t)key, (uint32_t)(key >> 32));
        word[4 * half] = w.x; word[4 * half + 1] = w.y; word[4 * half + 2] = w.z; word[4 * half + 3] = w.w;
    }
    auto result = [&](float value, uint32_t w, float beside) {     // (a dropped element is 0 whatever it holds)
        const float y = w >= A.below && A.scale != 0.f ? value * A.scale : 0.f;
        return A.residual ? y + beside : y;
    };
    if (whole) {
#pragma unroll
        for (int i = 0; i < kDropRun; i++) v[i] = result(v[i], word[i], r[i]);
        store_run<U, kDropRun>(out, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kDropRun; i++) {
        if (i < here) {
            *out = (U)result((float)*x, word[i], residual ? (float)*residual : 0.f);
            if (FLAT || ++column < A.dim) { x++; out++; if (residual) residual++; }
            else {                                                 // (the next row)
                column = 0;
                row++;
                x = (const T*)A.x + row * A.x_row;
                out = (U*)A.out + row * A.out_row;
                if (residual) residual = (const U*)A.residual + row * A.residual_row;
            }
        }
    }
}

}  // namespace pcr
