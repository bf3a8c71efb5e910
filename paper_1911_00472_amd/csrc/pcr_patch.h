// Ragged uint8 pictures -> normalised patch rows and their positions.
//
// Row r of picture i holds a patch as [channel][y][x], (pixel / 255 - mean) inv_std, written as one multiply-add of the pixel with
// inv_std / 255 and -mean inv_std (its error, 2^-24 of each of the two, is far below the rounding to 16 bits and within three units of 32).
// Bound by memory: a pixel byte in, two or four bytes out.  1024 photographs of 300 to 500 pixels a side, us (the bytes at the 5.0 TB/s of a large copy, which reads
// as much as it writes):
// patches of 14, bfloat 304, in windows of 2 x 2 319 (312), of 16 285 (305), of 8 300 (310), of 28 303; 512 of them in 32 bits, patches of 16 245 (253), of 14 247.
// An element a lane and loads of bytes took 1228 with patches of 14; eight pixels a lane with stores in pieces 504; one load of a lane under way at a time 340.
#pragma once
#include "pcr_vec.h"

namespace pcr {

constexpr int kPatchGroup = 64;                                // rows of a workgroup at most

struct PatchArgs {
    const uint8_t* pixels; const int32_t* shape; const int64_t* offset; const int64_t* first;
    int64_t n, rows, pixel_bytes;
    int64_t begin;                                             // workgroups of launches before this one
    int patch, merge, frames, group;
    uint32_t by_each, by_runs;                                 // 2^32 / (runs of a patch), 2^32 / (runs of a line of it), rounded up
    float scale[3], shift[3];
    void* out; int32_t* positions;
};

// The picture that row r belongs to: the last one whose first row is not behind r (64 places are asked at a time).  -1: none.
__device__ __forceinline__ int64_t picture_of(const PatchArgs& A, int64_t r) {
    const int lane = threadIdx.x & 63;
    int64_t low = 0, count = A.n;                             // first[low + j] for j < count may be the one; those before low are not behind r
    while (count > 0) {
        const int64_t step = (count + 63) / 64, at = lane * step;
        const bool before = at < count && A.first[low + at] <= r;
        const int k = __popcll(__ballot(before));             // (ascending: a run of ones)
        if (k == 0) break;
        low += (k - 1) * step;
        count = count - (k - 1) * step < step ? count - (k - 1) * step : step;
        if (step == 1) return low;
    }
    return -1;
}

// x / d for x d < 2^32, with the factor 2^32 / d rounded up (0: of d = 1).
__device__ __forceinline__ uint32_t quotient(uint32_t x, uint32_t factor) { return factor ? __umulhi(x, factor) : x; }

template <typename T> __device__ __forceinline__ void store_eight(T* out, const float (&v)[8]) {
    if constexpr (sizeof(T) == 2) store_run<T, 8>(out, v);
    else {
        const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
        store_run<T, 4>(out, a);
        store_run<T, 4>(out + 4, b);
    }
}

struct Patch { int64_t begin; int32_t row, column, H, W; };    // H = 0: a row of no picture

// The first n of eight values, element by element; n is the same for all of a patch's last runs.
template <typename T> __device__ __forceinline__ void store_some(T* out, const float (&v)[8], int n) {
#pragma unroll
    for (int i = 0; i < 8; i++) if (i < n) out[i] = (T)v[i];
}
// The same into LDS, two 16-bit elements at a time (n and the place are even).
template <typename T> __device__ __forceinline__ void stage_pairs(T* out, const float (&v)[8], int n) {
    typedef T Two __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 8; i += 2)
        if (i < n) {
            const Two two = {(T)v[i], (T)v[i + 1]};
            *reinterpret_cast<Two*>(out + i) = two;
        }
}

// A workgroup takes A.group rows that follow each other (of a line of patches mostly, so that the lines of memory that they share are read together);
// a lane takes eight pixels side by side of one line of a patch: a load of 8 C bytes at any address, a store of eight elements to each channel's part.
// STAGED: where lines do not consist of whole runs the stores would be in pieces of other sizes with gaps between them; they go to LDS then, and the
// workgroup's rows, which follow each other in memory, are written from there sixteen bytes a lane.
template <typename T, int C, bool STAGED>
__global__ __launch_bounds__(256) void k_patch_rows(PatchArgs A) {
    __shared__ Patch patches[kPatchGroup];
    extern __shared__ __attribute__((aligned(16))) uint8_t staged[];
    const int64_t r0 = (A.begin + blockIdx.x) * A.group;
    const int P = A.patch, m = A.merge, here = (int)min((int64_t)A.group, A.rows - r0);
    if (threadIdx.x < 64) {                                    // (a wavefront)
        int64_t i = picture_of(A, r0);
        if ((int)threadIdx.x < here) {
            const int64_t r = r0 + threadIdx.x;
            while (i + 1 < A.n && A.first[i + 1] <= r) i++;
            Patch p = {0, 0, 0, 0, 0};
            if (i >= 0) {
                const int H = A.shape[2 * i], W = A.shape[2 * i + 1];
                const int64_t begin = A.offset[i];
                if (H > 0 && W > 0 && begin >= 0 && (int64_t)H * W <= (A.pixel_bytes - begin) / C) {
                    const uint32_t cell = (uint32_t)(P * m), across = ((uint32_t)W + cell - 1) / cell, down = ((uint32_t)H + cell - 1) / cell;
                    const int64_t place = r - A.first[i];
                    if (place >= 0 && place < (int64_t)across * down * m * m) {
                        const int64_t window = place / (m * m);
                        const uint32_t inside = (uint32_t)(place - window * (m * m)), line = (uint32_t)(window / across);
                        p = {begin, (int)(line * m + inside / m), (int)((window - (int64_t)line * across) * m + inside % m), H, W};
                    }
                }
            }
            patches[threadIdx.x] = p;
            if (A.positions) {
                A.positions[r] = p.H ? (int32_t)(i % A.frames) : 0;
                A.positions[A.rows + r] = p.row;
                A.positions[2 * A.rows + r] = p.column;
            }
        }
    }
    __syncthreads();
    const uint32_t runs = (uint32_t)(P + 7) / 8, each = (uint32_t)P * runs, all = each * here;
    struct Item { uint32_t words[2 * C]; T* out; int n, there; };
    auto fetch = [&](uint32_t e, Item& I) {
        const uint32_t t = quotient(e, A.by_each), inside = e - t * each, y = quotient(inside, A.by_runs), x = (inside - y * runs) * 8;
        const Patch p = patches[t];
        const int64_t py = (int64_t)p.row * P + y, px = (int64_t)p.column * P + x;
        I.n = min(8, P - (int)x);
        I.there = py < p.H ? (int)max((int64_t)0, min((int64_t)I.n, p.W - px)) : 0;           // pixels that the picture has
        I.out = STAGED ? (T*)staged + (t * C * P + y) * P + x : (T*)A.out + ((r0 + t) * C * P + y) * P + x;
#pragma unroll
        for (int j = 0; j < 2 * C; j++) I.words[j] = 0;
        if (I.there) {
            const int64_t at = p.begin + (py * p.W + px) * C;
            if (at + 8 * C <= A.pixel_bytes) {
                struct __attribute__((packed, aligned(1))) Loose { uint32_t w[2 * C]; };
                const Loose v = *reinterpret_cast<const Loose*>(A.pixels + at);
#pragma unroll
                for (int j = 0; j < 2 * C; j++) I.words[j] = v.w[j];
            } else {                                           // the pixels' last bytes
#pragma unroll
                for (int j = 0; j < 8 * C; j++)
                    if (at + j < A.pixel_bytes) I.words[j / 4] |= (uint32_t)A.pixels[at + j] << 8 * (j % 4);
            }
        }
    };
    auto finish = [&](const Item& I) {
        T* out = I.out;
#pragma unroll
        for (int c = 0; c < C; c++) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int j = i * C + c;
                v[i] = i < I.there ? __builtin_fmaf((float)(I.words[j / 4] >> 8 * (j % 4) & 255), A.scale[c], A.shift[c]) : 0.f;
            }
            if (STAGED && sizeof(T) == 2 && P % 2 == 0) stage_pairs<T>(out, v, I.n);
            else if (!STAGED && I.n == 8) store_eight<T>(out, v);
            else store_some<T>(out, v, I.n);
            out += P * P;
        }
    };
    for (uint32_t e = threadIdx.x; e < all; e += 512) {        // two at a time: the loads of both are under way together
        Item I, J;
        fetch(e, I);
        const bool two = e + 256 < all;
        if (two) fetch(e + 256, J);
        finish(I);
        if (two) finish(J);
    }
    if (STAGED) {
        __syncthreads();
        typedef uint32_t Four __attribute__((ext_vector_type(4)));
        struct __attribute__((packed, aligned(2))) Loose { Four v; };
        const uint32_t bytes = (uint32_t)(here * C * P * P * sizeof(T)), whole = bytes / 16;
        uint8_t* to = (uint8_t*)A.out + r0 * C * P * P * (int64_t)sizeof(T);
        for (uint32_t e = threadIdx.x; e < whole; e += 256) reinterpret_cast<Loose*>(to)[e].v = reinterpret_cast<const Four*>(staged)[e];
        for (uint32_t e = whole * 16 / sizeof(T) + threadIdx.x; e < bytes / sizeof(T); e += 256) ((T*)to)[e] = ((const T*)staged)[e];
    }
}

}  // namespace pcr
