// Ragged uint8 pictures -> normalised patch rows and their positions.
//
// Row r of picture i holds a patch as [channel][y][x], (pixel / 255 - mean) inv_std, written as one multiply-add of the pixel with
// inv_std / 255 and -mean inv_std (its error, 2^-24 of each of the two, is far below the rounding to 16 bits and within three units of 32).
// Bound by memory: a pixel byte in, two or four bytes out.
#pragma once
#include "pcr_vec.h"

namespace pcr {

struct PatchArgs {
    const uint8_t* pixels; const int32_t* shape; const int64_t* offset; const int64_t* first;
    int64_t n, rows, pixel_bytes;
    int patch, merge, frames, channels;
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

template <typename T>
__global__ __launch_bounds__(256) void k_patch_rows(PatchArgs A) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= A.rows) return;
    const int lane = threadIdx.x & 63, P = A.patch, C = A.channels, m = A.merge, per = C * P * P;
    const int64_t i = picture_of(A, r);
    int H = 0, W = 0, row = 0, column = 0;
    int64_t begin = 0;
    bool mine = false;
    if (i >= 0) {
        H = A.shape[2 * i]; W = A.shape[2 * i + 1];
        begin = A.offset[i];
        if (H > 0 && W > 0) {
            const int64_t cell = (int64_t)P * m, place = r - A.first[i], across = (W + cell - 1) / cell, down = (H + cell - 1) / cell;
            const int64_t window = place / (m * m), inside = place % (m * m);
            if (window < across * down && begin >= 0) {
                mine = (int64_t)H * W * C <= A.pixel_bytes - begin;
                row = (int)(window / across * m + inside / m);
                column = (int)(window % across * m + inside % m);
            }
        }
    }
    if (A.positions && lane < 3) A.positions[lane * A.rows + r] = lane == 0 ? (mine ? (int32_t)(i % A.frames) : 0) : (mine ? (lane == 1 ? row : column) : 0);
    T* out = (T*)A.out + r * per;
    for (int f = lane; f < per; f += 64) {
        const int c = f / (P * P), y = f / P % P, x = f % P;
        const int64_t py = (int64_t)row * P + y, px = (int64_t)column * P + x;
        float v = 0.f;
        if (mine && py < H && px < W) v = __builtin_fmaf((float)A.pixels[begin + (py * W + px) * C + c], A.scale[c], A.shift[c]);
        out[f] = (T)v;
    }
}

}  // namespace pcr
