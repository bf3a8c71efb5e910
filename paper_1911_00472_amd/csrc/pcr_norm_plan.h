// How a call of group norm is divided: a host's program alone, compiled beside the kernels and by the tests.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/pcr.h"

namespace pcr {

constexpr int kNormThreads = 256;                                  // of two passes
constexpr int kNormTogether = 4;                                   // pixels of a thread whose loads are under way together
constexpr int kNormLong = 512;                                     // pixels that a thread adds up one after another, at most: in 32 bits its sums are off by 2^-16 of the magnitudes then
constexpr int kMergedChunks = 64;                                  // so many of a picture's chunks are joined by every workgroup that needs them

// What a call is made of.
struct NormPlan {
    int64_t chunk;                                                 // pixels of a workgroup
    int chunks, run;                                               // of a picture; channels that are loaded together
    int held, threads, block, blocks;                              // one pass: runs that a thread holds (0: two passes), threads and channels of a workgroup, workgroups of a picture
    int pack, turns;                                               // one pass: pictures of a workgroup side by side, and after one another
    bool many;                                                     // several pictures to a workgroup
    int64_t rows;                                                  // of channels' sums
    size_t part_bytes, sums_bytes, joined_bytes;
    size_t bytes() const { return part_bytes + sums_bytes + joined_bytes; }
    // LDS of a workgroup of one pass, in bytes; each: channels of a group.  (Forward: sums of 64 bits, and 16 bytes of a group.)
    size_t lds(int64_t each, bool back) const {
        const size_t groups = block / each, values = (size_t)threads * (each % run ? run : 1);
        return (back ? std::max(2 * values + pack * 2 * groups, (size_t)threads * run + block) : values * 2 + pack * 4 * groups) * sizeof(float);
    }
    // Whether the threads of a picture's part hold all of its pixels: lanes of a run of channels (rounded down), times what a thread holds.
    bool holds(int64_t pixels) const { return held && block && threads / pack / (block / run) * (int64_t)held >= pixels; }
};

inline bool multiple(const void* p, int64_t a, int64_t b, size_t size, int unit) { return ((uint64_t)(uintptr_t)p / size | (uint64_t)a | (uint64_t)b) % unit == 0; }

constexpr int64_t kSmallImages = 2048;                           // workgroups at least, where pictures share one

inline NormPlan plan_norm(const pcr_group_norm* N, bool back) {
    NormPlan P = {};
    const size_t size = N->dtype == PCR_FLOAT ? 4 : 2;
    // Runs of 16 bytes of channels, of two or of one.
    P.run = (int)(16 / size);
    for (; P.run > 1; P.run = P.run == 8 ? 2 : P.run >> 1) {
        if (N->channels % P.run) continue;
        if (multiple(N->x, N->x_image, N->x_pixel, size, P.run) && multiple(N->out, N->out_image, N->out_pixel, size, P.run) &&
            (!back || multiple(N->grad, N->grad_image, N->grad_pixel, size, P.run)))
            break;
    }
    const int64_t each = N->channels / N->groups;
    if (N->images && N->pixels) {
        // One pass: channels of whole groups and whole runs, 128 bytes of them where that many fit, fewer where there would be less than 256 workgroups.  A thread holds 16 runs at most (8 of
        // input and gradient each): with 32 there is one workgroup a compute unit, which loads, sums and stores one after another (64 pictures of 56 x 56 x 256 54 us and 48).
        const int64_t unit = each * P.run / std::__gcd(each, (int64_t)P.run), units = N->channels / unit;
        const int64_t target = 256, most = P.run * size < 16 ? 256 * 8 : 512 * (back ? 8 : 16);
        int64_t many = std::max<int64_t>(1, std::min<int64_t>((128 + unit * size - 1) / (unit * size), std::max<int64_t>(1, N->images * units / target)));
        const int64_t of_unit = N->pixels * (unit / P.run);
        while (many > 1 && of_unit * many > most) many >>= 1;
        many = std::min(many, units);
        // Many small pictures: where a picture has no more runs than a workgroup has threads (twice as many of fewer than 16 bytes), it has whole ones, side by side and after one another,
        // whose channels' sums are one row.  (us, with a picture or 128 bytes of its channels to a workgroup: 32768 of a pixel of 1024 channels 114, now 67, their gradient 440, 101;
        // 100000 of 2 x 2 x 32 324, 30, and 788, 46; 30000 of 3 x 3 x 108 285, 120, and 422, 178.)
        auto need = [&](int64_t threads, int64_t columns) { return (N->pixels + threads / columns - 1) / (threads / columns); };     // (lanes of a column are whole: 100 columns leave 56 threads of 256 without work)
        const bool whole = P.run * size == 16;
        const int64_t runs_held = whole ? 1 : 2;
        P.many = N->images >= kSmallImages && units * unit / P.run <= 256 && of_unit * units <= 256 * runs_held;
        if (P.many) many = units;
        const int64_t columns = many * unit / P.run;
        if (of_unit * many <= most && columns <= 256) {
            P.block = (int)(many * unit);
            P.blocks = (int)((units + many - 1) / many);
            P.threads = !whole || need(256, columns) <= 4 ? 256 : 512;
            // (512 runs of a picture are three of a thread where a pixel's runs do not divide the threads: 2 x 256 / 54 pixels of 54 runs on 4 lanes.)
            P.held = P.many ? (whole ? 1 : 3) : !whole ? 8 : P.threads == 256 ? 4 : back || need(512, columns) <= 8 ? 8 : 16;
            P.pack = 1;
            if (P.many)
                while (N->images >= 2 * P.pack * kSmallImages && 128 / P.pack >= columns && need(128 / P.pack, columns) <= runs_held) P.pack *= 2;
            if (!P.holds(N->pixels)) P.held = 0;
            P.turns = P.many ? (int)std::min<int64_t>(16, std::max<int64_t>(1, N->images / (P.pack * kSmallImages))) : 1;
            // Rows of 16 bytes of more than the caches hold.  (us in one pass / in two, runs of 8 channels and 4 of 32 bits: 64 pictures of 56 x 56 x 256 72 / 72 and their gradient 213 / 115;
            // 64 of 56 x 56 x 512 126 / 126 and 413 / 229; 96 of 60 x 60 x 192 88 / 88 and 272 / 171; 60 of 72 x 72 x 128 145 / 49 and 108 / 108; 32 bits, 64 of 56 x 56 x 128 68 / 68 and 138 / 110.)
            if (P.block < N->channels && P.block * (int64_t)size < 32 && N->images * N->pixels * N->channels * (int64_t)size > (64 << 20)) P.held = 0;
        }
    }
    if (P.held) {
        P.chunk = N->pixels;
        P.chunks = 1;
        P.rows = (N->images + P.pack * P.turns - 1) / (P.pack * P.turns);
        P.sums_bytes = back ? (size_t)P.rows * N->channels * 2 * sizeof(float) : 0;
        return P;
    }
    // Two passes.  Chunks of a picture's pixels: 768 workgroups in all, 512 of a gradient, of 16 pixels to a thread at least.  (us with 512 / 768 / 1024 / 2048: 64 pictures of
    // 112 x 112 x 64 59.8 / 57.9 / 59.3 / 64.6, gradient of 64 of 56 x 56 x 256 99 / 105 / 107 / 113, of 32 of 112 x 112 x 64 57 / 62 / 66 / 66.)
    const int64_t columns = std::min<int64_t>(N->channels / P.run, kNormThreads), lanes = kNormThreads / columns, step = kNormTogether * lanes;
    int64_t chunks = std::min<int64_t>(((back ? 512 : 768) + N->images - 1) / std::max<int64_t>(1, N->images), (N->pixels + 4 * step - 1) / (4 * step));
    chunks = std::max(std::max<int64_t>(1, chunks), std::min<int64_t>((N->pixels + kNormLong * lanes - 1) / (kNormLong * lanes), 1 << 30));
    P.chunk = ((N->pixels + chunks - 1) / chunks + step - 1) / step * step;
    P.chunks = N->pixels ? (int)((N->pixels + P.chunk - 1) / P.chunk) : 0;
    P.part_bytes = (size_t)N->images * P.chunks * N->groups * 2 * sizeof(float);
    P.rows = N->images * P.chunks;
    P.sums_bytes = back ? (size_t)P.rows * N->channels * 2 * sizeof(float) : 0;
    P.joined_bytes = back && P.chunks > kMergedChunks ? (size_t)N->images * N->groups * 2 * sizeof(float) : 0;
    return P;
}

}  // namespace pcr
