// Goes over calls of group norm and asks of every plan whether its workgroups and threads reach all pixels and channels of a picture.  Prints how many plans of each kind there were;
// a plan that does not reach everything is printed and ends the program with 1.
#include <stdio.h>

#include "../../paper_1911_00472_amd/csrc/pcr_norm_plan.h"

using namespace pcr;

static long counts[3];                                             // one pass, several pictures to a workgroup, two passes
static int bad;

static void look(int dtype, int64_t images, int64_t pixels, int64_t channels, int groups, int64_t pad, bool back) {
    pcr_group_norm n = {};
    n.dtype = n.weight_dtype = dtype;
    n.images = images; n.pixels = pixels; n.channels = channels; n.groups = groups;
    n.x_pixel = n.out_pixel = n.grad_pixel = channels + pad;
    n.x_image = n.out_image = n.grad_image = pixels * (channels + pad);
    const NormPlan P = plan_norm(&n, back);
    const int64_t size = dtype == PCR_FLOAT ? 4 : 2, each = channels / groups;
    bool ok = P.run >= 1 && P.run * size <= 16 && channels % P.run == 0 && n.x_pixel % P.run == 0;
    if (P.held) {
        counts[P.many]++;
        const int64_t columns = P.block / P.run, threads = P.threads / P.pack, lanes = columns ? threads / columns : 0;
        ok = ok && P.block % P.run == 0 && P.block % each == 0 && (int64_t)P.block * P.blocks >= channels && (int64_t)P.block * (P.blocks - 1) < channels;
        ok = ok && columns >= 1 && lanes >= 1 && lanes * P.held >= pixels && P.holds(pixels);
        ok = ok && P.threads == threads * P.pack && (threads & (threads - 1)) == 0 && P.rows * P.pack * P.turns >= images && (P.rows - 1) * P.pack * P.turns < images;
        ok = ok && (P.many ? P.blocks == 1 : P.pack == 1 && P.turns == 1);
        // what is launched: runs that a thread holds, and threads
        const bool whole = P.run * size == 16;
        ok = ok && (P.many ? P.threads == 256 && P.held == (whole ? 1 : 3) : P.threads == 256 ? P.held == (whole ? 4 : 8) : P.threads == 512 && whole && (P.held == 8 || (P.held == 16 && !back)));
        // what its kernels put into LDS
        const int64_t values = P.threads * (each % P.run == 0 ? 1 : P.run), of_block = P.block / each, lds = P.lds(each, back);
        ok = ok && lds >= (back ? 8 * (values + P.pack * of_block) : 8 * values + 16 * P.pack * of_block) && (!back || lds >= 4 * ((int64_t)P.threads * P.run + P.block)) && lds <= 160 * 1024;
    } else {
        counts[2]++;
        ok = ok && P.chunk >= 1 && P.chunks >= 1 && P.chunk * P.chunks >= pixels && P.chunk * (P.chunks - 1) < pixels && P.rows == images * P.chunks;
        ok = ok && P.part_bytes == (size_t)(images * P.chunks * groups * 8);
        // what a thread adds up one after another: the chunk's pixels over the lanes of a column
        ok = ok && P.chunk <= 512 * (256 / std::min<int64_t>(channels / P.run, 256));
    }
    ok = ok && P.sums_bytes == (back ? (size_t)P.rows * channels * 8 : 0);
    if (!ok && bad++ < 20)
        printf("lost: dtype %d, %lld images of %lld pixels, %lld channels (+ %lld) in %d groups, %s: runs of %d, %d held by %d threads, %d channels of a workgroup, %d side by side\n", dtype, (long long)images,
               (long long)pixels, (long long)channels, (long long)pad, groups, back ? "gradient" : "forward", P.run, P.held, P.threads, P.block, P.pack);
}

int main() {
    const int64_t images[] = {1, 7, 300, 2047, 2048, 4096, 10000, 100000};
    const int64_t wide[] = {1, 2, 3, 5, 6, 8, 9, 12, 16, 23, 31, 33, 49, 64, 85, 100, 128, 196, 256, 300, 511, 700, 1024, 3136, 12544, 50000, 3000000};
    for (int dtype = 0; dtype < 3; dtype++)
        for (int back = 0; back < 2; back++)
            for (int64_t n : images) {
                for (int64_t c = 1; c <= 620; c++)                 // every number of channels and of few pixels
                    for (int64_t p = 1; p <= 140; p += p < 48 ? 1 : 7)
                        for (int g : {1, 2, 3, 8, 32})
                            if (c % g == 0) look(dtype, n, p, c, g, 0, back);
                for (int64_t c = 1; c <= 16384; c += 1 + c / 9)    // wide ranges of both, with channels beside them that are not read
                    for (int64_t p : wide)
                        for (int64_t pad = 0; pad <= 4; pad += 1 + pad)
                            for (int g = 1; g <= 4096; g = 2 * g + (g == 1))
                                if (c % g == 0) look(dtype, n, p, c, g, pad, back);
            }
    printf("%ld %ld %ld\n", counts[0], counts[1], counts[2]);
    return bad != 0;
}
