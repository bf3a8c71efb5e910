// C ABI of the operators behind the decode (see include/pcr.h), patch rows and positions in queries and keys: checks of arguments, choice of a kernel,
// launches.  (Distillation: pcr_distill.hip.)
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "../../include/pcr.h"
#include "pcr_axes.h"
#include "pcr_host.h"
#include "pcr_patch.h"

using namespace pcr;

namespace {

// ---- rotation ----

// Whether every place of a side is a multiple of `unit` elements.
bool aligned(const void* p, int64_t b, int64_t t, int64_t h, size_t size, int unit) {
    return ((uint64_t)(uintptr_t)p / size | (uint64_t)b | (uint64_t)t | (uint64_t)h) % unit == 0;
}
bool within_32(int64_t stride) { return stride >= INT32_MIN && stride <= INT32_MAX; }

int check_rotation(const pcr_heads* q, const pcr_heads* k, const pcr_rotation* R, int dtype, bool back) {
    if (!q || !k || !R || !known_type(dtype)) return PCR_E_ARG;
    if (R->dim < 1 || R->dim > 512 || R->pairs < 0 || R->pairs > R->dim / 2 || R->axes < 1 || R->axes > 4) return PCR_E_RANGE;
    if (R->batch < 0 || R->tokens < 0 || R->tokens > kMaxGrid || R->batch > kMaxGrid) return PCR_E_RANGE;
    const pcr_heads* side[2] = {q, k};
    for (const pcr_heads* s : side) {
        if (s->heads < 0 || s->heads > 65536) return PCR_E_RANGE;
        if (s->heads && R->batch && R->tokens && (!s->in || !s->out || (back && !s->grad))) return PCR_E_ARG;
    }
    if (R->pairs && R->batch && R->tokens && (!R->position || !R->frequency || !R->axis)) return PCR_E_ARG;
    return PCR_OK;
}

template <typename T, int N, bool ADJ, int MODE> void launch_axes(const AxesArgs& A, int groups, hipStream_t s) {
    if constexpr (N <= 2) {
        if (A.slots > 64) {
            hipLaunchKernelGGL((k_axes<T, N, ADJ, MODE, 4>), dim3(groups, A.apart ? 2 : 1), dim3(256), (size_t)A.chunk * A.pairs * sizeof(float2), s, A);
            return;
        }
    }
    hipLaunchKernelGGL((k_axes<T, N, ADJ, MODE, 1>), dim3(groups, A.apart ? 2 : 1), dim3(256), (size_t)A.chunk * A.pairs * sizeof(float2), s, A);
}

constexpr int kBackGroups = 1024;                              // workgroups of a gradient: each leaves one sum of the weights' gradient a side

int run_axes(int device, const pcr_heads* q, const pcr_heads* k, const pcr_rotation* R, float eps, int inverse, int dtype, int weight_dtype, int mode,
             void* d_work, size_t work_bytes, hipStream_t s) {
    int rc = check_rotation(q, k, R, dtype, mode == kNormBack);
    if (rc) return rc;
    if (mode != kRotate && !known_type(weight_dtype)) return PCR_E_ARG;
    if (mode != kRotate && weight_dtype != PCR_FLOAT && weight_dtype != dtype) return PCR_E_ARG;
    if (mode != kRotate && !(eps >= 0.f && isfinite(eps))) return PCR_E_RANGE;
    const pcr_heads* side[2] = {q, k};
    const bool sums = mode == kNormBack && (q->weight_grad || k->weight_grad);
    AxesArgs A = {};
    if (R->batch * R->tokens > kMaxGrid) return PCR_E_RANGE;
    const size_t size = type_size(dtype);
    const bool back = mode == kNormBack;
    int64_t batch = R->batch, tokens = R->tokens;
    A.pos_a = R->axis_stride; A.pos_b = R->batch_stride; A.pos_t = R->token_stride;
    // Sequences whose tokens follow each other at one stride everywhere (always, if they are of one token) are one long sequence.
    bool one = tokens == 1 || A.pos_b == tokens * A.pos_t;
    for (const pcr_heads* H : side)
        if (H->heads && tokens != 1)
            one = one && H->in_batch == tokens * H->in_token && H->out_batch == tokens * H->out_token && (!back || H->grad_batch == tokens * H->grad_token);
    one = one && batch > 1;
    const bool single = one && tokens == 1;                    // the step from token to token is that from sequence to sequence
    if (single) A.pos_t = A.pos_b;
    if (one) { tokens *= batch; batch = 1; }
    for (int z = 0; z < 2; z++) {
        const pcr_heads& H = *side[z];
        HeadSide& S = A.side[z];
        S.in = H.in; S.grad = H.grad; S.out = H.out; S.weight = H.weight; S.heads = (int)H.heads;
        S.in_b = H.in_batch; S.in_t = single ? H.in_batch : H.in_token; S.in_h = H.in_head;
        S.out_b = H.out_batch; S.out_t = single ? H.out_batch : H.out_token; S.out_h = H.out_head;
        S.grad_b = H.grad_batch; S.grad_t = single ? H.grad_batch : H.grad_token; S.grad_h = H.grad_head;
        if (!S.heads) continue;
        if (batch == 1) S.in_b = S.out_b = S.grad_b = 0;       // (steps that are never taken neither move nor misalign anything)
        if (tokens == 1) S.in_t = S.out_t = S.grad_t = 0;
        if (S.heads == 1) S.in_h = S.out_h = S.grad_h = 0;
        A.far |= !within_32(S.in_t) || !within_32(S.in_h) || !within_32(S.out_t) || !within_32(S.out_h) || (back && (!within_32(S.grad_t) || !within_32(S.grad_h)));
    }
    // Runs of up to 16 bytes, as long as heads, pairs and alignment are multiples of them (of two, where those are one in memory).  A gradient's are of
    // four elements at most: with eight it has 140 registers, three wavefronts a SIMD (32768 tokens of 40 heads of 128, bfloat: 224 us, and 217).
    int N = back ? 4 : (int)(16 / size);
    for (; N > 1; N >>= 1) {
        bool fits = R->pairs % N == 0 && R->dim % (R->adjacent ? 2 * N : N) == 0;
        const int unit = R->adjacent ? std::min<int>(2 * N, (int)(16 / size)) : N;
        for (int z = 0; z < 2 && fits; z++) {
            const HeadSide& S = A.side[z];
            if (!S.heads) continue;
            fits = aligned(S.in, S.in_b, S.in_t, S.in_h, size, unit) && aligned(S.out, S.out_b, S.out_t, S.out_h, size, unit) &&
                   (!back || aligned(S.grad, S.grad_b, S.grad_t, S.grad_h, size, unit));
        }
        if (fits) break;
    }
    A.position = R->position; A.frequency = R->frequency; A.axis = R->axis;
    A.tokens = tokens; A.wide = R->wide; A.axes = R->axes; A.dim = R->dim; A.pairs = R->pairs;
    A.inverse = inverse; A.weight_float = weight_dtype == PCR_FLOAT; A.eps = eps; A.inv_dim = 1.f / R->dim;
    const int turned = 2 * R->pairs;
    A.slots = R->adjacent ? (R->dim + 2 * N - 1) / (2 * N) : R->pairs / N + (R->dim - turned + 2 * N - 1) / (2 * N);
    A.per_wave = std::max(1, 64 / A.slots);
    for (HeadSide& S : A.side) {
        if (!S.heads) continue;
        S.step_tokens = 4 * A.per_wave / S.heads; S.step_heads = 4 * A.per_wave % S.heads;
        S.by_heads = (uint32_t)(((1ull << 32) + S.heads - 1) / S.heads);
    }
    // Tokens of a workgroup at a time: rows of some 32 KB, 128 at least, as many as the table of sines holds, and as many as come to 1024 workgroups, which
    // fit side by side (2909 tokens of 26 heads, norm and rotation: 15.6 us with some more than that, 12.4).  (us with 64 / 128 / 256 / 512 rows: rows of 256
    // bytes 263 / 241 / 251 / 259, of 128 bytes 188 / 143 / 121 / 114.)  A gradient has 1024 workgroups at most, which leave sums: fewer of rows of 32 KB, down
    // to 128, where there are few tokens (us with rows of 16 / 32 / 64 KB: 3552 tokens of 19 heads of 64 19.0 / 18.7 / 23.9, 3160 of 18 of 128 22.6 / 18.3 / 19.5).
    const int64_t heads = std::max<int64_t>(1, q->heads + k->heads), all = batch * tokens;
    const int64_t row = (int64_t)(R->dim * size);
    const int64_t few = std::max<int64_t>(1, std::min<int64_t>(32768 / (row * heads), (all + 127) / 128));
    int64_t chunk = back ? std::max<int64_t>(few, (all + kBackGroups - 1) / kBackGroups) : std::min<int64_t>(std::max<int64_t>(128, 32768 / row) / heads, (all + 1023) / 1024);
    if (R->pairs) {
        // 32 KB of sines in gradients, and where 1024 workgroups come to it; 16 otherwise.  (Few heads: gradient of 2045759 tokens of one head of queries and keys 751
        // us with 32, 875 with 16, norm and rotation of 41828 tokens 16.1 and 18.9; rotation of 2 million, whose workgroups come and go, 396 and 357.)
        const bool all_at_once = back || (all + 1023) / 1024 * R->pairs <= kAxesTable;
        const int64_t most = (all_at_once ? kAxesTable : kAxesTable / 2) / R->pairs;
        if (chunk > most) {                                    // ... in whole steps of its wavefronts through the queries' rows (the last one 307 instead of 357)
            const int64_t step = 4 * A.per_wave, h = std::max<int64_t>(1, q->heads);
            chunk = most * h > step ? std::max<int64_t>(1, most * h / step * step / h) : most;
        }
    }
    chunk = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(chunk, 4096), tokens));
    A.chunk = (int)chunk;
    A.table_tokens = R->pairs ? 256 / R->pairs : 0;
    A.shares = tokens ? (tokens + chunk - 1) / chunk : 0;
    A.chunks = batch * A.shares;
    if (!A.shares) A.shares = 1;
    int groups = (int)std::min<int64_t>(A.chunks, back ? kBackGroups : groups_of_a_launch(256));
    // (us, one after the other / apart: norm and rotation of 256 tokens of 40 heads 6.7 / 6.2, of 1000 9.2 / 10.5; gradient of 64 tokens of 40 heads 14.4 / 10.4,
    // of 5006 of 31 of 64, 626 workgroups, 25.2 / 20.8, of 3000 of 56, 1000 workgroups, 37.2 / 38.3)
    A.apart = q->heads && k->heads && groups <= (back ? 768 : 512);
    if (sums) {
        size_t need = 0;
        pcr_norm_rotate_workspace(all, R->dim, &need);
        if (all && (!d_work || work_bytes < need)) return d_work ? PCR_E_RANGE : PCR_E_ARG;
        for (int z = 0; z < 2; z++) if (side[z]->weight_grad) A.side[z].part = (float*)d_work + (size_t)z * groups * R->dim;
    }
    const OnDevice on(device);
    if (!on.ok) return PCR_E_DEVICE;
    if (q->heads + k->heads == 0) groups = 0;
    if (groups) {
        with_type(dtype, [&](auto t) {
            typedef decltype(t) T;
            auto by_mode = [&](auto n, auto adj) {
                constexpr int M = decltype(n)::value;
                constexpr bool ADJ = decltype(adj)::value;
                if (mode == kRotate) launch_axes<T, M, ADJ, kRotate>(A, groups, s);
                else if (mode == kNorm) launch_axes<T, M, ADJ, kNorm>(A, groups, s);
                else if constexpr (M <= 4) launch_axes<T, M, ADJ, kNormBack>(A, groups, s);
            };
            auto by_pairs = [&](auto n) {
                if (R->adjacent) by_mode(n, std::true_type());
                else by_mode(n, std::false_type());
            };
            if (N == 8) { if constexpr (sizeof(T) == 2) by_pairs(std::integral_constant<int, 8>()); }
            else if (N == 4) by_pairs(std::integral_constant<int, 4>());
            else if (N == 2) by_pairs(std::integral_constant<int, 2>());
            else by_pairs(std::integral_constant<int, 1>());
        });
    }
    if (sums) {
        WeightSums W = {};
        for (int z = 0; z < 2; z++) { W.part[z] = A.side[z].part; W.out[z] = side[z]->weight_grad; }
        W.parts = groups; W.dim = R->dim;
        hipLaunchKernelGGL(k_weight_sums, dim3((R->dim + 15) / 16, 2), dim3(1024), 0, s, W);
    }
    return launched();
}

}  // namespace

extern "C" {

int pcr_patch_rows(int device_id, const uint8_t* d_pixels, size_t pixel_bytes, const int32_t* d_shape, const int64_t* d_offset, const int64_t* d_first, int64_t n,
                   int64_t rows, int patch, int merge, int frames, int channels, const float* mean, const float* inv_std, int dtype,
                   void* d_out, int32_t* d_positions, void* hip_stream) {
    if (!mean || !inv_std || !known_type(dtype)) return PCR_E_ARG;
    if (n < 0 || rows < 0 || patch < 1 || patch > 128 || merge < 1 || merge > 16 || frames < 1 || (channels != 1 && channels != 3)) return PCR_E_RANGE;
    if (rows > 4 * kMaxGrid) return PCR_E_RANGE;
    if (!d_offset || !d_first || (rows && !d_out) || (rows && n && (!d_pixels || !d_shape))) return PCR_E_ARG;
    if (!rows) return PCR_OK;
    PatchArgs A = {};
    A.pixels = d_pixels; A.shape = d_shape; A.offset = d_offset; A.first = d_first; A.n = n; A.rows = rows;
    A.pixel_bytes = (int64_t)std::min<size_t>(pixel_bytes, INT64_MAX);
    A.patch = patch; A.merge = merge; A.frames = frames; A.out = d_out; A.positions = d_positions;
    for (int c = 0; c < channels; c++) {
        A.scale[c] = (float)((double)inv_std[c] / 255.0);
        A.shift[c] = (float)(-(double)mean[c] * inv_std[c]);
    }
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    const uint32_t runs = (patch + 7) / 8, each = runs * patch;
    A.by_runs = (uint32_t)(((1ull << 32) + runs - 1) / runs);  // (of 1: 0)
    A.by_each = (uint32_t)(((1ull << 32) + each - 1) / each);
    // Stores go through LDS where lines are not of whole runs and a row fits there.  Rows of a workgroup: some 512 runs of eight pixels, two a thread (256 where 32-bit
    // elements are stored at once), in LDS no more than 10240 elements, eight together (16-byte stores then lie at multiples of 16).  us for 1024 photographs with 8 / 16 /
    // 24 rows of patches of 14: 406 / 319 / 350, of 16 - / 285 / 296; 512 of them in 32 bits, 14: 268 / 247 / -, 16: 245 / 250 / -.
    const size_t size = type_size(dtype), row_bytes = (size_t)channels * patch * patch * size;
    const bool staged = patch % 8 && row_bytes <= 61440;
    int64_t group = (dtype == PCR_FLOAT && !staged ? 256 : 512) / each;
    if (staged) group = std::min<int64_t>(group, 10240 * size / row_bytes);
    if (group > 8) group -= group % 8;
    A.group = (int)std::max<int64_t>(1, std::min<int64_t>(group, kPatchGroup));
    with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        auto launch = [&](auto c, auto s) {
            in_ranges((rows + A.group - 1) / A.group, 256, [&](int64_t begin, unsigned groups) {
                A.begin = begin;
                hipLaunchKernelGGL((k_patch_rows<T, decltype(c)::value, decltype(s)::value>), dim3(groups), dim3(256), staged ? A.group * row_bytes : 0, (hipStream_t)hip_stream, A);
            });
        };
        auto by_channels = [&](auto s) {
            if (channels == 3) launch(std::integral_constant<int, 3>(), s);
            else launch(std::integral_constant<int, 1>(), s);
        };
        if (staged) by_channels(std::true_type());
        else by_channels(std::false_type());
    });
    return launched();
}

int pcr_rotate_axes(int device_id, const pcr_heads* q, const pcr_heads* k, const pcr_rotation* rotation, int inverse, int dtype, void* hip_stream) {
    return run_axes(device_id, q, k, rotation, 0.f, inverse != 0, dtype, dtype, kRotate, nullptr, 0, (hipStream_t)hip_stream);
}

int pcr_norm_rotate(int device_id, const pcr_heads* q, const pcr_heads* k, const pcr_rotation* rotation, float eps, int dtype, int weight_dtype,
                    void* hip_stream) {
    return run_axes(device_id, q, k, rotation, eps, 0, dtype, weight_dtype, kNorm, nullptr, 0, (hipStream_t)hip_stream);
}

int pcr_norm_rotate_workspace(int64_t tokens, int dim, size_t* nbytes) {
    if (!nbytes) return PCR_E_ARG;
    if (tokens < 0 || dim < 1 || dim > 512) return PCR_E_RANGE;
    *nbytes = (size_t)2 * std::min<int64_t>(tokens, kBackGroups) * dim * sizeof(float);
    return PCR_OK;
}

int pcr_norm_rotate_backward(int device_id, const pcr_heads* q, const pcr_heads* k, const pcr_rotation* rotation, float eps, int dtype,
                             int weight_dtype, void* d_work, size_t work_bytes, void* hip_stream) {
    return run_axes(device_id, q, k, rotation, eps, 1, dtype, weight_dtype, kNormBack, d_work, work_bytes, (hipStream_t)hip_stream);
}

}  // extern "C"
