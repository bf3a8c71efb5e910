// C ABI of the layers of a network that trains on the pictures (see include/pcr.h): group norm with an activation, position bias, dropout.  Checks of arguments,
// choice of a kernel, launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "../../include/pcr.h"
#include "pcr_bias.h"
#include "pcr_dropout.h"
#include "pcr_group_norm.h"
#include "pcr_host.h"

using namespace pcr;

namespace {

// Working memory lies at a multiple of 16 bytes.
bool at_16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// ---- group norm ----

int check_norm(const pcr_group_norm* N, bool back) {
    if (!N || !known_type(N->dtype) || !known_type(N->weight_dtype) || (N->weight_dtype != PCR_FLOAT && N->weight_dtype != N->dtype)) return PCR_E_ARG;
    if (N->activation < PCR_ACT_NONE || N->activation > PCR_ACT_GELU) return PCR_E_ARG;
    if (N->channels < 1 || N->channels > 16384 || N->groups < 1 || N->groups > 4096 || N->channels % N->groups) return PCR_E_RANGE;
    if (N->images < 0 || N->pixels < 0 || N->images > kMaxGrid || N->pixels > (1ll << 40)) return PCR_E_RANGE;
    if (!back && !(N->eps >= 0.f && isfinite(N->eps))) return PCR_E_RANGE;
    if (N->images && N->pixels && (!N->x || !N->out || !N->stats || (back && !N->grad))) return PCR_E_ARG;
    return PCR_OK;
}

NormArgs norm_args(const pcr_group_norm* N, const NormPlan& P, void* d_work) {
    NormArgs A = {};
    A.x = N->x; A.grad = N->grad; A.weight = N->weight; A.bias = N->bias; A.out = N->out; A.stats = N->stats;
    A.part = (float*)d_work; A.sums = (float*)((char*)d_work + P.part_bytes); A.joined = (float*)((char*)A.sums + P.sums_bytes);
    A.images = N->images; A.pixels = N->pixels;
    A.x_image = N->x_image; A.x_pixel = N->x_pixel; A.grad_image = N->grad_image; A.grad_pixel = N->grad_pixel; A.out_image = N->out_image; A.out_pixel = N->out_pixel;
    A.chunk = P.chunk; A.chunks = P.chunks; A.channels = (int)N->channels; A.groups = N->groups; A.each = (int)(N->channels / N->groups);
    A.block = P.block; A.blocks = P.blocks; A.pack = P.pack; A.turns = P.turns;
    A.activation = N->activation; A.weight_float = N->weight_dtype == PCR_FLOAT; A.eps = N->eps;
    return A;
}
// ---- position bias ----

constexpr int64_t kBiasLds = 152 * 1024;                         // of a workgroup, at most
constexpr size_t kBiasTwo = 80 * 1024;                           // where two share a compute unit
constexpr size_t kBiasParts = 4ull << 30;                        // bytes of the shares' sums of a gradient, at most

int check_bias(const pcr_position_table* t, bool back) {
    if (!t || !known_type(t->dtype)) return PCR_E_ARG;
    if (!back && (!known_type(t->table_dtype) || (t->table_dtype != PCR_FLOAT && t->table_dtype != t->dtype))) return PCR_E_ARG;
    if (t->axes < 1 || t->axes > 4 || t->reach < 0 || t->reach > (1 << 24) || t->buckets < 1 || t->buckets > (1 << 24) || t->heads < 0 || t->heads > 65535) return PCR_E_RANGE;
    if (t->batch < 0 || t->queries < 0 || t->keys < 0 || t->batch > kMaxGrid || t->queries > kMaxGrid || t->keys > kMaxGrid) return PCR_E_RANGE;
    if (t->queries && t->keys && t->batch > (1ll << 50) / t->queries / t->keys) return PCR_E_RANGE;
    if (!t->query.segment != !t->key.segment) return PCR_E_ARG;
    if (t->batch && t->queries && t->keys && t->heads && (!t->query.position || !t->key.position || !t->map || !t->values || (!back && !t->table))) return PCR_E_ARG;
    return PCR_OK;
}
BiasArgs bias_args(const pcr_position_table* t) {
    BiasArgs A = {};
    const pcr_places* from[2] = {&t->query, &t->key};
    Places* to[2] = {&A.q, &A.k};
    for (int z = 0; z < 2; z++) {
        to[z]->position = from[z]->position; to[z]->segment = from[z]->segment;
        to[z]->axis = from[z]->axis_stride; to[z]->batch = from[z]->batch_stride; to[z]->token = from[z]->token_stride;
        to[z]->segment_batch = from[z]->segment_batch_stride; to[z]->segment_token = from[z]->segment_token_stride;
    }
    A.map = t->map; A.table = t->table; A.values = t->values;
    A.value_batch = t->value_batch; A.value_head = t->value_head; A.value_query = t->value_query;
    A.batch = t->batch; A.heads = t->heads; A.queries = t->queries; A.keys = t->keys; A.buckets = t->buckets;
    const int64_t V = 16 / (int64_t)type_size(t->dtype);
    A.runs = (A.keys + V - 1) / V;
    A.items = A.batch * A.queries * A.runs;
    A.axes = t->axes; A.reach = t->reach; A.wide = t->wide; A.table_float = t->table_dtype == PCR_FLOAT;
    return A;
}
void set_step(BiasArgs& A, int64_t step) {
    A.step_run = step % A.runs;
    A.step_query = step / A.runs % A.queries;
    A.step_batch = step / A.runs / A.queries;
}

// The axes, where there are up to three of 32-bit positions and every run of `run` keys lies in one piece; else 0.
int plain_axes(const pcr_position_table* t, int run) {
    const bool plain = !t->wide && t->keys >= run && t->key.token_stride == 1 && (!t->key.segment || t->key.segment_token_stride == 1);
    return plain && t->axes <= 3 ? t->axes : 0;
}

// How the gradient is divided: wavefronts (heads) of a workgroup, copies of a wavefront's bins, ranges of buckets (each goes through all items), shares of the items.
struct BiasPlan { int waves, copies, ranges; int64_t held, shares, items, runs; size_t lds, places_bytes, live_bytes, part_bytes; };
BiasPlan plan_bias(const pcr_position_table* t) {
    BiasPlan P = {};
    P.runs = (t->keys + kRun - 1) / kRun;
    P.items = t->batch * t->queries * P.runs;
    P.ranges = (int)((t->buckets + 4095) / 4096);
    P.held = (t->buckets + P.ranges - 1) / P.ranges;
    const int64_t elements = P.items * kRun, blocks = (P.items + 63) / 64, steps = (blocks + kBinItems - 1) / kBinItems;
    P.places_bytes = (size_t)blocks * 64 * sizeof(Places8);
    const size_t sums = (size_t)t->heads * t->buckets * sizeof(float);
    // Shares: of four values to a bin at least, of 16384 values one, whose sums are the result; as many as are resident together.  Copies: up to 1024 bins of a wavefront, 2048 where there
    // are more than 64 buckets, whose lanes meet more than once where differences are held at the reach (us with 1024 / 2048: four sequences of 32 x 32 patches, 12 heads, 31 x 31 buckets
    // 137 / 79, 15 x 15 75 / 61; 4096 tokens in 31 buckets 154 / 202), and an eighth of the share's values, as bins are cleared and summed.
    const int64_t most_shares = elements <= 16384 ? 1 : std::max<int64_t>(1, elements / std::max<int64_t>(4 * P.held, 4096));
    P.copies = 64;
    while (P.copies > 1 && bins_of(P.held, P.copies) > std::max<int64_t>(bins_of(P.held, 1), std::min<int64_t>(t->buckets <= 64 ? 1024 : 2048, elements / most_shares / 8))) P.copies >>= 1;
    auto bytes = [&](int64_t w) { return w * (bins_of(P.held, P.copies) + 64) * 8; };
    const int64_t head_blocks_8 = std::max<int64_t>(1, (t->heads + 7) / 8);
    P.waves = (int)std::max<int64_t>(1, (t->heads + head_blocks_8 - 1) / head_blocks_8);
    while (P.waves > 1 && bytes(P.waves) > kBiasLds) P.waves--;
    P.lds = (size_t)bytes(P.waves);
    const int64_t head_blocks = std::max<int64_t>(1, (t->heads + P.waves - 1) / P.waves);
    const int64_t resident = 256 * std::max<int64_t>(1, std::min<int64_t>(16 / P.waves, (int64_t)(160 * 1024 / P.lds)));
    P.shares = std::min<int64_t>(std::min<int64_t>(most_shares, steps), std::min<int64_t>(resident / head_blocks, (int64_t)(kBiasParts / std::max<size_t>(1, sums))));
    P.shares = std::max<int64_t>(1, P.shares);
    P.live_bytes = (size_t)(blocks + 1) / 2 * 2 * 8;
    P.part_bytes = P.shares == 1 ? 0 : (size_t)P.shares * sums;
    return P;
}

}  // namespace

extern "C" {

int pcr_group_norm_workspace(const pcr_group_norm* norm, int backward, size_t* nbytes) {
    if (!norm || !nbytes) return PCR_E_ARG;
    if (!known_type(norm->dtype)) return PCR_E_ARG;
    if (norm->channels < 1 || norm->channels > 16384 || norm->groups < 1 || norm->groups > 4096 || norm->channels % norm->groups || norm->images < 0 || norm->pixels < 0 ||
        norm->images > kMaxGrid || norm->pixels > (1ll << 40)) return PCR_E_RANGE;
    const NormPlan P = plan_norm(norm, backward != 0);
    *nbytes = P.bytes();
    return PCR_OK;
}

int pcr_group_norm_forward(int device_id, const pcr_group_norm* norm, void* d_work, size_t work_bytes, void* hip_stream) {
    const int rc = check_norm(norm, false);
    if (rc) return rc;
    if (!norm->images || !norm->pixels) return PCR_OK;
    const NormPlan P = plan_norm(norm, false);
    if (P.bytes() && !d_work) return PCR_E_ARG;
    if (work_bytes < P.bytes()) return PCR_E_RANGE;
    if (!at_16(d_work)) return PCR_E_ARG;
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    NormArgs A = norm_args(norm, P, d_work);
    const hipStream_t s = (hipStream_t)hip_stream;
    if (P.held) return run_norm_held(norm, P, A, s) ? launched() : PCR_E_DEVICE;
    with_run(norm->dtype, P.run, [&](auto t, auto v) {
        typedef decltype(t) T;
        constexpr int V = decltype(v)::value;
        in_ranges(A.images * A.chunks, kNormThreads, [&](int64_t begin, unsigned groups) {
            A.begin = begin;
            hipLaunchKernelGGL((k_norm_sums<T, V>), dim3(groups), dim3(kNormThreads), norm_sums_lds(V, A.groups), s, A);
        });
        if (A.chunks > kMergedChunks)
            in_ranges((A.images * A.groups + 3) / 4, 256, [&](int64_t begin, unsigned groups) {
                A.begin = begin;
                hipLaunchKernelGGL((k_norm_join<false>), dim3(groups), dim3(256), 0, s, A);
            });
        in_ranges(A.images * A.chunks, kNormThreads, [&](int64_t begin, unsigned groups) {
            A.begin = begin;
            if (A.each % V == 0) hipLaunchKernelGGL((k_norm_apply<T, V, true>), dim3(groups), dim3(kNormThreads), 2 * A.groups * sizeof(float), s, A);
            else if constexpr (V > 1) hipLaunchKernelGGL((k_norm_apply<T, V, false>), dim3(groups), dim3(kNormThreads), 2 * A.groups * sizeof(float), s, A);
        });
    });
    return launched();
}

int pcr_group_norm_backward(int device_id, const pcr_group_norm* norm, void* d_work, size_t work_bytes, void* hip_stream) {
    const int rc = check_norm(norm, true);
    if (rc) return rc;
    const NormPlan P = plan_norm(norm, true);
    const bool none = !norm->images || !norm->pixels;
    if (!none && !d_work) return PCR_E_ARG;
    if (!none && work_bytes < P.bytes()) return PCR_E_RANGE;
    if (!at_16(d_work)) return PCR_E_ARG;
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    NormArgs A = norm_args(norm, P, d_work);
    const hipStream_t s = (hipStream_t)hip_stream;
    if (!none && P.held) {
        if (!run_norm_back_held(norm, P, A, s)) return PCR_E_DEVICE;
    } else if (!none)
        with_run(norm->dtype, P.run, [&](auto t, auto v) {
            typedef decltype(t) T;
            constexpr int V = decltype(v)::value;
            const int block = std::min(A.channels, kNormThreads * V);
            in_ranges(A.images * A.chunks, kNormThreads, [&](int64_t begin, unsigned groups) {
                A.begin = begin;
                const size_t lds = (kNormThreads * V + 2 * A.groups + 2 * block) * sizeof(float);
                if (A.each % V == 0) hipLaunchKernelGGL((k_norm_back_sums<T, V, true>), dim3(groups), dim3(kNormThreads), lds, s, A);
                else if constexpr (V > 1) hipLaunchKernelGGL((k_norm_back_sums<T, V, false>), dim3(groups), dim3(kNormThreads), lds, s, A);
            });
            if (A.chunks > kMergedChunks)
                in_ranges((A.images * A.groups + 3) / 4, 256, [&](int64_t begin, unsigned groups) {
                    NormArgs J = A;
                    J.begin = begin;
                    J.stats = A.joined;
                    hipLaunchKernelGGL((k_norm_join<true>), dim3(groups), dim3(256), 0, s, J);
                });
            in_ranges(A.images * A.chunks, kNormThreads, [&](int64_t begin, unsigned groups) {
                A.begin = begin;
                if (A.each % V == 0) hipLaunchKernelGGL((k_norm_back_apply<T, V, true>), dim3(groups), dim3(kNormThreads), 2 * A.groups * sizeof(float), s, A);
                else if constexpr (V > 1) hipLaunchKernelGGL((k_norm_back_apply<T, V, false>), dim3(groups), dim3(kNormThreads), 2 * A.groups * sizeof(float), s, A);
            });
        });
    if (norm->weight_grad || norm->bias_grad) {
        NormWeightSums W = {A.sums, norm->weight_grad, norm->bias_grad, none ? 0 : P.rows, A.channels};
        hipLaunchKernelGGL(k_norm_weight_sums, dim3((2 * A.channels + 15) / 16), dim3(1024), 0, s, W);
    }
    return launched();
}

int pcr_position_bias(int device_id, const pcr_position_table* t, void* hip_stream) {
    const int rc = check_bias(t, false);
    if (rc) return rc;
    if (!t->batch || !t->queries || !t->keys || !t->heads) return PCR_OK;
    BiasArgs A = bias_args(t);
    const size_t size = type_size(t->dtype);
    const size_t map_bytes = (size_t)t->axes * (2 * t->reach + 1) * 4;
    auto lds = [&](int heads) { return ((size_t)(t->buckets + 2) * heads * size + 15) / 16 * 16 + map_bytes; };
    // Heads side by side: 16 bytes of them, fewer where fewer than two workgroups' tables fit (us with a limit of 72 / 80 KB: two sequences of 2048 tokens, 12 heads, 19321 buckets 98 / 85).
    // Workgroups of 1024 threads where a table takes more than 16 KB, and as many as fit side by side, as each loads its own (us with more than 36 / 16 KB: four sequences of
    // 2048, 3 heads, 3969 buckets 59 / 29; from 4 or 8 KB on the same).
    int together = (int)(16 / size);
    while (together > 1 && (together >= 2 * t->heads || lds(together) > kBiasTwo)) together >>= 1;
    const bool held = lds(together) <= (size_t)kBiasLds;
    if (!held) together = 4;
    const size_t bytes = held ? lds(together) : 0;
    const int threads = bytes > 16 * 1024 ? 1024 : 256;
    const int64_t most = bytes > kBiasTwo ? 256 : threads == 1024 ? 512 : 2048;
    const int64_t blocks = (t->heads + together - 1) / together;
    const int64_t groups = std::max<int64_t>(1, std::min<int64_t>((A.items + 2 * threads - 1) / (2 * threads), (most + blocks - 1) / blocks));
    set_step(A, groups * threads);
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    bool ok = true;
    with_type(t->dtype, [&](auto v) {
        typedef decltype(v) T;
        auto launch_axes = [&](auto h, auto in_lds, auto axes) {
            const auto kernel = k_bias<T, decltype(h)::value, decltype(in_lds)::value, decltype(axes)::value>;
            ok = allow_lds(kernel, bytes);
            if (ok) hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)blocks), dim3(threads), bytes, (hipStream_t)hip_stream, A);
        };
        const int plain = held ? plain_axes(t, (int)(16 / size)) : 0;
        auto launch = [&](auto h, auto in_lds) {
            if constexpr (decltype(in_lds)::value) {
                if (plain == 1) return launch_axes(h, in_lds, Int<1>());
                if (plain == 2) return launch_axes(h, in_lds, Int<2>());
                if (plain == 3) return launch_axes(h, in_lds, Int<3>());
            }
            launch_axes(h, in_lds, Int<0>());
        };
        if (!held) launch(Int<4>(), std::false_type());
        else if (together == 8) { if constexpr (sizeof(T) == 2) launch(Int<8>(), std::true_type()); }
        else if (together == 4) launch(Int<4>(), std::true_type());
        else if (together == 2) launch(Int<2>(), std::true_type());
        else launch(Int<1>(), std::true_type());
    });
    if (!ok) return PCR_E_DEVICE;
    return launched();
}

int pcr_position_bias_workspace(const pcr_position_table* t, size_t* nbytes) {
    if (!nbytes) return PCR_E_ARG;
    const int rc = check_bias(t, true);
    if (rc) return rc;
    const BiasPlan P = plan_bias(t);
    *nbytes = P.places_bytes + P.live_bytes + P.part_bytes;
    return PCR_OK;
}

int pcr_position_bias_backward(int device_id, const pcr_position_table* t, float* table_grad, void* d_work, size_t work_bytes, void* hip_stream) {
    const int rc = check_bias(t, true);
    if (rc) return rc;
    if (!t->heads) return PCR_OK;
    if (!table_grad) return PCR_E_ARG;
    const BiasPlan P = plan_bias(t);
    const bool none = !t->batch || !t->queries || !t->keys, direct = !none && P.shares == 1;
    if (!none && !d_work) return PCR_E_ARG;
    if (!none && work_bytes < P.places_bytes + P.live_bytes + P.part_bytes) return PCR_E_RANGE;
    if (!at_16(d_work)) return PCR_E_ARG;
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    const hipStream_t s = (hipStream_t)hip_stream;
    BiasArgs A = bias_args(t);
    A.runs = P.runs; A.items = P.items;
    A.places = (Places8*)d_work; A.live = (uint64_t*)((char*)d_work + P.places_bytes);
    A.part = direct ? table_grad : (float*)((char*)d_work + P.places_bytes + P.live_bytes);
    A.direct = direct; A.held_buckets = P.held; A.waves = P.waves; A.copies = P.copies;
    bool ok = true;
    if (!none) {
        auto steps = [&](int64_t items) { return Steps{(uint32_t)(items % A.runs), (uint32_t)(items / A.runs % A.queries), (uint32_t)(items / A.runs / A.queries)}; };
        A.near = steps(64);
        A.far = steps((P.shares - 1) * kBinItems * 64);
        const size_t map_bytes = (size_t)t->axes * (2 * t->reach + 1) * 4;
        const bool held_map = map_bytes <= 32 * 1024;
        const unsigned groups = (unsigned)std::min<int64_t>((P.items + 255) / 256, 4096);
        set_step(A, (int64_t)groups * 256);
        for (int r = 0; ok && r < P.ranges; r++) {
            A.first_bucket = r * P.held;
            A.held_buckets = std::min<int64_t>(P.held, t->buckets - A.first_bucket);
            const int plain = held_map ? plain_axes(t, kRun) : 0;
            auto places = [&](auto held, auto axes) {
                hipLaunchKernelGGL((k_bias_places<decltype(held)::value, decltype(axes)::value>), dim3(groups), dim3(256), decltype(held)::value ? map_bytes : 0, s, A);
            };
            if (!held_map) places(std::false_type(), Int<0>());
            else if (plain == 1) places(std::true_type(), Int<1>());
            else if (plain == 2) places(std::true_type(), Int<2>());
            else if (plain == 3) places(std::true_type(), Int<3>());
            else places(std::true_type(), Int<0>());
            with_type(t->dtype, [&](auto v) {
                typedef decltype(v) T;
                auto launch = [&](auto whole) {
                    const auto kernel = k_bias_bins<T, decltype(whole)::value>;
                    ok = allow_lds(kernel, P.lds);
                    if (ok) hipLaunchKernelGGL(kernel, dim3((unsigned)P.shares, (unsigned)((t->heads + P.waves - 1) / P.waves)), dim3(P.waves * 64), P.lds, s, A);
                };
                if (t->keys >= kRun) launch(std::true_type());
                else launch(std::false_type());
            });
        }
    }
    if (!ok) return PCR_E_DEVICE;
    if (direct) return launched();
    BiasSums S = {A.part, table_grad, none ? 0 : P.shares, t->heads, t->buckets, 0};
    in_ranges((t->heads * t->buckets + 63) / 64, 1024, [&](int64_t begin, unsigned groups) {
        S.begin = begin;
        hipLaunchKernelGGL(k_bias_sums, dim3(groups), dim3(1024), 0, s, S);
    });
    return launched();
}

int pcr_dropout_add(int device_id, const pcr_dropout* d, void* hip_stream) {
    if (!d || !known_type(d->dtype) || !known_type(d->out_dtype) || (d->dtype != d->out_dtype && d->dtype != PCR_FLOAT && d->out_dtype != PCR_FLOAT)) return PCR_E_ARG;
    if (d->rows < 0 || d->dim < 0 || d->call < 0 || d->call > 65535 || !(d->p >= 0.0 && d->p <= 1.0)) return PCR_E_RANGE;
    if (d->dim && d->rows > (1ll << 50) / d->dim) return PCR_E_RANGE;
    if (!d->rows || !d->dim) return PCR_OK;
    if (!d->x || !d->out || !d->seed) return PCR_E_ARG;
    DropArgs A = {};
    A.x = d->x; A.residual = d->residual; A.out = d->out; A.seed = d->seed; A.used = d->used;
    A.count = d->rows * d->dim; A.dim = d->dim; A.x_row = d->x_row; A.residual_row = d->residual_row; A.out_row = d->out_row;
    const double below = rint(d->p * 4294967296.0);
    A.below = below >= 4294967296.0 ? 0xffffffffu : (uint32_t)below;
    A.scale = below >= 4294967296.0 ? 0.f : (float)(1.0 / (1.0 - d->p));
    A.call = (uint32_t)d->call;
    const bool flat = d->rows == 1 || (d->x_row == d->dim && d->out_row == d->dim && (!d->residual || d->residual_row == d->dim));
    // (e / dim by a product is exact as long as both are below 2^32)
    A.by_dim = A.count < (1ll << 32) && d->dim > 1 ? ~0ull / (uint64_t)d->dim + 1 : 0;
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    auto launch = [&](auto t, auto u) {
        typedef decltype(t) T;
        typedef decltype(u) U;
        in_ranges((A.count + 256 * kDropRun - 1) / (256 * kDropRun), 256, [&](int64_t begin, unsigned groups) {
            A.begin = begin * 256;
            if (flat) hipLaunchKernelGGL((k_dropout<T, U, true>), dim3(groups), dim3(256), 0, (hipStream_t)hip_stream, A);
            else hipLaunchKernelGGL((k_dropout<T, U, false>), dim3(groups), dim3(256), 0, (hipStream_t)hip_stream, A);
        });
    };
    with_type(d->dtype, [&](auto t) {
        if (d->out_dtype == d->dtype) launch(t, t);
        else with_type(d->out_dtype, [&](auto u) {
            if constexpr ((sizeof(t) == 4) != (sizeof(u) == 4)) launch(t, u);
        });
    });
    return launched();
}

}  // extern "C"
