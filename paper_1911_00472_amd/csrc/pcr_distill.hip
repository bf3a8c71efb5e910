// C ABI of distillation from a teacher's top logits (see include/pcr.h): checks of arguments, choice of a kernel, launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "../../include/pcr.h"
#include "pcr_distill.h"
#include "pcr_host.h"

using namespace pcr;

namespace {

// Shares that a few rows are cut into: as many as fill the chip with some 2048 workgroups, none below 8192 classes.
int64_t parts_of(int64_t rows, int64_t V) {
    if (rows <= 0 || rows >= 512) return 1;
    return std::max<int64_t>(1, std::min<int64_t>(2048 / rows, V / 8192));
}
// Classes of a row that a team of 1024 threads holds in its registers.
constexpr int kMostRuns = 18;
int64_t most_held(size_t size) { return 1024 * kMostRuns * (int64_t)(16 / size); }
// Whether a loss (or a loss with its gradient) over few rows is made of shares of a row.  us, held / in shares, of rows of bfloat logits:
//                        1 row       24 rows      64 rows     128 rows
//   loss  65000      7.3/ 9.1     7.9/ 9.1     8.3/ 9.0     9.3/ 9.9      131071  10.5/ 8.8    10.8/ 8.8    12.0/10.3    14.6/13.1  (256 of 100000: 16.6/17.8)
//   step  65000     12.0/12.3    12.6/13.7    13.8/16.3    15.2/19.9      131071  18.1/12.4    19.1/15.9    21.5/20.6    24.2/28.0
bool in_shares(int64_t rows, int64_t V, size_t size, bool step) {
    if (parts_of(rows, V) == 1) return false;
    return V > most_held(size) || (V * (int64_t)size > 131072 && rows <= (step ? 64 : 128));
}

int check_distill(const pcr_distill* d) {
    if (!d || !known_type(d->dtype) || !known_type(d->top_dtype)) return PCR_E_ARG;
    if (d->rows < 0 || d->rows > kMaxGrid || d->classes < 1 || d->classes > kMaxGrid || d->top < 1 || d->top > 1024) return PCR_E_RANGE;
    if (!(d->temperature > 0.f) || !isfinite(d->temperature) || !isfinite(d->distill_part) || !isfinite(d->label_part)) return PCR_E_RANGE;
    if (d->rows && (!d->logits || !d->top_index || !d->top_logits)) return PCR_E_ARG;
    return PCR_OK;
}

DistillArgs distill_args(const pcr_distill* d) {
    DistillArgs A = {};
    A.logits = d->logits; A.top_index = d->top_index; A.top_logits = d->top_logits; A.labels = d->labels;
    A.row_stride = d->row_stride; A.rows = d->rows; A.V = d->classes; A.chunk = d->classes; A.chunks = 1;
    A.K = d->top; A.top_dtype = d->top_dtype; A.wide = d->index_wide;
    A.T = d->temperature; A.inv_T = 1.f / d->temperature; A.a = d->distill_part; A.b = d->label_part;
    A.two = d->labels && d->label_part != 0.f;
    return A;
}

void cut(DistillArgs& A, int64_t parts) {
    A.chunk = ((A.V + parts - 1) / parts + 63) / 64 * 64;
    A.chunks = (int)((A.V + A.chunk - 1) / A.chunk);
}

template <typename T, int TEAM, int MODE> void launch_team(DistillArgs A, hipStream_t s) {
    const size_t lds = (size_t)(16 + entry_floats(A.K, A.chunk)) * sizeof(float);
    in_ranges(A.rows * A.chunks, TEAM, [&](int64_t first, unsigned groups) {
        A.first = first;
        if (A.two && A.T != 1.f) hipLaunchKernelGGL((k_distill<T, TEAM, true, MODE>), dim3(groups), dim3(TEAM), lds, s, A);
        else hipLaunchKernelGGL((k_distill<T, TEAM, false, MODE>), dim3(groups), dim3(TEAM), lds, s, A);
    });
}
// The gradient from saved sums of rows for more than a wavefront, and (MODE kLoss, kStep) rows too long for a team's registers, read twice.
template <int MODE> void launch_distill(const DistillArgs& A, int dtype, hipStream_t s) {
    with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const int64_t bytes = std::min(A.chunk, A.V) * (int64_t)sizeof(T);
        if constexpr (MODE == kGrad) {
            if (bytes <= 65536) return launch_team<T, 256, MODE>(A, s);
        }
        launch_team<T, 1024, MODE>(A, s);
    });
}
// A team that holds a row in its registers, the smallest there is: false if there is none.
template <typename T, int TEAM, int R, int MODE> bool launch_rows(DistillArgs A, hipStream_t s) {
    constexpr int N = 16 / sizeof(T);
    if (A.V > (int64_t)TEAM * R * N) return false;             // (elements in front of and behind the runs are held beside them)
    const int teams = TEAM < 256 ? 256 / TEAM : 1, threads = TEAM < 256 ? 256 : TEAM;
    const size_t lds = (size_t)teams * (6 * (TEAM / 64) + entry_floats(A.K, A.V)) * sizeof(float);
    in_ranges((A.rows + teams - 1) / teams, threads, [&](int64_t first, unsigned groups) {
        A.first = first;
        if (!A.two || A.T == 1.f) hipLaunchKernelGGL((k_distill_rows<T, TEAM, R, kOneSum, MODE>), dim3(groups), dim3(threads), lds, s, A);
        else if (MODE != kGrad && A.T == 2.f) hipLaunchKernelGGL((k_distill_rows<T, TEAM, R, MODE == kGrad ? kTwoSums : kSquare, MODE>), dim3(groups), dim3(threads), lds, s, A);
        else if (MODE != kGrad && A.T == 4.f) hipLaunchKernelGGL((k_distill_rows<T, TEAM, R, MODE == kGrad ? kTwoSums : kFourth, MODE>), dim3(groups), dim3(threads), lds, s, A);
        else hipLaunchKernelGGL((k_distill_rows<T, TEAM, R, kTwoSums, MODE>), dim3(groups), dim3(threads), lds, s, A);
    });
    return true;
}
// Whether rows go to a wavefront each: short ones, unless there are so few that a workgroup each is done sooner.  (us, wavefronts / workgroups of 256, gradient
// from saved sums over rows of 3000 classes with 256 entries: 1 row 7.9 / 5.7, 64 9.0 / 5.4, 1024 11.2 / 7.3, 4096 18.9 / 24.7; of 500 classes with 10
// entries: 1024 5.5 / 5.5, 4096 6.8 / 16.7.)
bool by_wavefronts(int64_t rows, int64_t V, size_t size) { return V * (int64_t)size <= 8192 && rows > (V * (int64_t)size > 4096 ? 1024 : 256); }
template <int MODE> bool launch_resident(const DistillArgs& A, int dtype, hipStream_t s) {
    bool held = false;
    with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        if (by_wavefronts(A.rows, A.V, sizeof(T))) held = launch_rows<T, 64, 4, MODE>(A, s) || launch_rows<T, 64, 8, MODE>(A, s);
        if constexpr (MODE != kGrad)                           // (longer rows are written as fast as they are read again)
            held = held || launch_rows<T, 256, 4, MODE>(A, s) || launch_rows<T, 256, 8, MODE>(A, s) || launch_rows<T, 512, 8, MODE>(A, s) ||
                   launch_rows<T, 512, 16, MODE>(A, s) || launch_rows<T, 1024, 16, MODE>(A, s) || launch_rows<T, 1024, kMostRuns, MODE>(A, s);
    });
    return held;
}
// The sums of rows in shares, and the loss.
void launch_shares(DistillArgs A, int64_t parts, int dtype, hipStream_t s) {
    cut(A, parts);
    with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const unsigned groups = (unsigned)(A.rows * A.chunks);
        if (A.two && A.T != 1.f) {
            hipLaunchKernelGGL((k_distill_part<T, true>), dim3(groups), dim3(256), 0, s, A);
            hipLaunchKernelGGL((k_distill_join<T, true>), dim3((unsigned)A.rows), dim3(64), 0, s, A);
        } else {
            hipLaunchKernelGGL((k_distill_part<T, false>), dim3(groups), dim3(256), 0, s, A);
            hipLaunchKernelGGL((k_distill_join<T, false>), dim3((unsigned)A.rows), dim3(64), 0, s, A);
        }
    });
}

int check_work(bool shares, int64_t rows, int64_t V, void* d_work, size_t work_bytes) {
    if (!shares) return PCR_OK;
    size_t need = 0;
    pcr_distill_workspace(rows, V, &need);
    return !d_work ? PCR_E_ARG : work_bytes < need ? PCR_E_RANGE : PCR_OK;
}

}  // namespace

extern "C" {

int pcr_distill_workspace(int64_t rows, int64_t classes, size_t* nbytes) {
    if (!nbytes) return PCR_E_ARG;
    if (rows < 0 || classes < 1) return PCR_E_RANGE;
    const bool shares = in_shares(rows, classes, 2, false) || in_shares(rows, classes, 4, false);     // (of a step as well: its rows are fewer)
    *nbytes = shares ? (size_t)rows * (3 * parts_of(rows, classes) + 2) * sizeof(float) : 0;
    return PCR_OK;
}

int pcr_distill_forward(int device_id, const pcr_distill* d, float* loss, float* sums, void* d_work, size_t work_bytes, void* hip_stream) {
    int rc = check_distill(d);
    if (rc) return rc;
    if (d->rows && (!loss || !sums)) return PCR_E_ARG;
    const bool shares = in_shares(d->rows, d->classes, type_size(d->dtype), false);
    rc = check_work(shares, d->rows, d->classes, d_work, work_bytes);
    if (rc || !d->rows) return rc;
    DistillArgs A = distill_args(d);
    A.loss = loss; A.sums = sums; A.part = (float*)d_work;
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    if (shares) launch_shares(A, parts_of(A.rows, A.V), d->dtype, (hipStream_t)hip_stream);
    else if (!launch_resident<kLoss>(A, d->dtype, (hipStream_t)hip_stream)) launch_distill<kLoss>(A, d->dtype, (hipStream_t)hip_stream);
    return launched();
}

int pcr_distill_backward(int device_id, const pcr_distill* d, const float* sums, const float* row_grad, void* out, int64_t out_stride, void* hip_stream) {
    int rc = check_distill(d);
    if (!rc && d->rows && (!sums || !row_grad || !out)) rc = PCR_E_ARG;
    if (rc || !d->rows) return rc;
    DistillArgs A = distill_args(d);
    A.sums_in = sums; A.row_grad = row_grad; A.out = out; A.out_stride = out_stride;
    cut(A, parts_of(A.rows, A.V));
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    if (!launch_resident<kGrad>(A, d->dtype, (hipStream_t)hip_stream)) launch_distill<kGrad>(A, d->dtype, (hipStream_t)hip_stream);
    return launched();
}

int pcr_distill_step(int device_id, const pcr_distill* d, const float* row_weight, float* loss, void* out, int64_t out_stride, void* d_work,
                     size_t work_bytes, void* hip_stream) {
    int rc = check_distill(d);
    if (rc) return rc;
    if (d->rows && (!row_weight || !loss || !out)) return PCR_E_ARG;
    const bool shares = in_shares(d->rows, d->classes, type_size(d->dtype), true);
    rc = check_work(shares, d->rows, d->classes, d_work, work_bytes);
    if (rc || !d->rows) return rc;
    DistillArgs A = distill_args(d);
    A.row_grad = row_weight; A.loss = loss; A.out = out; A.out_stride = out_stride;
    const OnDevice on(device_id);
    if (!on.ok) return PCR_E_DEVICE;
    if (shares) {
        const int64_t parts = parts_of(A.rows, A.V);
        A.part = (float*)d_work;
        A.sums = A.part + 3 * A.rows * parts;
        launch_shares(A, parts, d->dtype, (hipStream_t)hip_stream);
        A.sums_in = A.sums;
        cut(A, parts);
        launch_distill<kGrad>(A, d->dtype, (hipStream_t)hip_stream);
    } else if (!launch_resident<kStep>(A, d->dtype, (hipStream_t)hip_stream)) launch_distill<kStep>(A, d->dtype, (hipStream_t)hip_stream);
    return launched();
}

}  // extern "C"
