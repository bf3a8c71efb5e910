// Group norm in one pass: its kernels and their launches.
#include "pcr_norm_held.h"

bool pcr::run_norm_held(const pcr_group_norm* N, const NormPlan& P, NormArgs A, hipStream_t s) { return run_held<false>(N, P, A, s); }
