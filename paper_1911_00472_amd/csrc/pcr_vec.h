// Element types of the operators behind the decode, their vectors in memory, and sums over a group of lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcr {

// A run of N elements as it lies in memory; aligned to an element only, so that any row may be read with it.  (The compiler makes one load of
// up to 16 bytes of it; the hardware takes any alignment, at full speed where the address is a multiple of the run's size.)
template <typename T, int N> struct Run {
    typedef T Vec __attribute__((ext_vector_type(N)));
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { Vec v; };
};
template <typename T> struct Run<T, 1> {
    typedef T Vec;
    struct Loose { T v; };
};

template <typename T, int N> __device__ __forceinline__ void load_run(const T* p, float (&x)[N]) {
    const typename Run<T, N>::Vec v = reinterpret_cast<const typename Run<T, N>::Loose*>(p)->v;
    if constexpr (N == 1) x[0] = (float)v;
    else {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = (float)v[i];
    }
}
// Rounds to the nearest, ties to even: the one rounding of a result.
template <typename T, int N> __device__ __forceinline__ void store_run(T* p, const float (&x)[N]) {
    typename Run<T, N>::Vec v;
    if constexpr (N == 1) v = (T)x[0];
    else {
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = (T)x[i];
    }
    reinterpret_cast<typename Run<T, N>::Loose*>(p)->v = v;
}

// v of another lane: the neighbour's, one of the other pair of four lanes, of the other four of eight, of the other eight of sixteen (the last two mirrored).
enum { kNeighbour = 0xb1, kPairOfFour = 0x4e, kFourOfEight = 0x141, kEightOfSixteen = 0x140 };
template <int FROM> __device__ __forceinline__ float across(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), FROM, 0xf, 0xf, true));
}
// Maximum or sum over a wavefront, the same bits in all lanes.
template <bool MAX> __device__ __forceinline__ float both(float a, float b) { return MAX ? fmaxf(a, b) : a + b; }
template <bool MAX> __device__ __forceinline__ float wave_join(float v) {
    v = both<MAX>(v, across<kNeighbour>(v));
    v = both<MAX>(v, across<kPairOfFour>(v));
    v = both<MAX>(v, across<kFourOfEight>(v));
    v = both<MAX>(v, across<kEightOfSixteen>(v));
    v = both<MAX>(v, __shfl_xor(v, 16));
    return both<MAX>(v, __shfl_xor(v, 32));
}

inline bool known_type(int dtype) { return dtype >= 0 && dtype <= 2; }
inline size_t type_size(int dtype) { return dtype == 0 ? 4 : 2; }

}  // namespace pcr
