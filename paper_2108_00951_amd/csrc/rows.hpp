// Rows of fp32 or bf16 elements as packs of a thread's registers, for the
// kernels that stream whole rows (embed.hip, norm.hip, adamw.hip).
#pragma once

#include "device_common.hpp"

namespace efs {

// N consecutive elements at any address that their type allows: one access as
// wide as they are, since the hardware asks for no more alignment than that.
template <typename T, int N>
struct PackOf {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Elements a lane takes at once from a row of T where it also handles rows of
// F: 16 bytes of the wider type.
template <typename T, typename F>
constexpr int kPack = sizeof(T) == 2 && sizeof(F) == 2 ? 8 : 4;

template <int N, typename T>
__device__ __forceinline__ void load_pack(const T *p, float (&v)[N]) {
    const typename PackOf<T, N>::type a = *reinterpret_cast<const typename PackOf<T, N>::type *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = float(a[i]);
}

// The first `left` (at least 1) of them, zeros behind; a whole pack if left >= N.
template <int N, typename T>
__device__ __forceinline__ void load_pack(const T *p, int left, float (&v)[N]) {
    if (left >= N) return load_pack(p, v);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < left ? float(p[i]) : 0.0f;
}

// bf16 results are rounded here, to nearest even.
template <int N, typename T>
__device__ __forceinline__ void store_pack(T *p, int left, const float (&v)[N]) {
    if (left >= N) {
        typename PackOf<T, N>::type a;
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = T(v[i]);
        *reinterpret_cast<typename PackOf<T, N>::type *>(p) = a;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = T(v[i]);
    }
}

// Sum over the wave, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

}  // namespace efs
