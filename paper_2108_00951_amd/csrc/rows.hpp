// Rows of fp32 or bf16 elements as packs of a thread's registers, for the
// kernels that stream whole rows (embed.hip, norm.hip, adamw.hip).
#pragma once

#include "device_common.hpp"

namespace efs {

// N consecutive elements at any address that their type allows: one access as
// wide as they are, since the hardware asks for no more alignment than that.
template <typename T, int N>
struct PackOf {
    typedef T type __attribute__((ext_vector_type(N)));
    typedef T loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T, int N>
using Pack = typename PackOf<T, N>::type;

// Elements a lane takes at once from a row of T where it also handles rows of
// F: 16 bytes of the wider type.
template <typename T, typename F>
constexpr int kPack = sizeof(T) == 2 && sizeof(F) == 2 ? 8 : 4;

// The first `left` (at least 1) elements from p on, zeros behind; a whole pack if
// left >= N.
template <int N, typename T>
__device__ __forceinline__ Pack<T, N> load_raw(const T *p, int left) {
    Pack<T, N> v;
    if (left >= N) return *reinterpret_cast<const typename PackOf<T, N>::loose *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < left ? p[i] : T(0.0f);
    return v;
}

template <int N, typename T>
__device__ __forceinline__ void load_pack(const T *p, int left, float (&v)[N]) {
    const Pack<T, N> a = load_raw<N>(p, left);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = float(a[i]);
}

// What a call writes from here on does not stay in the 256 MB of the Infinity Cache
// until it is read: it is stored past the caches (norm of 16,384 x 4,096 bf16 and its
// gradients 144 -> 134 us, gradient of 131,072 x 2,048 266 -> 236; below, 33,278 x 650
// in 16 us through them and 23 past them).
constexpr int64_t kPastCaches = int64_t(128) << 20;

// bf16 results are rounded here, to nearest even.
template <int N, typename T>
__device__ __forceinline__ void store_pack(T *p, int left, const float (&v)[N], bool past = false) {
    if (left >= N) {
        Pack<T, N> a;
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = T(v[i]);
        typename PackOf<T, N>::loose *to = reinterpret_cast<typename PackOf<T, N>::loose *>(p);
        if (past) {
            asm volatile("");   // (both keep the two stores from becoming one)
            __builtin_nontemporal_store(a, to);
            asm volatile("");
        } else {
            *to = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = T(v[i]);
    }
}

// Lane permutations within the wave without LDS: pairs, fours, eights, sixteens
// mirrored, and the last lane of a row of 16 (of 32) to the next (to the upper half).
constexpr int kDppPairs = 0xB1, kDppFours = 0x4E, kDppEights = 0x141, kDppSixteens = 0x140, kDppNextRow = 0x142,
              kDppUpperHalf = 0x143;

// (lanes of rows that are left out get 0)
template <int kControl, int kRows = 0xf>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), kControl, kRows, 0xf, kRows == 0xf));
}

template <int kControl, int kRows = 0xf>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(dpp<kControl, kRows>(__float_as_uint(v)));
}

// Sum over the wave, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp<kDppPairs>(v);
    v += dpp<kDppFours>(v);
    v += dpp<kDppEights>(v);
    v += dpp<kDppSixteens>(v);
    v += dpp<kDppNextRow, 0xa>(v);
    v += dpp<kDppUpperHalf, 0xc>(v);
    return __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(v)), kWave - 1)));
}

// Largest over the wave, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, dpp<kDppPairs>(v));
    v = max(v, dpp<kDppFours>(v));
    v = max(v, dpp<kDppEights>(v));
    v = max(v, dpp<kDppSixteens>(v));
    v = max(v, dpp<kDppNextRow, 0xa>(v));
    v = max(v, dpp<kDppUpperHalf, 0xc>(v));
    return uint32_t(__builtin_amdgcn_readlane(int(v), kWave - 1));
}

}  // namespace efs
