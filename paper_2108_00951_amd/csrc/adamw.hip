// AdamW over many tensors at once.
//
//   m = b1 m + (1 - b1) g ;  v = b2 v + ((1 - b2) g) g
//   x = (1 - gamma decay) x - alpha (m / (root sqrt(v) + eps))
//   alpha = gamma / (1 - b1^t) ;  root = 1 / sqrt(1 - b2^t)
//
// each operation rounded to fp32 by itself.  Bytes bound it: 28 of an element
// with states of 32 bits (g, x, m, v in; x, m, v out), 16 with states of 8.
// A launch takes the tensors of its arguments, kTensors at most, one tile of
// kTile elements a workgroup, whichever tensor it lies in.
//
// States of 8 bits.  A block of kStateBlock elements shares a scale for m and one
// for r = sqrt(v), powers of two that put the block's largest in [2^7, 2^8).
// m takes a sign, 4 bits of exponent and 3 below the leading one; r, which has
// no sign, 4 and 4: values from 2^-6 on in full, below in steps of 2^-9 (2^-10),
// which is 2^-17 (2^-18) of the block's largest.  r and not v, since 18 bits of
// range of r are 36 of v; and a value of r above 0 stays above 0, so that no
// element ever divides by eps alone.  Values are rounded at random, up as often as
// they are near to the upper one: what b2 = 0.999 adds to r in a step is a
// hundredth of a step of its 8 bits, which rounding to nearest would drop
// for good.  The random bits are a hash of seed, tensor, step and element.
#include "rows.hpp"
#include "launch.hpp"

#include <math.h>

namespace efs {

namespace {

constexpr int kTensors = 64;           // of one launch: 3.6 KB of arguments
constexpr int kTiles = kTile / (kBlock * 4);
constexpr int kStateBlock = kAdamwBlock;
static_assert(kStateBlock == kWave * 4, "a wave holds a block of a state");

struct Tensor {
    const void *g;
    float *x;
    void *m, *v;
    __bf16 *copy;
    int32_t size;
    float decay;
    uint32_t ordinal;     // in the caller's list
    uint32_t first;       // tile
};

// What a step multiplies by.
struct Rates {
    float b1, c1, b2, c2, alpha, root, eps, gain;   // gain: of g
    double gamma;                                   // 1 - gamma decay is a tensor's own
    uint32_t key;                                   // of the random bits, before the tensor's ordinal
};

struct Step {
    Tensor tensor[kTensors];
    Rates rates;
    const int64_t *step;      // on the device, NULL: rates are complete
    const float *factors;     // on the device, may be NULL
    int64_t given;            // the step where it is not on the device
    float gamma;
    uint32_t seed;
    int32_t count;
};

// b^t by squaring, in binary64.
__host__ __device__ inline double power(double b, int64_t t) {
    double p = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) p *= b;
    return p;
}

// The rates of a step; the same operations on the host and on the device.
__host__ __device__ inline void set_step(Rates &r, float gamma, float factor, int64_t step, uint32_t seed) {
    r.gamma = double(gamma) * double(factor);
    r.alpha = float(r.gamma / (1.0 - power(double(r.b1), step)));
    r.root = float(1.0 / sqrt(1.0 - power(double(r.b2), step)));
    r.key = seed + uint32_t(step) * 0xA54FF53Bu;   // (the constants here: fractional bits of square roots)
}

__device__ __forceinline__ uint32_t mixed(uint32_t z) {
    z ^= z >> 16;
    z *= 0x6A09E667u;
    z ^= z >> 15;
    z *= 0xBB67AE85u;
    return z ^ (z >> 16);
}

constexpr uint32_t kInfinity = 0x7f800000u, kMagnitude = 0x7fffffffu;
constexpr uint32_t kNanM = 0x7fu, kNanR = 0xffu;

// The code of a magnitude, of kMantissa bits below the leading one and 4 of
// exponent, rounded up with the share `dither` / 2^16; e: the block's exponent,
// magnitudes are below 2^(e + 1).  In full: fp32's own bits, moved and cut ...
template <int kMantissa>
__device__ __forceinline__ uint32_t encode(uint32_t bits, uint32_t dither, int e) {
    return (bits + (dither << (7 - kMantissa)) - (uint32_t(113 + e) << 23)) >> (23 - kMantissa);
}

// ... and below 2^-6 of the scale in steps of its last bit there.
__device__ __forceinline__ uint32_t least_in_full(int e) { return uint32_t(114 + e) << 23; }

template <int kMantissa>
__device__ __forceinline__ uint32_t encode_small(float y, uint32_t dither, float up) {
    return uint32_t(__fadd_rn(__fmul_rn(__fmul_rn(y, up), 0x1p6f * float(1 << kMantissa)), __fmul_rn(float(dither), 0x1p-16f)));
}

__device__ __forceinline__ float two_to(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }

// The exponent of a block's scale from its largest finite magnitude; those below
// 2^-95 are small beside the scale.
__device__ __forceinline__ int scale_exponent(uint32_t largest) { return max(int(largest >> 23) - 127, -95); }

// The largest finite magnitude of a block.
__device__ __forceinline__ uint32_t top_of(const uint32_t (&bits)[4], bool &whole) {
    uint32_t top = wave_max(max(max(bits[0], bits[1]), max(bits[2], bits[3])));
    whole = top < kInfinity;
    if (!whole) {   // (the same for the wave)
        top = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, bits[i] < kInfinity ? bits[i] : 0u);
        top = wave_max(top);
    }
    return top;
}

// One lane's four elements of a block: its m and r >= 0 into codes; the block's
// scales.  What few blocks have (NaN, infinities, values that are small beside the
// scale) is left to branches that the whole wave takes or not.
__device__ __forceinline__ void pack_block(const float (&m)[4], const float (&r)[4], const uint32_t (&random)[4],
                                           uint32_t &m_codes, uint32_t &r_codes, float &m_scale, float &r_scale) {
    uint32_t mb[4], rb[4], c[4], d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) mb[i] = __float_as_uint(m[i]) & kMagnitude, rb[i] = __float_as_uint(r[i]);
    bool whole_m, whole_r;
    const int em = scale_exponent(top_of(mb, whole_m)), er = scale_exponent(top_of(rb, whole_r));
    m_scale = two_to(em - 7), r_scale = two_to(er - 7);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c[i] = encode<3>(mb[i], random[i] & 0xffffu, em);
        d[i] = encode<4>(rb[i], random[i] >> 16, er);
    }
    const uint32_t least_m = least_in_full(em), least_r = least_in_full(er);
    if (__any(min(min(mb[0], mb[1]), min(mb[2], mb[3])) < least_m)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t small = encode_small<3>(fabsf(m[i]), random[i] & 0xffffu, two_to(7 - em));
            c[i] = mb[i] < least_m ? small : c[i];
        }
    }
    if (__any(min(min(rb[0], rb[1]), min(rb[2], rb[3])) < least_r)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t small = max(encode_small<4>(r[i], random[i] >> 16, two_to(7 - er)), rb[i] != 0u ? 1u : 0u);
            d[i] = rb[i] < least_r ? small : d[i];
        }
    }
    if (!whole_m || !whole_r) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = mb[i] < kInfinity ? c[i] : kNanM;
            d[i] = rb[i] < kInfinity ? d[i] : kNanR;
        }
    }
    m_codes = r_codes = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m_codes |= (c[i] | ((__float_as_uint(m[i]) >> 24) & 0x80u)) << (8 * i);
        r_codes |= d[i] << (8 * i);
    }
}

// The values of a lane's four codes.  Those of m are the 8-bit floats of 4 and 3
// bits that the hardware knows.
__device__ __forceinline__ void values_of_m(uint32_t codes, float scale, float (&m)[4]) {
    m[0] = __builtin_amdgcn_cvt_f32_fp8(int(codes), 0);
    m[1] = __builtin_amdgcn_cvt_f32_fp8(int(codes), 1);
    m[2] = __builtin_amdgcn_cvt_f32_fp8(int(codes), 2);
    m[3] = __builtin_amdgcn_cvt_f32_fp8(int(codes), 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = __fmul_rn(m[i], scale);
}

// Those of r as fp32's own exponent and mantissa bits, 2^120 too small; there also
// the small ones are right, as subnormals.
__device__ __forceinline__ void values_of_r(uint32_t codes, float scale, float (&r)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t bits = (i < 3 ? codes << (19 - 8 * i) : codes >> 5) & (0xffu << 19);
        const float v = __fmul_rn(__uint_as_float(bits), 0x1p120f);
        r[i] = __fmul_rn(v > 256.0f ? NAN : v, scale);   // (kNanR; no other code is above 256)
    }
}

// The step of one element; returns the new x.
__device__ __forceinline__ float advance(const Rates &c, float keep, float g, float x, float &m, float &v) {
    m = __fadd_rn(__fmul_rn(c.b1, m), __fmul_rn(c.c1, g));
    v = __fadd_rn(__fmul_rn(c.b2, v), __fmul_rn(__fmul_rn(c.c2, g), g));
    const float den = __fadd_rn(__fmul_rn(sqrtf(v), c.root), c.eps);
    return __fsub_rn(__fmul_rn(x, keep), __fmul_rn(c.alpha, m / den));
}

// The tensor in which a tile lies, of those of the arguments.
template <typename List>
__device__ __forceinline__ int tensor_of(const List &a, uint32_t tile) {
    int lo = 0, hi = a.count;   // the last whose first tile is at or before it
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.tensor[mid].first <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename G, bool kBytes, bool kDevice>
__global__ __launch_bounds__(kBlock) void adamw_kernel(const Step a) {
    const Tensor t = a.tensor[tensor_of(a, blockIdx.x)];
    const int64_t tile0 = int64_t(blockIdx.x - t.first) * kTile;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int blocks = (t.size + kStateBlock - 1) / kStateBlock;
    const G *g = static_cast<const G *>(t.g);

    // a wave's share is kTiles blocks of 256 elements, four of a lane's each
    float gv[kTiles][4], xv[kTiles][4], mv[kTiles][4], vv[kTiles][4];
    int left[kTiles];
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
        const int block = int(tile0 / kStateBlock) + wave * kTiles + k;
        const int64_t at = int64_t(block) * kStateBlock + lane * 4;
        left[k] = int(min(int64_t(4), t.size - at));
#pragma unroll
        for (int i = 0; i < 4; ++i) gv[k][i] = xv[k][i] = mv[k][i] = vv[k][i] = 0.0f;
        if (kBytes && block < blocks) {
            const uint8_t *m8 = static_cast<const uint8_t *>(t.m), *r8 = static_cast<const uint8_t *>(t.v);
            const uint32_t mc = *reinterpret_cast<const uint32_t *>(m8 + at), rc = *reinterpret_cast<const uint32_t *>(r8 + at);
            values_of_m(mc, reinterpret_cast<const float *>(m8 + int64_t(blocks) * kStateBlock)[block], mv[k]);
            values_of_r(rc, reinterpret_cast<const float *>(r8 + int64_t(blocks) * kStateBlock)[block], vv[k]);
#pragma unroll
            for (int i = 0; i < 4; ++i) vv[k][i] = __fmul_rn(vv[k][i], vv[k][i]);
        }
        if (left[k] > 0) {
            load_pack<4>(g + at, left[k], gv[k]);
            load_pack<4>(t.x + at, left[k], xv[k]);
            if (!kBytes) {
                load_pack<4>(static_cast<const float *>(t.m) + at, left[k], mv[k]);
                load_pack<4>(static_cast<const float *>(t.v) + at, left[k], vv[k]);
            }
        }
    }

    Rates c = a.rates;
    if (kDevice) {   // the step's rates are computed by one wave, beside the loads
        __shared__ Rates s_rates;
        if (wave == 0) {
            const int64_t step = a.step != nullptr ? *a.step : a.given;
            if (a.factors != nullptr) c.gain = a.factors[1];
            set_step(c, a.gamma, a.factors != nullptr ? a.factors[0] : 1.0f, step < 1 ? 1 : step, a.seed);
            if (lane == 0) s_rates = c;
        }
        __syncthreads();
        c = s_rates;
    }
    const float keep = float(1.0 - c.gamma * double(t.decay));
    const uint32_t key = mixed(c.key + t.ordinal * 0x3C6EF373u);

#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
        const int block = int(tile0 / kStateBlock) + wave * kTiles + k;
        const int64_t at = int64_t(block) * kStateBlock + lane * 4;
        if (block >= blocks) break;   // the whole wave's
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (kDevice) gv[k][i] = __fmul_rn(gv[k][i], c.gain);
            xv[k][i] = advance(c, keep, gv[k][i], xv[k][i], mv[k][i], vv[k][i]);
        }
        if (kBytes) {
            uint32_t random[4], mc, rc;
            float r[4], ms, rs;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                random[i] = mixed((uint32_t(at + i) * 0x9E3779B1u) ^ key);
                const bool in = i < left[k];   // what lies behind the tensor is zero
                mv[k][i] = in ? mv[k][i] : 0.0f;
                r[i] = in ? sqrtf(vv[k][i]) : 0.0f;
            }
            pack_block(mv[k], r, random, mc, rc, ms, rs);
            uint8_t *m8 = static_cast<uint8_t *>(t.m), *r8 = static_cast<uint8_t *>(t.v);
            *reinterpret_cast<uint32_t *>(m8 + at) = mc;
            *reinterpret_cast<uint32_t *>(r8 + at) = rc;
            if (lane == 0) {
                reinterpret_cast<float *>(m8 + int64_t(blocks) * kStateBlock)[block] = ms;
                reinterpret_cast<float *>(r8 + int64_t(blocks) * kStateBlock)[block] = rs;
            }
        }
        if (left[k] <= 0) continue;
        store_pack<4>(t.x + at, left[k], xv[k]);
        if (t.copy != nullptr) store_pack<4>(t.copy + at, left[k], xv[k]);
        if (!kBytes) {
            store_pack<4>(static_cast<float *>(t.m) + at, left[k], mv[k]);
            store_pack<4>(static_cast<float *>(t.v) + at, left[k], vv[k]);
        }
    }
}

// States of 8 bits from values of 32 and back: what a program does when it saves
// or loads them.
struct StateTensor {
    float *m, *v;
    void *m8, *v8;
    int32_t size;
    uint32_t first;
};

struct States {
    StateTensor tensor[kTensors];
    int32_t count;
};

template <bool kWrite>
__global__ __launch_bounds__(kBlock) void adamw_state_kernel(const States a) {
    const StateTensor t = a.tensor[tensor_of(a, blockIdx.x)];
    const int64_t tile0 = int64_t(blockIdx.x - t.first) * kTile;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int blocks = (t.size + kStateBlock - 1) / kStateBlock;
    uint8_t *m8 = static_cast<uint8_t *>(t.m8), *r8 = static_cast<uint8_t *>(t.v8);
    float *m_scale = reinterpret_cast<float *>(m8 + int64_t(blocks) * kStateBlock);
    float *r_scale = reinterpret_cast<float *>(r8 + int64_t(blocks) * kStateBlock);
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
        const int block = int(tile0 / kStateBlock) + wave * kTiles + k;
        const int64_t at = int64_t(block) * kStateBlock + lane * 4;
        const int left = int(min(int64_t(4), t.size - at));
        if (block >= blocks) break;
        if (kWrite) {   // rounded to nearest, ties up
            const uint32_t half[4] = {0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
            float m[4] = {0.0f, 0.0f, 0.0f, 0.0f}, r[4] = {0.0f, 0.0f, 0.0f, 0.0f}, ms, rs;
            uint32_t mc, rc;
            if (left > 0) {
                load_pack<4>(t.m + at, left, m);
                load_pack<4>(t.v + at, left, r);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = sqrtf(r[i]);
            pack_block(m, r, half, mc, rc, ms, rs);
            *reinterpret_cast<uint32_t *>(m8 + at) = mc;
            *reinterpret_cast<uint32_t *>(r8 + at) = rc;
            if (lane == 0) m_scale[block] = ms, r_scale[block] = rs;
        } else if (left > 0) {
            const uint32_t mc = *reinterpret_cast<const uint32_t *>(m8 + at), rc = *reinterpret_cast<const uint32_t *>(r8 + at);
            float m[4], v[4];
            values_of_m(mc, m_scale[block], m);
            values_of_r(rc, r_scale[block], v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __fmul_rn(v[i], v[i]);
            store_pack<4>(t.m + at, left, m);
            store_pack<4>(t.v + at, left, v);
        }
    }
}

uint32_t tiles_of(int64_t size) { return uint32_t((size + kTile - 1) / kTile); }

template <typename G>
void step(const Step &a, uint32_t tiles, bool bytes, bool device, hipStream_t stream) {
    if (bytes && device) adamw_kernel<G, true, true><<<tiles, kBlock, 0, stream>>>(a);
    else if (bytes) adamw_kernel<G, true, false><<<tiles, kBlock, 0, stream>>>(a);
    else if (device) adamw_kernel<G, false, true><<<tiles, kBlock, 0, stream>>>(a);
    else adamw_kernel<G, false, false><<<tiles, kBlock, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs &c, hipStream_t stream) {
    Step a;
    a.rates.b1 = c.beta1, a.rates.c1 = float(1.0 - double(c.beta1));
    a.rates.b2 = c.beta2, a.rates.c2 = float(1.0 - double(c.beta2));
    a.rates.eps = c.eps, a.rates.gain = 1.0f;
    a.step = c.step_device, a.factors = c.factors, a.gamma = c.gamma, a.seed = c.seed;
    a.given = c.step;
    const bool device = c.step_device != nullptr || c.factors != nullptr;
    set_step(a.rates, c.gamma, 1.0f, c.step, c.seed);
    for (int32_t i = 0; i < c.count;) {
        uint32_t tiles = 0;
        for (a.count = 0; i < c.count && a.count < kTensors; ++i) {
            if (c.size[i] == 0) continue;
            Tensor &t = a.tensor[a.count++];
            t.g = c.g[i], t.x = c.x[i], t.m = c.m[i], t.v = c.v[i];
            t.copy = c.copy != nullptr ? static_cast<__bf16 *>(c.copy[i]) : nullptr;
            t.size = int32_t(c.size[i]), t.decay = c.decay != nullptr ? c.decay[i] : 0.0f;
            t.ordinal = uint32_t(i), t.first = tiles;
            tiles += tiles_of(t.size);
        }
        if (a.count == 0) break;
        if (c.bf16) step<__bf16>(a, tiles, c.bytes, device, stream);
        else step<float>(a, tiles, c.bytes, device, stream);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

size_t adamw_state_size(int64_t size) {
    const int64_t blocks = (size + kStateBlock - 1) / kStateBlock;
    return size_t(blocks) * (kStateBlock + sizeof(float));
}

hipError_t launch_adamw_state(bool write, float *const *m, float *const *v, void *const *m8, void *const *v8,
                              const int64_t *size, int32_t count, hipStream_t stream) {
    States a;
    for (int32_t i = 0; i < count;) {
        uint32_t tiles = 0;
        for (a.count = 0; i < count && a.count < kTensors; ++i) {
            if (size[i] == 0) continue;
            a.tensor[a.count++] = StateTensor{m[i], v[i], m8[i], v8[i], int32_t(size[i]), tiles};
            tiles += tiles_of(size[i]);
        }
        if (a.count == 0) break;
        if (write) adamw_state_kernel<true><<<tiles, kBlock, 0, stream>>>(a);
        else adamw_state_kernel<false><<<tiles, kBlock, 0, stream>>>(a);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace efs
