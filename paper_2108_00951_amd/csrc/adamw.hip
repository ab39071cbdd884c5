// AdamW over many tensors at once.
//
//   m = b1 m + (1 - b1) g ;  v = b2 v + ((1 - b2) g) g
//   x = (1 - gamma decay) x - alpha (m / (root sqrt(v) + eps))
//   alpha = gamma / (1 - b1^t) ;  root = 1 / sqrt(1 - b2^t)
//
// each operation rounded to fp32 by itself.  Bytes bound it: 28 of an element
// with states of 32 bits (g, x, m, v in; x, m, v out), 16 with states of 8.  Measured
// on one MI355X: 37 M elements of 161 tensors, 32 bits, 198 us (5.3 TB/s, two
// launches); 134 M, 8 bits, bf16 g and copy (16 bytes an element too) 370 to 440 us
// (5.8 to 4.9 TB/s), where the vector units are busy throughout: 92 instructions an
// element, of which the square root, the division and the hash are half; 97 short
// vectors 5.0 us.
// A launch takes the tensors of its arguments, kTensors at most, one tile of
// kStepTile elements a workgroup, whichever tensor it lies in.
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

constexpr int kTensors = 112;          // of one launch: 3.9 KB of arguments
constexpr int kStateBlock = kAdamwBlock;
static_assert(kStateBlock == kWave * 4, "a wave holds a block of a state");
// Four times as much a workgroup (217 instead of 204 us for 37 M elements of 161
// tensors, 680 instead of 597 for 134 M with states of 8 bits) leaves each wave
// more registers to wait for and the chip fewer waves.
constexpr int kStepTile = kBlock * 4;

constexpr uint32_t kMaxTiles = 1u << 23;   // of one launch, whose threads are counted in 32 bits

// States are read again a step later, after all else has passed the caches.  x and its
// copy may be read sooner; through the caches they gain nothing: a step of 10.5 M elements
// and a pass over the copy behind it 53 us, past the caches 55, of 1 M 9.4 and 9.4, of 42 M
// 257 and 254.
constexpr bool kPast = true;

constexpr int32_t kNone = INT32_MIN;   // no tensor of an optional list

// The tensors of a launch: list l's tensor i starts at[l][i] units of unit[l] bytes
// behind (or before) its first one at base[l], so that a launch holds many.
template <int kLists>
struct Tensors {
    char *base[kLists];
    int32_t unit[kLists];
    int32_t at[kLists][kTensors];
    int32_t size[kTensors];
    uint32_t first[kTensors];     // tile
    int32_t count;
    uint32_t ordinal;             // of the first in the caller's list

    template <typename T>
    __device__ __forceinline__ T *pointer(int list, int i) const {
        return reinterpret_cast<T *>(base[list] + int64_t(at[list][i]) * unit[list]);
    }
};

// The tensor in which a tile lies: the last whose first tile is at or before it
// (one that is empty starts where the next one does).
template <int kLists>
__device__ __forceinline__ int tensor_of(const Tensors<kLists> &a, uint32_t tile) {
    static_assert(kTensors <= 2 * kWave, "two tensors a lane");
    const int lane = threadIdx.x & (kWave - 1);
    int before = int(__popcll(__ballot(lane < a.count && a.first[min(lane, kTensors - 1)] <= tile)));
    if (a.count > kWave)
        before += int(__popcll(__ballot(lane + kWave < a.count && a.first[min(lane + kWave, kTensors - 1)] <= tile)));
    return __builtin_amdgcn_readfirstlane(before - 1);
}

// What a step multiplies by.
struct Rates {
    float b1, c1, b2, c2, alpha, root, eps, gain;   // gain: of g
    double gamma;                                   // 1 - gamma decay is a tensor's own
    uint32_t key;                                   // of the random bits, before the tensor's ordinal
};

enum { kG, kX, kM, kV, kCopy, kStepLists };

struct Step {
    Tensors<kStepLists> tensors;
    float decay[kTensors];
    Rates rates;
    const int64_t *step;      // on the device, NULL: rates are complete
    const float *factors;     // on the device, may be NULL
    int64_t given;            // the step where it is not on the device
    float gamma;
    uint32_t seed;
};
static_assert(sizeof(Step) <= 4096, "a launch's arguments");

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
constexpr uint32_t kTopM = 0x77u, kTopR = 0xefu;   // the largest below 2^8 of the scale

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
    // (the products are exact: the scale and the share are powers of two)
    return uint32_t(fmaf(float(dither), 0x1p-16f, __fmul_rn(y, up * (0x1p6f * float(1 << kMantissa)))));
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
    for (int i = 0; i < 4; ++i) mb[i] = __float_as_uint(m[i]) & kMagnitude, rb[i] = __float_as_uint(r[i]) & kMagnitude;
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
    // up to 2^128, which is infinite, no m is rounded, nor r to 2^64, whose square v is
    if (em == 127 || er == 63) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = em == 127 ? min(c[i], kTopM) : c[i];
            d[i] = er == 63 ? min(d[i], kTopR) : d[i];
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

// A wave's block of 256 elements of a tensor, four of a lane's each, `left` of which
// are there (kWhole: all of the wave's).
template <typename G, bool kBytes, bool kDevice, bool kWhole>
__device__ __forceinline__ void step_block(const Step &a, const Rates &c, int which, int64_t tile0, int left) {
    const Tensors<kStepLists> &t = a.tensors;
    const int lane = threadIdx.x & (kWave - 1), off = threadIdx.x * 4, count = kWhole ? 4 : left;
    const int block = int(tile0 / kStateBlock) + int(threadIdx.x) / kWave;
    const G *g = t.template pointer<const G>(kG, which) + tile0;   // (of the workgroup; off is a thread's)
    float *x = t.template pointer<float>(kX, which) + tile0;
    float *m32 = t.template pointer<float>(kM, which) + tile0, *v32 = t.template pointer<float>(kV, which) + tile0;
    uint8_t *m8 = t.template pointer<uint8_t>(kM, which) + tile0, *r8 = t.template pointer<uint8_t>(kV, which) + tile0;
    // the scales lie behind the codes
    const int64_t scales = (int64_t(t.size[which] - 1) / kStateBlock + 1) * kStateBlock - tile0;
    float *m_scale = reinterpret_cast<float *>(m8 + scales) + block, *r_scale = reinterpret_cast<float *>(r8 + scales) + block;

    float gv[4], xv[4], mv[4], vv[4];
    if (!kWhole)
#pragma unroll
        for (int i = 0; i < 4; ++i) gv[i] = xv[i] = mv[i] = vv[i] = 0.0f;
    if (kBytes) {
        values_of_m(*reinterpret_cast<const uint32_t *>(m8 + off), *m_scale, mv);
        values_of_r(*reinterpret_cast<const uint32_t *>(r8 + off), *r_scale, vv);
#pragma unroll
        for (int i = 0; i < 4; ++i) vv[i] = __fmul_rn(vv[i], vv[i]);
    }
    if (kWhole || left > 0) {
        load_pack<4>(g + off, count, gv);
        load_pack<4>(x + off, count, xv);
        if (!kBytes) {
            load_pack<4>(m32 + off, count, mv);
            load_pack<4>(v32 + off, count, vv);
        }
    }
    const float keep = float(1.0 - c.gamma * double(a.decay[which]));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (kDevice) gv[i] = __fmul_rn(gv[i], c.gain);
        xv[i] = advance(c, keep, gv[i], xv[i], mv[i], vv[i]);
    }
    if (kBytes) {
        const uint32_t key = mixed(c.key + (t.ordinal + uint32_t(which)) * 0x3C6EF373u);
        const uint32_t index = (uint32_t(tile0) + uint32_t(off)) * 0x9E3779B1u;
        uint32_t random[4], mc, rc;
        float r[4], ms, rs;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            random[i] = mixed((index + uint32_t(i) * 0x9E3779B1u) ^ key);
            const bool in = kWhole || i < left;   // what lies behind the tensor is zero
            mv[i] = in ? mv[i] : 0.0f;
            r[i] = in ? sqrtf(vv[i]) : 0.0f;
        }
        pack_block(mv, r, random, mc, rc, ms, rs);
        *reinterpret_cast<uint32_t *>(m8 + off) = mc;
        *reinterpret_cast<uint32_t *>(r8 + off) = rc;
        if (lane == 0) *m_scale = ms, *r_scale = rs;
    }
    if (!kWhole && left <= 0) return;
    store_pack<4>(x + off, count, xv, kPast);
    if (t.at[kCopy][which] != kNone)
        store_pack<4>(t.template pointer<__bf16>(kCopy, which) + tile0 + off, count, xv, kPast);
    if (!kBytes) {
        store_pack<4>(m32 + off, count, mv, kPast);
        store_pack<4>(v32 + off, count, vv, kPast);
    }
}

template <typename G, bool kBytes, bool kDevice>
__global__ __launch_bounds__(kBlock) void adamw_kernel(const Step a) {
    Rates c = a.rates;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    if (kDevice) {   // the step's rates, by one wave
        __shared__ Rates s_rates;
        if (wave == 0) {
            const int64_t step = a.step != nullptr ? *a.step : a.given;
            if (a.factors != nullptr) c.gain = a.factors[1];
            set_step(c, a.gamma, a.factors != nullptr ? a.factors[0] : 1.0f, step < 1 ? 1 : step, a.seed);
            if (threadIdx.x == 0) s_rates = c;
        }
        __syncthreads();
        c = s_rates;
    }
    const int which = tensor_of(a.tensors, blockIdx.x);
    const int64_t tile0 = int64_t(blockIdx.x - a.tensors.first[which]) * kStepTile;
    const int rest = int(min(int64_t(kStepTile), a.tensors.size[which] - tile0));   // of the workgroup's elements
    if (rest >= (wave + 1) * kStateBlock)
        step_block<G, kBytes, kDevice, true>(a, c, which, tile0, 4);
    else if (rest > wave * kStateBlock)
        step_block<G, kBytes, kDevice, false>(a, c, which, tile0, rest - int(threadIdx.x) * 4);
}

// States of 8 bits from values of 32 and back: what a program does when it saves
// or loads them.
enum { kM32, kV32, kM8, kV8, kStateLists };

struct States {
    Tensors<kStateLists> tensors;
};

template <bool kWrite>
__global__ __launch_bounds__(kBlock) void adamw_state_kernel(const States a) {
    const int which = tensor_of(a.tensors, blockIdx.x);
    const int32_t size = a.tensors.size[which], blocks = (size - 1) / kStateBlock + 1;   // (a size may be the largest)
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int block = int(blockIdx.x - a.tensors.first[which]) * kWaves + wave;
    if (block >= blocks) return;
    const int64_t at = int64_t(block) * kStateBlock + lane * 4;
    const int left = int(min(int64_t(4), size - at));
    float *m32 = a.tensors.template pointer<float>(kM32, which) + at, *v32 = a.tensors.template pointer<float>(kV32, which) + at;
    uint8_t *m8 = a.tensors.template pointer<uint8_t>(kM8, which), *r8 = a.tensors.template pointer<uint8_t>(kV8, which);
    float *m_scale = reinterpret_cast<float *>(m8 + int64_t(blocks) * kStateBlock) + block;
    float *r_scale = reinterpret_cast<float *>(r8 + int64_t(blocks) * kStateBlock) + block;
    if (kWrite) {   // rounded to nearest, ties up
        const uint32_t half[4] = {0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
        float m[4] = {}, r[4] = {}, ms, rs;
        uint32_t mc, rc;
        if (left > 0) {
            load_pack<4>(m32, left, m);
            load_pack<4>(v32, left, r);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = sqrtf(r[i]);
        pack_block(m, r, half, mc, rc, ms, rs);
        *reinterpret_cast<uint32_t *>(m8 + at) = mc;
        *reinterpret_cast<uint32_t *>(r8 + at) = rc;
        if (lane == 0) *m_scale = ms, *r_scale = rs;
    } else if (left > 0) {
        float m[4], v[4];
        values_of_m(*reinterpret_cast<const uint32_t *>(m8 + at), *m_scale, m);
        values_of_r(*reinterpret_cast<const uint32_t *>(r8 + at), *r_scale, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __fmul_rn(v[i], v[i]);
        store_pack<4>(m32, left, m, kPast);
        store_pack<4>(v32, left, v, kPast);
    }
}

const void *const *list_of(const void *list) { return static_cast<const void *const *>(list); }

// The next launch's tensors, from tensor i on: as many as fit.  Returns their tiles.
template <int kLists>
uint32_t take(Tensors<kLists> &a, const void *const *const (&lists)[kLists], const int64_t *size, int32_t count, int32_t &i) {
    uint32_t tiles = 0;
    a.ordinal = uint32_t(i);
    for (int l = 0; l < kLists; ++l) a.base[l] = nullptr;
    for (a.count = 0; i < count && a.count < kTensors; ++i, ++a.count) {
        bool fits = true;
        for (int l = 0; l < kLists; ++l) {
            char *p = size[i] > 0 && lists[l] != nullptr ? static_cast<char *>(const_cast<void *>(lists[l][i])) : nullptr;
            a.at[l][a.count] = kNone;
            if (p == nullptr) continue;
            if (a.base[l] == nullptr) a.base[l] = p;
            // (of whole elements: a list is aligned to its type)
            const int64_t far = (p - a.base[l]) / a.unit[l];
            fits = fits && far > INT32_MIN && far <= INT32_MAX && far * a.unit[l] == p - a.base[l];
            a.at[l][a.count] = int32_t(far);
        }
        const uint32_t more = uint32_t((size[i] + kStepTile - 1) / kStepTile);
        if (!fits || (a.count > 0 && tiles + more > kMaxTiles)) break;
        a.size[a.count] = int32_t(size[i]);
        a.first[a.count] = tiles;
        tiles += more;
    }
    return tiles;
}

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
    const int units[kStepLists] = {c.bf16 ? 2 : 4, 4, c.bytes ? 16 : 4, c.bytes ? 16 : 4, 2};
    for (int l = 0; l < kStepLists; ++l) a.tensors.unit[l] = units[l];
    const void *const *const lists[kStepLists] = {c.g, list_of(c.x), list_of(c.m), list_of(c.v), list_of(c.copy)};
    for (int32_t i = 0; i < c.count;) {
        const int32_t from = i;
        const uint32_t tiles = take(a.tensors, lists, c.size, c.count, i);
        for (int32_t k = from; k < i; ++k) a.decay[k - from] = c.decay != nullptr ? c.decay[k] : 0.0f;
        if (tiles == 0) continue;
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
    for (int l = 0; l < kStateLists; ++l) a.tensors.unit[l] = l == kM32 || l == kV32 ? 4 : 16;
    const void *const *const lists[kStateLists] = {list_of(m), list_of(v), list_of(m8), list_of(v8)};
    for (int32_t i = 0; i < count;) {
        const uint32_t tiles = take(a.tensors, lists, size, count, i);
        if (tiles == 0) continue;
        if (write) adamw_state_kernel<true><<<tiles, kBlock, 0, stream>>>(a);
        else adamw_state_kernel<false><<<tiles, kBlock, 0, stream>>>(a);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace efs
