// The AdamW update with both moments in 8 bits.
//
//   x = f g,  m = b1 m + (1 - b1) x,  v = b2 v + (1 - b2) (x x),  w -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay w)
//
// m and v are codes with a power of two for every 64 elements (include/alch.h has the formats).  A power of two makes the division by the
// scale exact, so that a code is what fp32 arithmetic and 16 random bits say, bit for bit.  Rounding is stochastic: v changes by
// 1 - b2 (0.1 to 5 %) of itself a step and codes are 6 to 12 % apart, so that the nearest code would be the old one for ever.  v has no
// sign and spends that bit on its exponent: the square roots that the update divides by span 2^15 in a block besides the eight smallest
// codes, where four bits of exponent would leave 2^7.
//
// Bound by memory: 16 bytes an element with a master copy (28 with fp32 moments).  The random bits are computed, 14 operations an
// element, not read.  218 M elements with master copies: 607 us, 5.8 TB/s (1.9 times less than with fp32 moments at a copy's rate).  In bf16 without
// master copies there are 10 bytes an element for the same arithmetic, and the vector units bound it: 67 M elements 140 us, 4.8 TB/s.
#include <algorithm>
#include <float.h>
#include <math.h>

#include "chunk_table.h"
#include "kernels.h"

namespace alch {

static constexpr int kBlock = ALCH_ADAMW8_BLOCK;
// Elements of a chunk.  A work-group's look for its chunk is 150 instructions of each wavefront, which several rounds share.
static constexpr int kChunk = 4096;

typedef float f32x4_a __attribute__((ext_vector_type(4)));
typedef float f32x2_a __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4_a __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_a __attribute__((ext_vector_type(4)));

// Pointers out of the table: without the address space they would be flat ones, whose loads also wait for LDS.
template <typename T> using Global = __attribute__((address_space(1))) T*;
template <typename T>
__device__ __forceinline__ Global<T> global(T* p) { return (Global<T>)p; }

struct Adamw8Args {
    const alch_adamw8_tensor* tensors;
    int n;
    float lr, c1, c2;           // 1 / (1 - b1^step), sqrt(1 / (1 - b2^step))
    float b1, b2, d1, d2, eps;  // d = 1 - b
    double beta1, beta2;        // for a step that is known on the device only
    uint32_t seed, step;
    const float *schedule, *grad_factor;
};
struct Rates {
    float factor, lr, c1, c2;
    uint32_t key;
};

__host__ __device__ inline double correction(double beta, double step) { return 1.0 / (1.0 - pow(beta, step)); }  // (as in the update with fp32 moments)

__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

// kPer consecutive elements, of which n are there; kFull: all of them.
typedef __bf16 bf16x8_a __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2_a __attribute__((ext_vector_type(2)));
template <bool kFull, int kPer>
__device__ __forceinline__ void load(Global<const float> p, int n, float (&x)[kPer]) {
    if constexpr (kFull) {
#pragma unroll
        for (int k = 0; k < kPer; k += 4) {
            const f32x4_a v = __builtin_nontemporal_load((Global<const f32x4_a>)(p + k));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[k + e] = v[e];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = e < n ? p[e] : 0.f;
}
template <bool kFull, int kPer>
__device__ __forceinline__ void load(Global<const __bf16> p, int n, float (&x)[kPer]) {
    if constexpr (kFull && kPer == 8) {
        const bf16x8_a v = __builtin_nontemporal_load((Global<const bf16x8_a>)p);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
        return;
    } else if constexpr (kFull) {
        const bf16x4_a v = __builtin_nontemporal_load((Global<const bf16x4_a>)p);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (float)v[e];
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = e < n ? (float)p[e] : 0.f;
}
template <bool kFull, int kPer>
__device__ __forceinline__ void store(Global<float> p, const float (&x)[kPer], int n) {
    if constexpr (kFull) {
#pragma unroll
        for (int k = 0; k < kPer; k += 4) __builtin_nontemporal_store(f32x4_a{x[k], x[k + 1], x[k + 2], x[k + 3]}, (Global<f32x4_a>)(p + k));
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) p[e] = x[e];
}
template <bool kFull, int kPer>
__device__ __forceinline__ void store(Global<__bf16> p, const float (&x)[kPer], int n) {
    if constexpr (kFull && kPer == 8) {
        bf16x8_a v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
        __builtin_nontemporal_store(v, (Global<bf16x8_a>)p);
        return;
    } else if constexpr (kFull) {
        __builtin_nontemporal_store(bf16x4_a{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]}, (Global<bf16x4_a>)p);
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) p[e] = (__bf16)x[e];
}
template <bool kFull, int kPer>
__device__ __forceinline__ void load_codes(Global<const uint8_t> p, int n, uint32_t (&w)[kPer / 4]) {
    if constexpr (kFull && kPer == 8) {
        const u32x2_a v = __builtin_nontemporal_load((Global<const u32x2_a>)p);
        w[0] = v[0];
        w[1] = v[1];
        return;
    } else if constexpr (kFull) {
        w[0] = __builtin_nontemporal_load((Global<const uint32_t>)p);
        return;
    }
#pragma unroll
    for (int k = 0; k < kPer / 4; ++k) w[k] = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) w[e / 4] |= (uint32_t)p[e] << (8 * (e & 3));
}
template <bool kFull, int kPer>
__device__ __forceinline__ void store_codes(Global<uint8_t> p, const uint32_t (&w)[kPer / 4], int n) {
    if constexpr (kFull && kPer == 8) {
        __builtin_nontemporal_store(u32x2_a{w[0], w[1]}, (Global<u32x2_a>)p);
        return;
    } else if constexpr (kFull) {
        __builtin_nontemporal_store(w[0], (Global<uint32_t>)p);
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) p[e] = (uint8_t)(w[e / 4] >> (8 * (e & 3)));
}

__device__ __forceinline__ float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_bits(float f) { return __builtin_bit_cast(uint32_t, f); }
__device__ __forceinline__ float scale_of(uint32_t byte) { return byte == 255u ? __builtin_nanf("") : as_float(byte << 23); }
__device__ __forceinline__ f32x4_a from_m(uint32_t codes) {
    const f32x2_a a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    return f32x4_a{a[0], a[1], b[0], b[1]};
}
// 2^-112 times the codes' values (those below 8 are denormal numbers here).
__device__ __forceinline__ f32x4_a from_v(uint32_t codes) {
    constexpr uint32_t kMask = 0x0ff00000u;
    return f32x4_a{as_float(codes << 20 & kMask), as_float(codes << 12 & kMask), as_float(codes << 4 & kMask), as_float(codes >> 4 & kMask)};
}

// y >= 0 (its bits, and itself) as a code in the byte above bit 20 whose smallest normal value is 2^kLowest: 3 bits of mantissa, rounded up where the
// 20 bits behind them and the random ones carry.  Below 2^kLowest the codes are as far apart as in the next binade, and y is moved there
// by adding 2^kLowest; of the two readings the right one is the larger (they meet at 2^kLowest, where the slopes of bits over value cross).
template <int kLowest>
__device__ __forceinline__ uint32_t to_code(float y, uint32_t random16) {
    constexpr float kSmall = kLowest == -6 ? 0x1p-6f : 0x1p-14f;
    constexpr uint32_t kBias = (uint32_t)(126 + kLowest) << 23;
    static_assert(kLowest == -6 || kLowest == -14, "");
    const uint32_t bits = max(as_bits(y), as_bits(y + kSmall) - (8u << 20));
    return (bits + ((random16 << 4) - kBias)) >> 20;
}
__device__ __forceinline__ uint32_t bytes4(const u32x4_a& c, uint32_t select) {  // the byte that select names of each
    const uint32_t low = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u + select * 0x0101u), high = __builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400u + select * 0x0101u);
    return __builtin_amdgcn_perm(high, low, 0x05040100u);
}

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, kCtrl, 0xf, 0xf, false);
    return v > o ? v : o;
}
template <int kPer>
__device__ __forceinline__ uint32_t max_of_block(uint32_t v) {  // over the lanes that share one: 16 of four elements, 8 of eight
    v = dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v)));
    return kPer == 4 ? dpp_max<0x140>(v) : v;
}

// The scale byte of a block whose largest magnitude has these bits, its largest value going to 2^kAbove and more.
template <int kAbove>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    const int exponent = (int)(most >> 23);
    return exponent == 255 ? 255u : (uint32_t)max(exponent - kAbove, 1);
}
__device__ __forceinline__ float inverse(uint32_t byte) { return as_float((254u - min(byte, 253u)) << 23); }

// sqrt(v) and the quotient of the update are the instructions', one unit in the last place each: the step is off by 0.89 units of 2^-24 of itself (root
// mean square; 3.7 at most), by 0.73 (2.8) with sqrtf and a division, which take 660 us for 607 (218 M elements with master copies), 160 for 138 (67 M
// in bf16 alone).  Moments and their codes have no part in it.
// The root takes denormal numbers for 0, so that where a wavefront has numbers near them these are moved.
template <int kPer>
__device__ __forceinline__ void root(const float (&v)[kPer], float (&r)[kPer]) {
    constexpr uint32_t kNear = 0x10000000u;  // 2^-95
    uint32_t least = 0xffffffffu;
#pragma unroll
    for (int e = 0; e < kPer; ++e) least = min(least, as_bits(v[e]) - 1u);  // (0 is no such number)
    if (__builtin_expect(__any(least < kNear), 0)) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) r[e] = v[e] < as_float(kNear) ? __builtin_amdgcn_sqrtf(v[e] * 0x1p64f) * 0x1p-32f : __builtin_amdgcn_sqrtf(v[e]);
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) r[e] = __builtin_amdgcn_sqrtf(v[e]);
}

// What all tensors of a call are, if they are alike: a kernel of its own has the registers of that form alone.
enum Kind { kAny, kBf16, kBf16Master, kF32 };

// A round of 256 * kPer elements.  Eight elements a lane share more of what a block takes; where fp32 is read beside them its loads then leave
// every other 16 bytes to the next one, so that they pay for bf16 alone (67 M elements without master copies: 146 us with four, 140 with eight).
template <typename T, bool kMaster, int kPer, bool kFull>
__device__ __forceinline__ void adamw8(const alch_adamw8_tensor& t, long long begin, int elements, const Adamw8Args& a, const Rates& r) {
#pragma clang fp contract(off)
    constexpr int kWords = kPer / 4;
    const int own = threadIdx.x * kPer, n = kFull ? kPer : min(max(elements - own, 0), kPer);
    const long long at = begin + own, block = begin / kBlock + own / kBlock;  // (begin is a multiple of a block)
    const bool there = kFull || (own & ~(kBlock - 1)) < elements;  // some of its block is
    const auto grad = global(static_cast<const T*>(t.grad)) + at;
    const auto param = global(static_cast<T*>(t.param)) + at;
    const auto master = global(t.master) + at;
    const auto mp = global(t.m) + at, vp = global(t.v) + at;
    const auto msp = global(t.m_scale) + block, vsp = global(t.v_scale) + block;
    float g[kPer], w[kPer], m[kPer], v[kPer];
    uint32_t mc[kWords], vc[kWords], ms = 0, vs = 0;
    load<kFull>((Global<const T>)grad, n, g);
    if constexpr (kMaster) load<kFull>((Global<const float>)master, n, w);
    else load<kFull>((Global<const T>)param, n, w);
    load_codes<kFull, kPer>((Global<const uint8_t>)mp, n, mc);
    load_codes<kFull, kPer>((Global<const uint8_t>)vp, n, vc);
    if (there) {
        ms = *msp;
        vs = *vsp;
    }
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        const f32x4_a x = from_m(mc[k]), y = from_v(vc[k]);
#pragma unroll
        for (int e = 0; e < 4; ++e) m[4 * k + e] = x[e], v[4 * k + e] = y[e];
    }
    // b1 m and b2 v.  A power of two and a beta as one factor round as one after the other do, unless the factor leaves the normal numbers: for m with scale
    // bytes of 1 (of blocks that are 0, mostly), for betas below a half with some more, for v with a beta below 2^-112, and beyond 2^30.
    float fm, fv = as_float((vs + 112u) << 23) * a.b2;
    if (vs == 0u) fv = 0.f;
    if (vs == 255u) fv = __builtin_nanf("");
    const float sm = scale_of(ms);
    fm = sm * a.b1;
    uint32_t codes = 0;
#pragma unroll
    for (int k = 0; k < kWords; ++k) codes |= mc[k];
    const float low_m = a.b1 > 0.f ? 0x1p-126f : 0.f, low_v = a.b2 > 0.f ? 0x1p-126f : 0.f;  // (0 times anything is 0)
    if (__builtin_expect(__any((fm < low_m && codes != 0u) || (fv < low_v && vs != 0u) || (vs > 142u && vs != 255u)), 0)) {
        const float sv = scale_of(vs);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            m[e] = m[e] * sm * a.b1;
            v[e] = v[e] * 0x1p112f * sv * a.b2;
        }
        fm = fv = 1.f;
    }
    uint32_t most_m = 0, most_v = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const float x = g[e] * r.factor;
        m[e] = m[e] * fm + x * a.d1;
        v[e] = v[e] * fv + x * x * a.d2;
        if (!kFull && e >= n) m[e] = v[e] = 0.f;  // (behind the tensor; a block that is NaN would make these NaN too)
        most_m = max(most_m, as_bits(m[e]) & 0x7fffffffu);
        most_v = max(most_v, as_bits(v[e]));
    }
    // (a v that is NaN may have its sign bit set)
    const uint32_t nms = scale_byte<7>(max_of_block<kPer>(most_m)), nvs = scale_byte<15>(max_of_block<kPer>(most_v) & 0x7fffffffu);
    const float im = inverse(nms), iv = inverse(nvs);
    const unsigned long long first = (unsigned long long)(t.first + at);
    const uint32_t upper = (uint32_t)((unsigned long long)(t.first + begin) >> 32);
    uint32_t random[kPer];
    if (__builtin_expect((uint32_t)((unsigned long long)(t.first + begin + 256 * kPer - 1) >> 32) == upper, 1)) {
        const uint32_t key = (uint32_t)__builtin_amdgcn_readfirstlane((int)mix(r.key ^ upper));
#pragma unroll
        for (int e = 0; e < kPer; ++e) random[e] = mix((uint32_t)first + e + key);
    } else {  // the numbers' upper half changes among these
#pragma unroll
        for (int e = 0; e < kPer; ++e) random[e] = mix((uint32_t)(first + e) + mix(r.key ^ (uint32_t)((first + e) >> 32)));
    }
    uint32_t nm[kWords], nv[kWords], zero = 0;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        u32x4_a cm, cv, ym;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float y = m[4 * k + e] * im;
            ym[e] = as_bits(y);
            cm[e] = to_code<-6>(fabsf(y), random[4 * k + e] & 0xffffu);
            cv[e] = to_code<-14>(v[4 * k + e] * iv, random[4 * k + e] >> 16);
        }
        nm[k] = bytes4(cm, 0) | (bytes4(ym, 3) & 0x80808080u);
        nv[k] = bytes4(cv, 0);
        zero |= (nv[k] - 0x01010101u) & ~nv[k] & 0x80808080u;  // (whether a byte is 0)
    }
    if (__builtin_expect(__any(zero), 0)) {  // 0 for 0 alone
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (v[e] > 0.f && (nv[e / 4] >> (8 * (e & 3)) & 0xffu) == 0u) nv[e / 4] |= 1u << (8 * (e & 3));
    }
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        if (nms == 255u) nm[k] = 0x7f7f7f7fu;
        if (nvs == 255u) nv[k] = 0xffffffffu;
    }
    store_codes<kFull, kPer>(mp, nm, n);
    store_codes<kFull, kPer>(vp, nv, n);
    if (there && (own & (kBlock - 1)) == 0) {
        *msp = (uint8_t)nms;
        *vsp = (uint8_t)nvs;
    }
    float q[kPer];
    root(v, q);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const float change = m[e] * r.c1 * __builtin_amdgcn_rcpf(fmaf(q[e], r.c2, a.eps));
        w[e] = fmaf(-r.lr, fmaf(t.weight_decay, w[e], change), w[e]);
    }
    if constexpr (kMaster) store<kFull>(master, w, n);
    store<kFull>(param, w, n);
}
// A chunk by rounds.  Where the tensor ends in a round, the wavefronts before that end take their elements whole (434 bf16 adapters of 2944 elements and more:
// 13.7 us, 19.3 with every wavefront element by element).
template <typename T, bool kMaster, int kPer = 4>
__device__ __forceinline__ void adamw8_chunk(const alch_adamw8_tensor& t, long long begin, const Adamw8Args& a, const Rates& r) {
    constexpr int kRound = 256 * kPer, kWave = 64 * kPer;
    const int left = (int)min((long long)t.n - begin, (long long)kChunk), before = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * kWave;
    if (left == kChunk) {
#pragma unroll 1
        for (int at = 0; at < kChunk; at += kRound) adamw8<T, kMaster, kPer, true>(t, begin + at, kRound, a, r);
        return;
    }
#pragma unroll 1
    for (int at = 0; at < left; at += kRound) {
        const int own = left - at - before;
        if (own >= kWave) adamw8<T, kMaster, kPer, true>(t, begin + at, kRound, a, r);
        else if (own > 0) adamw8<T, kMaster, kPer, false>(t, begin + at, min(kRound, left - at), a, r);
    }
}

template <bool kFew, Kind kKind>
__global__ __launch_bounds__(256) void k_adamw8(Adamw8Args a) {
    __shared__ int first[kFew ? 1 : kMaxTensors + 1];
    __shared__ float shared_c[3];
    const float factor = a.grad_factor ? *a.grad_factor : 1.f;
    if (!(fabsf(factor) < INFINITY)) return;            // (the gradients are of no use: nothing changes)
    if (a.schedule && !(a.schedule[1] >= 1.f)) return;  // (nor is this a step)
    if (a.schedule && threadIdx.x == 0) {
        const double step = a.schedule[1];
        shared_c[0] = a.schedule[0];
        shared_c[1] = (float)correction(a.beta1, step);
        shared_c[2] = (float)sqrt(correction(a.beta2, step));
    }
    const ChunkTable<alch_adamw8_tensor, kFew> table(a.tensors, a.n, [](int) { return kChunk; }, first);
    if (a.schedule) __syncthreads();  // (its rates have been written)
    const uint32_t step = a.schedule ? (uint32_t)(unsigned long long)a.schedule[1] : a.step;
    const Rates r{factor, a.schedule ? shared_c[0] : a.lr, a.schedule ? shared_c[1] : a.c1, a.schedule ? shared_c[2] : a.c2, mix(a.seed ^ mix(step))};
    for (int c = blockIdx.x; c < table.chunks; c += gridDim.x) {
        const auto k = table.find(c);
        const long long begin = (long long)k.index * kChunk;
        if constexpr (kKind == kBf16) adamw8_chunk<__bf16, false, 8>(k.t, begin, a, r);
        else if constexpr (kKind == kBf16Master) adamw8_chunk<__bf16, true>(k.t, begin, a, r);
        else if constexpr (kKind == kF32) adamw8_chunk<float, false>(k.t, begin, a, r);
        else if (k.t.dtype == ALCH_BF16) {
            if (k.t.master) adamw8_chunk<__bf16, true>(k.t, begin, a, r);
            else adamw8_chunk<__bf16, false>(k.t, begin, a, r);
        } else {
            if (k.t.master) adamw8_chunk<float, true>(k.t, begin, a, r);
            else adamw8_chunk<float, false>(k.t, begin, a, r);
        }
    }
}

template <bool kFew>
static void (*kernel_of(Kind kind))(Adamw8Args) {
    return kind == kBf16 ? k_adamw8<kFew, kBf16> : kind == kBf16Master ? k_adamw8<kFew, kBf16Master> : kind == kF32 ? k_adamw8<kFew, kF32> : k_adamw8<kFew, kAny>;
}

int launch_adamw8(int n_tensors, const alch_adamw8_tensor* tensors, const alch_adamw8_tensor* host, const alch_adamw& p, uint32_t seed,
                  hipStream_t stream) {
    long long chunks = 0;
    double bytes = 0;
    bool kinds[4] = {};
    for (int i = 0; i < n_tensors; ++i) {
        if (host[i].n > 0) kinds[host[i].dtype == ALCH_BF16 ? (host[i].master ? kBf16Master : kBf16) : host[i].master ? kAny : kF32] = true;
        chunks += (host[i].n + kChunk - 1) / kChunk;
        const double E = (double)dtype_size((alch_dtype)host[i].dtype);
        bytes += (double)host[i].n * (2 * E + 4 + 4.0 / kBlock + (host[i].master ? 8 : E));
    }
    if (chunks == 0) return ALCH_OK;
    TraceScope ts(kTraceUpdate, 0.0, bytes, stream);
    const Adamw8Args a{tensors, n_tensors, (float)p.lr, p.schedule ? 0.f : (float)correction(p.beta1, p.step),
                       p.schedule ? 0.f : (float)sqrt(correction(p.beta2, p.step)),
                       (float)p.beta1, (float)p.beta2, (float)(1.0 - p.beta1), (float)(1.0 - p.beta2), p.eps > 0.0 ? std::max((float)p.eps, FLT_MIN) : 0.f,
                       p.beta1, p.beta2, seed, (uint32_t)p.step, p.schedule, p.grad_factor};
    const Kind kind = kinds[kAny] || kinds[kBf16] + kinds[kBf16Master] + kinds[kF32] > 1 ? kAny : kinds[kBf16] ? kBf16 : kinds[kBf16Master] ? kBf16Master : kF32;
    const auto kernel = n_tensors <= 64 ? kernel_of<true>(kind) : kernel_of<false>(kind);
    kernel<<<(int)std::min<long long>(chunks, kMaxChunkBlocks), 256, 0, stream>>>(a);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
