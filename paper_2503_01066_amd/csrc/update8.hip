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
// element, not read.
#include <algorithm>
#include <math.h>

#include "chunk_table.h"
#include "kernels.h"

namespace alch {

static constexpr int kBlock = ALCH_ADAMW8_BLOCK;
static constexpr int kChunk = 1024;  // elements, four a thread: 16 blocks, a block a row of 16 lanes

typedef float f32x4_a __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4_a __attribute__((ext_vector_type(4)));

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

__device__ __forceinline__ f32x4_a load4(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const f32x4_a*>(p)); }
__device__ __forceinline__ f32x4_a load4(const __bf16* p) {
    return __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const bf16x4_a*>(p)), f32x4_a);
}
__device__ __forceinline__ void store4(float* p, f32x4_a v) { __builtin_nontemporal_store(v, reinterpret_cast<f32x4_a*>(p)); }
__device__ __forceinline__ void store4(__bf16* p, f32x4_a v) {
    __builtin_nontemporal_store(__builtin_convertvector(v, bf16x4_a), reinterpret_cast<bf16x4_a*>(p));
}
// Four consecutive elements, of which n are there.
template <typename V, typename T>
__device__ __forceinline__ V load_some(const T* p, int n) {
    V v = {};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) v[e] = p[e];
    return v;
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, f32x4_a v, int n) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) p[e] = (T)v[e];
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n) {
    if (n == 4) return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) w |= (uint32_t)p[e] << (8 * e);
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t w, int n) {
    if (n == 4) {
        __builtin_nontemporal_store(w, reinterpret_cast<uint32_t*>(p));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) p[e] = (uint8_t)(w >> (8 * e));
}

__device__ __forceinline__ float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_bits(float f) { return __builtin_bit_cast(uint32_t, f); }
__device__ __forceinline__ float scale_of(uint32_t byte) { return byte == 255u ? __builtin_nanf("") : as_float(byte << 23); }
// (codes below 8 are denormal numbers here, which the product makes normal)
__device__ __forceinline__ float from_m(uint32_t code) {
    return (code & 0x7fu) == 0x7fu ? __builtin_nanf("") : as_float((code & 0x80u) << 24 | (code & 0x7fu) << 20) * 0x1p120f;
}
__device__ __forceinline__ float from_v(uint32_t code) { return as_float(code << 20) * 0x1p112f; }

// y >= 0 as a code whose smallest normal value is 2^kLowest: 3 bits of mantissa, rounded up where the 20 bits behind them and the random
// ones carry.  Below 2^kLowest the codes are evenly spaced, as they are in the next binade: there the value is moved.
template <int kLowest>
__device__ __forceinline__ uint32_t to_code(float y, uint32_t random16) {
#pragma clang fp contract(off)
    constexpr float kSmall = kLowest == -6 ? 0x1p-6f : 0x1p-14f;
    constexpr uint32_t kBias = (126 + kLowest) * 8;
    static_assert(kLowest == -6 || kLowest == -14, "");
    const bool small = y < kSmall;
    const uint32_t bits = as_bits(small ? y + kSmall : y);
    return ((bits + (random16 << 4)) >> 20) - (small ? kBias + 8 : kBias);
}

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, kCtrl, 0xf, 0xf, false);
    return v > o ? v : o;
}
__device__ __forceinline__ uint32_t max_of_16(uint32_t v) { return dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v)))); }

// The scale byte of a block whose largest magnitude has these bits, its largest value going to 2^kAbove and more.
template <int kAbove>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    const int exponent = (int)(most >> 23);
    return exponent == 255 ? 255u : (uint32_t)max(exponent - kAbove, 1);
}
__device__ __forceinline__ float inverse(uint32_t byte) { return as_float((254u - min(byte, 253u)) << 23); }

template <typename T, bool kMaster>
__device__ __forceinline__ void adamw8(const alch_adamw8_tensor& t, long long begin, int elements, const Adamw8Args& a, const Rates& r) {
#pragma clang fp contract(off)
    const int own = threadIdx.x * 4, n = min(max(elements - own, 0), 4);
    const long long at = begin + own, block = at / kBlock;
    const bool there = (own & ~(kBlock - 1)) < elements;  // some of its block is
    f32x4_a g = {}, w = {};
    uint32_t mc = 0, vc = 0, ms = 0, vs = 0;
    const T* grad = static_cast<const T*>(t.grad) + at;
    T* param = static_cast<T*>(t.param) + at;
    if (n == 4) {
        g = load4(grad);
        if constexpr (kMaster) w = load4(t.master + at);
        else w = load4(param);
    } else if (n > 0) {
        g = load_some<f32x4_a>(grad, n);
        if constexpr (kMaster) w = load_some<f32x4_a>(t.master + at, n);
        else w = load_some<f32x4_a>(param, n);
    }
    if (n > 0) {
        mc = load_codes(t.m + at, n);
        vc = load_codes(t.v + at, n);
    }
    if (there) {
        ms = t.m_scale[block];
        vs = t.v_scale[block];
    }
    const float sm = scale_of(ms), sv = scale_of(vs);
    f32x4_a m, v;
    uint32_t most_m = 0, most_v = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = g[e] * r.factor;
        m[e] = from_m(mc >> (8 * e) & 0xffu) * sm * a.b1 + x * a.d1;
        v[e] = from_v(vc >> (8 * e) & 0xffu) * sv * a.b2 + x * x * a.d2;
        if (e >= n) m[e] = v[e] = 0.f;  // (behind the tensor: a block that is NaN makes these NaN too, which would not matter)
        most_m = max(most_m, as_bits(m[e]) & 0x7fffffffu);
        most_v = max(most_v, as_bits(v[e]) & 0x7fffffffu);
        w[e] -= r.lr * (m[e] * r.c1 / (sqrtf(v[e]) * r.c2 + a.eps) + t.weight_decay * w[e]);
    }
    const uint32_t nms = scale_byte<7>(max_of_16(most_m)), nvs = scale_byte<15>(max_of_16(most_v));
    const float im = inverse(nms), iv = inverse(nvs);
    uint32_t nm = 0, nv = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned long long number = (unsigned long long)(t.first + at + e);
        const uint32_t random = mix((uint32_t)number + ((number >> 32) ? mix(r.key ^ (uint32_t)(number >> 32)) : mix(r.key)));
        const float y = m[e] * im;
        uint32_t c = to_code<-6>(fabsf(y), random & 0xffffu) | (as_bits(y) >> 31 << 7);
        if (nms == 255u) c = 127u;
        nm |= c << (8 * e);
        c = to_code<-14>(v[e] * iv, random >> 16);
        if (v[e] > 0.f && c == 0u) c = 1u;
        if (nvs == 255u) c = 255u;
        nv |= c << (8 * e);
    }
    if (n > 0) {
        store_codes(t.m + at, nm, n);
        store_codes(t.v + at, nv, n);
    }
    if (there && (own & (kBlock - 1)) == 0) {
        t.m_scale[block] = (uint8_t)nms;
        t.v_scale[block] = (uint8_t)nvs;
    }
    if (n == 4) {
        if constexpr (kMaster) store4(t.master + at, w);
        store4(param, w);
    } else if (n > 0) {
        if constexpr (kMaster) store_some(t.master + at, w, n);
        store_some(param, w, n);
    }
}

template <bool kFew>
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
        const int elements = (int)min((long long)kChunk, (long long)k.t.n - begin);
        if (k.t.dtype == ALCH_BF16) {
            if (k.t.master) adamw8<__bf16, true>(k.t, begin, elements, a, r);
            else adamw8<__bf16, false>(k.t, begin, elements, a, r);
        } else {
            if (k.t.master) adamw8<float, true>(k.t, begin, elements, a, r);
            else adamw8<float, false>(k.t, begin, elements, a, r);
        }
    }
}

int launch_adamw8(int n_tensors, const alch_adamw8_tensor* tensors, const alch_adamw8_tensor* host, const alch_adamw& p, uint32_t seed,
                  hipStream_t stream) {
    long long chunks = 0;
    double bytes = 0;
    for (int i = 0; i < n_tensors; ++i) {
        chunks += (host[i].n + kChunk - 1) / kChunk;
        const double E = (double)dtype_size((alch_dtype)host[i].dtype);
        bytes += (double)host[i].n * (2 * E + 4 + 4.0 / kBlock + (host[i].master ? 8 : E));
    }
    if (chunks == 0) return ALCH_OK;
    TraceScope ts(kTraceUpdate, 0.0, bytes, stream);
    const Adamw8Args a{tensors, n_tensors, (float)p.lr, p.schedule ? 0.f : (float)correction(p.beta1, p.step),
                       p.schedule ? 0.f : (float)sqrt(correction(p.beta2, p.step)),
                       (float)p.beta1, (float)p.beta2, (float)(1.0 - p.beta1), (float)(1.0 - p.beta2), (float)p.eps, p.beta1, p.beta2,
                       seed, (uint32_t)p.step, p.schedule, p.grad_factor};
    const auto kernel = n_tensors <= 64 ? k_adamw8<true> : k_adamw8<false>;
    kernel<<<(int)std::min<long long>(chunks, kMaxChunkBlocks), 256, 0, stream>>>(a);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
