// The clipped policy loss of sampled tokens with its KL term (preference alignment on served responses), from rows of logits.
//
//   logz = log sum_v exp(x_v),  logp = x_label - logz,  ratio = exp(logp - old),  u = ratio A,  b = clamp(ratio, 1 - lo, 1 + hi) A
//   kl = exp(ref - logp) - (ref - logp) - 1,   loss = sum w (-min(u, b) + c kl)
//   dx_v = d ((v == label) - exp(x_v - logz)),   d = w (-(b < u ? 0 : u) + c (1 - exp(ref - logp)))
//
// A row of logits is one softmax, and its gradient needs the row's sum alone: bound by memory, a row read once and written once.
// Four forms:
//   held   a work-group a row, which stays in its registers between the sum and the gradient (up to 256 KB; rows longer than that also in LDS, up to
//          400 KB; what they have beyond is read twice);
//   stay   rows of 128 to 256 KB: a row is half of a compute unit's registers, so that no second work-group fits that could load while
//          this one computes.  One work-group a unit stays and has the next row on its way, 9 of 16 pieces to LDS, the others to registers;
//   few    few rows: several work-groups share one, in two launches with the parts' sums between them;
//   parts  the forward alone (and few rows whose parts are long): nothing is held, small work-groups go over a row, or its part, in one pass.
// A row is summed without its label: beside a p of all but 1 (most tokens that were sampled) the others' sum r is what logp = -log(1 + r) and
// 1 - p = r / (1 + r) are made of, and 1 + r would lose it.  The row kernels leave x_label - max and the sum of every item; the loss is made of
// them in 64 bits by one launch, where terms of either sign cancel and a rounding of logp to fp32 would be seen.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace alch {

typedef float f32x4_p __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_p __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4_p __attribute__((ext_vector_type(4)));
typedef int i32x4_p __attribute__((ext_vector_type(4)));

static constexpr float kLog2e = 1.4426950408889634f;
static constexpr float kLog2eRest = 1.9259629e-8f;  // log2 e - kLog2e
static constexpr double kLog2eDouble = 1.4426950408889634;
static constexpr int kGridMax = 1 << 20;  // work-groups of a launch; rows behind them are gone over in rounds

struct PolicyArgs {
    const int* label;
    const float *old_logp, *advantage, *weight, *ref_logp;
    float low, high, kl_coef;  // 1 - clip_low, 1 + clip_high
    double exact_low, exact_high;  // the same, for the loss
    float *own, *sum;  // of every item: its label's logit less the row's largest, and the sum of exponentials; of a label that is the largest, of the others

    PolicyArgs from(int m) const {  // of the items behind the first m
        return {label + m, old_logp + m, advantage + m, weight + m, ref_logp ? ref_logp + m : nullptr, low, high, kl_coef,
                exact_low, exact_high, own + m, sum + m};
    }
};

static constexpr float kNoPower = 0x1p30f;  // a power of two that stands for infinity
// 2^(x log2 e - power), log2 e in two parts: the product alone would lose as much as x is large
__device__ __forceinline__ float grown2(float x, float power) {
    return __builtin_amdgcn_exp2f(fmaf(x, kLog2eRest, fmaf(x, kLog2e, -power)));
}
// d of the gradient: d 2^shift, the power of two only where the number leaves fp32.
struct Slope {
    float d, shift;
};
// With e^m taken out, m the larger of the exponents: what p makes small again is not lost, and a logit of -inf has 0 times a number.
__device__ __forceinline__ Slope far_slope(const PolicyArgs& a, float w, float A, float old, float ref, float logp, bool cut) {
    const bool with_kl = a.ref_logp && a.kl_coef != 0.f;
    const float up = logp - old, far = ref - logp, m = fmaxf(fmaxf(up, with_kl ? far : 0.f), 0.f);
    const auto without_m = [m](float x) { return x == m ? 1.f : expf(x - m); };
    float d = cut ? 0.f : -0.25f * A * without_m(up);  // (a quarter: the sum does not overflow)
    if (with_kl) d -= 0.25f * a.kl_coef * (without_m(far) - without_m(0.f));
    const float power = fminf(ceilf(m * kLog2e), kNoPower);
    const int exponents = __builtin_amdgcn_frexp_expf(d) + __builtin_amdgcn_frexp_expf(w) + 2;
    d = __builtin_amdgcn_frexp_mantf(d) * __builtin_amdgcn_frexp_mantf(w);
    return {power < kNoPower ? d * grown2(m, power) : d, power + (float)exponents};
}
// From an item's log-probability.
__device__ __forceinline__ Slope slope(const PolicyArgs& a, float w, float A, float old, float ref, float logp) {
    const float ratio = expf(logp - old);
    const float bounded = ratio < a.low ? a.low : ratio > a.high ? a.high : ratio;  // (NaN stays)
    const float u = ratio * A;
    const bool cut = A == 0.f || bounded * A < u;
    float d = cut ? 0.f : -u;
    if (a.ref_logp && a.kl_coef != 0.f) d -= a.kl_coef * expm1f(ref - logp);
    d *= w;
    return __builtin_expect(fabsf(d) < INFINITY, 1) ? Slope{d, 0.f} : far_slope(a, w, A, old, ref, logp, cut);
}
__device__ __forceinline__ Slope slope(const PolicyArgs& a, int m, float logp) {
    return slope(a, a.weight[m], a.advantage[m], a.old_logp[m], a.ref_logp ? a.ref_logp[m] : 0.f, logp);
}
__device__ __forceinline__ bool scores(const PolicyArgs& a, int m, int vocab) { return (unsigned)a.label[m] < (unsigned)vocab && a.weight[m] != 0.f; }

// v of the lane that a DPP pattern names; other's value in rows of 16 lanes outside of the mask.
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ float from_lane(float other, float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, other), __builtin_bit_cast(int, v), kCtrl, kRows, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63)); }
// Over a wavefront: neighbours, pairs, quads, halves of a row of 16 lanes; then row by row into the last one.
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, from_lane<0xB1>(v, v));
    v = fmaxf(v, from_lane<0x4E>(v, v));
    v = fmaxf(v, from_lane<0x141>(v, v));
    v = fmaxf(v, from_lane<0x140>(v, v));
    v = fmaxf(v, from_lane<0x142, 0xa>(v, v));
    return last_lane(fmaxf(v, from_lane<0x143, 0xc>(v, v)));
}
// Sums in 64 bits: beside a term of 1 every addition in fp32 loses 2^-24, ten of them are seen in the loss of a few items.
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ double from_lane(double v) {  // 0 in rows outside of the mask
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
    const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, kCtrl, kRows, 0xf, false);
    const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), kCtrl, kRows, 0xf, false);
    return __builtin_bit_cast(double, (unsigned long long)high << 32 | low);
}
__device__ __forceinline__ double wave_sum(double v) {
    v += from_lane<0xB1>(v);
    v += from_lane<0x4E>(v);
    v += from_lane<0x141>(v);
    v += from_lane<0x140>(v);
    v += from_lane<0x142, 0xa>(v);
    v += from_lane<0x143, 0xc>(v);
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
    const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63), high = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, (unsigned long long)high << 32 | low);
}
// Over a work-group, the result for everybody.  red: a number a wavefront, of each call its own.
template <int kThreads>
__device__ __forceinline__ float group_max(float v, float* red) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) v = fmaxf(v, red[w]);
    return v;
}
template <int kThreads>
__device__ __forceinline__ double group_sum(double v, double* red) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) v += red[w];
    return v;
}

static constexpr float kScoresNothing = -1.f;  // in the place of a sum
// What the loss is made of, of an item that scores: own - log(sum) is its log-probability, -log(1 + sum) where own is 0.  An fp32 logit's difference from the
// largest one is rounded, and the sum takes what that leaves, r: log(sum (1 - r)) = log(sum) - r.  (Of 16 bits the difference is exact, or as
// far as it matters.)
template <typename T>
__device__ __forceinline__ void put_item(const PolicyArgs& a, int m, float label_logit, float base, float label_part, double rest) {
    const float own = label_logit - base;
    double sum = own == 0.f ? rest : rest + label_part;
    if constexpr (sizeof(T) == 4) {
        const float part = own - label_logit, r = (label_logit - (own - part)) + (-base - part);
        if (fabsf(r) < 1e-3f) sum -= sum * r;  // (far beyond that, or none where there is an infinity)
    }
    a.own[m] = own;
    a.sum[m] = (float)sum;
}

// ---- a row in pieces ---------------------------------------------------------------------------
// Of 16 bytes, at multiples of 16: rows of an odd vocabulary begin anywhere.  What lies before the first and behind the last piece, less than a
// piece each, is an element each of the first 16 threads.
template <typename T> struct Piece;
template <> struct Piece<__bf16> {
    typedef bf16x8_p type;
    static constexpr int n = 8;
};
template <> struct Piece<float> {
    typedef f32x4_p type;
    static constexpr int n = 4;
};

struct RowCut {
    int head, pieces;  // elements before the first piece, pieces
};
template <typename T>
__device__ __forceinline__ RowCut cut_row(const T* x, int vocab) {
    constexpr int n = Piece<T>::n;
    const int head = min((int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T), vocab);
    return {head, (vocab - head) / n};
}
// The element of its own that a thread has, or -1.
template <typename T>
__device__ __forceinline__ int extra_of(const RowCut& c, int vocab) {
    const int tid = threadIdx.x;
    if (tid < 8) return tid < c.head ? tid : -1;
    const int e = c.head + c.pieces * Piece<T>::n + tid - 8;
    return tid < 16 && e < vocab ? e : -1;
}

// The piece that the label is in, or -1.  It is left out of the sums; its other elements, one each of the first threads, are added to them.
template <typename T>
__device__ __forceinline__ int label_piece(const RowCut& c, int label) {
    const int e = label - c.head;
    return e >= 0 && e < c.pieces * Piece<T>::n ? e / Piece<T>::n : -1;
}
// The element of a thread among them, or -1; `first`: of which thread on.
template <typename T>
__device__ __forceinline__ int beside_label(const RowCut& c, int piece, int label, int first = 0) {
    const int k = (int)threadIdx.x - first, e = c.head + piece * Piece<T>::n + k;
    return piece >= 0 && (unsigned)k < (unsigned)Piece<T>::n && e != label ? e : -1;
}

// exp(x - base) to a rounding or two: log2 e in two parts.  (What the first alone leaves is the same side's in every term of a sum: 1.3e-8 of x - base.)
__device__ __forceinline__ float grown_exactly(float x, float base) {
    const float d = x - base;
    return __builtin_amdgcn_exp2f(fmaf(d, kLog2e, d * kLog2eRest));
}

template <typename T, typename V>
__device__ __forceinline__ float piece_max(const V& x, float most) {
#pragma unroll
    for (int e = 0; e < Piece<T>::n; ++e) most = fmaxf(most, (float)x[e]);
    return most;
}
__device__ __forceinline__ float sum_of(const float (&v)[4]) { return (v[0] + v[1]) + (v[2] + v[3]); }
__device__ __forceinline__ float sum_of(const float (&v)[8]) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
template <typename T, typename V>
__device__ __forceinline__ double piece_sum(const V& x, float base) {
    float v[Piece<T>::n];
#pragma unroll
    for (int e = 0; e < Piece<T>::n; ++e) v[e] = grown_exactly((float)x[e], base);
    return sum_of(v);
}
// scale 2^shift exp(x - base); at_label in the label's place.  bf16: the scale goes into the exponent, whose rounding (2^-20 of the result where it has 5
// bits before the point) is far below the result's own of 2^-9.
struct GradOf {
    float base, scale, shift, log2_scale, at_label;
    uint32_t sign;
};
// rest: the sum of the others' exponentials, sum: with the label's (0: nothing that the gradient depends on).  In the label's place d (1 - p) by the one of
// its two forms that rounds the smaller part.
__device__ __forceinline__ GradOf grad_of(float label_logit, float base, float label_part, float rest, float sum, Slope s) {
    if (sum == 0.f) s = {0.f, 0.f};
    float scale = sum == 0.f ? 0.f : -s.d / sum, at_label = label_part < rest ? fmaf(scale, label_part, s.d) : -scale * rest;
    if (__builtin_expect(s.shift != 0.f, 0)) {  // (the scale to 1 and more, so that a product is not beyond fp32 before it has to be)
        at_label = label_logit == -INFINITY ? 0.f : ldexpf(at_label, (int)s.shift);
        const int e = __builtin_amdgcn_frexp_expf(scale) - 1;
        scale = ldexpf(scale, -e);
        s.shift += (float)e;
    }
    return {base, scale, s.shift, __builtin_amdgcn_logf(fabsf(scale)) + s.shift, at_label, __builtin_bit_cast(uint32_t, scale) & 0x80000000u};
}
__device__ __forceinline__ float single_grad(float x, const GradOf& o) { return o.scale * __builtin_amdgcn_exp2f(fmaf(x - o.base, kLog2e, o.shift)); }
template <typename T, typename V>
__device__ __forceinline__ V piece_grad(const V& x, const GradOf& o) {
    V g;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < Piece<T>::n; ++e) g[e] = (T)__builtin_amdgcn_exp2f(fmaf((float)x[e] - o.base, kLog2e, o.log2_scale));
        return __builtin_bit_cast(V, __builtin_bit_cast(u32x4_p, g) ^ (o.sign | o.sign >> 16));
    } else {
#pragma unroll
        for (int e = 0; e < Piece<T>::n; ++e) g[e] = single_grad((float)x[e], o);
        return g;
    }
}

// e: the label's place in the piece, where it is there: in one piece of a row.
template <typename T, typename V>
__device__ __forceinline__ V with_label(V g, int e, float at_label) {
    if ((unsigned)e < (unsigned)Piece<T>::n) {
#pragma unroll
        for (int i = 0; i < Piece<T>::n; ++i)
            if (i == e) g[i] = (T)at_label;
    }
    return g;
}

template <typename V>
__device__ __forceinline__ V load_piece(const void* p) {
    return __builtin_bit_cast(V, __builtin_nontemporal_load(static_cast<const u32x4_p*>(p)));
}
template <typename V>
__device__ __forceinline__ V load_again(const void* p) {  // (of what will be read once more: it may stay in the caches)
    return __builtin_bit_cast(V, *static_cast<const u32x4_p*>(p));
}
typedef u32x4_p u32x4_any __attribute__((aligned(2)));  // (rows of the gradient may begin elsewhere than those of the logits)
template <typename V>
__device__ __forceinline__ void store_piece(void* p, const V& v) {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_p, v), static_cast<u32x4_any*>(p));
}

__device__ __forceinline__ i32x4_p resource(const void* p, int bytes) {  // reads past the bytes are zero, writes dropped
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    i32x4_p r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    r[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu));
    r[2] = __builtin_amdgcn_readfirstlane(bytes);
    r[3] = 0x00020000;
    return r;
}

// 16 bytes a lane, from `offset` of the resource on, to `lds` and the wavefront's lanes one after another.  (s_nop: such a load takes one wait state after a
// scalar write of m0)
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, const i32x4_p& src) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(src) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_offset(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

// ---- a sum in one pass -------------------------------------------------------------------------
// With the largest logit so far and the power of two above its exponential, by which the terms are scaled; where a larger one comes the sum is moved by
// the difference of the powers, exactly.
// Beyond it a power is no longer exact (masks of the type's lowest value, for one).
static constexpr float kPowerMost = 1048576.f;
__device__ __forceinline__ float power(float most) { return fabsf(most) <= kPowerMost ? ceilf(most * kLog2e) : 0.f; }
__device__ __forceinline__ double moved(double sum, float from, float to) { return ldexp(sum, (int)(from - to)); }
// Adds pieces to the sum s of a thread whose largest logit so far is most, scaled by at.
template <typename T, typename V, int kBatch>
__device__ __forceinline__ void add_pieces(V (&x)[kBatch], float& most, float& at, double& s) {
    float higher = most;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) higher = piece_max<T>(x[k], higher);
    const float to = power(higher);
    if (to != at && most != -INFINITY) s = moved(s, at, to);
    most = higher;
    at = to;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
        asm volatile("" : "+v"(x[k]));
        float v[Piece<T>::n];
#pragma unroll
        for (int e = 0; e < Piece<T>::n; ++e) v[e] = grown2((float)x[k][e], at);
        s += sum_of(v);
    }
}
// Whether sums of threads that have such powers are whole: a thread all of whose logits are below -kPowerMost has added nothing, and 128 below the
// largest one that is no loss (e^-128 a term).
__device__ __forceinline__ bool by_powers(float base) { return base >= 128.f - kPowerMost && base <= kPowerMost; }
// The factor of a sum scaled by the power of two above exp(base), relative to exp(base): where by_powers(base).
__device__ __forceinline__ double from_power(float base) { return exp2((double)power(base) - (double)base * kLog2eDouble); }

// ---- held --------------------------------------------------------------------------------------
// 6000 x 50257 bf16 with gradient 220 us (5.2 TB/s of logits and gradient: a copy's rate), 9000 x 16000 105 us (5.2).  The second bound keeps 32 KB
// rows at six wavefronts a SIMD: left to itself the compiler takes 182 registers for 2500 x 7001 fp32, two wavefronts, and 53 us in place of 34.
// kLds: so many pieces a thread more are in LDS, and what a row has beyond those is read twice, for its sum in one pass; the second time most of it comes
// from the L2 (3000 x 128256 fp32, a fifth of each row read again: 571 us, 5.1 TB/s; without LDS, and with a pass more for the largest
// logit, 821).
template <typename T, int kThreads, int kHeld, int kLds = 0>
__global__ __launch_bounds__(kThreads, kHeld <= 8 ? 6 : 4) void k_policy_held(const T* logits, long long ld, int vocab, PolicyArgs a, T* dlogits, long long ld_grad) {
    typedef typename Piece<T>::type V;
    constexpr int n = Piece<T>::n, kBatch = 2;
    __shared__ float red[kThreads / 64];
    __shared__ double red_sum[2][kThreads / 64];
    __shared__ __attribute__((aligned(1024))) V lower[kLds > 0 ? kLds * kThreads : 1];
    const int m = blockIdx.x, tid = threadIdx.x;
    const T* row = logits + m * ld;
    T* out = dlogits + m * ld_grad;
    const RowCut c = cut_row(row, vocab);
    const int extra = extra_of<T>(c, vocab);
    const T* body = row + c.head;
    if (!scores(a, m, vocab)) {
        if (tid == 0) a.own[m] = 0.f, a.sum[m] = kScoresNothing;
        const V zero = {};
        for (int p = tid; p < c.pieces; p += kThreads) store_piece(out + c.head + (long long)p * n, zero);
        if (extra >= 0) out[extra] = (T)0.f;
        return;
    }
    V x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (tid + k * kThreads < c.pieces) x[k] = load_piece<V>(body + (tid + k * kThreads) * n);
    if constexpr (kLds > 0) {  // (each wavefront what its own lanes will use)
        const i32x4_p src = resource(body, c.pieces * 16);
        const uint32_t lds = lds_offset(lower) + (uint32_t)__builtin_amdgcn_readfirstlane(tid >> 6) * 1024u;
#pragma unroll
        for (int k = 0; k < kLds; ++k) load_to_lds(lds + k * kThreads * 16, (uint32_t)(tid + (kHeld + k) * kThreads) * 16u, src);
    }
    const int label = a.label[m], without = label_piece<T>(c, label), beside = beside_label<T>(c, without, label);
    const float xe = extra >= 0 ? (float)row[extra] : -INFINITY, xl = (float)row[label], xb = beside >= 0 ? (float)row[beside] : -INFINITY;
    float most = xe;
    float rest_most = -INFINITY, at = 0.f;
    double again = 0.0;
    if constexpr (kLds > 0) {
        V least;
#pragma unroll
        for (int e = 0; e < n; ++e) least[e] = (T)-INFINITY;
        for (int p = tid + (kHeld + kLds) * kThreads; p < c.pieces; p += kBatch * kThreads) {
            V y[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                y[k] = p + k * kThreads < c.pieces && p + k * kThreads != without ? load_again<V>(body + (long long)(p + k * kThreads) * n) : least;
            add_pieces<T>(y, rest_most, at, again);
        }
        most = fmaxf(fmaxf(most, rest_most), fmaxf(xl, xb));
    }
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (tid + k * kThreads < c.pieces) most = piece_max<T>(x[k], most);
    if constexpr (kLds > 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll 1
        for (int k = 0; k < kLds; ++k)
            if (tid + (kHeld + k) * kThreads < c.pieces) most = piece_max<T>(lower[k * kThreads + tid], most);
    }
    most = group_max<kThreads>(most, red);
    const float base = most == -INFINITY ? 0.f : most;  // (without a finite logit the sum is 0, or NaN)
    double s = (extra == label ? 0.f : grown_exactly(xe, base)) + grown_exactly(xb, base);
    // (the empty asm keeps the row packed in registers: without it the compiler carries converted copies across)
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        asm volatile("" : "+v"(x[k]));
        if (tid + k * kThreads < c.pieces && tid + k * kThreads != without) s += piece_sum<T>(x[k], base);
    }
    if constexpr (kLds > 0) {
#pragma unroll 1
        for (int k = 0; k < kLds; ++k)
            if (tid + (kHeld + k) * kThreads < c.pieces && tid + (kHeld + k) * kThreads != without) s += piece_sum<T>(lower[k * kThreads + tid], base);
    }
    double others = group_sum<kThreads>(s, red_sum[0]);
    if constexpr (kLds > 0) {
        if (c.pieces > (kHeld + kLds) * kThreads) {
            if (by_powers(base)) {
                others += group_sum<kThreads>(rest_most == -INFINITY ? again : moved(again, at, power(base)), red_sum[1]) * from_power(base);
            } else {  // (the powers say nothing: once more, from the largest one)
                double once = 0.0;
                for (int p = tid + (kHeld + kLds) * kThreads; p < c.pieces; p += kThreads)
                    if (p != without) once += piece_sum<T>(load_again<V>(body + (long long)p * n), base);
                others += group_sum<kThreads>(once, red_sum[1]);
            }
        }
    }
    const float label_part = grown_exactly(xl, base);
    if (tid == 0) put_item<T>(a, m, xl, base, label_part, others);
    const float rest = (float)others, sum = rest + label_part;
    const GradOf grad = grad_of(xl, base, label_part, rest, sum, slope(a, m, xl - base - logf(sum)));
    const auto put = [&](int p, const V& v) {
        store_piece(out + c.head + (long long)p * n, with_label<T>(piece_grad<T>(v, grad), label - c.head - p * n, grad.at_label));
    };
    // (each thread writes what it has read: in place nobody reads what another one has written)
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        asm volatile("" : "+v"(x[k]));
        if (tid + k * kThreads < c.pieces) put(tid + k * kThreads, x[k]);
    }
    if constexpr (kLds > 0) {
#pragma unroll 1
        for (int k = 0; k < kLds; ++k)
            if (tid + (kHeld + k) * kThreads < c.pieces) put(tid + (kHeld + k) * kThreads, lower[k * kThreads + tid]);
#pragma unroll 4
        for (int p = tid + (kHeld + kLds) * kThreads; p < c.pieces; p += kThreads) put(p, load_piece<V>(body + (long long)p * n));
    }
    if (extra >= 0) out[extra] = (T)(extra == label ? grad.at_label : single_grad(xe, grad));
}

// ---- stay --------------------------------------------------------------------------------------
// 6001 x 128256 bf16 with gradient: 580 us, 652 by the kernel above.  What the loop must not do is wait for everything between a row's fetch and its
// stores: a single element converted where it is loaded, or an item by a vector load, costs 3 to 13 % (100352 columns 466 us, 496).
static constexpr int kStayThreads = 1024, kStayPieces = 16, kStayLds = 9, kStayRegs = kStayPieces - kStayLds;
static constexpr int kStayRows = 1024;  // of a work-group in a launch
static constexpr int kHeldBytes = kStayThreads * kStayPieces * 16;  // the longest row that a work-group holds

// The rows of work-group b of n: list[0 .. counted) score, list[kStayRows - 1] downwards the others do not.  Either kind is dealt out in turn, from the
// first work-group and from the last one: a row that scores costs twice as much as one that is only written.  With the rows in turn whatever they are
// 6001 of them take 601, 572 and 512 us where 0.1, 0.3 and 0.6 do not score, so dealt 592, 521 and 442; where all do, 2 us more.
struct Dealt {
    int counted, others;
};
__device__ __forceinline__ Dealt deal_rows(const PolicyArgs& a, int rows, int vocab, unsigned b, unsigned n, int* list, int (*counts)[64]) {
    constexpr int kLoads = 4;  // (a count of each wavefront and load is a lane of the scan)
    static_assert(kLoads * (kStayThreads / 64) == 64, "");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int before = 0, turn = 0;
    for (int base = 0; base < rows; base += kLoads * kStayThreads, turn ^= 1) {
        int label[kLoads];
        float weight[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int m = min(base + k * kStayThreads + tid, rows - 1);
            label[k] = a.label[m];
            weight[k] = a.weight[m];
        }
        unsigned long long which[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) which[k] = __ballot(base + k * kStayThreads + tid < rows && (unsigned)label[k] < (unsigned)vocab && weight[k] != 0.f);
        if (lane == 0) {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) counts[turn][k * (kStayThreads / 64) + wave] = __popcll(which[k]);
        }
        __syncthreads();
        const int own = counts[turn][lane];
        int sum = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d, 64);
            if (lane >= d) sum += o;
        }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int m = base + k * kStayThreads + tid;
            const int at = before + __builtin_amdgcn_readlane(sum - own, k * (kStayThreads / 64) + wave) + __popcll(which[k] & ((1ull << lane) - 1));
            if (which[k] >> lane & 1) {
                if ((unsigned)at % n == b) list[(unsigned)at / n] = m;
            } else if (m < rows && (unsigned)(m - at) % n == n - 1 - b) {
                list[kStayRows - 1 - (unsigned)(m - at) / n] = m;
            }
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    __syncthreads();
    const auto share = [n](unsigned all, unsigned first) { return (int)((all + n - 1 - first) / n); };
    return {share(before, b), share(rows - before, n - 1 - b)};
}

template <typename T>
__global__ __launch_bounds__(kStayThreads) void k_policy_stay(const T* logits, long long ld, int rows, int vocab, PolicyArgs a, T* dlogits, long long ld_grad) {
    typedef typename Piece<T>::type V;
    typedef std::conditional_t<sizeof(T) == 2, unsigned short, unsigned int> Bits;
    constexpr int n = Piece<T>::n;
    __shared__ __attribute__((aligned(1024))) V ahead[kStayLds * kStayThreads];
    __shared__ float red[kStayThreads / 64];
    __shared__ double red_sum[kStayThreads / 64];
    __shared__ int list[kStayRows], counts[2][64];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Dealt mine = deal_rows(a, rows, vocab, blockIdx.x, gridDim.x, list, counts);
    const int total = mine.counted + mine.others;
    if (total == 0) return;
    const uint32_t lds0 = lds_offset(ahead) + (uint32_t)wave * 1024u;
    struct Item {  // of the row that is on its way
        int row, label;
        float weight, advantage, old_logp, ref_logp;
        bool counted;
    };
    // A few rows that do not score go first, or the last rows that do would wait for their stores (1000 rows, a tenth: 126 us, last 132); many go last,
    // where all work-groups only write (6001 rows, six tenths: 442 us, first 475).
    const int from = 4 * mine.others > total ? mine.counted : 0;
    const auto item_of = [&](int i) {  // (by scalar loads: a vector load here would be waited for with the stores before it)
        const bool other = i >= from && i < from + mine.others;
        const int m = i >= total ? 0 : __builtin_amdgcn_readfirstlane(list[other ? kStayRows - 1 - (i - from) : i < from ? i : i - mine.others]);
        const auto at = [m](const auto* p) { return ((const __attribute__((address_space(4))) std::remove_cv_t<std::remove_pointer_t<decltype(p)>>*)(uintptr_t)p)[m]; };
        return Item{m, at(a.label), at(a.weight), at(a.advantage), at(a.old_logp), a.ref_logp ? at(a.ref_logp) : 0.f, i < total && !other};
    };
    V next[kStayRegs];
    Bits xe_next, xl_next;  // what this thread has beside its pieces, and the label's logit: as loaded, for the row's own turn to look at
    // an element before or behind the pieces, or of the label's piece
    const auto single_of = [&](const RowCut& c, int label) { return tid < 16 ? extra_of<T>(c, vocab) : beside_label<T>(c, label_piece<T>(c, label), label, 16); };
    // The loads of a row: a wavefront fetches what its own lanes will use.  kStayPieces of them are issued whether or not the row reaches
    // as far, or is wanted at all.
    const auto fetch = [&](const Item& i) {
        const T* row = logits + (long long)i.row * ld;
        const RowCut c = cut_row(row, vocab);
        const int bytes = i.counted ? c.pieces * 16 : 0;
        xe_next = reinterpret_cast<const Bits*>(row)[max(single_of(c, i.counted ? i.label : -1), 0)];
        xl_next = reinterpret_cast<const Bits*>(row)[i.counted ? i.label : 0];
        const i32x4_p src = resource(row + c.head, bytes);
        uint32_t at = (uint32_t)tid * 16u;
        asm volatile("" : "+v"(at));  // (one register, not one per piece kept across the loop)
#pragma unroll
        for (int k = 0; k < kStayLds; ++k) load_to_lds(lds0 + k * kStayThreads * 16, at + k * kStayThreads * 16, src);
#pragma unroll
        for (int k = 0; k < kStayRegs; ++k)
            next[k] = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(row) + c.head, 0, bytes, 0x00020000),
                                                                                  at + (kStayLds + k) * kStayThreads * 16, 0, 0));
    };
    Item item = item_of(0), item1 = item_of(1);
    fetch(item);
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0), known to the compiler: inside the loop it then counts the stores, too
    for (int i = 0; i < total; ++i) {
        // the row's loads have landed; the last kStayPieces stores of the row before may still be on their way
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kStayPieces) : "memory");
        const Item item2 = item_of(i + 2);
        const int r = item.row;
        const RowCut c = cut_row(logits + (long long)r * ld, vocab);
        const int extra = extra_of<T>(c, vocab);
        T* out = dlogits + (long long)r * ld_grad;
        const auto dst = __builtin_amdgcn_make_buffer_rsrc(out + c.head, 0, c.pieces * 16, 0x00020000);
        if (!item.counted) {
            fetch(item1);
            if (tid == 0) a.own[r] = 0.f, a.sum[r] = kScoresNothing;
            if (extra >= 0) out[extra] = (T)0.f;
            int at = tid;
            asm volatile("" : "+v"(at) :: "memory");
#pragma unroll
            for (int k = 0; k < kStayPieces; ++k) __builtin_amdgcn_raw_buffer_store_b128(u32x4_p{0, 0, 0, 0}, dst, (at + k * kStayThreads) * 16, 0, 0);
            item = item1;
            item1 = item2;
            continue;
        }
        V x[kStayPieces];
#pragma unroll
        for (int k = 0; k < kStayLds; ++k) x[k] = ahead[k * kStayThreads + tid];
#pragma unroll
        for (int k = 0; k < kStayRegs; ++k) x[kStayLds + k] = next[k];
        asm volatile("" : "+v"(xe_next), "+v"(xl_next));
        const int single = single_of(c, item.label), without = label_piece<T>(c, item.label);
        const float xe = single >= 0 ? (float)__builtin_bit_cast(T, xe_next) : -INFINITY, xl = (float)__builtin_bit_cast(T, xl_next);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int k = 0; k < kStayPieces; ++k) asm volatile("" : "+v"(x[k]));  // (in registers before the next row overwrites them)
        fetch(item1);
        float most = xe;
#pragma unroll
        for (int k = 0; k < kStayPieces; ++k)
            if (tid + k * kStayThreads < c.pieces) most = piece_max<T>(x[k], most);
        most = group_max<kStayThreads>(most, red);
        const float base = most == -INFINITY ? 0.f : most;
        double s = single == item.label ? 0.f : grown_exactly(xe, base);
        int own = tid;
        asm volatile("" : "+v"(own));  // (as above)
#pragma unroll
        for (int k = 0; k < kStayPieces; ++k) {
            asm volatile("" : "+v"(x[k]));
            if (own + k * kStayThreads < c.pieces && own + k * kStayThreads != without) s += piece_sum<T>(x[k], base);
        }
        const double others = group_sum<kStayThreads>(s, red_sum);
        const float label_part = grown_exactly(xl, base);
        const float rest = (float)others, sum = rest + label_part;
        const GradOf grad = grad_of(xl, base, label_part, rest, sum, slope(a, item.weight, item.advantage, item.old_logp, item.ref_logp, xl - base - logf(sum)));
        // (what is stored beside the pieces goes first: the wait above counts the last kStayPieces stores)
        if (tid == 0) put_item<T>(a, r, xl, base, label_part, others);
        if (extra >= 0) out[extra] = (T)(extra == item.label ? grad.at_label : single_grad(xe, grad));
        int at = tid;
        asm volatile("" : "+v"(at) :: "memory");
#pragma unroll
        for (int k = 0; k < kStayPieces; ++k) {
            asm volatile("" : "+v"(x[k]));
            const V g = with_label<T>(piece_grad<T>(x[k], grad), item.label - c.head - (at + k * kStayThreads) * n, grad.at_label);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_p, g), dst, (at + k * kStayThreads) * 16, 0, 0);
        }
        item = item1;
        item1 = item2;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// ---- parts -------------------------------------------------------------------------------------
// Nothing of a part is held, so that work-groups are small and many rows are on their way at once: 6001 x 128256 bf16 without gradient 272 us, 5.7 TB/s
// read.
static constexpr int kPartThreads = 256, kPartBatch = 8;
static constexpr int kMaxParts = 64, kMaxPartials = 1024;  // of a row; of a call

struct Partial {  // of a part: its largest logit, and its sum of exponentials, the label's left out, relative to that one (0: there is nothing finite else)
    float most;
    double sum;
};
// The pieces of part j of n.
__device__ __forceinline__ void part_of(int pieces, int j, int n, int* begin, int* end) {
    const int each = (pieces + n - 1) / n;
    *begin = min(j * each, pieces);
    *end = min(*begin + each, pieces);
}
// A row of its parts, one to a lane of a wavefront (kMaxParts at most).  base is the largest logit (0: there is none), the others' sum relative to it.
struct Whole {
    float base, rest;
};
__device__ __forceinline__ double part_in(const Partial& p, float base) {  // (a part of NaN alone has no largest one either)
    return p.most == -INFINITY ? p.sum : p.sum * exp2(((double)p.most - (double)base) * kLog2eDouble);
}
__device__ __forceinline__ Whole whole_row(const Partial& p) {
    const float most = wave_max(p.most), base = most == -INFINITY ? 0.f : most;
    return {base, (float)wave_sum(part_in(p, base))};
}

// Part j of row m is work-group m * parts + j's; parts == 1: the row is whole, and its sum goes to where k_policy_sums finds it.
template <typename T>
__global__ __launch_bounds__(kPartThreads) void k_policy_parts(const T* logits, long long ld, int rows, int vocab, PolicyArgs a, int parts,
                                                               Partial* __restrict__ partial) {
    typedef typename Piece<T>::type V;
    constexpr int n = Piece<T>::n;
    __shared__ float red[kPartThreads / 64];
    __shared__ double red_sum[2][kPartThreads / 64];
    const int tid = threadIdx.x;
    V least;
#pragma unroll
    for (int e = 0; e < n; ++e) least[e] = (T)-INFINITY;
    for (long long b = blockIdx.x; b < (long long)rows * parts; b += gridDim.x) {
        const int m = (int)(b / parts), j = (int)(b % parts);
        const T* row = logits + m * ld;
        if (!scores(a, m, vocab)) {
            if (tid == 0 && parts == 1) a.own[m] = 0.f, a.sum[m] = kScoresNothing;
            continue;
        }
        const RowCut c = cut_row(row, vocab);
        int p, end;
        part_of(c.pieces, j, parts, &p, &end);
        const int label = a.label[m], without = label_piece<T>(c, label);
        p += tid;
        const T* body = row + c.head;
        // (what is outside of the pieces, and of the label's piece, is the first part's)
        const int single = j > 0 ? -1 : tid < 16 ? extra_of<T>(c, vocab) : beside_label<T>(c, without, label, 16);
        const float xe = single >= 0 ? (float)row[single] : -INFINITY;
        const auto load = [&](V (&x)[kPartBatch], int at) {
            if ((unsigned)(without - at + tid) < (unsigned)(kPartBatch * kPartThreads)) {  // (of one batch: 1501 x 32000 bf16 26.9 us, 28.1 if of all)
#pragma unroll
                for (int k = 0; k < kPartBatch; ++k) x[k] = at + k * kPartThreads < end && at + k * kPartThreads != without ? load_piece<V>(body + (long long)(at + k * kPartThreads) * n) : least;
                return;
            }
#pragma unroll
            for (int k = 0; k < kPartBatch; ++k) x[k] = at + k * kPartThreads < end ? load_piece<V>(body + (long long)(at + k * kPartThreads) * n) : least;
        };
        V next[kPartBatch];
        load(next, p);
        const float xl = j == 0 ? (float)row[label] : -INFINITY;
        float most = fmaxf(xe, xl), at = power(most);
        double s = single >= 0 && single != label ? grown2(xe, at) : 0.f;
        for (; p < end; p += kPartBatch * kPartThreads) {
            V x[kPartBatch];
#pragma unroll
            for (int k = 0; k < kPartBatch; ++k) x[k] = next[k];
            load(next, p + kPartBatch * kPartThreads);
            add_pieces<T>(x, most, at, s);
        }
        const float group = group_max<kPartThreads>(most, red), base = group == -INFINITY ? 0.f : group;
        double total = group_sum<kPartThreads>(most == -INFINITY ? s : moved(s, at, power(group)), red_sum[0]);
        if (by_powers(base)) {
            total *= from_power(base);
        } else {  // (the powers say nothing: once more, from the largest one)
            double once = single >= 0 && single != label ? grown_exactly(xe, base) : 0.f;
            int q, to;
            part_of(c.pieces, j, parts, &q, &to);
            for (q += tid; q < to; q += kPartThreads)
                if (q != without) once += piece_sum<T>(load_piece<V>(body + (long long)q * n), base);
            total = group_sum<kPartThreads>(once, red_sum[1]);
        }
        if (tid == 0) {
            if (parts > 1) {
                partial[b] = {group, total};
                if (j == 0) a.own[m] = xl;
            } else {
                put_item<T>(a, m, xl, base, grown_exactly(xl, base), total);
            }
        }
    }
}

// The parts of few rows: kHeld pieces a thread, which are on their way before the item has been looked at.  (Latency is all there is here: 17 x 128256 bf16,
// both launches 14.1 us with the kernel above and the item first, so 10.7; 9.4 since the loss has its items ahead, too.)
template <typename T, int kHeld>
__global__ __launch_bounds__(kPartThreads) void k_policy_few(const T* logits, long long ld, int vocab, PolicyArgs a, int parts, Partial* __restrict__ partial) {
    typedef typename Piece<T>::type V;
    constexpr int n = Piece<T>::n;
    __shared__ float red[kPartThreads / 64];
    __shared__ double red_sum[kPartThreads / 64];
    const int tid = threadIdx.x, m = (int)blockIdx.x / parts, j = (int)blockIdx.x % parts;
    const T* row = logits + m * ld;
    const RowCut c = cut_row(row, vocab);
    int begin, end;
    part_of(c.pieces, j, parts, &begin, &end);
    const T* body = row + c.head;
    V x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (begin + tid + k * kPartThreads < end) x[k] = load_piece<V>(body + (long long)(begin + tid + k * kPartThreads) * n);
    const int extra = j == 0 ? extra_of<T>(c, vocab) : -1, label = a.label[m];
    const float xe = extra >= 0 ? (float)row[extra] : -INFINITY, weight = a.weight[m];
    if ((unsigned)label >= (unsigned)vocab || weight == 0.f) return;
    const int without = label_piece<T>(c, label), beside = without >= begin && without < end ? beside_label<T>(c, without, label) : -1;
    const float xl = j == 0 ? (float)row[label] : -INFINITY, xb = beside >= 0 ? (float)row[beside] : -INFINITY;
    float most = xe;
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (begin + tid + k * kPartThreads < end) most = piece_max<T>(x[k], most);
    most = group_max<kPartThreads>(most, red);
    const float base = most == -INFINITY ? 0.f : most;
    double s = (extra >= 0 && extra != label ? grown_exactly(xe, base) : 0.f) + grown_exactly(xb, base);
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (begin + tid + k * kPartThreads < end && begin + tid + k * kPartThreads != without) s += piece_sum<T>(x[k], base);
    const double sum = group_sum<kPartThreads>(s, red_sum);
    if (tid == 0) {
        partial[blockIdx.x] = {most, sum};
        if (j == 0) a.own[m] = xl;
    }
}

// ---- the loss ----------------------------------------------------------------------------------
// Its four sums, in a fixed order and in 64 bits, by one work-group.
static constexpr int kSumThreads = 1024, kSumGroups = 256;
struct PolicySums {
    double loss, surrogate, kl, clipped;
    __device__ __forceinline__ void add(const PolicySums& o) {
        loss += o.loss;
        surrogate += o.surrogate;
        kl += o.kl;
        clipped += o.clipped;
    }
};
struct ItemIn {  // (loaded at once and first: one behind the other, and behind the logarithm, they would be most of a small call)
    float own, sum, weight, advantage, old_logp, ref_logp;
    int label;
};
__device__ __forceinline__ ItemIn load_item(const PolicyArgs& a, int m) {
    return {a.own[m], a.sum[m], a.weight[m], a.advantage[m], a.old_logp[m], a.ref_logp ? a.ref_logp[m] : 0.f, a.label[m]};
}
// (own and sum as put_item leaves them)
__device__ __forceinline__ PolicySums item_sums(const PolicyArgs& a, int m, const ItemIn& in, double own, double sum, float* __restrict__ logp_out) {
    PolicySums s = {};
    double logp = 0.0;
    if (!(sum < 0.0)) {
        if (sum == 0.0 && own != 0.0) {  // (its logits are all -inf)
            logp = own;
        } else {
            // (a small sum by its series: 2^-40 of it are left out)
            logp = own == 0.0 && sum < 0x1p-20 ? sum * (0.5 * sum - 1.0) : own - log(own == 0.0 ? 1.0 + sum : sum);
            const double w = in.weight, A = in.advantage, ratio = exp(logp - (double)in.old_logp);
            const double bounded = ratio < a.exact_low ? a.exact_low : ratio > a.exact_high ? a.exact_high : ratio;
            const double u = A == 0.0 ? 0.0 : ratio * A, b = A == 0.0 ? 0.0 : bounded * A;
            const bool cut = b < u;
            s.surrogate = w * (cut ? -b : -u);
            s.clipped = cut ? w : 0.0;
            s.loss = s.surrogate;
            if (a.ref_logp) {
                const double far = (double)in.ref_logp - logp;
                s.kl = w * (far == INFINITY ? far : expm1(far) - far);  // (a label that the logits forbid)
                if (a.kl_coef != 0.f) s.loss += (double)a.kl_coef * s.kl;
            }
        }
    }
    if (logp_out) logp_out[m] = (float)logp;
    return s;
}
template <int kThreads>
__device__ __forceinline__ void group_sums(const PolicySums& s, double (*red)[4], double* out) {  // to [4]
    double of[4] = {s.loss, s.surrogate, s.kl, s.clipped};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        of[i] = wave_sum(of[i]);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][i] = of[i];
    }
    __syncthreads();
    if (threadIdx.x >= 4) return;
    double t = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) t += red[w][threadIdx.x];
    out[threadIdx.x] = t;
}
template <int kThreads>
__device__ __forceinline__ void put_sums(const PolicySums& s, double (*red)[4], float* __restrict__ loss_out) {
    __shared__ double total[4];
    group_sums<kThreads>(s, red, total);
    if (threadIdx.x < 4) loss_out[threadIdx.x] = (float)total[threadIdx.x];
}
// Thread `first` of `stride`: its items' share.
__device__ __forceinline__ PolicySums items_sums(const PolicyArgs& a, int n, int first, int stride, float* __restrict__ logp_out) {
    PolicySums s = {};
    for (unsigned m = first; m < (unsigned)n; m += stride) {  // (n may be 2^31 - 1)
        const ItemIn in = load_item(a, (int)m);
        s.add(item_sums(a, (int)m, in, in.own, in.sum, logp_out));
    }
    return s;
}
// The same of rows that were summed in parts (own is the label's logit as it stands), by a work-group.  Parts are joined by as many lanes as there
// are, several rows at once: a 64-bit exponential each is what this takes.
template <int kThreads>
__device__ __forceinline__ PolicySums parts_sums(const PolicyArgs& a, int n, int vocab, int parts, const Partial* __restrict__ partial,
                                                 float* __restrict__ logp_out) {
    __shared__ double joined[kMaxPartials / 2];
    __shared__ float largest[kMaxPartials / 2];
    const int lanes = parts <= 1 ? 1 : 1 << (32 - __builtin_clz(parts - 1)), tid = threadIdx.x, j = tid & (lanes - 1), rows = kThreads / lanes;
    constexpr int kAhead = 4;
    const ItemIn mine = load_item(a, min(tid, n - 1));
    for (int first = 0; first < n; first += rows * kAhead) {
        Partial p[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int m = first + k * rows + tid / lanes;
            p[k] = m < n && j < parts ? partial[m * parts + j] : Partial{-INFINITY, 0.0};  // (of rows that do not score: whatever was there)
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int m = first + k * rows + tid / lanes;
            if (first + k * rows >= n) break;
            float most = p[k].most;
            for (int d = lanes >> 1; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
            const float base = most == -INFINITY ? 0.f : most;
            double sum = part_in(p[k], base);
            for (int d = lanes >> 1; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
            if (m < n && j == 0) {
                joined[m] = sum;
                largest[m] = base;
            }
        }
    }
    __syncthreads();
    PolicySums s = {};
    for (int m = tid; m < n; m += kThreads) {
        const ItemIn in = m == tid ? mine : load_item(a, m);
        const bool counted = (unsigned)in.label < (unsigned)vocab && in.weight != 0.f;
        const double own = counted ? (double)in.own - (double)largest[m] : 0.0;
        s.add(item_sums(a, m, in, own, !counted ? (double)kScoresNothing : own == 0.0 ? joined[m] : joined[m] + grown_exactly(in.own, largest[m]), logp_out));
    }
    return s;
}
__global__ __launch_bounds__(kSumThreads) void k_policy_sums(PolicyArgs a, int n, int vocab, int parts, const Partial* __restrict__ partial,
                                                             float* __restrict__ logp_out, float* __restrict__ loss_out) {
    __shared__ double red[kSumThreads / 64][4];
    if (parts > 1) put_sums<kSumThreads>(parts_sums<kSumThreads>(a, n, vocab, parts, partial, logp_out), red, loss_out);
    else put_sums<kSumThreads>(items_sums(a, n, threadIdx.x, kSumThreads, logp_out), red, loss_out);
}

// Many items: a work-group to each kSumThreads of them (64-bit logarithms and exponentials take 18 us for 6001 items by one), and one that adds theirs.
__global__ __launch_bounds__(kSumThreads) void k_policy_sums_of(PolicyArgs a, int n, float* __restrict__ logp_out, double (*__restrict__ sums)[4]) {
    __shared__ double red[kSumThreads / 64][4];
    group_sums<kSumThreads>(items_sums(a, n, blockIdx.x * kSumThreads + threadIdx.x, gridDim.x * kSumThreads, logp_out), red, sums[blockIdx.x]);
}
__global__ __launch_bounds__(64) void k_policy_sums_join(const double (*__restrict__ sums)[4], int n, float* __restrict__ loss_out) {
    const int i = threadIdx.x & 3;
    double t = 0.0;
    for (int k = threadIdx.x >> 2; k < n; k += 16) t += sums[k][i];
#pragma unroll
    for (int d = 4; d < 64; d <<= 1) t += __shfl_xor(t, d, 64);
    if (threadIdx.x < 4) loss_out[i] = (float)t;
}
static void launch_sums(const PolicyArgs& a, int n, void* scratch, float* logp_out, float* loss_out, hipStream_t stream) {
    if (n <= 3 * kSumThreads) {  // (1501 items: 5.5 us, 10 by two launches)
        k_policy_sums<<<1, kSumThreads, 0, stream>>>(a, n, 0, 0, nullptr, logp_out, loss_out);
        return;
    }
    const int groups = (int)std::min(((long long)n + kSumThreads - 1) / kSumThreads, (long long)kSumGroups);
    const auto sums = static_cast<double(*)[4]>(scratch);
    k_policy_sums_of<<<groups, kSumThreads, 0, stream>>>(a, n, logp_out, sums);
    k_policy_sums_join<<<1, 64, 0, stream>>>(sums, groups, loss_out);
}

// The gradient of rows that were summed in parts, a work-group a part, and by the first work-group the loss.  What a part begins with is on its way
// before the row's sum is known.
template <typename T>
__global__ __launch_bounds__(kPartThreads) void k_policy_part_grads(const T* logits, long long ld, int vocab, PolicyArgs a, int rows, int parts,
                                                                    const Partial* __restrict__ partial, T* dlogits, long long ld_grad,
                                                                    float* __restrict__ logp_out, float* __restrict__ loss_out) {
    typedef typename Piece<T>::type V;
    constexpr int n = Piece<T>::n, kHeld = 2;
    __shared__ double red[kPartThreads / 64][4];
    const int tid = threadIdx.x, b = (int)blockIdx.x - 1;
    if (b < 0) {
        put_sums<kPartThreads>(parts_sums<kPartThreads>(a, rows, vocab, parts, partial, logp_out), red, loss_out);
        return;
    }
    const int m = b / parts, j = b % parts;
    const T* row = logits + m * ld;
    T* out = dlogits + m * ld_grad;
    const RowCut c = cut_row(row, vocab);
    int begin, end;
    part_of(c.pieces, j, parts, &begin, &end);
    const T* body = row + c.head;
    V x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (begin + tid + k * kPartThreads < end) x[k] = load_piece<V>(body + (long long)(begin + tid + k * kPartThreads) * n);
    const int extra = j == 0 ? extra_of<T>(c, vocab) : -1, label = a.label[m], lane = tid & 63;
    const float xe = extra >= 0 ? (float)row[extra] : 0.f, weight = a.weight[m], advantage = a.advantage[m], old_logp = a.old_logp[m];
    const float ref_logp = a.ref_logp ? a.ref_logp[m] : 0.f, own = a.own[m];  // (own, and the parts below: of a row that does not score anything)
    const Partial part = lane < parts ? partial[(long long)m * parts + lane] : Partial{-INFINITY, 0.0};
    GradOf grad = {};
    bool some = false;  // logits that the gradient depends on
    if ((unsigned)label < (unsigned)vocab && weight != 0.f) {
        const Whole w = whole_row(part);
        const float label_part = grown_exactly(own, w.base), sum = w.rest + label_part;
        some = sum != 0.f;
        if (some) grad = grad_of(own, w.base, label_part, w.rest, sum, slope(a, weight, advantage, old_logp, ref_logp, own - w.base - logf(sum)));
    }
    const auto put = [&](int p, const V& v) {
        V g = {};
        if (some) g = with_label<T>(piece_grad<T>(v, grad), label - c.head - p * n, grad.at_label);
        store_piece(out + c.head + (long long)p * n, g);
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (begin + tid + k * kPartThreads < end) put(begin + tid + k * kPartThreads, x[k]);
#pragma unroll 4
    for (int p = begin + tid + kHeld * kPartThreads; p < end; p += kPartThreads) put(p, load_piece<V>(body + (long long)p * n));
    if (extra >= 0) out[extra] = (T)(!some ? 0.f : extra == label ? grad.at_label : single_grad(xe, grad));
}

// Parts of each row of a call: 8 KB to a work-group, kMaxPartials in all.  1: rows as a whole, of which 256 and more (128 short ones) fill the card, 320
// where a work-group's registers are not enough for one.  With gradient, bf16, vocabulary 128256, in parts and whole: 64 rows 20.9 us and 49, 200 rows
// 38.4 and 49, 400 rows 65 and 50; fp32: 260 rows 66 and 74, 400 rows 97 and 82, 500 rows 115 and 95.  The work-group that forms the loss joins all of
// them meanwhile, so that many rows have fewer: 20 x 128256 fp32 in 32 parts 10.5 us, in 51 12.8; 64 x 32000 fp32 in parts of 16 KB 9.2, of 8 KB 10.7.
static int parts_of(int rows, int vocab, size_t element, bool grad) {
    const long long bytes = (long long)vocab * (long long)element;
    if (rows > (bytes <= kHeldBytes / 2 ? 128 : bytes <= kHeldBytes ? 256 : 320)) return 1;
    const int most = std::max(std::min(rows > 8 ? kMaxParts / 2 : kMaxParts, kMaxPartials / rows), 1);
    const auto of = [&](long long each) { return (int)std::min<long long>((bytes + each - 1) / each, most); };
    return grad && rows * of(8192) > kMaxPartials / 2 ? of(16384) : of(8192);
}

size_t policy_scratch_bytes() { return std::max(kMaxPartials * sizeof(Partial), kSumGroups * 4 * sizeof(double)); }
size_t policy_loss_workspace_bytes(int n_items, int vocab) {
    (void)vocab;
    return round_up((size_t)(n_items > 0 ? n_items : 1) * 2 * sizeof(float), 256) + policy_scratch_bytes();
}

static PolicyArgs policy_args(const alch_policy& p, int item0, float* own, float* sum) {
    const double low = 1.0 - (double)p.clip_low, high = 1.0 + (double)p.clip_high;
    return PolicyArgs{p.label, p.old_logp, p.advantage, p.weight, p.ref_logp, (float)low, (float)high, p.kl_coef, low, high, own, sum}.from(item0);
}

template <typename T>
static void launch_held(const T* logits, long long ld, int rows, int vocab, const PolicyArgs& a, T* dlogits, long long ld_grad, hipStream_t stream) {
    const int pieces = vocab / Piece<T>::n + 1;
    const auto go = [&](auto kernel, int threads) {
        for (long long r = 0; r < rows; r += kGridMax)
            kernel<<<(int)std::min<long long>(rows - r, kGridMax), threads, 0, stream>>>(logits + r * ld, ld, vocab, a.from((int)r), dlogits + r * ld_grad, ld_grad);
    };
    if (pieces <= 256) go(k_policy_held<T, 256, 1>, 256);
    else if (pieces <= 256 * 4) go(k_policy_held<T, 256, 4>, 256);
    else if (pieces <= 256 * 8) go(k_policy_held<T, 256, 8>, 256);
    else if (pieces <= 256 * 16) go(k_policy_held<T, 256, 16>, 256);
    else if (pieces <= 512 * 16) go(k_policy_held<T, 512, 16>, 512);
    else if (pieces <= 1024 * 16) go(k_policy_held<T, 1024, 16>, 1024);
    else go(k_policy_held<T, 1024, 16, 9>, 1024);
}

template <typename T>
static int launch_rows(const T* logits, long long ld, int rows, int vocab, const PolicyArgs& a, T* dlogits, long long ld_grad, Partial* partial,
                       float* logp_out, float* loss_out, hipStream_t stream) {
    int n_cu = 0;
    ALCH_TRY(compute_units(&n_cu));
    const int pieces = vocab / Piece<T>::n + 1, parts = loss_out ? parts_of(rows, vocab, sizeof(T), dlogits) : 1;
    if (parts > 1 || !dlogits) {
        const int held = (pieces + parts * kPartThreads - 1) / (parts * kPartThreads);  // of a part, a thread
        if (parts > 1 && held <= 2) k_policy_few<T, 2><<<rows * parts, kPartThreads, 0, stream>>>(logits, ld, vocab, a, parts, partial);
        else if (parts > 1 && held <= 8) k_policy_few<T, 8><<<rows * parts, kPartThreads, 0, stream>>>(logits, ld, vocab, a, parts, partial);
        else k_policy_parts<<<(int)std::min<long long>((long long)rows * parts, kGridMax), kPartThreads, 0, stream>>>(logits, ld, rows, vocab, a, parts, partial);
        if (dlogits)
            k_policy_part_grads<<<rows * parts + 1, kPartThreads, 0, stream>>>(logits, ld, vocab, a, rows, parts, partial, dlogits, ld_grad, logp_out, loss_out);
        else if (parts > 1)
            k_policy_sums<<<1, kSumThreads, 0, stream>>>(a, rows, vocab, parts, partial, logp_out, loss_out);
        else if (loss_out)
            launch_sums(a, rows, partial, logp_out, loss_out, stream);
        return ALCH_OK;
    }
    // pieces of both matrices' rows begin together, and the row fits
    const bool alike = (ld - ld_grad) * (long long)sizeof(T) % 16 == 0;
    if (alike && pieces > 512 * 16 && pieces <= kStayThreads * kStayPieces) {
        const int most = (kStayRows - 1) * n_cu;  // (of both kinds together a work-group may have one more than its share)
        for (long long r = 0; r < rows; r += most)
            k_policy_stay<<<(int)std::min<long long>(rows - r, n_cu), kStayThreads, 0, stream>>>(logits + r * ld, ld, (int)std::min<long long>(rows - r, most), vocab,
                                                                                                 a.from((int)r), dlogits + r * ld_grad, ld_grad);
    } else {
        launch_held<T>(logits, ld, rows, vocab, a, dlogits, ld_grad, stream);
    }
    if (loss_out) launch_sums(a, rows, partial, logp_out, loss_out, stream);
    return ALCH_OK;
}

int launch_policy(alch_dtype dt, const void* logits, long long ld, int rows, int vocab, const alch_policy& p, int item0, void* dlogits, long long ld_grad,
                  float* own, float* sum, void* scratch, float* loss_out, hipStream_t stream) {
    if (rows <= 0) return loss_out ? launch_policy_sums(p, own, sum, scratch, loss_out, stream) : ALCH_OK;
    const double E = (double)dtype_size(dt);
    TraceScope ts(kTraceCrossEntropy, 0.0, (double)rows * vocab * E * (dlogits ? 2 : 1), stream);
    const PolicyArgs a = policy_args(p, item0, own, sum);
    Partial* partial = static_cast<Partial*>(scratch);
    if (dt == ALCH_BF16)
        ALCH_TRY(launch_rows(static_cast<const __bf16*>(logits), ld, rows, vocab, a, static_cast<__bf16*>(dlogits), ld_grad, partial, p.logp_out, loss_out, stream));
    else
        ALCH_TRY(launch_rows(static_cast<const float*>(logits), ld, rows, vocab, a, static_cast<float*>(dlogits), ld_grad, partial, p.logp_out, loss_out, stream));
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

int launch_policy_sums(const alch_policy& p, float* own, float* sum, void* scratch, float* loss_out, hipStream_t stream) {
    launch_sums(policy_args(p, 0, own, sum), p.n_items, scratch, p.logp_out, loss_out, stream);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
