// The clipped policy loss of sampled tokens with its KL term (preference alignment on served responses), from rows of logits.
//
//   logz = log sum_v exp(x_v),  logp = x_label - logz,  ratio = exp(logp - old),  u = ratio A,  b = clamp(ratio, 1 - lo, 1 + hi) A
//   kl = exp(ref - logp) - (ref - logp) - 1,   loss = sum w (-min(u, b) + c kl)
//   dx_v = d ((v == label) - exp(x_v - logz)),   d = w (-(b < u ? 0 : u) + c (1 - exp(ref - logp)))
//
// A row of logits is one softmax, and its gradient needs the row's sum alone: bound by memory, a row read once and written once.
// Three kernels:
//   held   a work-group a row, which stays in its registers between the sum and the gradient (up to 256 KB; what a row has beyond them is
//          read twice);
//   stay   rows of 128 to 256 KB: a row is half of a compute unit's registers, so that no second work-group fits that could load while
//          this one computes.  One work-group a unit stays and has the next row on its way, 9 of 16 pieces to LDS, the others to registers;
//   parts  few rows: several work-groups share one, in two launches with the parts' sums between them.
// The row kernels leave x_label - max and the sum of exponentials of every item; the loss is made of them in 64 bits by one launch, where
// terms of either sign cancel and a rounding of logp to fp32 would be seen.
#include "kernels.h"

namespace alch {

typedef float f32x4_p __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_p __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4_p __attribute__((ext_vector_type(4)));
typedef int i32x4_p __attribute__((ext_vector_type(4)));

static constexpr float kLog2e = 1.4426950408889634f;

struct PolicyArgs {
    const int* label;
    const float *old_logp, *advantage, *weight, *ref_logp;
    float low, high, kl_coef;  // 1 - clip_low, 1 + clip_high
    float *own, *sum;          // of every item: its label's logit less the row's largest, and the sum of exponentials (0: it scores nothing)
};

// d of the gradient, from an item's log-probability.
__device__ __forceinline__ float slope(const PolicyArgs& a, float w, float A, float old, float ref, float logp) {
    const float ratio = expf(logp - old);
    const float bounded = ratio < a.low ? a.low : ratio > a.high ? a.high : ratio;  // (NaN stays)
    const float u = ratio * A;
    float d = A == 0.f || bounded * A < u ? 0.f : -u;
    if (a.ref_logp && a.kl_coef != 0.f) d -= a.kl_coef * expm1f(ref - logp);
    return w * d;
}
__device__ __forceinline__ float slope(const PolicyArgs& a, int m, float logp) {
    return slope(a, a.weight[m], a.advantage[m], a.old_logp[m], a.ref_logp ? a.ref_logp[m] : 0.f, logp);
}
__device__ __forceinline__ bool scores(const PolicyArgs& a, int m, int vocab) { return (unsigned)a.label[m] < (unsigned)vocab && a.weight[m] != 0.f; }

template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}
// Over a work-group, the result for everybody.  red: a float a wavefront, of each call its own.
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
__device__ __forceinline__ float group_sum(float v, float* red) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) v += red[w];
    return v;
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

// exp(x - base)
__device__ __forceinline__ float grown(float x, float base) { return __builtin_amdgcn_exp2f((x - base) * kLog2e); }

template <typename T, typename V>
__device__ __forceinline__ float piece_max(const V& x, float most) {
#pragma unroll
    for (int e = 0; e < Piece<T>::n; ++e) most = fmaxf(most, (float)x[e]);
    return most;
}
// Adds to a sum for every element of a piece: the sums are shorter, and do not wait for one another.
template <typename T, typename V>
__device__ __forceinline__ void piece_sum(const V& x, float base, float (&s)[4]) {
#pragma unroll
    for (int e = 0; e < Piece<T>::n; ++e) s[e & 3] += grown((float)x[e], base);
}
template <typename T, typename V>
__device__ __forceinline__ V piece_grad(const V& x, float base, float scale) {
    V g;
#pragma unroll
    for (int e = 0; e < Piece<T>::n; ++e) g[e] = (T)(scale * grown((float)x[e], base));
    return g;
}

template <typename V>
__device__ __forceinline__ V load_piece(const void* p) {
    return __builtin_bit_cast(V, __builtin_nontemporal_load(static_cast<const u32x4_p*>(p)));
}
typedef u32x4_p u32x4_any __attribute__((aligned(2)));  // (rows of the gradient may begin elsewhere than those of the logits)
template <typename V>
__device__ __forceinline__ void store_piece(void* p, const V& v) {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_p, v), static_cast<u32x4_any*>(p));
}

// ---- held --------------------------------------------------------------------------------------
template <typename T, int kThreads, int kHeld, bool kGrad>
__global__ __launch_bounds__(kThreads) void k_policy_held(const T* logits, long long ld, int vocab, PolicyArgs a, T* dlogits, long long ld_grad) {
    typedef typename Piece<T>::type V;
    constexpr int n = Piece<T>::n;
    __shared__ float red[2][kThreads / 64];
    const int m = blockIdx.x, tid = threadIdx.x;
    const T* row = logits + m * ld;
    T* out = kGrad ? dlogits + m * ld_grad : nullptr;
    const RowCut c = cut_row(row, vocab);
    const int extra = extra_of<T>(c, vocab);
    const T* body = row + c.head;
    if (!scores(a, m, vocab)) {
        if (tid == 0) a.own[m] = 0.f, a.sum[m] = 0.f;
        if constexpr (kGrad) {
            const V zero = {};
            for (int p = tid; p < c.pieces; p += kThreads) store_piece(out + c.head + p * n, zero);
            if (extra >= 0) out[extra] = (T)0.f;
        }
        return;
    }
    V x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (tid + k * kThreads < c.pieces) x[k] = load_piece<V>(body + (tid + k * kThreads) * n);
    const float xe = extra >= 0 ? (float)row[extra] : -INFINITY, xl = (float)row[a.label[m]];
    float most = xe;
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (tid + k * kThreads < c.pieces) most = piece_max<T>(x[k], most);
    for (int p = tid + kHeld * kThreads; p < c.pieces; p += kThreads) most = piece_max<T>(load_piece<V>(body + p * n), most);
    most = group_max<kThreads>(most, red[0]);
    const float base = most == -INFINITY ? 0.f : most;  // (without a finite logit the sum is 0, or NaN)
    float s[4] = {grown(xe, base), 0.f, 0.f, 0.f};
    // (the empty asm keeps the row packed in registers: without it the compiler carries converted copies across)
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        asm volatile("" : "+v"(x[k]));
        if (tid + k * kThreads < c.pieces) piece_sum<T>(x[k], base, s);
    }
    for (int p = tid + kHeld * kThreads; p < c.pieces; p += kThreads) piece_sum<T>(load_piece<V>(body + p * n), base, s);
    const float sum = group_sum<kThreads>((s[0] + s[1]) + (s[2] + s[3]), red[1]);
    if (tid == 0) {
        a.own[m] = sum == 0.f ? -INFINITY : xl - base;
        a.sum[m] = sum;
    }
    if constexpr (kGrad) {
        const float logp = xl - base - logf(sum), d = sum == 0.f ? 0.f : slope(a, m, logp), scale = sum == 0.f ? 0.f : -d / sum;
        const float at_label = sum == 0.f ? 0.f : d * -expm1f(logp);  // (1 - p without the difference)
        const int label = a.label[m];
        // (each thread writes what it has read: in place nobody reads what another one has written)
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            asm volatile("" : "+v"(x[k]));
            const int p = tid + k * kThreads;
            if (p >= c.pieces) continue;
            V g = piece_grad<T>(x[k], base, scale);
            const int e = label - c.head - p * n;
            if ((unsigned)e < (unsigned)n) g[e] = (T)at_label;
            store_piece(out + c.head + p * n, g);
        }
        for (int p = tid + kHeld * kThreads; p < c.pieces; p += kThreads) {
            V g = piece_grad<T>(load_piece<V>(body + p * n), base, scale);
            const int e = label - c.head - p * n;
            if ((unsigned)e < (unsigned)n) g[e] = (T)at_label;
            store_piece(out + c.head + p * n, g);
        }
        if (extra >= 0) out[extra] = (T)(extra == label ? at_label : scale * grown(xe, base));
    }
}

// ---- the loss ----------------------------------------------------------------------------------
// Its four sums, in a fixed order and in 64 bits, by one work-group.
static constexpr int kSumThreads = 1024;
struct PolicySums {
    double loss, surrogate, kl, clipped;
};
__device__ __forceinline__ PolicySums item_sums(const PolicyArgs& a, int m, double own, double sum, float* __restrict__ logp_out) {
    PolicySums s = {};
    double logp = 0.0;
    if (sum != 0.0 || own != 0.0) {  // (0, 0: it does not score; its logits are all -inf: -inf, 0)
        if (sum == 0.0) {
            logp = own;
        } else {
            logp = own - log(sum);
            const double w = a.weight[m], A = a.advantage[m], ratio = exp(logp - (double)a.old_logp[m]);
            const double bounded = ratio < (double)a.low ? (double)a.low : ratio > (double)a.high ? (double)a.high : ratio;
            const double u = A == 0.0 ? 0.0 : ratio * A, b = A == 0.0 ? 0.0 : bounded * A;
            const bool cut = b < u;
            s.surrogate = w * (cut ? -b : -u);
            s.clipped = cut ? w : 0.0;
            s.loss = s.surrogate;
            if (a.ref_logp) {
                const double far = (double)a.ref_logp[m] - logp;
                s.kl = w * (expm1(far) - far);
                if (a.kl_coef != 0.f) s.loss += (double)a.kl_coef * s.kl;
            }
        }
    }
    if (logp_out) logp_out[m] = (float)logp;
    return s;
}
template <int kThreads>
__device__ __forceinline__ void put_sums(PolicySums s, double (*red)[4], float* __restrict__ loss_out) {
    double of[4] = {s.loss, s.surrogate, s.kl, s.clipped};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) of[i] += __shfl_xor(of[i], d, 64);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][i] = of[i];
    }
    __syncthreads();
    if (threadIdx.x >= 4) return;
    double t = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) t += red[w][threadIdx.x];
    loss_out[threadIdx.x] = (float)t;
}
__global__ __launch_bounds__(kSumThreads) void k_policy_sums(PolicyArgs a, int n, float* __restrict__ logp_out, float* __restrict__ loss_out) {
    __shared__ double red[kSumThreads / 64][4];
    PolicySums s = {};
    for (int m = threadIdx.x; m < n; m += kSumThreads) {
        const PolicySums t = item_sums(a, m, a.own[m], a.sum[m], logp_out);
        s.loss += t.loss;
        s.surrogate += t.surrogate;
        s.kl += t.kl;
        s.clipped += t.clipped;
    }
    put_sums<kSumThreads>(s, red, loss_out);
}

size_t policy_loss_workspace_bytes(int n_items, int vocab) {
    (void)vocab;
    return round_up((size_t)(n_items > 0 ? n_items : 1) * 2 * sizeof(float), 256);
}

static PolicyArgs policy_args(const alch_policy& p, int item0, float* own, float* sum) {
    return {p.label + item0, p.old_logp + item0, p.advantage + item0, p.weight + item0, p.ref_logp ? p.ref_logp + item0 : nullptr,
            1.f - p.clip_low, 1.f + p.clip_high, p.kl_coef, own + item0, sum + item0};
}

template <typename T, bool kGrad>
static void launch_held(const T* logits, long long ld, int rows, int vocab, const PolicyArgs& a, T* dlogits, long long ld_grad, hipStream_t stream) {
    const int pieces = vocab / Piece<T>::n + 1;
    const auto go = [&](auto kernel, int threads) { kernel<<<rows, threads, 0, stream>>>(logits, ld, vocab, a, dlogits, ld_grad); };
    if (pieces <= 256) go(k_policy_held<T, 256, 1, kGrad>, 256);
    else if (pieces <= 256 * 4) go(k_policy_held<T, 256, 4, kGrad>, 256);
    else if (pieces <= 256 * 8) go(k_policy_held<T, 256, 8, kGrad>, 256);
    else if (pieces <= 256 * 16) go(k_policy_held<T, 256, 16, kGrad>, 256);
    else if (pieces <= 512 * 16) go(k_policy_held<T, 512, 16, kGrad>, 512);
    else go(k_policy_held<T, 1024, 16, kGrad>, 1024);
}

template <typename T>
static void launch_rows(const T* logits, long long ld, int rows, int vocab, const PolicyArgs& a, T* dlogits, long long ld_grad, hipStream_t stream) {
    if (dlogits) launch_held<T, true>(logits, ld, rows, vocab, a, dlogits, ld_grad, stream);
    else launch_held<T, false>(logits, ld, rows, vocab, a, dlogits, ld_grad, stream);
}

int launch_policy_rows(alch_dtype dt, const void* logits, long long ld, int rows, int vocab, const alch_policy& p, int item0, void* dlogits,
                       long long ld_grad, float* own, float* sum, hipStream_t stream) {
    if (rows <= 0) return ALCH_OK;
    const double E = (double)dtype_size(dt);
    TraceScope ts(kTraceCrossEntropy, 0.0, (double)rows * vocab * E * (dlogits ? 2 : 1), stream);
    const PolicyArgs a = policy_args(p, item0, own, sum);
    if (dt == ALCH_BF16) launch_rows(static_cast<const __bf16*>(logits), ld, rows, vocab, a, static_cast<__bf16*>(dlogits), ld_grad, stream);
    else launch_rows(static_cast<const float*>(logits), ld, rows, vocab, a, static_cast<float*>(dlogits), ld_grad, stream);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

int launch_policy_sums(const alch_policy& p, float* own, float* sum, float* loss_out, hipStream_t stream) {
    k_policy_sums<<<1, kSumThreads, 0, stream>>>(policy_args(p, 0, own, sum), p.n_items, p.logp_out, loss_out);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
