// The clipped policy loss of sampled tokens with its KL term (preference alignment on served responses), from rows of logits.
//
//   logz = log sum_v exp(x_v),  logp = x_label - logz,  ratio = exp(logp - old),  u = ratio A,  b = clamp(ratio, 1 - lo, 1 + hi) A
//   kl = exp(ref - logp) - (ref - logp) - 1,   loss = sum w (-min(u, b) + c kl)
//   dx_v = d ((v == label) - exp(x_v - logz)),   d = w (-(b < u ? 0 : u) + c (1 - exp(ref - logp)))
//
// A row of logits is one softmax, and its gradient needs the normaliser alone: bound by memory, a row read once and written once.
#include "kernels.h"

namespace alch {

typedef float f32x4_p __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_p __attribute__((ext_vector_type(8)));

static constexpr int kThreads = 1024;
static constexpr float kLog2e = 1.4426950408889634f;

struct PolicyArgs {
    const int* label;
    const float *old_logp, *advantage, *weight, *ref_logp;
    float low, high, kl_coef;  // 1 - clip_low, 1 + clip_high
    float* logp_out;
    float* terms;  // [4, stride]: w * loss, w * surrogate, w * kl, w * clipped of every item
    long long stride;
};

// What an item adds to the sums, and the factor of its gradient.
struct Scored {
    float loss, surrogate, kl, clipped, d;
};
__device__ __forceinline__ Scored score(const PolicyArgs& a, int m, float logp) {
    const float w = a.weight[m], A = a.advantage[m], ratio = expf(logp - a.old_logp[m]);
    const float bounded = ratio < a.low ? a.low : ratio > a.high ? a.high : ratio;  // (NaN stays)
    const float u = A == 0.f ? 0.f : ratio * A, b = A == 0.f ? 0.f : bounded * A;
    const bool cut = b < u;
    Scored s;
    float d = cut ? 0.f : -u;
    s.surrogate = cut ? -b : -u;
    s.kl = 0.f;
    if (a.ref_logp) {
        const float far = a.ref_logp[m] - logp, grown = expm1f(far);
        s.kl = grown - far;
        if (a.kl_coef != 0.f) d -= a.kl_coef * grown;
    }
    s.loss = w * (s.surrogate + (a.kl_coef != 0.f ? a.kl_coef * s.kl : 0.f));
    s.surrogate *= w;
    s.kl *= w;
    s.clipped = cut ? w : 0.f;
    s.d = w * d;
    return s;
}
__device__ __forceinline__ void put_terms(const PolicyArgs& a, int m, float logp, const Scored& s) {
    a.terms[m] = s.loss;
    a.terms[a.stride + m] = s.surrogate;
    a.terms[2 * a.stride + m] = s.kl;
    a.terms[3 * a.stride + m] = s.clipped;
    if (a.logp_out) a.logp_out[m] = logp;
}
__device__ __forceinline__ bool scores(const PolicyArgs& a, int m, int vocab) { return (unsigned)a.label[m] < (unsigned)vocab && a.weight[m] != 0.f; }

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

template <typename T>
__global__ __launch_bounds__(kThreads) void k_policy_rows(const T* logits, long long ld, int vocab, PolicyArgs a, T* dlogits, long long ld_grad) {
    __shared__ float red[2][kThreads / 64];
    const int m = blockIdx.x, tid = threadIdx.x;
    const T* x = logits + m * ld;
    T* out = dlogits ? dlogits + m * ld_grad : nullptr;
    const bool counted = scores(a, m, vocab);
    float most = -INFINITY, base = 0.f, sum = 0.f, logp = 0.f;
    Scored s = {};
    if (counted) {
        for (int v = tid; v < vocab; v += kThreads) most = fmaxf(most, (float)x[v]);
        most = wave_max(most);
        if ((tid & 63) == 0) red[0][tid >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) most = fmaxf(most, red[0][i]);
        base = most == -INFINITY ? 0.f : most;  // (without a finite logit the sum is 0, or NaN)
        for (int v = tid; v < vocab; v += kThreads) sum += __builtin_amdgcn_exp2f(((float)x[v] - base) * kLog2e);
        sum = wave_sum(sum);
        if ((tid & 63) == 0) red[1][tid >> 6] = sum;
        const float own = (float)x[a.label[m]];
        __syncthreads();  // (everybody has read the label's logit before it may be overwritten)
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) sum += red[1][i];
        if (sum == 0.f) {
            logp = -INFINITY;
        } else {
            logp = own - base - logf(sum);
            s = score(a, m, logp);
        }
    }
    if (tid == 0) put_terms(a, m, logp, s);
    if (!out) return;
    const float scale = -s.d / sum;
    for (int v = tid; v < vocab; v += kThreads) {
        float g = 0.f;
        if (counted && sum != 0.f)  // (1 - p of the label without the difference)
            g = v == a.label[m] ? s.d * -expm1f(logp) : scale * __builtin_amdgcn_exp2f(((float)x[v] - base) * kLog2e);
        out[v] = (T)g;
    }
}

// The four sums, in a fixed order and in 64 bits: terms of either sign cancel.
__global__ __launch_bounds__(kThreads) void k_policy_sums(const float* __restrict__ terms, long long stride, int n, float* __restrict__ loss_out) {
    __shared__ double red[kThreads / 64];
    const int tid = threadIdx.x;
    double s = 0.0;
    for (int m = tid; m < n; m += kThreads) s += (double)terms[blockIdx.x * stride + m];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((tid & 63) == 0) red[tid >> 6] = s;
    __syncthreads();
    if (tid != 0) return;
    s = 0.0;
    for (int i = 0; i < kThreads / 64; ++i) s += red[i];
    loss_out[blockIdx.x] = (float)s;
}

size_t policy_loss_workspace_bytes(int n_items, int vocab) {
    (void)vocab;
    return round_up((size_t)(n_items > 0 ? n_items : 1) * 4 * sizeof(float), 256);
}

// Rows of a call whose items are item0 .. item0 + rows - 1 of policy; terms [4, stride] are indexed by item.
int launch_policy_rows(alch_dtype dt, const void* logits, long long ld, int rows, int vocab, const alch_policy& p, int item0, void* dlogits,
                       long long ld_grad, float* terms, long long stride, hipStream_t stream) {
    if (rows <= 0) return ALCH_OK;
    const double E = (double)dtype_size(dt);
    TraceScope ts(kTraceCrossEntropy, 0.0, (double)rows * vocab * E * (dlogits ? 2 : 1), stream);
    const PolicyArgs a{p.label + item0, p.old_logp + item0, p.advantage + item0, p.weight + item0, p.ref_logp ? p.ref_logp + item0 : nullptr,
                       1.f - p.clip_low, 1.f + p.clip_high, p.kl_coef, p.logp_out ? p.logp_out + item0 : nullptr, terms + item0, stride};
    if (dt == ALCH_BF16)
        k_policy_rows<__bf16><<<rows, kThreads, 0, stream>>>(static_cast<const __bf16*>(logits), ld, vocab, a, static_cast<__bf16*>(dlogits), ld_grad);
    else
        k_policy_rows<float><<<rows, kThreads, 0, stream>>>(static_cast<const float*>(logits), ld, vocab, a, static_cast<float*>(dlogits), ld_grad);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

int launch_policy_sums(const float* terms, long long stride, int n_items, float* loss_out, hipStream_t stream) {
    k_policy_sums<<<4, kThreads, 0, stream>>>(terms, stride, n_items, loss_out);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
