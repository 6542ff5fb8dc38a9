// Behind the gradients: their norm over all tensors, clipping, and the AdamW update of the weights.
//
//   norm = sqrt(sum g^2), factor = max_norm / norm where norm > max_norm, else 1 (NaN where the norm is no finite number)
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,  w -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay w)
//
// Both are bound by memory: one pass over the gradients for the norm, one for what uses the factor.  All tensors of a call share
// its launches: they are cut into chunks, and every work-group finds the tensor of a chunk in a table of the tensors' first
// chunks, which it makes in LDS from the tensors' lengths.
#include <algorithm>
#include <math.h>

#include "kernels.h"

namespace alch {

static constexpr int kMaxTensors = ALCH_MAX_TENSORS;
static constexpr int kNormBlocks = 1024;

typedef float f32x4_u __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_u __attribute__((ext_vector_type(8)));

// first[i] = chunks of the tensors before i, first[n] = all of them.  Work-groups of 256 threads.
template <typename Tensor>
__device__ __forceinline__ void chunk_table(const Tensor* __restrict__ tensors, int n, int chunk, int* first /*[n + 1]*/) {
    __shared__ int wave_total[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int carry = 0;
    for (int base = 0; base < n; base += 256) {
        const int i = base + tid, own = i < n ? (int)((tensors[i].n + chunk - 1) / chunk) : 0;
        int inc = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(inc, d, 64);
            if (lane >= d) inc += o;
        }
        if (lane == 63) wave_total[wave] = inc;
        __syncthreads();
        int before = carry;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) before += wave_total[w];
            carry += wave_total[w];
        }
        if (i < n) first[i] = before + inc - own;
        __syncthreads();
    }
    if (tid == 0) first[n] = carry;
    __syncthreads();
}

// The tensor of a chunk: the last one whose first chunk is not behind it (of empty ones, which begin where the next one does,
// the last, which is not empty).  64 candidates at a time.
__device__ __forceinline__ int tensor_of(const int* first, int n, int chunk) {
    const int lane = threadIdx.x & 63;
    int lo = 0, step = 1;
    while (step * 64 < n) step *= 64;
    for (; step >= 1; step /= 64) {
        const int i = lo + lane * step;
        lo += (__popcll(__ballot(i < n && first[i] <= chunk)) - 1) * step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ double block_sum(double v, double* red /*[4]*/) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Eight elements of a tensor from element at on, as fp32; what lies behind its end counts as 0.
__device__ __forceinline__ void load8(const void* p, int dtype, long long at, int count, float (&x)[8]) {
    if (count >= 8) {
        if (dtype == ALCH_BF16) {
            const bf16x8_u v = *reinterpret_cast<const bf16x8_u*>(static_cast<const __bf16*>(p) + at);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
        } else {
            const f32x4_u *q = reinterpret_cast<const f32x4_u*>(static_cast<const float*>(p) + at);
            const f32x4_u a = q[0], b = q[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = e >= count ? 0.f : dtype == ALCH_BF16 ? (float)static_cast<const __bf16*>(p)[at + e] : static_cast<const float*>(p)[at + e];
    }
}
__device__ __forceinline__ void store8(void* p, int dtype, long long at, int count, const float (&x)[8]) {
    if (count >= 8) {
        if (dtype == ALCH_BF16) {
            bf16x8_u v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
            *reinterpret_cast<bf16x8_u*>(static_cast<__bf16*>(p) + at) = v;
        } else {
            f32x4_u a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) { a[e] = x[e]; b[e] = x[4 + e]; }
            f32x4_u* q = reinterpret_cast<f32x4_u*>(static_cast<float*>(p) + at);
            q[0] = a;
            q[1] = b;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < count) {
                if (dtype == ALCH_BF16) static_cast<__bf16*>(p)[at + e] = (__bf16)x[e];
                else static_cast<float*>(p)[at + e] = x[e];
            }
    }
}

// ---- norm and clipping --------------------------------------------------------------------
static constexpr int kClipChunk = 8192;  // elements

// The squares are added in 64 bits: no gradient of finite numbers overflows there, none vanishes, and the order of the additions
// (that of the chunks, which differs with the lengths of the tensors) is not seen in a norm of 32 bits.
__global__ __launch_bounds__(256) void k_norm(const alch_grad_tensor* __restrict__ tensors, int n, double* __restrict__ partial) {
    __shared__ int first[kMaxTensors + 1];
    __shared__ double red[4];
    chunk_table(tensors, n, kClipChunk, first);
    const int chunks = first[n];
    double s = 0.0;
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = tensor_of(first, n, c);
        const alch_grad_tensor a = tensors[t];
        const long long begin = (long long)(c - first[t]) * kClipChunk;
        const int len = (int)min((long long)kClipChunk, (long long)a.n - begin);
#pragma unroll 4
        for (int i = threadIdx.x * 8; i < len; i += 2048) {
            float x[8];
            load8(a.grad, a.dtype, begin + i, len - i, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) s += (double)x[e] * (double)x[e];
        }
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ float clip_factor(double sum, float max_norm, float* norm_out) {
    const double norm = sqrt(sum);
    const float factor = !(norm < INFINITY) ? NAN : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
    if (norm_out) {
        norm_out[0] = (float)norm;
        norm_out[1] = factor;
    }
    return factor;
}

__global__ __launch_bounds__(256) void k_norm_finish(const double* __restrict__ partial, int blocks, float max_norm, float* __restrict__ norm_out) {
    __shared__ double red[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < blocks; i += 256) s += partial[i];
    s = block_sum(s, red);
    if (threadIdx.x == 0) clip_factor(s, max_norm, norm_out);
}

__global__ __launch_bounds__(256) void k_clip(const alch_grad_tensor* __restrict__ tensors, int n, const float* __restrict__ norm) {
    __shared__ int first[kMaxTensors + 1];
    chunk_table(tensors, n, kClipChunk, first);
    const int chunks = first[n];
    const float factor = norm[1];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = tensor_of(first, n, c);
        const alch_grad_tensor a = tensors[t];
        if (!a.out) continue;
        const long long begin = (long long)(c - first[t]) * kClipChunk;
        const int len = (int)min((long long)kClipChunk, (long long)a.n - begin);
        for (int i = threadIdx.x * 8; i < len; i += 2048) {
            float x[8];
            load8(a.grad, a.dtype, begin + i, len - i, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= factor;
            store8(a.out, a.dtype, begin + i, len - i, x);
        }
    }
}

size_t grad_clip_workspace_bytes() { return kNormBlocks * sizeof(double); }

int launch_grad_clip(int n_tensors, const alch_grad_tensor* tensors, const alch_grad_tensor* host, float max_norm, float* norm_out, void* workspace,
                     hipStream_t stream) {
    long long chunks = 0;
    double bytes = 0;
    bool any_out = false;
    for (int i = 0; i < n_tensors; ++i) {
        chunks += (host[i].n + kClipChunk - 1) / kClipChunk;
        any_out = any_out || (host[i].out && host[i].n > 0);
        bytes += (double)host[i].n * dtype_size((alch_dtype)host[i].dtype) * (host[i].out ? 2 : 1);
    }
    TraceScope ts(kTraceUpdate, 0.0, bytes, stream);
    double* partial = static_cast<double*>(workspace);
    const int blocks = (int)std::min<long long>(std::max<long long>(chunks, 1), kNormBlocks);
    k_norm<<<blocks, 256, 0, stream>>>(tensors, n_tensors, partial);
    k_norm_finish<<<1, 256, 0, stream>>>(partial, blocks, max_norm, norm_out);
    if (any_out) k_clip<<<(int)std::min<long long>(chunks, 2048), 256, 0, stream>>>(tensors, n_tensors, norm_out);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

// ---- AdamW --------------------------------------------------------------------------------
static constexpr int kAdamwChunk = 2048;  // elements: eight a thread

struct AdamwArgs {
    const alch_adamw_tensor* tensors;
    int n;
    float lr, c1, c2;        // c = 1 / (1 - b^step)
    float b1, b2, d1, d2, eps;  // d = 1 - b
    double beta1, beta2;     // for a step that is known on the device only
    const float *schedule, *grad_factor;
};

// 1 / (1 - b^t), in 64 bits: for b = 0.999 and t = 1 three of seven digits are lost in 32.
__host__ __device__ inline float correction(double beta, double step) { return (float)(1.0 / (1.0 - pow(beta, step))); }

__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a) {
    __shared__ int first[kMaxTensors + 1];
    __shared__ float shared_c[3];
    const float factor = a.grad_factor ? *a.grad_factor : 1.f;
    if (!(fabsf(factor) < INFINITY)) return;  // (the gradients are of no use: nothing changes)
    if (a.schedule && threadIdx.x == 0) {
        const double step = a.schedule[1];
        shared_c[0] = a.schedule[0];
        shared_c[1] = correction(a.beta1, step);
        shared_c[2] = correction(a.beta2, step);
    }
    chunk_table(a.tensors, a.n, kAdamwChunk, first);
    const int chunks = first[a.n];
    const float lr = a.schedule ? shared_c[0] : a.lr, c1 = a.schedule ? shared_c[1] : a.c1, c2 = a.schedule ? shared_c[2] : a.c2;
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int ti = tensor_of(first, a.n, c);
        const alch_adamw_tensor t = a.tensors[ti];
        const long long at = (long long)(c - first[ti]) * kAdamwChunk + threadIdx.x * 8;
        const int count = (int)min((long long)8, (long long)t.n - at);
        if (count <= 0) continue;
        float g[8], m[8], v[8], w[8];
        load8(t.grad, t.dtype, at, count, g);
        load8(t.m, ALCH_F32, at, count, m);
        load8(t.v, ALCH_F32, at, count, v);
        if (t.master) load8(t.master, ALCH_F32, at, count, w);
        else load8(t.param, t.dtype, at, count, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = g[e] * factor;
            m[e] = a.b1 * m[e] + a.d1 * x;
            v[e] = a.b2 * v[e] + a.d2 * x * x;
            w[e] -= lr * (m[e] * c1 / (sqrtf(v[e] * c2) + a.eps) + t.weight_decay * w[e]);
        }
        store8(t.m, ALCH_F32, at, count, m);
        store8(t.v, ALCH_F32, at, count, v);
        if (t.master) store8(t.master, ALCH_F32, at, count, w);
        store8(t.param, t.dtype, at, count, w);
    }
}

int launch_adamw(int n_tensors, const alch_adamw_tensor* tensors, const alch_adamw_tensor* host, const alch_adamw& p, hipStream_t stream) {
    long long chunks = 0;
    double bytes = 0;
    for (int i = 0; i < n_tensors; ++i) {
        chunks += (host[i].n + kAdamwChunk - 1) / kAdamwChunk;
        const double E = (double)dtype_size((alch_dtype)host[i].dtype);
        bytes += (double)host[i].n * (2 * E + 16 + (host[i].master ? 8 : E));
    }
    if (chunks == 0) return ALCH_OK;
    TraceScope ts(kTraceUpdate, 0.0, bytes, stream);
    const AdamwArgs a{tensors, n_tensors, (float)p.lr, p.schedule ? 0.f : correction(p.beta1, p.step), p.schedule ? 0.f : correction(p.beta2, p.step),
                      (float)p.beta1, (float)p.beta2, (float)(1.0 - p.beta1), (float)(1.0 - p.beta2), (float)p.eps, p.beta1, p.beta2,
                      p.schedule, p.grad_factor};
    k_adamw<<<(int)std::min<long long>(chunks, 2048), 256, 0, stream>>>(a);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
