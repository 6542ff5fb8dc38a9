// Behind the gradients: their norm over all tensors, clipping, and the AdamW update of the weights.
//
//   norm = sqrt(sum g^2), factor = max_norm / norm where norm > max_norm, else 1 (NaN where the norm is no finite number)
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,  w -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay w)
//
// Both are bound by memory: one pass over the gradients for the norm, one for what uses the factor.  All tensors of a call share
// its launches: they are cut into chunks, and every work-group finds the tensor of a chunk in a table that it makes of the tensors'
// lengths.
#include <algorithm>
#include <math.h>

#include "chunk_table.h"
#include "kernels.h"

namespace alch {

static constexpr int kNormBlocks = 1024;

typedef float f32x4_u __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_u __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ double block_sum(double v, double* red /*[4]*/) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// ---- norm and clipping --------------------------------------------------------------------
// A chunk is kBatch pieces of 16 bytes a thread, 16 KB (4 KB: 436 MB 242 instead of 209 us, and the 4 MB of a small fp32 layer, which
// then are chunks for all compute units, 8.7 instead of 7.9).  Both kernels deal the chunks out in the same order, so that what
// fits into an XCD's L2 is there when it is clipped.  Loads and stores are non-temporal: with ordinary stores the norm of 436 MB
// behind a clipping takes 105 us instead of 73, with ordinary loads beside them the clipping 139 instead of 125.
static constexpr int kBatch = 4;

struct ClipChunk {
    const char* grad;
    char* out;
    int elements, dtype;
};
__host__ __device__ inline int clip_elements(int dtype) { return 256 * kBatch * (dtype == ALCH_BF16 ? 8 : 4); }
template <bool kFew>
__device__ __forceinline__ ClipChunk clip_chunk(const ChunkTable<alch_grad_tensor, kFew>& table, int c) {
    const auto k = table.find(c);
    const int chunk = clip_elements(k.t.dtype);
    const long long begin = (long long)k.index * chunk, at = begin * (k.t.dtype == ALCH_BF16 ? 2 : 4);
    return {static_cast<const char*>(k.t.grad) + at, k.t.out ? static_cast<char*>(k.t.out) + at : nullptr, (int)min((long long)chunk, (long long)k.t.n - begin),
            k.t.dtype};
}
// The pieces of a thread.  Of a tensor's last chunk those that lie in it as a whole, the others are zero; behind them at most one
// element a thread, *rest (its index, or -1), *r.  Returns whether the chunk is whole.
__device__ __forceinline__ bool clip_load(const ClipChunk& c, f32x4_u (&v)[kBatch], int* rest, float* r) {
    const f32x4_u* p = reinterpret_cast<const f32x4_u*>(c.grad) + threadIdx.x;
    if (c.elements == clip_elements(c.dtype)) {
#pragma unroll
        for (int b = 0; b < kBatch; ++b) v[b] = __builtin_nontemporal_load(p + 256 * b);
        return true;
    }
    const int n = c.dtype == ALCH_BF16 ? 8 : 4, pieces = c.elements / n;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) v[b] = (int)threadIdx.x + 256 * b < pieces ? __builtin_nontemporal_load(p + 256 * b) : f32x4_u{0.f, 0.f, 0.f, 0.f};
    *rest = pieces * n + (int)threadIdx.x;
    if (*rest >= c.elements) *rest = -1;
    else *r = c.dtype == ALCH_BF16 ? (float)reinterpret_cast<const __bf16*>(c.grad)[*rest] : reinterpret_cast<const float*>(c.grad)[*rest];
    return false;
}

// The squares are added in 64 bits: no gradient of finite numbers overflows there, none vanishes, and the order of the
// additions (which differs with the lengths of the tensors) is not seen in a norm of 32 bits.  They cost nothing beside the
// loads (436 MB: 73.9 us, 73.1 with sums in fp32).
template <bool kFew>
__global__ __launch_bounds__(256) void k_norm(const alch_grad_tensor* __restrict__ tensors, int n, double* __restrict__ partial) {
    __shared__ int first[kFew ? 1 : kMaxTensors + 1];
    __shared__ double red[4];
    const ChunkTable<alch_grad_tensor, kFew> table(tensors, n, clip_elements, first);
    const int chunks = table.chunks;
    double s = 0.0;
    ClipChunk next = {};
    if ((int)blockIdx.x < chunks) next = clip_chunk(table, blockIdx.x);
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const ClipChunk a = next;
        f32x4_u v[kBatch];
        int rest = -1;
        float r = 0.f;
        clip_load(a, v, &rest, &r);
        // (while these are on their way where the table is in registers: they are flat loads, the compiler cannot know where a pointer out of
        // memory points, and a look into LDS waits for those too)
        if (c + (int)gridDim.x < chunks) next = clip_chunk(table, c + gridDim.x);
        if (a.dtype == ALCH_BF16) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const bf16x8_u x = __builtin_bit_cast(bf16x8_u, v[b]);
#pragma unroll
                for (int e = 0; e < 8; ++e) s += (double)(float)x[e] * (double)(float)x[e];
            }
        } else {
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s += (double)v[b][e] * (double)v[b][e];
        }
        if (rest >= 0) s += (double)r * (double)r;
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The factor from the sums that k_norm left, by every work-group for itself and in the same order: a launch for it alone costs more.
struct NormSums {
    double of[kNormBlocks / 256];
};
__device__ __forceinline__ NormSums norm_sums(const double* __restrict__ partial, int blocks) {
    NormSums s;
#pragma unroll
    for (int i = 0; i < kNormBlocks / 256; ++i) s.of[i] = (int)threadIdx.x + 256 * i < blocks ? partial[threadIdx.x + 256 * i] : 0.0;
    return s;
}
__device__ __forceinline__ float clip_factor(const NormSums& sums, float max_norm, float* __restrict__ norm_out) {
    __shared__ double red[4];
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kNormBlocks / 256; ++i) s += sums.of[i];
    const double norm = sqrt(block_sum(s, red));
    const float factor = !(norm < INFINITY) ? NAN : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        norm_out[0] = (float)norm;
        norm_out[1] = factor;
    }
    return factor;
}

template <bool kFew>
__global__ __launch_bounds__(256) void k_clip(const alch_grad_tensor* __restrict__ tensors, int n, const double* __restrict__ partial, int blocks,
                                              float max_norm, float* __restrict__ norm_out) {
    __shared__ int first[kFew ? 1 : kMaxTensors + 1];
    const NormSums sums = norm_sums(partial, blocks);
    const ChunkTable<alch_grad_tensor, kFew> table(tensors, n, clip_elements, first);
    const int chunks = table.chunks;
    ClipChunk a = clip_chunk(table, blockIdx.x);  // (no more work-groups than chunks)
    float factor = 0.f;
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        f32x4_u v[kBatch];
        int rest = -1;
        float r = 0.f;
        const bool full = a.out && clip_load(a, v, &rest, &r);
        ClipChunk next = {};
        if (c + (int)gridDim.x < chunks) next = clip_chunk(table, c + gridDim.x);  // (behind the loads, which the compiler waits for here)
        if (c == (int)blockIdx.x) factor = clip_factor(sums, max_norm, norm_out);
        if (a.out && !(a.out == a.grad && factor == 1.f)) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (a.dtype == ALCH_BF16) {
                    bf16x8_u x = __builtin_bit_cast(bf16x8_u, v[b]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = (__bf16)((float)x[e] * factor);
                    v[b] = __builtin_bit_cast(f32x4_u, x);
                } else {
                    v[b] *= factor;
                }
            }
            f32x4_u* out = reinterpret_cast<f32x4_u*>(a.out) + threadIdx.x;
            if (full) {
#pragma unroll
                for (int b = 0; b < kBatch; ++b) __builtin_nontemporal_store(v[b], out + 256 * b);
            } else {
                const int pieces = a.elements / (a.dtype == ALCH_BF16 ? 8 : 4);
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if ((int)threadIdx.x + 256 * b < pieces) __builtin_nontemporal_store(v[b], out + 256 * b);
            }
            if (rest >= 0) {
                if (a.dtype == ALCH_BF16) reinterpret_cast<__bf16*>(a.out)[rest] = (__bf16)(r * factor);
                else reinterpret_cast<float*>(a.out)[rest] = r * factor;
            }
        }
        a = next;
    }
}

__global__ __launch_bounds__(256) void k_norm_finish(const double* __restrict__ partial, int blocks, float max_norm, float* __restrict__ norm_out) {
    clip_factor(norm_sums(partial, blocks), max_norm, norm_out);
}

size_t grad_clip_workspace_bytes() { return kNormBlocks * sizeof(double); }

int launch_grad_clip(int n_tensors, const alch_grad_tensor* tensors, const alch_grad_tensor* host, float max_norm, float* norm_out, void* workspace,
                     hipStream_t stream) {
    double bytes = 0;
    long long chunks = 0;
    bool any_out = false;
    for (int i = 0; i < n_tensors; ++i) {
        const int chunk = clip_elements(host[i].dtype);
        chunks += (host[i].n + chunk - 1) / chunk;
        any_out = any_out || (host[i].out && host[i].n > 0);
        bytes += (double)host[i].n * dtype_size((alch_dtype)host[i].dtype);
    }
    TraceScope ts(kTraceUpdate, 0.0, bytes * (any_out ? 3 : 1), stream);
    double* partial = static_cast<double*>(workspace);
    const int blocks = (int)std::min<long long>(std::max<long long>(chunks, 1), kNormBlocks);
    const bool few = n_tensors <= 64;
    const auto norm = few ? k_norm<true> : k_norm<false>;
    const auto clip = few ? k_clip<true> : k_clip<false>;
    norm<<<blocks, 256, 0, stream>>>(tensors, n_tensors, partial);
    // a work-group a chunk where the table costs little: 436 MB of nine tensors 204 us, 215 with 1024 work-groups that walk the chunks;
    // 42 MB of 448 tensors 27.9 and 26.3
    if (any_out)
        clip<<<few ? (int)std::min<long long>(chunks, kMaxChunkBlocks) : blocks, 256, 0, stream>>>(tensors, n_tensors, partial, blocks, max_norm, norm_out);
    else
        k_norm_finish<<<1, 256, 0, stream>>>(partial, blocks, max_norm, norm_out);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

// ---- AdamW --------------------------------------------------------------------------------
// Elements of a chunk, four a thread, and a work-group a chunk: 218 M elements 1054 us, 1079 with two pieces a thread, 1192 with 2048
// work-groups that walk the chunks.
static constexpr int kAdamwChunk = 1024;

struct AdamwArgs {
    const alch_adamw_tensor* tensors;
    int n;
    float lr, c1, c2;        // 1 / (1 - b1^step), sqrt(1 / (1 - b2^step))
    float b1, b2, d1, d2, eps;  // d = 1 - b
    double beta1, beta2;     // for a step that is known on the device only
    const float *schedule, *grad_factor;
};

// 1 / (1 - b^t), in 64 bits: for b = 0.999 and t = 1 three of seven digits are lost in 32.
__host__ __device__ inline double correction(double beta, double step) { return 1.0 / (1.0 - pow(beta, step)); }

// Four elements a lane, so that the 64 lanes of a load of fp32 read 1 KB without a gap (eight a lane, as two loads of every other
// 16 bytes, cost 10 % with non-temporal loads).
__device__ __forceinline__ f32x4_u load4(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const f32x4_u*>(p)); }
__device__ __forceinline__ f32x4_u load4(const __bf16* p) {
    return __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const bf16x4_u*>(p)), f32x4_u);
}
__device__ __forceinline__ void store4(float* p, f32x4_u v) { __builtin_nontemporal_store(v, reinterpret_cast<f32x4_u*>(p)); }
__device__ __forceinline__ void store4(__bf16* p, f32x4_u v) {
    __builtin_nontemporal_store(__builtin_convertvector(v, bf16x4_u), reinterpret_cast<bf16x4_u*>(p));
}

struct AdamwChunk {
    alch_adamw_tensor t;
    long long at;
    int elements;
};
template <bool kFew>
__device__ __forceinline__ AdamwChunk adamw_chunk(const ChunkTable<alch_adamw_tensor, kFew>& table, int c) {
    const auto k = table.find(c);
    const long long at = (long long)k.index * kAdamwChunk;
    return {k.t, at, (int)min((long long)kAdamwChunk, (long long)k.t.n - at)};
}

struct AdamwRates {
    float factor, lr, c1, c2;
};
__device__ __forceinline__ void adamw_element(const AdamwArgs& a, const AdamwRates& r, float decay, float g, float& m, float& v, float& w) {
    const float x = g * r.factor;
    m = a.b1 * m + a.d1 * x;
    v = a.b2 * v + a.d2 * x * x;
    w -= r.lr * (m * r.c1 / (sqrtf(v) * r.c2 + a.eps) + decay * w);
}

template <typename T, bool kMaster>
__device__ __forceinline__ void adamw(const AdamwChunk& k, const AdamwArgs& a, const AdamwRates& r) {
    T* param = static_cast<T*>(k.t.param) + k.at;
    const T* grad = static_cast<const T*>(k.t.grad) + k.at;
    float *m = k.t.m + k.at, *v = k.t.v + k.at, *master = kMaster ? k.t.master + k.at : nullptr;
    const int at = threadIdx.x * 4;
    if (at + 4 <= k.elements) {
        const f32x4_u g4 = load4(grad + at);
        f32x4_u m4 = load4(m + at), v4 = load4(v + at), w4;
        if constexpr (kMaster) w4 = load4(master + at);
        else w4 = load4(param + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float me = m4[e], ve = v4[e], we = w4[e];
            adamw_element(a, r, k.t.weight_decay, g4[e], me, ve, we);
            m4[e] = me; v4[e] = ve; w4[e] = we;
        }
        store4(m + at, m4);
        store4(v + at, v4);
        if constexpr (kMaster) store4(master + at, w4);
        store4(param + at, w4);
    }
    const int i = (k.elements & ~3) + (int)threadIdx.x;  // behind the last whole piece
    if (i < k.elements) {
        float me = m[i], ve = v[i], we = kMaster ? master[i] : (float)param[i];
        adamw_element(a, r, k.t.weight_decay, (float)grad[i], me, ve, we);
        m[i] = me;
        v[i] = ve;
        if constexpr (kMaster) master[i] = we;
        param[i] = (T)we;
    }
}

template <bool kFew>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a) {
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
    const ChunkTable<alch_adamw_tensor, kFew> table(a.tensors, a.n, [](int) { return kAdamwChunk; }, first);
    if (a.schedule) __syncthreads();  // (its rates have been written)
    const AdamwRates r{factor, a.schedule ? shared_c[0] : a.lr, a.schedule ? shared_c[1] : a.c1, a.schedule ? shared_c[2] : a.c2};
    for (int c = blockIdx.x; c < table.chunks; c += gridDim.x) {
        const AdamwChunk k = adamw_chunk(table, c);
        if (k.t.dtype == ALCH_BF16) {
            if (k.t.master) adamw<__bf16, true>(k, a, r);
            else adamw<__bf16, false>(k, a, r);
        } else {
            if (k.t.master) adamw<float, true>(k, a, r);
            else adamw<float, false>(k, a, r);
        }
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
    const AdamwArgs a{tensors, n_tensors, (float)p.lr, p.schedule ? 0.f : (float)correction(p.beta1, p.step),
                      p.schedule ? 0.f : (float)sqrt(correction(p.beta2, p.step)),
                      (float)p.beta1, (float)p.beta2, (float)(1.0 - p.beta1), (float)(1.0 - p.beta2), (float)p.eps, p.beta1, p.beta2,
                      p.schedule, p.grad_factor};
    const auto kernel = n_tensors <= 64 ? k_adamw<true> : k_adamw<false>;
    kernel<<<(int)std::min<long long>(chunks, kMaxChunkBlocks), 256, 0, stream>>>(a);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
