// Embedding rows in front of layer 0 and the gradient of their table behind it.
//
//   forward   X[t] = scale * W[id_t]                          (a zero row where id_t is outside 0 .. vocab-1)
//   backward  dW[v] (+)= scale * sum over t with id_t = v of dX[t]
//
// Both are bound by memory.  The backward pass needs the tokens of a row next to one another: they are sorted by id (stable,
// so that every sum runs over ascending tokens and results repeat bit for bit; no float atomics), and the sorted tokens are
// cut into parts of equal length, so that one id that half of a batch shares is no longer a chain than any other.
#include <algorithm>

#include "kernels.h"

namespace alch {

typedef unsigned int u32x4_e __attribute__((ext_vector_type(4)));

// ---- forward ----------------------------------------------------------------------------

// kVec elements a lane (16 bytes, or single elements where rows are not made of aligned 16-byte pieces), lanes_per_row lanes
// (a power of two) share a row.
template <typename T, int kVec>
__global__ __launch_bounds__(256) void k_embed(const int* __restrict__ ids, const T* __restrict__ W, T* __restrict__ X, int n_tokens, int vocab,
                                               int hidden, float scale, int log_lanes) {
    typedef T vec __attribute__((ext_vector_type(kVec)));
    const int lanes = 1 << log_lanes, rows = 256 >> log_lanes, c0 = (threadIdx.x & (lanes - 1)) * kVec;
    for (long long t = (long long)blockIdx.x * rows + (threadIdx.x >> log_lanes); t < n_tokens; t += (long long)gridDim.x * rows) {
        const int id = ids[t];
        const bool valid = (unsigned)id < (unsigned)vocab;
        const T* src = W + (long long)(valid ? id : 0) * hidden;
        T* dst = X + t * hidden;
        for (int c = c0; c < hidden; c += lanes * kVec) {
            vec v = {};
            if (valid) {
                v = *reinterpret_cast<const vec*>(src + c);
#pragma unroll
                for (int e = 0; e < kVec; ++e) v[e] = (T)((float)v[e] * scale);
            }
            *reinterpret_cast<vec*>(dst + c) = v;
        }
    }
}

template <typename T>
static void embed_launch(const int* ids, const void* W, void* X, int n, int vocab, int hidden, float scale, hipStream_t stream) {
    constexpr int kVec = 16 / sizeof(T);
    const bool vec = hidden % kVec == 0;
    const int pieces = vec ? hidden / kVec : hidden;
    int log_lanes = 0;
    while (log_lanes < 8 && (1 << log_lanes) < pieces) ++log_lanes;
    const int grid = std::min(ceil_div(n, 256 >> log_lanes), 1 << 20);
    if (vec)
        k_embed<T, kVec><<<grid, 256, 0, stream>>>(ids, (const T*)W, (T*)X, n, vocab, hidden, scale, log_lanes);
    else
        k_embed<T, 1><<<grid, 256, 0, stream>>>(ids, (const T*)W, (T*)X, n, vocab, hidden, scale, log_lanes);
}

int launch_embed(alch_dtype dt, const int* ids, const void* W, void* X, int n_tokens, int vocab, int hidden, float scale, hipStream_t stream) {
    if (n_tokens <= 0) return ALCH_OK;
    TraceScope ts(kTraceEmbed, (double)n_tokens * hidden, 2.0 * n_tokens * hidden * dtype_size(dt), stream);
    if (dt == ALCH_BF16)
        embed_launch<__bf16>(ids, W, X, n_tokens, vocab, hidden, scale, stream);
    else
        embed_launch<float>(ids, W, X, n_tokens, vocab, hidden, scale, stream);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

// ---- backward: tokens sorted by id --------------------------------------------------------
// A radix sort from the lowest digit, two launches a digit: counts of the digits in every block of tokens, then every block
// finds the places of its tokens from the counts of all blocks (at most kSortBlocks of them) and writes them there.  An id
// outside the table counts as `vocab`: it is sorted behind all others.
static constexpr int kSortBlocks = 512;
static constexpr int kDigitBits = 10;

struct SortPlan {
    int bits, passes, digit;  // of the key, digits, bits a digit
    int per_block, blocks;    // tokens
};
static SortPlan plan_sort(int n, int vocab) {
    SortPlan p;
    p.bits = 1;
    while (p.bits < 31 && (1u << p.bits) <= (unsigned)vocab) ++p.bits;
    p.passes = ceil_div(p.bits, kDigitBits);
    p.digit = ceil_div(p.bits, p.passes);
    p.per_block = std::max(1024, (int)round_up((size_t)ceil_div(n, kSortBlocks), 256));
    p.blocks = ceil_div(n, p.per_block);
    return p;
}

__device__ __forceinline__ int key_of(int id, int vocab) { return (unsigned)id < (unsigned)vocab ? id : vocab; }

__global__ __launch_bounds__(256) void k_sort_count(const int* __restrict__ keys, int n, int vocab, int shift, int bins, int per_block,
                                                    int* __restrict__ counts) {
    __shared__ int hist[1 << kDigitBits];
    for (int b = threadIdx.x; b < bins; b += 256) hist[b] = 0;
    __syncthreads();
    const int begin = blockIdx.x * per_block, end = min(n, begin + per_block);
    for (int t = begin + threadIdx.x; t < end; t += 256) atomicAdd(&hist[(key_of(keys[t], vocab) >> shift) & (bins - 1)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += 256) counts[(long long)blockIdx.x * bins + b] = hist[b];
}

// tokens == null: the order before the first digit.  where (may be null): where[v] = some token with id v; nothing else of it is
// written, a reader checks what it finds there against the ids.
__global__ __launch_bounds__(256) void k_sort_place(const int* __restrict__ keys, const int* __restrict__ tokens, int n, int vocab, int shift,
                                                    int digit_bits, int per_block, const int* __restrict__ counts, int blocks,
                                                    int* __restrict__ keys_out, int* __restrict__ tokens_out, int* __restrict__ where) {
    constexpr int kBins = 1 << kDigitBits;
    __shared__ int base[kBins];             // tokens of lower digits, and of this digit in blocks before this one
    __shared__ int place[4][kBins];         // first place of this digit's tokens of every wavefront
    __shared__ int sums[4];
    const int bins = 1 << digit_bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before[kBins / 256], total[kBins / 256];
#pragma unroll
    for (int j = 0; j < kBins / 256; ++j) {
        const int b = tid + 256 * j;
        before[j] = total[j] = 0;
        if (b < bins) {
            for (int k = 0; k < blocks; ++k) {
                const int c = counts[(long long)k * bins + b];
                total[j] += c;
                if (k < (int)blockIdx.x) before[j] += c;
            }
            base[b] = total[j];
        }
#pragma unroll
        for (int w = 0; w < 4; ++w)
            if (b < bins) place[w][b] = 0;
    }
    __syncthreads();
    // exclusive scan over the digits, kBins / 256 consecutive ones a thread
    int own[kBins / 256], run = 0;
#pragma unroll
    for (int j = 0; j < kBins / 256; ++j) {
        const int b = tid * (kBins / 256) + j;
        own[j] = run;
        run += b < bins ? base[b] : 0;
    }
    int inc = run;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(inc, d, 64);
        if (lane >= d) inc += o;
    }
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    int ahead = inc - run;
    for (int w = 0; w < wave; ++w) ahead += sums[w];
#pragma unroll
    for (int j = 0; j < kBins / 256; ++j) {
        const int b = tid * (kBins / 256) + j;
        if (b < bins) base[b] = ahead + own[j];
    }
    // every wavefront counts its quarter of the block
    const int quarter = per_block / 4, begin = blockIdx.x * per_block + wave * quarter, end = min(n, begin + quarter);
    for (int t = begin + lane; t < end; t += 64) atomicAdd(&place[wave][(key_of(keys[t], vocab) >> shift) & (bins - 1)], 1);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kBins / 256; ++j) {
        const int b = tid + 256 * j;
        if (b < bins) {
            int at = base[b] + before[j];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int c = place[w][b];
                place[w][b] = at;
                at += c;
            }
        }
    }
    __syncthreads();
    // 64 tokens at a time, in their order: a lane's place is behind the lanes before it that have the same digit
    volatile int* mine = place[wave];
    for (int t0 = begin; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        const bool live = t < end;
        const int key = live ? key_of(keys[t], vocab) : 0, digit = (key >> shift) & (bins - 1);
        unsigned long long same = __ballot(live);
        for (int b = 0; b < digit_bits; ++b) {
            const unsigned long long set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const int at = live ? mine[digit] : 0;
        __builtin_amdgcn_wave_barrier();  // (a wavefront's LDS accesses are carried out in their order)
        if (live && rank == 0) mine[digit] = at + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (live) {
            const int token = tokens ? tokens[t] : t;
            keys_out[at + rank] = key;
            tokens_out[at + rank] = token;
            if (where && key < vocab) where[key] = token;
        }
    }
}

// ---- backward: sums ----------------------------------------------------------------------
// kPart sorted tokens a wavefront and 64 * kVec columns.  A row whose tokens lie in one part is finished here; what crosses
// into other parts is left as fp32 sums, [part][0] of the row that came from the part before, [part][1] of the one that
// begins here and goes on.
static constexpr int kPart = 32;

template <typename T, int kVec>
__device__ __forceinline__ void store_row(T* dst, const float (&s)[kVec], float scale, int accumulate) {
    typedef T vec __attribute__((ext_vector_type(kVec)));
    vec o;
    if (accumulate) {
        o = *reinterpret_cast<const vec*>(dst);
#pragma unroll
        for (int e = 0; e < kVec; ++e) o[e] = (T)((float)o[e] + scale * s[e]);
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) o[e] = (T)(scale * s[e]);
    }
    *reinterpret_cast<vec*>(dst) = o;
}

template <typename T, int kVec>
__global__ __launch_bounds__(256) void k_embed_sums(const int* __restrict__ keys, const int* __restrict__ tokens, int n, int vocab, int hidden,
                                                    const T* __restrict__ dX, float scale, int accumulate, T* __restrict__ dW,
                                                    float* __restrict__ partial, int stride, int tiles, long long units) {
    typedef T vec __attribute__((ext_vector_type(kVec)));
    const int lane = threadIdx.x & 63;
    for (long long u = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (long long)gridDim.x * 4) {
        const int part = __builtin_amdgcn_readfirstlane((int)(u / tiles)), tile = __builtin_amdgcn_readfirstlane((int)(u % tiles));
        const int p0 = part * kPart, count = min(kPart, n - p0), c = (tile * 64 + lane) * kVec;
        const bool in = c < hidden;
        // the keys of the part, of its neighbours, and the tokens
        const int my_key = lane < count ? keys[p0 + lane] : -1, my_token = lane < count ? tokens[p0 + lane] : 0;
        const int key_before = p0 > 0 ? keys[p0 - 1] : -1, key_behind = p0 + count < n ? keys[p0 + count] : -1;
        float s[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) s[e] = 0.f;
        bool begins = __builtin_amdgcn_readlane(my_key, 0) != key_before;
        for (int i = 0; i < count; ++i) {
            const int key = __builtin_amdgcn_readlane(my_key, i);
            if (key >= vocab) break;  // padding: behind all others
            const int token = __builtin_amdgcn_readlane(my_token, i);
            if (in) {
                const vec v = *reinterpret_cast<const vec*>(dX + (long long)token * hidden + c);
#pragma unroll
                for (int e = 0; e < kVec; ++e) s[e] += (float)v[e];
            }
            const int next = i + 1 < count ? __builtin_amdgcn_readlane(my_key, i + 1) : key_behind;
            if (next != key || i + 1 == count) {
                const bool ends = next != key;
                if (in) {
                    if (begins && ends) {
                        store_row<T, kVec>(dW + (long long)key * hidden + c, s, scale, accumulate);
                    } else {
                        float* p = partial + ((long long)part * 2 + (begins ? 1 : 0)) * stride + c;
#pragma unroll
                        for (int e = 0; e < kVec; ++e) p[e] = s[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < kVec; ++e) s[e] = 0.f;
                begins = true;
            }
        }
    }
}

// Rows that lie in several parts: the part in which a row begins adds what the parts behind it have of it, in their order.
// One work-group a part and 256 columns, four wavefronts with a quarter of the parts each.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_join(const int* __restrict__ keys, int n, int vocab, int hidden, float scale, int accumulate,
                                                    T* __restrict__ dW, const float* __restrict__ partial, int stride, int parts) {
    __shared__ float red[4][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c0 = blockIdx.y * 256;
    for (int part = blockIdx.x; part < parts - 1; part += gridDim.x) {
        const int p0 = part * kPart, key = keys[p0 + kPart - 1];
        if (key >= vocab || keys[p0 + kPart] != key) continue;                  // no row goes on
        if (keys[p0] == key && p0 > 0 && keys[p0 - 1] == key) continue;          // it began before this part
        int more = 0;                                                            // parts behind this one that it lies in
        for (int base = part + 1; base < parts; base += 64) {
            const unsigned long long other = __ballot(base + lane >= parts || keys[(long long)min(base + lane, parts - 1) * kPart] != key);
            more += other ? __ffsll(other) - 1 : 64;
            if (other) break;
        }
        // pieces 0 .. more: the part's own, then theirs
        const int pieces = more + 1, per = (pieces + 3) / 4, first = wave * per, last = min(pieces, first + per);
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i = first; i < last; ++i) {
            const float* p = partial + ((long long)(part + i) * 2 + (i == 0 ? 1 : 0)) * stride + c0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c0 + 64 * j + lane < hidden) s[j] += p[64 * j + lane];
        }
        __syncthreads();  // (the sums of the row before have been read)
#pragma unroll
        for (int j = 0; j < 4; ++j) red[wave][64 * j + lane] = s[j];
        __syncthreads();
        const int c = c0 + threadIdx.x;
        if (c < hidden) {
            const float sum = red[0][threadIdx.x] + red[1][threadIdx.x] + red[2][threadIdx.x] + red[3][threadIdx.x];
            T* dst = dW + (long long)key * hidden + c;
            *dst = (T)(accumulate ? (float)*dst + scale * sum : scale * sum);
        }
    }
}

// Rows that no token has: zeros.  where[v] is whatever the workspace held unless a token has id v.
template <typename T, int kVec>
__global__ __launch_bounds__(256) void k_embed_zero(const int* __restrict__ ids, int n, const int* __restrict__ where, int vocab, int hidden,
                                                    T* __restrict__ dW) {
    typedef T vec __attribute__((ext_vector_type(kVec)));
    for (int v = blockIdx.x; v < vocab; v += gridDim.x) {
        const int t = n > 0 ? where[v] : -1;
        if ((unsigned)t < (unsigned)n && ids[t] == v) continue;
        const vec zero = {};
        for (int c = threadIdx.x * kVec; c < hidden; c += 256 * kVec) *reinterpret_cast<vec*>(dW + (long long)v * hidden + c) = zero;
    }
}

struct EmbedPlan {
    SortPlan sort;
    int *keys[2], *tokens[2], *counts, *where;
    float* partial;
    int parts, stride;
    size_t bytes;
};
static EmbedPlan plan_embed(int vocab, int hidden, int n, void* ws, size_t ws_bytes) {
    Arena a(ws, ws_bytes);
    EmbedPlan p;
    n = n > 0 ? n : 1;
    p.sort = plan_sort(n, vocab);
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = static_cast<int*>(a.take((size_t)n * sizeof(int)));
        p.tokens[i] = static_cast<int*>(a.take((size_t)n * sizeof(int)));
    }
    p.counts = static_cast<int*>(a.take(((size_t)p.sort.blocks << p.sort.digit) * sizeof(int)));
    p.where = static_cast<int*>(a.take((size_t)vocab * sizeof(int)));
    p.parts = ceil_div(n, kPart);
    p.stride = (int)round_up((size_t)hidden, 8);
    p.partial = static_cast<float*>(a.take((size_t)p.parts * 2 * p.stride * sizeof(float)));
    p.bytes = round_up(a.used, 256);
    return p;
}

size_t embed_backward_workspace_bytes(int vocab, int hidden, int n_tokens) { return plan_embed(vocab, hidden, n_tokens, nullptr, 0).bytes; }

template <typename T>
static void embed_backward_launch(const EmbedPlan& p, const int* ids, const T* dX, int n, int vocab, int hidden, float scale, int accumulate,
                                  T* dW, hipStream_t stream) {
    constexpr int kVec = 16 / sizeof(T);
    const bool vec = hidden % kVec == 0;
    const int *keys = ids, *tokens = nullptr;
    if (n > 0) {
        const int bins = 1 << p.sort.digit;
        for (int i = 0; i < p.sort.passes; ++i) {
            const int shift = i * p.sort.digit;
            k_sort_count<<<p.sort.blocks, 256, 0, stream>>>(keys, n, vocab, shift, bins, p.sort.per_block, p.counts);
            k_sort_place<<<p.sort.blocks, 256, 0, stream>>>(keys, tokens, n, vocab, shift, p.sort.digit, p.sort.per_block, p.counts, p.sort.blocks,
                                                            p.keys[i & 1], p.tokens[i & 1], i == 0 && !accumulate ? p.where : nullptr);
            keys = p.keys[i & 1];
            tokens = p.tokens[i & 1];
        }
    }
    if (!accumulate) {
        const int grid = std::min(vocab, 1 << 20);
        if (vec)
            k_embed_zero<T, kVec><<<grid, 256, 0, stream>>>(ids, n, p.where, vocab, hidden, dW);
        else
            k_embed_zero<T, 1><<<grid, 256, 0, stream>>>(ids, n, p.where, vocab, hidden, dW);
    }
    if (n <= 0) return;
    const int tiles = ceil_div(hidden, 64 * (vec ? kVec : 1));
    const long long units = (long long)p.parts * tiles;
    const int grid = (int)std::min<long long>((units + 3) / 4, 1 << 20);
    if (vec)
        k_embed_sums<T, kVec><<<grid, 256, 0, stream>>>(keys, tokens, n, vocab, hidden, dX, scale, accumulate, dW, p.partial, p.stride, tiles, units);
    else
        k_embed_sums<T, 1><<<grid, 256, 0, stream>>>(keys, tokens, n, vocab, hidden, dX, scale, accumulate, dW, p.partial, p.stride, tiles, units);
    if (p.parts > 1)
        k_embed_join<T><<<dim3(std::min(p.parts - 1, 1 << 16), ceil_div(hidden, 256)), 256, 0, stream>>>(keys, n, vocab, hidden, scale, accumulate, dW,
                                                                                                        p.partial, p.stride, p.parts);
}

int launch_embed_backward(alch_dtype dt, const int* ids, const void* dX, int n_tokens, int vocab, int hidden, float scale, int accumulate,
                          void* dW, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const EmbedPlan p = plan_embed(vocab, hidden, n_tokens, workspace, workspace_bytes);
    TraceScope ts(kTraceEmbed, (double)n_tokens * hidden, ((double)n_tokens + (accumulate ? 0 : vocab)) * hidden * dtype_size(dt), stream);
    if (dt == ALCH_BF16)
        embed_backward_launch<__bf16>(p, ids, (const __bf16*)dX, n_tokens, vocab, hidden, scale, accumulate, (__bf16*)dW, stream);
    else
        embed_backward_launch<float>(p, ids, (const float*)dX, n_tokens, vocab, hidden, scale, accumulate, (float*)dW, stream);
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
