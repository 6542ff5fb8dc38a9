// Records in 8 bits: the kept rows of activations as int8 codes with an fp32 scale for every 64 elements, and back (Section 4.1 of the
// paper: what serving leaves behind is kept until it is trained on).
//
//   a = max |x| of a group,  scale = a / 127,  code = rint(x * (127 / a));   x' = code * scale
//
// Each rounding is made where the definition has it (no fused multiply-add between the product and rint), so that codes and scales
// are defined bit for bit.  int8 with the group's own scale: an activation of normal distribution comes back to 0.5 % in the 2-norm,
// 8-bit floats with 3 bits of mantissa leave 2.6 %.
//
// Both directions are bound by memory: a kept element is 2 bytes read and 1 1/16 written, and the reverse.  A quarter of 70001 tokens of 38912 bf16
// elements: 358 us, 5.8 TB/s; 8192 rows of them back: 175 us, 5.6 TB/s.
#include <algorithm>

#include "kernels.h"
#include "mask_scan.h"

namespace alch {

static constexpr int kGroup = ALCH_Q8_GROUP, kThreads = 256;
static constexpr int kMaxPerLaunch = 16;        // streams of a launch
// Up to so many rows the streams of a row have a work-group each, one behind the other's latency otherwise; fewer where every work-group looks through the
// mask.  Six bf16 streams, packed: 450 rows of 256 to 1024 elements 9.0 us, so 5.3; 500 rows of 1024 to 14336 22.2 and 17.5, 1000 of them 28 and 37.
// Expanded: 700 rows of 256 to 1024 6.1 and 3.7; 1500 of 1024 to 14336 36 and 35; 3000 of 512 to 8192 38.6 and 41.  Short rows, four to a work-group:
// expanded up to four times as many (8095 of 256 to 1024 21.9 and 19.6), packed not (2000 of 8000 tokens 11.6 and 13.3).
static constexpr int kFewRows = 2048, kFewOfScan = 512;
static constexpr int kGridMax = 1 << 20;        // work-groups of a launch; rows behind them are gone over in rounds
static constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: below it 127 / a would leave fp32

typedef float f32x4_q __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_q __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2_q __attribute__((ext_vector_type(2)));

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, kCtrl, 0xf, 0xf, false);
    return v > o ? v : o;
}
// Over each eight lanes: neighbours, pairs, quads.
__device__ __forceinline__ uint32_t max_of_8(uint32_t v) {
    v = dpp_max<0xB1>(v);
    v = dpp_max<0x4E>(v);
    return dpp_max<0x141>(v);
}
__device__ __forceinline__ uint32_t max_of_16(uint32_t v) { return dpp_max<0x140>(max_of_8(v)); }

struct GroupScale {
    float scale, r;
    bool fine;  // no infinity and no NaN
};
__device__ __forceinline__ GroupScale group_scale(uint32_t bits) {  // of the largest magnitude
    const float a = __builtin_bit_cast(float, bits);
    GroupScale s;
    s.fine = bits < 0x7f800000u;
    s.r = s.fine && a >= kTiny ? 127.f / a : 0.f;
    s.scale = !s.fine ? __builtin_nanf("") : a >= kTiny ? a / 127.f : 0.f;
    return s;
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
// rint(x r) in the low byte: 1.5 * 2^23 added, the last bit of the sum is 1
__device__ __forceinline__ uint32_t code_of(float x, float r) {
#pragma clang fp contract(off)
    const float y = x * r;
    return __builtin_bit_cast(uint32_t, y + 12582912.f);
}
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
    const bf16x8_q v = __builtin_bit_cast(bf16x8_q, __builtin_nontemporal_load(reinterpret_cast<const f32x4_q*>(p)));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const f32x4_q a = __builtin_nontemporal_load(reinterpret_cast<const f32x4_q*>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const f32x4_q*>(p) + 1);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
    bf16x8_q v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
    __builtin_nontemporal_store(__builtin_bit_cast(f32x4_q, v), reinterpret_cast<f32x4_q*>(p));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    __builtin_nontemporal_store(f32x4_q{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4_q*>(p));
    __builtin_nontemporal_store(f32x4_q{x[4], x[5], x[6], x[7]}, reinterpret_cast<f32x4_q*>(p) + 1);
}

// ---- a row, by kLanes threads: a work-group, or a wavefront where rows are short ------------------
// Eight elements a lane, so that a group is eight lanes and its maximum three steps of neighbours; kBatch pieces a thread are on their way at
// once (a row of 14336 elements: two rounds).
static constexpr int kBatch = 4;
template <int kLanes, typename T>
__device__ __forceinline__ void quantise_row_pieces(const T* __restrict__ src, int8_t* __restrict__ codes, float* __restrict__ scales, long long width, int lane) {
    const long long pieces = width >> 3;
    for (long long base = 0; base < pieces; base += kLanes * kBatch) {
        float x[kBatch][8];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const long long p = base + b * kLanes + lane;
            if (p < pieces) load8(src + p * 8, x[b]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) x[b][e] = 0.f;
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (base + b * kLanes >= pieces) break;
            const long long p = base + b * kLanes + lane;
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, magnitude(x[b][e]));
            const GroupScale s = group_scale(max_of_8(most));
            uint32_t c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = code_of(x[b][e], s.r);
            u32x2_q w = {bytes4(c[0], c[1], c[2], c[3]), bytes4(c[4], c[5], c[6], c[7])};
            if (!s.fine) w = u32x2_q{0, 0};
            if (p < pieces) {
                __builtin_nontemporal_store(w, reinterpret_cast<u32x2_q*>(codes + p * 8));
                if ((lane & 7) == 0) scales[p >> 3] = s.scale;
            }
        }
    }
}
// Rows that are not made of aligned pieces: four elements a lane, wherever they begin, and a group is a row of 16 lanes.
template <typename T>
struct Four {
    typedef T type __attribute__((ext_vector_type(4)));
    typedef type any __attribute__((aligned(sizeof(T))));
};
typedef uint32_t u32_any __attribute__((aligned(1)));
static constexpr int kQuads = 2;
template <int kLanes, typename T>
__device__ __forceinline__ void quantise_row_elements(const T* __restrict__ src, int8_t* __restrict__ codes, float* __restrict__ scales, long long width, int lane) {
    for (long long base = 0; base < width; base += kLanes * 4 * kQuads) {
        float x[kQuads][4];
        int n[kQuads];
#pragma unroll
        for (int b = 0; b < kQuads; ++b) {
            const long long at = base + (b * kLanes + lane) * 4;
            n[b] = (int)max(min(width - at, 4LL), 0LL);
            typename Four<T>::type v = {};
            if (n[b] == 4) v = *reinterpret_cast<const typename Four<T>::any*>(src + at);
            else if (n[b] > 0)
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < n[b]) v[e] = src[at + e];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[b][e] = (float)v[e];
        }
#pragma unroll
        for (int b = 0; b < kQuads; ++b) {
            const long long at = base + (b * kLanes + lane) * 4;
            if (base + b * kLanes * 4 >= width) break;
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) most = max(most, magnitude(x[b][e]));
            const GroupScale s = group_scale(max_of_16(most));
            uint32_t w = bytes4(code_of(x[b][0], s.r), code_of(x[b][1], s.r), code_of(x[b][2], s.r), code_of(x[b][3], s.r));
            if (!s.fine) w = 0;
            if (n[b] == 4) *reinterpret_cast<u32_any*>(codes + at) = w;
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < n[b]) codes[at + e] = (int8_t)(w >> (8 * e));
            if ((lane & 15) == 0 && n[b] > 0) scales[at / kGroup] = s.scale;
        }
    }
}

template <int kLanes, typename T>
__device__ __forceinline__ void expand_row_pieces(const int8_t* __restrict__ codes, const float* __restrict__ scales, T* __restrict__ dst, long long width, int lane) {
    const long long pieces = width >> 3;
    for (long long base = 0; base < pieces; base += kLanes * kBatch) {
        u32x2_q c[kBatch];
        float s[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const long long p = base + b * kLanes + lane;
            c[b] = u32x2_q{0, 0};
            s[b] = 0.f;
            if (codes && p < pieces) {
                c[b] = __builtin_nontemporal_load(reinterpret_cast<const u32x2_q*>(codes + p * 8));
                s[b] = scales[p >> 3];
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const long long p = base + b * kLanes + lane;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)(int8_t)(c[b][e >> 2] >> (8 * (e & 3))) * s[b];
            if (p < pieces) store8(dst + p * 8, x);
        }
    }
}
template <int kLanes, typename T>
__device__ __forceinline__ void expand_row_elements(const int8_t* __restrict__ codes, const float* __restrict__ scales, T* __restrict__ dst, long long width, int lane) {
    for (long long at = lane * 4; at < width; at += kLanes * 4) {
        const int n = (int)min(width - at, 4LL);
        const float s = codes ? scales[at / kGroup] : 0.f;
        uint32_t c = 0;
        if (codes) {
            if (n == 4) c = *reinterpret_cast<const u32_any*>(codes + at);
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < n) c |= (uint32_t)(uint8_t)codes[at + e] << (8 * e);
        }
        typename Four<T>::type v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (T)((float)(int8_t)(c >> (8 * e)) * s);
        if (n == 4) *reinterpret_cast<typename Four<T>::any*>(dst + at) = v;
        else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) dst[at + e] = v[e];
    }
}

// ---- kernels -----------------------------------------------------------------------------------
struct Q8Stream {  // of either direction: codes and scales dense, the tensor's rows `stride` bytes apart
    char* tensor;
    int8_t* codes;
    float* scales;
    long long width, stride;
    int bf16, pieces;
};
struct Q8Args {
    Q8Stream s[kMaxPerLaunch];
    int n;
};

template <int kLanes>
__device__ __forceinline__ void quantise_row(const Q8Stream& s, long long from, long long to, int lane) {
    const char* src = s.tensor + from * s.stride;
    int8_t* codes = s.codes + to * s.width;
    float* scales = s.scales + to * ((s.width + kGroup - 1) / kGroup);
    if (s.bf16) {
        if (s.pieces) quantise_row_pieces<kLanes>(reinterpret_cast<const __bf16*>(src), codes, scales, s.width, lane);
        else quantise_row_elements<kLanes>(reinterpret_cast<const __bf16*>(src), codes, scales, s.width, lane);
    } else {
        if (s.pieces) quantise_row_pieces<kLanes>(reinterpret_cast<const float*>(src), codes, scales, s.width, lane);
        else quantise_row_elements<kLanes>(reinterpret_cast<const float*>(src), codes, scales, s.width, lane);
    }
}
template <int kLanes>
__device__ __forceinline__ void expand_row(const Q8Stream& s, long long from, long long to, int lane) {  // from < 0: zeros
    char* dst = s.tensor + to * s.stride;
    const int8_t* codes = from < 0 ? nullptr : s.codes + from * s.width;
    const float* scales = s.scales + (from < 0 ? 0 : from) * ((s.width + kGroup - 1) / kGroup);
    if (s.bf16) {
        if (s.pieces) expand_row_pieces<kLanes>(codes, scales, reinterpret_cast<__bf16*>(dst), s.width, lane);
        else expand_row_elements<kLanes>(codes, scales, reinterpret_cast<__bf16*>(dst), s.width, lane);
    } else {
        if (s.pieces) expand_row_pieces<kLanes>(codes, scales, reinterpret_cast<float*>(dst), s.width, lane);
        else expand_row_elements<kLanes>(codes, scales, reinterpret_cast<float*>(dst), s.width, lane);
    }
}

// Which of the rows of its work-group a thread is at, and its lane there.  (Rows of a whole work-group stay in scalar registers: 70001 tokens 410 us
// where they were not.)
template <int kLanes>
__device__ __forceinline__ int row_of() { return kLanes == kThreads ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / kLanes); }
template <int kLanes>
__device__ __forceinline__ int lane_of() { return kLanes == kThreads ? (int)threadIdx.x : (int)threadIdx.x & (kLanes - 1); }

// A work-group a row, or four rows (the grid is sized for the most rows that the call can produce).  kept_index NULL: every token, n_rows of them.  An
// index that is no token of the batch (of a call that had no room for it) leaves its row as it was.
template <int kLanes>
__global__ __launch_bounds__(kThreads) void k_gather_q8(Q8Args a, const int* __restrict__ kept_index, const int* __restrict__ n_kept_and_status,
                                                        long long n_rows, int T) {
    constexpr int kRows = kThreads / kLanes;
    if (kept_index) n_rows = min(n_rows, (long long)n_kept_and_status[0]);
    const int lane = lane_of<kLanes>();
    for (long long r = (long long)blockIdx.x * kRows + row_of<kLanes>(); r < n_rows; r += (long long)gridDim.x * kRows) {
        const int t = __builtin_amdgcn_readfirstlane(kept_index ? kept_index[r] : (int)r);  // (a row's address in vector registers: 398 us for 377)
        if ((unsigned)t >= (unsigned)T) continue;
        for (int k = blockIdx.y; k < a.n; k += gridDim.y) quantise_row<kLanes>(a.s[k], t, r, lane);
    }
}

// Scan and rows of a batch of at most 4096 * kLoads tokens in one launch: every work-group finds its rows' tokens in the mask by itself, the first
// one writes the counts; blockIdx.y deals out the streams of a row.
template <int kLoads, int kLanes>
__global__ __launch_bounds__(kScanThreads) void k_pack_small_q8(Q8Args a, const uint8_t* __restrict__ mask, int T, const int* __restrict__ cu_seqlens,
                                                                int n_bounds, int* __restrict__ kept_index, int* __restrict__ cu_kept,
                                                                int* __restrict__ n_kept_and_status, long long capacity) {
    constexpr int kRows = kScanThreads / kLanes;
    __shared__ int token[kRows];
    __shared__ int prefix[kLoads * kScanThreads];
    __shared__ unsigned short kept_bits[kLoads * kScanThreads];
    const int tid = threadIdx.x, r0 = blockIdx.x * kRows;
    const bool first = blockIdx.x == 0 && blockIdx.y == 0;
    uint32_t bits[kLoads];
    int count[kLoads], carry = 0;
#pragma unroll
    for (int l = 0; l < kLoads; ++l) count[l] = nonzero_bytes16(mask, (l * kScanThreads + tid) * kTokPerThread, T, bits[l]);
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
        int total;
        const int ex = carry + block_exclusive_scan(count[l], total);
        if (first) {
            prefix[l * kScanThreads + tid] = ex;
            kept_bits[l * kScanThreads + tid] = (unsigned short)bits[l];
        }
        // its tokens among the rows of this work-group
        uint32_t left = bits[l];
        for (int i = ex; i < min(ex + count[l], r0 + kRows); ++i, left &= left - 1) {
            if (i < r0) continue;
            const int t = (l * kScanThreads + tid) * kTokPerThread + __ffs(left) - 1;
            token[i - r0] = t;
            if (blockIdx.y == 0 && i < capacity) kept_index[i] = t;
        }
        carry += total;
    }
    __syncthreads();
    if (first) {
        if (tid == 0) {
            n_kept_and_status[0] = carry;
            n_kept_and_status[1] = (long long)carry > capacity ? 1 : 0;
        }
        for (int s = tid; s < n_bounds; s += kScanThreads) {
            const int end = cu_seqlens[s], owner = end / kTokPerThread;
            int n = carry;
            if (owner < kLoads * kScanThreads) n = prefix[owner] + __popc(kept_bits[owner] & ((1u << (end % kTokPerThread)) - 1u));
            cu_kept[s] = n;
        }
    }
    const int row = row_of<kLanes>(), r = r0 + row;
    if (r >= carry || r >= capacity) return;
    const int t = __builtin_amdgcn_readfirstlane(token[row]);
    for (int k = blockIdx.y; k < a.n; k += gridDim.y) quantise_row<kLanes>(a.s[k], t, r, lane_of<kLanes>());
}

template <int kLanes>
__global__ __launch_bounds__(kThreads) void k_expand(Q8Args a, const int* __restrict__ rows, long long n_rows, long long n_src_rows) {
    constexpr int kRows = kThreads / kLanes;
    const int lane = lane_of<kLanes>();
    for (long long r = (long long)blockIdx.x * kRows + row_of<kLanes>(); r < n_rows; r += (long long)gridDim.x * kRows) {
        long long from = rows ? rows[r] : r;
        if (from < 0 || from >= n_src_rows) from = -1;
        for (int k = blockIdx.y; k < a.n; k += gridDim.y) expand_row<kLanes>(a.s[k], from, r, lane);
    }
}

static bool made_of_pieces(const void* tensor, const void* codes, long long width, size_t stride) {
    return width % 8 == 0 && stride % 16 == 0 && aligned16(tensor) && aligned16(codes);
}
// Streams base .. of a call, at most kMaxPerLaunch of them.
static Q8Args q8_args(int n, const alch_q8_stream* streams, int base) {
    Q8Args a;
    a.n = n - base < kMaxPerLaunch ? n - base : kMaxPerLaunch;
    for (int k = 0; k < a.n; ++k) {
        const alch_q8_stream& s = streams[base + k];
        a.s[k] = {const_cast<char*>(static_cast<const char*>(s.src)), s.codes, s.scales, s.width, (long long)s.src_row_stride_bytes, s.dtype == ALCH_BF16,
                  made_of_pieces(s.src, s.codes, s.width, s.src_row_stride_bytes)};
    }
    return a;
}

static double row_bytes(int n_streams, const alch_q8_stream* streams) {  // of a kept row: their number is on the device
    double bytes = 0;
    for (int k = 0; k < n_streams; ++k) bytes += (double)streams[k].width * (dtype_size((alch_dtype)streams[k].dtype) + 1 + 4.0 / kGroup);
    return bytes;
}

// Whether a wavefront is enough for a row: up to so many elements.  487 + 163 fp32 elements, 2501 rows of 5003 tokens: 8.5 us, 12.0 with a work-group a row.
static constexpr int kShortRow = 1024;
static bool short_rows(const Q8Args& a) {
    bool all = true;
    for (int k = 0; k < a.n; ++k) all = all && a.s[k].width <= kShortRow;
    return all;
}
// The grid for so many rows, of a launch whose work-groups have one or four of them each.
static dim3 rows_grid(long long rows, bool four, int streams, bool dealt) {
    const long long groups = four ? (rows + 3) / 4 : rows;
    return dim3((unsigned)std::min<long long>(groups, kGridMax), dealt ? streams : 1);
}

int launch_gather_q8(int T, int n_streams, const alch_q8_stream* streams, long long capacity, const int* kept_index, const int* n_kept_and_status,
                     hipStream_t stream) {
    const long long max_rows = T < capacity ? T : capacity;
    if (max_rows == 0 || n_streams == 0) return ALCH_OK;
    TraceScope ts(kTracePackGather, 0.0, row_bytes(n_streams, streams), stream);
    for (int base = 0; base < n_streams; base += kMaxPerLaunch) {
        const Q8Args a = q8_args(n_streams, streams, base);
        const bool four = short_rows(a);
        const auto kernel = four ? k_gather_q8<64> : k_gather_q8<kThreads>;
        kernel<<<rows_grid(max_rows, four, a.n, max_rows <= kFewRows), kThreads, 0, stream>>>(a, kept_index, n_kept_and_status, max_rows, T);
    }
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

int launch_pack_q8(const uint8_t* mask, int T, const int* cu_seqlens, int n_seqs, int n_streams, const alch_q8_stream* streams, long long capacity,
                   int* kept_index, int* cu_kept, int* n_kept_and_status, void* workspace, hipStream_t stream) {
    const long long max_rows = T < capacity ? T : capacity;
    if (T <= 2 * kTokPerBlock && max_rows > 0 && n_streams > 0 && n_streams <= kMaxPerLaunch) {
        TraceScope ts(kTracePackGather, 0.0, row_bytes(n_streams, streams), stream);
        const Q8Args a = q8_args(n_streams, streams, 0);
        const bool four = short_rows(a), one = T <= kTokPerBlock;
        const auto kernel = four ? (one ? k_pack_small_q8<1, 64> : k_pack_small_q8<2, 64>) : one ? k_pack_small_q8<1, kThreads> : k_pack_small_q8<2, kThreads>;
        kernel<<<rows_grid(max_rows, four, n_streams, max_rows <= kFewOfScan), kScanThreads, 0, stream>>>(a, mask, T, cu_seqlens, n_seqs + 1, kept_index, cu_kept, n_kept_and_status, capacity);
        ALCH_HIP_TRY(hipGetLastError());
        return ALCH_OK;
    }
    ALCH_TRY(launch_pack(mask, T, cu_seqlens, n_seqs, 0, nullptr, capacity, kept_index, cu_kept, n_kept_and_status, workspace, stream));
    return launch_gather_q8(T, n_streams, streams, capacity, kept_index, n_kept_and_status, stream);
}

int launch_expand(long long n_rows, const int* rows, long long n_src_rows, int n_tensors, const alch_q8_tensor* tensors, hipStream_t stream) {
    if (n_rows == 0 || n_tensors == 0) return ALCH_OK;
    double bytes = 0;
    for (int k = 0; k < n_tensors; ++k) bytes += (double)n_rows * tensors[k].width * (dtype_size((alch_dtype)tensors[k].dtype) + 1 + 4.0 / kGroup);
    TraceScope ts(kTracePackGather, 0.0, bytes, stream);
    for (int base = 0; base < n_tensors; base += kMaxPerLaunch) {
        Q8Args a;
        a.n = n_tensors - base < kMaxPerLaunch ? n_tensors - base : kMaxPerLaunch;
        for (int k = 0; k < a.n; ++k) {
            const alch_q8_tensor& t = tensors[base + k];
            a.s[k] = {static_cast<char*>(t.dst), const_cast<int8_t*>(t.codes), const_cast<float*>(t.scales), t.width, (long long)t.dst_row_stride_bytes,
                      t.dtype == ALCH_BF16, made_of_pieces(t.dst, t.codes, t.width, t.dst_row_stride_bytes)};
        }
        const bool four = short_rows(a);
        const auto kernel = four ? k_expand<64> : k_expand<kThreads>;
        kernel<<<rows_grid(n_rows, four, a.n, n_rows <= (four ? 4 : 1) * kFewRows), kThreads, 0, stream>>>(a, rows, n_rows, n_src_rows);
    }
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
