// Embedding rows in front of layer 0 and the gradient of their table behind it.
//
//   forward   X[t] = scale * W[id_t]                          (a zero row where id_t is outside 0 .. vocab-1)
//   backward  dW[v] (+)= scale * sum over t with id_t = v of dX[t]
//
// Both are bound by memory.  The backward pass needs the tokens of a row next to one another: they are sorted by id (stable,
// so that every sum runs over ascending tokens and results repeat bit for bit; no float atomics), and the sorted tokens are
// cut into parts of equal length, so that one id that half of a batch shares is summed by as many wavefronts as its tokens need.  What
// stays a chain is the sum of these pieces: a quarter of an id's parts behind one another, for every 256 columns.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace alch {

// kVec elements of a row, 16 bytes (single elements where a row has fewer): rows of any width lie one behind the other, so that they
// need not begin at a multiple of 16 bytes.  The last piece of a row is moved back to end with it and overlaps the one before.
template <typename T, int kVec>
struct Piece {
    typedef T type __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
};

// A work-group goes over 8 KB of rows that lie behind one another, two pieces a thread: `1 << log_lanes` threads to a row, one row
// in `segments` work-groups where it is longer, with three pieces a thread where that saves one (50,000 rows of 10 KB copied in 130 us
// with two, 120 with three).  Work-groups with more, or with fewer that have more of them under way, are slower: 70,001 rows of 8 KB
// copied in 131 us, with two rows a work-group 143, with four 146.
struct RowGrid {
    int log_lanes, per, segments, blocks;
    bool pairs;  // of zeros: see zero_block
};
static RowGrid row_grid(long long rows, int hidden, int vec) {
    RowGrid g;
    const int pieces = ceil_div(hidden, vec);
    g.log_lanes = 0;
    while (g.log_lanes < 8 && (2 << g.log_lanes) < pieces) ++g.log_lanes;
    g.per = ceil_div(pieces, 3 << g.log_lanes) < ceil_div(pieces, 2 << g.log_lanes) ? 3 : 2;
    g.segments = ceil_div(pieces, g.per << g.log_lanes);
    g.pairs = false;
    g.blocks = (int)((rows + (256 >> g.log_lanes) - 1) / (256 >> g.log_lanes) * g.segments);  // (at most 2^30: 2^40 elements)
    return g;
}
// First row of a work-group, and its part of it.
__device__ __forceinline__ long long first_row(const RowGrid& g, int block, int* segment) {
    const int group = g.segments == 1 ? block : block / g.segments;
    *segment = block - group * g.segments;
    return (long long)group * (256 >> g.log_lanes);
}
static constexpr int kMaxBlocks = 1 << 23;  // of a launch; what is more is gone over in rounds

// ---- forward ----------------------------------------------------------------------------
// kWide: a wavefront has one row, whose id is then read as a scalar.
template <typename T, int kVec, bool kWide>
__global__ __launch_bounds__(256) void k_embed(const int* __restrict__ ids, const T* __restrict__ W, T* __restrict__ X, int n_tokens, int vocab,
                                               int hidden, float scale, RowGrid g) {
    typedef typename Piece<T, kVec>::type vec;
    const int lane = threadIdx.x & ((1 << g.log_lanes) - 1);
    for (int b = blockIdx.x; b < g.blocks; b += gridDim.x) {
        int segment;
        long long t = first_row(g, b, &segment) + (threadIdx.x >> g.log_lanes);
        if (kWide) t = __builtin_amdgcn_readfirstlane((int)t);
        if (t >= n_tokens) continue;
        const int id = ids[t], c0 = ((segment * g.per << g.log_lanes) + lane) * kVec, step = kVec << g.log_lanes;
        const int end = min(hidden, c0 + g.per * step);
        const bool valid = (unsigned)id < (unsigned)vocab;
        const T* src = W + (long long)(valid ? id : 0) * hidden;
        vec v[3] = {};
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (valid && c0 + j * step < end) v[j] = *reinterpret_cast<const vec*>(src + min(c0 + j * step, hidden - kVec));
#pragma unroll
        for (int j = 0; j < 3; ++j) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[j][e] = (T)((float)v[j][e] * scale);  // (by 1: the same bits, but a signalling NaN's)
            if (!valid) v[j] = vec{};  // (also where the scale is negative or no number)
            if (c0 + j * step < end) __builtin_nontemporal_store(v[j], reinterpret_cast<vec*>(X + t * hidden + min(c0 + j * step, hidden - kVec)));
        }
    }
}

// f(type, pieces of how many elements) for rows of a type and width
template <typename F>
static void with_pieces(alch_dtype dt, int hidden, F f) {
    using std::integral_constant;
    if (dt == ALCH_BF16) hidden >= 8 ? f(__bf16{}, integral_constant<int, 8>{}) : f(__bf16{}, integral_constant<int, 1>{});
    else hidden >= 4 ? f(float{}, integral_constant<int, 4>{}) : f(float{}, integral_constant<int, 1>{});
}

int launch_embed(alch_dtype dt, const int* ids, const void* W, void* X, int n_tokens, int vocab, int hidden, float scale, hipStream_t stream) {
    if (n_tokens <= 0) return ALCH_OK;
    TraceScope ts(kTraceEmbed, (double)n_tokens * hidden, 2.0 * n_tokens * hidden * dtype_size(dt), stream);
    with_pieces(dt, hidden, [&](auto type, auto vec) {
        typedef decltype(type) T;
        constexpr int kVec = decltype(vec)::value;
        const RowGrid g = row_grid(n_tokens, hidden, kVec);
        const int grid = std::min(g.blocks, kMaxBlocks);
        if (g.log_lanes >= 6)
            k_embed<T, kVec, true><<<grid, 256, 0, stream>>>(ids, (const T*)W, (T*)X, n_tokens, vocab, hidden, scale, g);
        else
            k_embed<T, kVec, false><<<grid, 256, 0, stream>>>(ids, (const T*)W, (T*)X, n_tokens, vocab, hidden, scale, g);
    });
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

// ---- backward: tokens sorted by id --------------------------------------------------------
// A radix sort from the lowest digit.  The first launch counts the lowest digits in every block of tokens; one launch a digit then
// finds the places of a block's tokens from the counts of all blocks, writes them there, and counts the next digit for the blocks
// that they come to lie in (whole numbers: the order of these atomics is not seen).  An id outside the table counts as `vocab`:
// it is sorted behind all others.
static constexpr int kSortBlocks = 512;  // at most
static constexpr int kDigitBits = 10;    // at most
static constexpr int kSortBlockMin = 512;  // tokens

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
    p.per_block = std::max(kSortBlockMin, (int)round_up((size_t)ceil_div(n, kSortBlocks), 256));
    p.blocks = ceil_div(n, p.per_block);
    return p;
}

__device__ __forceinline__ int key_of(int id, int vocab) { return (unsigned)id < (unsigned)vocab ? id : vocab; }

// where (may be null): where[v] = some token with id v; nothing else of it is written, a reader checks what it finds there
// against the ids.  clear: the counts of the digits behind the lowest one.
__global__ __launch_bounds__(256) void k_sort_count(const int* __restrict__ ids, int n, int vocab, int bins, int per_block, int* __restrict__ counts,
                                                    int* __restrict__ clear, int n_clear, int* __restrict__ where) {
    __shared__ int hist[1 << kDigitBits];
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n_clear; i += gridDim.x * 256) clear[i] = 0;
    for (int b = threadIdx.x; b < bins; b += 256) hist[b] = 0;
    __syncthreads();
    const int begin = blockIdx.x * per_block, end = min(n, begin + per_block);
    for (int t = begin + threadIdx.x; t < end; t += 256) {
        const int key = key_of(ids[t], vocab);
        atomicAdd(&hist[key & (bins - 1)], 1);
        if (where && key < vocab) where[key] = t;
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += 256) counts[(long long)blockIdx.x * bins + b] = hist[b];
}

// Zeros a work-group's rows of a table, the block-th of the grid; present(row): whether a token has it.  g.pairs: a thread's first two
// pieces lie next to one another, instead of a row of threads' first pieces before their second ones.
template <typename T, int kVec, typename F>
__device__ __forceinline__ void zero_block(T* __restrict__ dW, int block, int vocab, int hidden, const RowGrid& g, F present) {
    typedef typename Piece<T, kVec>::type vec;
    int segment;
    const long long row = first_row(g, block, &segment) + (threadIdx.x >> g.log_lanes);
    const auto zero = [&](long long r) {
        if (r >= vocab || present(r)) return;
        const int lane = threadIdx.x & ((1 << g.log_lanes) - 1), first = segment * g.per << g.log_lanes;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const int c = (first + (g.pairs && j < 2 ? 2 * lane + j : (j << g.log_lanes) + lane)) * kVec;
            if (j < g.per && c < hidden) *reinterpret_cast<vec*>(dW + r * hidden + min(c, hidden - kVec)) = vec{};
        }
    };
    if (g.log_lanes >= 6) zero(__builtin_amdgcn_readfirstlane((int)row));  // (one row a wavefront: looked up as scalars)
    else zero(row);
}

// Whether a launch that mostly zeros does so in pairs: tables beyond the last-level cache (256 MB) whose rows fill their work-groups.
// us of a whole backward pass of 9000 tokens, in pairs / not: rows of 8 KB 82 MB 57.4 / 53.6, 246 MB 72.7 / 64.6, 492 MB 114 / 119, 1.05 GB
// 198 / 212; of 4 KB 1.05 GB 191 / 202; of 16 KB 983 MB 209 / 216; of 2 KB 614 MB 118 / 119; of 10 KB 1.02 GB 229 / 224, of 7 KB 919 MB 194 / 183.
// Beside the sums of few tokens or the joins not in pairs serves better (1.05 GB, 64 tokens 160 / 166, 487 tokens 184 / 172, 1000 tokens 212 / 164).
static bool zero_in_pairs(const RowGrid& g, long long rows, int hidden, int vec, size_t size) {
    return g.per == 2 && rows * hidden * (long long)size > 256LL << 20 && hidden % (vec * (2 << g.log_lanes)) == 0;
}

// Blocks begin .. end-1 of the table's grid.
struct ZeroRows {
    int n, vocab;  // tokens
    RowGrid grid;
    int begin, end;
};
template <typename T, int kVec>
__device__ __forceinline__ void zero_rows(const ZeroRows& z, const int* __restrict__ ids, const int* __restrict__ where, T* __restrict__ dW, int hidden,
                                          int block, int blocks) {
    for (int b = z.begin + block; b < z.end; b += blocks)
        zero_block<T, kVec>(dW, b, z.vocab, hidden, z.grid, [&](long long row) {
            const int t = z.n > 0 ? where[row] : -1;  // (whatever the workspace held where no token has this id)
            return (unsigned)t < (unsigned)z.n && ids[t] == (int)row;
        });
}
template <typename T, int kVec>
__global__ __launch_bounds__(256) void k_embed_zero(ZeroRows z, const int* __restrict__ ids, const int* __restrict__ where, T* __restrict__ dW, int hidden) {
    zero_rows<T, kVec>(z, ids, where, dW, hidden, blockIdx.x, gridDim.x);
}

// Up to kRankTokens tokens for every digit that their sort would have are sorted by one launch: a token's place is the number of
// tokens with a lower id, and of those with the same one before it.  A work-group finds the places of 64 tokens, a token a lane; its
// wavefronts go over a sixteenth of all tokens each, 64 of them with one load, and compare them with their own one after the other.
// us of a backward pass with this sort / the radix sort, rows of 8 KB: 17 bits of id, accumulated 2500 tokens 23.6 / 32.8, 8192 52.8 / 55.3,
// 12,000 67.4 / 64.0; 10 bits (rows of 4 KB) 4096 26.5 / 25.9, 6000 30.5 / 27.8.  A table that is written can be zeroed beside the launches of
// the radix sort, which is more where it is large: 2300 and 8192 tokens, 82 MB 28.7 / 36.5 and 49.6 / 49.9, 330 MB 66 / 72 and 87.1 / 86.9, 600 MB
// 125 / 116 and 147 / 132, 1.05 GB 199 / 180 and 229 / 199.
static constexpr int kRankTokens = 4096;
static constexpr long long kRankTable = 384LL << 20;  // bytes
__global__ __launch_bounds__(1024) void k_sort_rank(const int* __restrict__ ids, int n, int vocab, int* __restrict__ keys_out, int* __restrict__ tokens_out,
                                                    int* __restrict__ where) {
    __shared__ int counts[16][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), block = blockIdx.x, t = block * 64 + lane;
    const auto key_at = [&](int i) { return i < n ? min((unsigned)ids[i], (unsigned)vocab) : 0xffffffffu; };  // (none is counted behind the last)
    const unsigned key = key_at(t);
    const int chunks = (n + 63) / 64, per = (chunks + 15) / 16, end = min(chunks, (wave + 1) * per);
    int count = 0;
    unsigned next = key_at(wave * per * 64 + lane);
    for (int c = wave * per; c < end; ++c) {
        const unsigned others = next;
        next = key_at((c + 1) * 64 + lane);
        if (c == block) {
#pragma unroll
            for (int i = 0; i < 64; ++i) count += (unsigned)__builtin_amdgcn_readlane((int)others, i) < key + (i < lane);
        } else {
            const unsigned limit = key + (c < block);  // (a key is at most 2^31 - 1)
#pragma unroll
            for (int i = 0; i < 64; ++i) count += (unsigned)__builtin_amdgcn_readlane((int)others, i) < limit;
        }
    }
    counts[wave][lane] = count;
    __syncthreads();
    if (wave != 0 || t >= n) return;
    int at = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) at += counts[w][lane];
    keys_out[at] = (int)key;
    tokens_out[at] = t;
    if (where && key < (unsigned)vocab) where[key] = t;
}

struct SortPass {
    const int *keys, *tokens;  // tokens null: the order before the first digit, keys are the ids then
    int *keys_out, *tokens_out;
    const int* counts;         // [block][digit]
    int* next_counts;          // of the next digit, null for the last one
    int n, vocab, shift, digit_bits, per_block, blocks;
};

// The work-groups behind the sort's own zero rows of the table meanwhile: the sort is a chain of latencies on a few compute units.
// kRun consecutive digits a thread.
template <typename T, int kVec, int kRun>
__global__ __launch_bounds__(256) void k_sort_place(SortPass a, ZeroRows z, const int* __restrict__ ids, const int* __restrict__ where,
                                                    T* __restrict__ dW, int hidden) {
    if ((int)blockIdx.x >= a.blocks) {
        zero_rows<T, kVec>(z, ids, where, dW, hidden, blockIdx.x - a.blocks, gridDim.x - a.blocks);
        return;
    }
    constexpr int kBins = 256 * kRun;
    __shared__ int place[4][kBins];  // first place of this digit's tokens of every wavefront
    __shared__ int sums[4];
    const int bins = 1 << a.digit_bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b0 = tid * kRun;
    // tokens of a digit in all blocks, and in those before this one
    int before[kRun], total[kRun], run = 0;
#pragma unroll
    for (int j = 0; j < kRun; ++j) before[j] = total[j] = 0;
    if (b0 < bins) {
#pragma unroll 8
        for (int k = 0; k < a.blocks; ++k)
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                const int c = a.counts[(long long)k * bins + b0 + j];
                total[j] += c;
                before[j] += k < (int)blockIdx.x ? c : 0;
            }
    }
#pragma unroll
    for (int j = 0; j < kRun; ++j) run += total[j];
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int j = 0; j < kRun; ++j) place[w][b0 + j] = 0;
    int inc = run;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(inc, d, 64);
        if (lane >= d) inc += o;
    }
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    int ahead = inc - run;  // tokens of lower digits
    for (int w = 0; w < wave; ++w) ahead += sums[w];
    // every wavefront counts its quarter of the block
    const int quarter = a.per_block / 4, begin = blockIdx.x * a.per_block + wave * quarter, end = min(a.n, begin + quarter);
    for (int t = begin + lane; t < end; t += 64) atomicAdd(&place[wave][(key_of(a.keys[t], a.vocab) >> a.shift) & (bins - 1)], 1);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
        int at = ahead + before[j];
        ahead += total[j];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int c = place[w][b0 + j];
            place[w][b0 + j] = at;
            at += c;
        }
    }
    __syncthreads();
    // 64 tokens at a time, in their order: a lane's place is behind the lanes before it that have the same digit
    volatile int* mine = place[wave];
    for (int t0 = begin; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        const bool live = t < end;
        const int key = live ? key_of(a.keys[t], a.vocab) : 0, digit = (key >> a.shift) & (bins - 1);
        const int token = live && a.tokens ? a.tokens[t] : t;
        unsigned long long same = __ballot(live);
        for (int b = 0; b < a.digit_bits; ++b) {
            const unsigned long long set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const int at = (live ? mine[digit] : 0) + rank;
        __builtin_amdgcn_wave_barrier();  // (a wavefront's LDS accesses are carried out in their order)
        if (live && rank == 0) mine[digit] = at + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (live) {
            a.keys_out[at] = key;
            a.tokens_out[at] = token;
            if (a.next_counts) atomicAdd(&a.next_counts[(long long)(at / a.per_block) * bins + ((key >> (a.shift + a.digit_bits)) & (bins - 1))], 1);
        }
    }
}

// ---- backward: sums ----------------------------------------------------------------------
// A wavefront takes the rows whose tokens begin among its `part` sorted tokens (at most kPart), in 64 * kVec columns, and sums
// each to its end, also past its own tokens.  (A work-group of its own each: they end at different times.)  Only rows of more than
// two parts' tokens are cut: every wavefront sums those among its own tokens and leaves them in fp32, [part][1] where the row begins
// here, [part][0] where it came from the part before.
static constexpr int kPart = 32, kPartMin = 8;
__host__ __device__ inline int longest_whole(int part_len) { return 2 * part_len; }  // at most 64: the keys that a wavefront looks at

template <typename T, int kVec, typename V>
__device__ __forceinline__ void store_own(T* p, const V& v, int skip) {
    if (skip == 0) {
        __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            if (e >= skip) p[e] = v[e];
    }
}

template <typename T, int kVec, bool kAccumulate>
__global__ __launch_bounds__(64) void k_embed_sums(const int* __restrict__ keys, const int* __restrict__ tokens, int n, int vocab, int hidden,
                                                    const T* __restrict__ dX, float scale, T* __restrict__ dW, float* __restrict__ partial,
                                                    int* __restrict__ cut, int stride, int part_len, int tiles, long long units) {
    typedef typename Piece<T, kVec>::type vec;
    constexpr int kBatch = 8;  // rows that are on their way while as many are summed
    const int lane = threadIdx.x;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int part = __builtin_amdgcn_readfirstlane((int)(u / tiles)), tile = __builtin_amdgcn_readfirstlane((int)(u % tiles));
        const int p0 = part * part_len, own = (tile * 64 + lane) * kVec;
        const int longest = longest_whole(part_len);
        const bool in = own < hidden;
        // the last lane of a row may have fewer columns of its own: it reads some of the lane's before it too, and stores none of them
        const int c = min(own, hidden - kVec);
        // keys of the 64 tokens before the part, of its own and those behind it up to 128; -1 where there are none
        const int kb = p0 - 64 + lane >= 0 ? keys[p0 - 64 + lane] : -1;
        const int k0 = p0 + lane < n ? keys[p0 + lane] : -1, k1 = p0 + 64 + lane < n ? keys[p0 + 64 + lane] : -1;
        const int t0 = p0 + lane < n ? tokens[p0 + lane] : 0, t1 = p0 + 64 + lane < n ? tokens[p0 + 64 + lane] : 0;
        const int key_first = __builtin_amdgcn_readlane(k0, 0);
        // bit i: the row of token i ends with it
        const int behind0 = __shfl_down(k0, 1, 64), behind1 = __shfl_down(k1, 1, 64), k1_first = __builtin_amdgcn_readlane(k1, 0);
        const unsigned long long ends0 = __ballot((lane == 63 ? k1_first : behind0) != k0);
        const unsigned long long ends1 = __ballot((lane == 63 ? -2 : behind1) != k1);
        // (an index of a row's last token from i on; the rows that are asked for end before token 127, or are long)
        const auto end_of = [&](int i) {
            const unsigned long long lo = i < 64 ? ends0 >> i : 0, hi = i < 64 ? ends1 : ends1 >> (i - 64);
            return lo ? i + __ffsll(lo) - 1 : (i < 64 ? 64 : i) + (hi ? __ffsll(hi) - 1 : 63);
        };
        int begin = 0, end = min(part_len, n - p0), first_slot = -1, last_slot = -1;
        const unsigned long long padded = __ballot(k0 < 0 || k0 >= vocab);
        if (padded) end = min(end, __ffsll(padded) - 1);  // padding: behind all others
        if (end > 0) {
            const unsigned long long others = __ballot(kb != key_first);
            const int back = others ? __clzll(others) : 64;  // tokens of the first row before the part
            if (back > 0) {
                const int last = end_of(0);
                if (back + last + 1 > longest) first_slot = 0;
                else begin = last + 1;
            }
            // the row of the part's last token, if it goes on and is not the first one cut above
            const int last = end_of(end - 1);
            if (last >= end) {
                const int key = __builtin_amdgcn_readlane(k0, end - 1);
                const unsigned long long same = __ballot(lane < end && k0 == key);
                const int start = __ffsll(same) - 1;
                if (start > 0 || back == 0) {
                    if (last - start + 1 > longest) last_slot = 1;
                    else end = last + 1;
                }
            }
        }
        if (tile == 0 && lane == 0) cut[part] = last_slot == 1;
        float s[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) s[e] = 0.f;
        // Read with all lanes running and before a choice is made: what lanes that a branch has switched off hold in a register that
        // was written inside it is not defined, and a lane is read whether it is switched off or not.
        const auto at = [&](int v0, int v1, int i) {
            const int a = __builtin_amdgcn_readlane(v0, i & 63), b = __builtin_amdgcn_readlane(v1, i & 63);
            return i < 64 ? a : b;
        };
        const auto ends_at = [&](int i) { return ((i < 64 ? ends0 : ends1) >> (i & 63) & 1) != 0; };
        const auto load = [&](int g, vec (&row)[kBatch], vec (&old)[kBatch]) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int i = g + j;
                if (i < end) {
                    const int token = at(t0, t1, i), key = at(k0, k1, i);
                    row[j] = in ? __builtin_nontemporal_load(reinterpret_cast<const vec*>(dX + (long long)token * hidden + c)) : vec{};
                    if constexpr (kAccumulate)
                        if (ends_at(i)) old[j] = in ? *reinterpret_cast<const vec*>(dW + (long long)key * hidden + c) : vec{};
                }
            }
        };
        const auto sum = [&](int g, const vec (&row)[kBatch], const vec (&old)[kBatch]) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int i = g + j;
                if (i < end) {
#pragma unroll
                    for (int e = 0; e < kVec; ++e) s[e] += (float)row[j][e];
                    const bool ends = ends_at(i);
                    const int key = at(k0, k1, i);
                    if (ends || i + 1 == end) {
                        const int slot = first_slot >= 0 ? first_slot : !ends ? last_slot : -1;
                        if (in && slot >= 0) {
                            float* p = partial + ((long long)part * 2 + slot) * stride + c;
#pragma unroll
                            for (int e = 0; e < kVec; ++e)
                                if (c + e >= own) p[e] = s[e];
                        } else if (in) {
                            vec o;
#pragma unroll
                            for (int e = 0; e < kVec; ++e) o[e] = (T)(kAccumulate ? (float)old[j][e] + scale * s[e] : scale * s[e]);
                            store_own<T, kVec>(dW + (long long)key * hidden + c, o, own - c);
                        }
                        first_slot = -1;
#pragma unroll
                        for (int e = 0; e < kVec; ++e) s[e] = 0.f;
                    }
                }
            }
        };
        vec row_a[kBatch], row_b[kBatch], old_a[kBatch], old_b[kBatch];
        load(begin, row_a, old_a);
        for (int g = begin; g < end; g += 2 * kBatch) {
            load(g + kBatch, row_b, old_b);
            sum(g, row_a, old_a);
            load(g + 2 * kBatch, row_a, old_a);
            sum(g + kBatch, row_b, old_b);
        }
    }
}

// The rows that were cut: the part in which a row begins adds what the parts behind it have of it, in their order.  A work-group
// looks at kJoinParts parts, in 256 columns; its four wavefronts take a quarter of a row's parts each.  The work-groups from `blocks`
// on zero rows, where the sort has left that to this launch.
static constexpr int kJoinParts = 16;
template <typename T, int kVec>
__global__ __launch_bounds__(256) void k_embed_join(const int* __restrict__ keys, int n, int hidden, float scale, int accumulate, T* __restrict__ dW,
                                                    const float* __restrict__ partial, const int* __restrict__ cut, int stride, int part_len, int parts,
                                                    int slices, int blocks, ZeroRows z, const int* __restrict__ ids, const int* __restrict__ where) {
    if ((int)blockIdx.x >= blocks) {
        zero_rows<T, kVec>(z, ids, where, dW, hidden, blockIdx.x - blocks, gridDim.x - blocks);
        return;
    }
    typedef float vec __attribute__((ext_vector_type(4)));
    __shared__ vec red[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c0 = (int)blockIdx.x % slices * 256, base = (int)blockIdx.x / slices * kJoinParts;
    unsigned long long todo = __ballot(lane < kJoinParts && base + lane < parts && cut[base + lane]);
    for (; todo; todo &= todo - 1) {
        const int part = base + __ffsll(todo) - 1, key = keys[(part + 1) * part_len];  // (a cut row goes on behind its part)
        int more = 0;                                                                  // parts behind this one that it lies in
        for (int b = part + 1; b < parts; b += 64) {
            const unsigned long long other = __ballot(b + lane >= parts || keys[(long long)min(b + lane, parts - 1) * part_len] != key);
            more += other ? __ffsll(other) - 1 : 64;
            if (other) break;
        }
        // pieces 0 .. more: the part's own, then theirs
        const int per = (more + 4) / 4, first = wave * per, last = min(more + 1, first + per);
        vec s = {0.f, 0.f, 0.f, 0.f};
        const float* p = partial + (long long)part * 2 * stride + c0 + 4 * lane;
        if (c0 + 4 * lane < stride) {
#pragma unroll 8
            for (int i = first; i < last; ++i) s += *reinterpret_cast<const vec*>(p + ((long long)i * 2 + (i == 0 ? 1 : 0)) * stride);
        }
        __syncthreads();  // (the sums of the row before have been read)
        red[wave][lane] = s;
        __syncthreads();
        const int c = c0 + threadIdx.x;
        if (c < hidden) {
            const float* r = reinterpret_cast<const float*>(red) + threadIdx.x;
            const float sum = (r[0] + r[256]) + (r[512] + r[768]);
            T* dst = dW + (long long)key * hidden + c;
            *dst = (T)(accumulate ? (float)*dst + scale * sum : scale * sum);
        }
    }
}

// ---- backward of few tokens: one launch ----------------------------------------------------
// A work-group a token (or, kByRow, a row of a table that has fewer rows than there are tokens) and 64 * kVec columns.  Each of its
// wavefronts compares the id with a part of all tokens' and sums the rows of those that have it.  By token nothing is done if one of
// them comes before the token; its own row is on its way meanwhile, as is what it is added to.  The work-groups behind these zero the
// rows that no token has, and find out from the ids which those are.
static constexpr int kFewTokens = 2048, kFewTokensByRow = 8192;
static constexpr int kTokenWaves = 4, kRowWaves = 8;
static constexpr long long kFewPairs = 1 << 23, kFewUnits = 1 << 12;
// Where comparing all ids with one another, once in every tile of columns, costs less than a sort and the launches behind it; ids as
// texts have them, us by this kernel / with the sort:
//   by token, table of 128,256 rows     1024 tokens    2048       3000
//     hidden 256 (one tile), fp32         7.1 / 15.9   8.1 / 17.7   12.3 / 20.5
//     1024 (two), bf16                    7.1 / 16.9  12.9 / 18.4   20.9 / 21.7
//     4096 (eight)                       17.7 / 17.4  41.3 / 20.7
//   by row, table of 1000 rows          1024           4096       8192
//     hidden 256, fp32                    6.4 / 14.3   8.8 / 21.7   18.5 / 22.3
//     1024                                8.4 / 15.4  15.3 / 22.9
//     4096                               25.0 / 16.7
// One id alone shared by 1024 tokens 20.5 / 14.9 by token, by 4096 50 / 27 by row: that is a chain of rows here.
static bool few_tokens(int n, int tiles) { return n <= kFewTokens && (long long)n * n * tiles <= kFewPairs; }
static bool few_rows(int n, int vocab, int tiles) {
    return vocab < n && n <= kFewTokensByRow && (long long)vocab * tiles <= kFewUnits && (long long)n * vocab * tiles <= kFewPairs;
}

template <typename T, int kVec, bool kAccumulate, bool kByRow>
__global__ __launch_bounds__(kByRow ? 64 * kRowWaves : 64 * kTokenWaves) void k_embed_few(const int* __restrict__ ids, int n, int vocab, int hidden, const T* __restrict__ dX, float scale,
                                                   T* __restrict__ dW, int tiles, int units, RowGrid g) {
    typedef typename Piece<T, kVec>::type vec;
    constexpr int kBatch = 16, kWaves = kByRow ? kRowWaves : kTokenWaves;
    __shared__ unsigned short list[(kByRow ? kFewTokensByRow : kFewTokens) + 64 * kWaves];  // the tokens that have the id, ascending in every part
    __shared__ float red[kWaves - 1][64 * kVec];
    __shared__ int found[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if constexpr (!kAccumulate && !kByRow) {
        if ((int)blockIdx.x >= units) {
            __shared__ unsigned present[256 / 32];  // of the work-group's rows
            for (int b = blockIdx.x - units; b < g.blocks; b += gridDim.x - units) {
                const int rows = 256 >> g.log_lanes;
                int segment;
                const long long row0 = first_row(g, b, &segment);
                __syncthreads();  // (what the round before had here has been read)
                if (tid < 256 / 32) present[tid] = 0;
                __syncthreads();
                for (int t = tid; t < n; t += 64 * kWaves) {
                    const long long r = ids[t] - row0;
                    if (r >= 0 && r < rows) atomicOr(&present[r >> 5], 1u << (r & 31));
                }
                __syncthreads();
                zero_block<T, kVec>(dW, b, vocab, hidden, g, [&](long long row) { return (present[(row - row0) >> 5] >> ((row - row0) & 31) & 1) != 0; });
            }
            return;
        }
    }
    const int unit = blockIdx.x / tiles, own = ((int)blockIdx.x % tiles * 64 + lane) * kVec, token = kByRow ? -1 : unit, id = kByRow ? unit : ids[unit];
    if (!kByRow && (unsigned)id >= (unsigned)vocab) return;
    const bool in = own < hidden;
    const int c = min(own, hidden - kVec);  // (as in k_embed_sums)
    T* dst = dW + (long long)id * hidden + c;
    vec old = {}, row0 = {};
    if (in && wave == 0) {
        if (kAccumulate) old = *reinterpret_cast<const vec*>(dst);
        if (!kByRow) row0 = *reinterpret_cast<const vec*>(dX + (long long)token * hidden + c);
    }
    const int part = (n + 64 * kWaves - 1) / (64 * kWaves) * 64, begin = wave * part, end = min(n, begin + part);
    unsigned short* mine = list + begin;
    int count = 0;
    unsigned long long earlier = 0;
#pragma unroll 4
    for (int t0 = begin; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        const bool same = t < end && ids[t] == id && t != token;
        const unsigned long long set = __ballot(same);
        if (!kByRow) earlier |= __ballot(same && t < token);
        if (same) mine[count + __popcll(set & ((1ull << lane) - 1))] = (unsigned short)t;
        count += __popcll(set);
    }
    if (lane == 0) found[wave] = earlier ? -1 : count;
    __syncthreads();
    int others = 0;  // tokens of the other wavefronts
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (!kByRow && found[w] < 0) return;
        if (w > 0) others += found[w];
    }
    const bool absent = kByRow && found[0] + others == 0;
    if (kAccumulate && absent) return;
    float s[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) s[e] = (float)row0[e];
    for (int i = 0; i < count; i += kBatch) {
        vec row[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (i + j < count && in) row[j] = *reinterpret_cast<const vec*>(dX + (long long)mine[i + j] * hidden + c);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (i + j < count)
#pragma unroll
                for (int e = 0; e < kVec; ++e) s[e] += (float)row[j][e];
    }
    if (others) {
        if (wave > 0)
#pragma unroll
            for (int e = 0; e < kVec; ++e) red[wave - 1][64 * e + lane] = s[e];
        __syncthreads();
    }
    if (wave > 0 || !in) return;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        if (others)
#pragma unroll
            for (int w = 0; w < kWaves - 1; ++w) s[e] += red[w][64 * e + lane];
        old[e] = (T)(kAccumulate ? (float)old[e] + scale * s[e] : absent ? 0.f : scale * s[e]);
    }
    store_own<T, kVec>(dst, old, own - c);
}

struct EmbedPlan {
    SortPlan sort;
    int *keys[2], *tokens[2], *counts, *where, *cut;
    float* partial;
    int part_len, parts, stride;
    size_t counts_a_pass, bytes;
};
// A workspace for n tokens serves every smaller batch too: blocks of the sort and parts are longer, and therefore fewer, behind some n,
// so that room is taken for the most that any batch of up to n tokens has.
static EmbedPlan plan_embed(int vocab, int hidden, int n, void* ws, size_t ws_bytes) {
    Arena a(ws, ws_bytes);
    EmbedPlan p;
    n = n > 0 ? n : 1;
    p.sort = plan_sort(n, vocab);
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = static_cast<int*>(a.take((size_t)n * sizeof(int)));
        p.tokens[i] = static_cast<int*>(a.take((size_t)n * sizeof(int)));
    }
    p.counts_a_pass = (size_t)p.sort.blocks << p.sort.digit;
    const size_t most_blocks = std::min(ceil_div(n, kSortBlockMin), kSortBlocks);
    p.counts = static_cast<int*>(a.take((most_blocks << p.sort.digit) * p.sort.passes * sizeof(int)));
    p.where = static_cast<int*>(a.take((size_t)vocab * sizeof(int)));
    // parts as long as leaves 4096 wavefronts (of 512 columns): shorter ones are more loads of keys and more cut rows, longer ones too few
    // wavefronts for the memory; us with parts of 8 / 32, rows of 8 KB: 3000 tokens 25.7 / 36.9, 10,000 62 / 61, 70,001 249 / 207
    constexpr int kWavefronts = 4096;
    const int tiles = ceil_div(hidden, 512);
    p.part_len = kPart;
    while (p.part_len > kPartMin && (long long)ceil_div(n, p.part_len) * tiles < kWavefronts) p.part_len /= 2;
    p.parts = ceil_div(n, p.part_len);
    // (parts shorter than kPart are taken where there are fewer than kWavefronts / tiles of twice their length)
    const size_t most_parts = std::max(ceil_div(n, kPart), std::min(ceil_div(n, kPartMin), 2 * ((kWavefronts - 1) / tiles)));
    p.cut = static_cast<int*>(a.take(most_parts * sizeof(int)));
    p.stride = (int)round_up((size_t)hidden, 8);
    p.partial = static_cast<float*>(a.take(most_parts * 2 * p.stride * sizeof(float)));
    p.bytes = round_up(a.used, 256);
    return p;
}

size_t embed_backward_workspace_bytes(int vocab, int hidden, int n_tokens) { return plan_embed(vocab, hidden, n_tokens, nullptr, 0).bytes; }

template <typename T, int kVec>
static void embed_backward_launch(const EmbedPlan& p, const int* ids, const T* dX, int n, int vocab, int hidden, float scale, int accumulate,
                                  T* dW, hipStream_t stream) {
    const RowGrid table = row_grid(accumulate ? 0 : vocab, hidden, kVec);
    ZeroRows z{n, vocab, table, 0, 0};
    z.grid.pairs = zero_in_pairs(table, vocab, hidden, kVec, sizeof(T));
    if (n <= 0) {
        z.end = table.blocks;
        if (z.end) k_embed_zero<T, kVec><<<std::min(z.end, kMaxBlocks), 256, 0, stream>>>(z, ids, p.where, dW, hidden);
        return;
    }
    const int tiles = ceil_div(hidden, 64 * kVec);
    const bool by_row = few_rows(n, vocab, tiles);
    if (by_row || few_tokens(n, tiles)) {
        const int units = (by_row ? vocab : n) * tiles, grid = units + (by_row ? 0 : std::min(table.blocks, kMaxBlocks));
        const auto launch = [&](auto kernel) { kernel<<<grid, 64 * (by_row ? kRowWaves : kTokenWaves), 0, stream>>>(ids, n, vocab, hidden, dX, scale, dW, tiles, units, table); };
        if (by_row) accumulate ? launch(k_embed_few<T, kVec, true, true>) : launch(k_embed_few<T, kVec, false, true>);
        else accumulate ? launch(k_embed_few<T, kVec, true, false>) : launch(k_embed_few<T, kVec, false, false>);
        return;
    }
    const int *keys = ids, *tokens = nullptr;
    if (n <= kRankTokens * p.sort.passes && (accumulate || (long long)vocab * hidden * (long long)sizeof(T) <= kRankTable)) {
        k_sort_rank<<<ceil_div(n, 64), 1024, 0, stream>>>(ids, n, vocab, p.keys[0], p.tokens[0], accumulate ? nullptr : p.where);
        keys = p.keys[0];
        tokens = p.tokens[0];
    } else {
        const SortPlan& o = p.sort;
        const int bins = 1 << o.digit;
        k_sort_count<<<o.blocks, 256, 0, stream>>>(ids, n, vocab, bins, o.per_block, p.counts, p.counts + p.counts_a_pass,
                                                   (int)(p.counts_a_pass * (o.passes - 1)), accumulate ? nullptr : p.where);
        for (int i = 0; i < o.passes; ++i) {
            int* counts = p.counts + p.counts_a_pass * i;
            const SortPass s{keys, tokens, p.keys[i & 1], p.tokens[i & 1], counts, i + 1 < o.passes ? counts + p.counts_a_pass : nullptr,
                             n, vocab, i * o.digit, o.digit, o.per_block, o.blocks};
            z.begin = z.end;  // every launch its share of the rows
            z.end = (int)((long long)table.blocks * (i + 1) / o.passes);
            const int grid = o.blocks + std::min(z.end - z.begin, kMaxBlocks);
            if (o.digit == 10) k_sort_place<T, kVec, 4><<<grid, 256, 0, stream>>>(s, z, ids, p.where, dW, hidden);
            else if (o.digit == 9) k_sort_place<T, kVec, 2><<<grid, 256, 0, stream>>>(s, z, ids, p.where, dW, hidden);
            else k_sort_place<T, kVec, 1><<<grid, 256, 0, stream>>>(s, z, ids, p.where, dW, hidden);
            keys = p.keys[i & 1];
            tokens = p.tokens[i & 1];
        }
    }
    z.begin = z.end;  // what is left goes beside the joins
    z.end = table.blocks;
    z.grid.pairs = false;
    const long long units = (long long)p.parts * tiles;
    const int grid = (int)std::min<long long>(units, kMaxBlocks);
    const auto sums = accumulate ? k_embed_sums<T, kVec, true> : k_embed_sums<T, kVec, false>;
    sums<<<grid, 64, 0, stream>>>(keys, tokens, n, vocab, hidden, dX, scale, dW, p.partial, p.cut, p.stride, p.part_len, tiles, units);
    const int slices = ceil_div(hidden, 256), joins = n > longest_whole(p.part_len) ? ceil_div(p.parts, kJoinParts) * slices : 0;
    const int zeros = std::min(z.end - z.begin, kMaxBlocks);
    if (joins + zeros > 0)
        k_embed_join<T, kVec><<<joins + zeros, 256, 0, stream>>>(keys, n, hidden, scale, accumulate, dW, p.partial, p.cut, p.stride, p.part_len, p.parts,
                                                                 slices, joins, z, ids, p.where);
}

int launch_embed_backward(alch_dtype dt, const int* ids, const void* dX, int n_tokens, int vocab, int hidden, float scale, int accumulate,
                          void* dW, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const EmbedPlan p = plan_embed(vocab, hidden, n_tokens, workspace, workspace_bytes);
    TraceScope ts(kTraceEmbed, (double)n_tokens * hidden, ((double)n_tokens + (accumulate ? 0 : vocab)) * hidden * dtype_size(dt), stream);
    with_pieces(dt, hidden, [&](auto type, auto vec) {
        typedef decltype(type) T;
        embed_backward_launch<T, decltype(vec)::value>(p, ids, static_cast<const T*>(dX), n_tokens, vocab, hidden, scale, accumulate, static_cast<T*>(dW), stream);
    });
    ALCH_HIP_TRY(hipGetLastError());
    return ALCH_OK;
}

}  // namespace alch
