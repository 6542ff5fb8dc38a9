// Calls over tables of tensors: all tensors share a call's launches, they are cut into chunks, and every work-group finds the tensor of a
// chunk in a table that it makes of the tensors' lengths.
#pragma once
#include "common.h"

namespace alch {

static constexpr int kMaxTensors = ALCH_MAX_TENSORS;
static constexpr int kMaxChunkBlocks = 1 << 22;  // of a launch; chunks behind them are gone over in rounds

// Which tensor a chunk belongs to, and which of its chunks it is.  Up to 64 tensors (kFew) every wavefront holds the table in
// registers, a tensor a lane, so that a chunk's address is one load behind the launch; more of them have their first chunks in LDS.
// Work-groups of 256 threads, all of which make the table and look chunks up together.
template <typename Tensor, bool kFew>
struct ChunkTable {
    struct Chunk {
        Tensor t;
        int index;
    };
    static constexpr int kWords = sizeof(Tensor) / 4;
    const Tensor* tensors;
    int n, chunks;
    int* first;         // [kMaxTensors + 1]: chunks of the tensors before, of all of them behind the last
    int words[kWords];  // kFew: the lane's tensor,
    int before;         // the chunks of those before it

    template <typename F>
    static __device__ __forceinline__ int count(const Tensor& t, F chunk_of) {
        const int chunk = chunk_of(t.dtype);  // (a power of two)
        return (int)((t.n + chunk - 1) >> (31 - __clz(chunk)));
    }
    static __device__ __forceinline__ int inclusive(int v) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(v, d, 64);
            if (lane >= d) v += o;
        }
        return v;
    }
    template <typename F>
    __device__ __forceinline__ ChunkTable(const Tensor* __restrict__ tensors_, int n_, F chunk_of, int* first_) : tensors(tensors_), n(n_), first(first_) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        if constexpr (kFew) {
            Tensor t = {};
            if (lane < n) t = tensors[lane];
            __builtin_memcpy(words, &t, sizeof(Tensor));
            const int own = lane < n ? count(t, chunk_of) : 0, inc = inclusive(own);
            before = inc - own;
            chunks = __builtin_amdgcn_readlane(inc, 63);
        } else {
            __shared__ int wave_total[4];
            int carry = 0;
            for (int base = 0; base < n; base += 256) {
                const int i = base + tid, own = i < n ? count(tensors[i], chunk_of) : 0, inc = inclusive(own);
                if (lane == 63) wave_total[wave] = inc;
                __syncthreads();
                int ahead = carry;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    if (w < wave) ahead += wave_total[w];
                    carry += wave_total[w];
                }
                if (i < n) first[i] = ahead + inc - own;
                __syncthreads();
            }
            chunks = carry;
        }
    }
    // The last tensor whose first chunk is not behind it (of empty ones, which begin where the next one does, the last, which is not
    // empty), among 64 at a time.
    __device__ __forceinline__ Chunk find(int c) const {
        const int lane = threadIdx.x & 63;
        if constexpr (kFew) {
            const int at = __popcll(__ballot(lane < n && before <= c)) - 1;
            int w[kWords];
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = __builtin_amdgcn_readlane(words[i], at);
            Chunk r;
            __builtin_memcpy(&r.t, w, sizeof(Tensor));
            r.index = c - __builtin_amdgcn_readlane(before, at);
            return r;
        } else {
            int at = 0, step = 1;
            while (step * 64 < n) step *= 64;
            for (; step >= 1; step /= 64) {
                const int i = at + lane * step;
                at += (__popcll(__ballot(i < n && first[i] <= c)) - 1) * step;
            }
            at = __builtin_amdgcn_readfirstlane(at);
            return {tensors[at], c - first[at]};
        }
    }
};

}  // namespace alch
