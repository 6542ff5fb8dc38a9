// Reading a byte mask of tokens: sixteen to a thread, and the scan of a work-group's counts.
#pragma once
#include "common.h"

namespace alch {

static constexpr int kTokPerThread = 16;
static constexpr int kScanThreads = 256;
static constexpr int kTokPerBlock = kTokPerThread * kScanThreads;  // 4096

// 0x80 in every byte of w that is not zero
__device__ __forceinline__ uint32_t nonzero_flags(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w) & 0x80808080u; }

__device__ __forceinline__ int nonzero_bytes16(const uint8_t* __restrict__ mask, int t0, int T, uint32_t& bits) {
    // bits: bit i set <=> mask[t0+i] != 0 (tokens beyond T count as dropped)
    bits = 0;
    if (t0 + kTokPerThread <= T) {
        uint4 v = *reinterpret_cast<const uint4*>(mask + t0);
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)  // the flags of four bytes, moved together by one multiplication
            bits |= ((((nonzero_flags(w[i]) >> 7) * 0x01020408u) >> 24) & 0xfu) << (4 * i);
    } else {
        for (int i = 0; i < kTokPerThread; ++i)
            if (t0 + i < T && mask[t0 + i] != 0) bits |= 1u << i;
    }
    return __popc(bits);
}

__device__ __forceinline__ int wave_inclusive_scan(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        int o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}

// Exclusive scan of one int per thread over a block of kScanThreads; returns the exclusive
// prefix, writes the block total to `total`.
__device__ __forceinline__ int block_exclusive_scan(int v, int& total) {
    __shared__ int wave_sum[kScanThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int inc = wave_inclusive_scan(v);
    if (lane == 63) wave_sum[wave] = inc;
    __syncthreads();
    int before = 0, tot = 0;
#pragma unroll
    for (int w = 0; w < kScanThreads / 64; ++w) {
        int s = wave_sum[w];
        if (w < wave) before += s;
        tot += s;
    }
    total = tot;
    __syncthreads();
    return before + inc - v;
}

}  // namespace alch
