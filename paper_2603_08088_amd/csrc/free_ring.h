// The ring of free blocks (eagletv.h, "Beam decoding over a paged cache") and sums over a workgroup of W wavefronts.
#pragma once
#include "etv_common.h"

namespace etv {

struct Ring {
    long n, first, count;
    bool valid;
    int32_t raw[2];
    __device__ Ring(const int32_t *state, int num_blocks) : n(num_blocks) {
        raw[0] = state[0], raw[1] = state[1];
        valid = raw[0] >= 0 && raw[0] < num_blocks && raw[1] >= 0 && raw[1] <= num_blocks;
        first = valid ? raw[0] : 0;
        count = valid ? raw[1] : 0;
    }
    // free blocks to take, and room for blocks to put behind them: none of either in a state that is not one
    __device__ long room() const { return valid ? n - count : 0; }
    // where entry i lies, 0 <= i < n
    __device__ long place(long i) const {
        const long x = first + i;
        return x >= n ? x - n : x;
    }
    __device__ void leave(int32_t *out, long taken, long given) const {
        out[0] = valid ? (int32_t)place(taken) : raw[0];
        out[1] = valid ? (int32_t)(count - taken + given) : raw[1];
    }
};

// Sum of v over the workgroup; every thread calls it.
template <int W>
__device__ __forceinline__ long block_sum(long v) {
    __shared__ long s_part[W];
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    __syncthreads();  // the last call's readers are done
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < W; w++) v += s_part[w];
    return v;
}

// `carry` plus the sum of v over the threads before and with each (whose total stays below 2^31); carry grows by that total.  Every thread
// calls it.
template <int W>
__device__ __forceinline__ long block_scan_sum(int v, long &carry) {
    __shared__ int s_wave[W];
    int x = wave_scan_sum(v), all = 0;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s_wave[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; w++) {
        if (w < (int)(threadIdx.x >> 6)) x += s_wave[w];
        all += s_wave[w];
    }
    const long before = carry;
    carry += all;
    return before + x;
}

}  // namespace etv
