// What the two kernels of low-rank adapters share (k14_adapters.cu: any rows; k15_adapter_tiles.cu: long inputs, few adapters at a time).
#pragma once
#include <limits.h>

#include "kernels.h"
#include "ptx.cuh"

namespace muxq {
namespace adapters {

// The adapter of a row: its slot, INT_MAX without one.  *bad: the slot or its rank is out of range (the row then counts as one without).
__device__ __forceinline__ int adapter_of(int slot, const int32_t *ranks, int slots, int max_rank, int *rank, bool *bad) {
    *rank = 0;
    *bad = slot < -1 || slot >= slots;
    if (*bad || slot < 0) return INT_MAX;
    const int r = ranks ? ranks[slot] : max_rank;
    *bad = r < 0 || r > max_rank;
    if (*bad || r == 0) return INT_MAX;
    *rank = r;
    return slot;
}

// A row of T before the second product: the powers of two that bring its largest value into [2^13, 2^14) and back (a row of nothing but tiny
// values stays below), and a value as two fp16 numbers.
__device__ __forceinline__ void row_factors(float most, float *up, float *down) {
    int e = 13 - ((int)(__float_as_uint(most) >> 23) - 127);
    if (e > 100) e = most == 0.0f ? 0 : 100;
    *up = __uint_as_float((uint32_t)(127 + e) << 23);
    *down = __uint_as_float((uint32_t)(127 - e) << 23);
}
__device__ __forceinline__ void split(float x, __half *hi, __half *lo) {
    *hi = __float2half_rn(x);
    *lo = __float2half_rn(x - __half2float(*hi));
}

constexpr int kWindow = 128, kWindowAdapters = 4;
constexpr int kWindowRanks = 256;  // columns of tensor memory for T, and rows of A in two stages
struct WindowAdapters {  // of 128 rows
    int count;           // adapters
    int uneven;          // whether one of their ranks ends inside a step of 16 that is not the last of max_rank
    int slot[kWindowAdapters], rank[kWindowAdapters];
    int next[kWindowAdapters + 1];
    int8_t index[kWindow];  // by row: which of them, -1 none
};
// Whether k_adapter_tiles takes the window that begins at row m0: up to four adapters that together fit kWindowRanks.  Called by
// all threads of a CTA, at least 128; *mine: the calling thread's row's adapter among the window's.
__device__ __forceinline__ bool window_adapters(WindowAdapters *w, const int32_t *row_slot, const int32_t *ranks, int slots, int max_rank, int m0, int M,
                                                int *mine, bool *bad) {
    const int tid = threadIdx.x, r16 = (max_rank + 15) & ~15;
    const int most = kWindowRanks / r16 < kWindowAdapters ? kWindowRanks / r16 : kWindowAdapters;
    if (tid <= kWindowAdapters) w->next[tid] = INT_MAX;
    int key = INT_MAX, rank = 0, prev = -1, n = 0;
    *mine = -1;
    *bad = false;
    if (tid < kWindow && tid < M - m0) key = adapter_of(row_slot[m0 + tid], ranks, slots, max_rank, &rank, bad);
    const bool uneven = key != INT_MAX && rank % 16 != 0 && rank != max_rank;
    const int any_uneven = __syncthreads_or(uneven);
    for (; n <= most; ++n) {
        const int low = __reduce_min_sync(0xffffffffu, key > prev ? key : INT_MAX);
        if ((tid & 31) == 0 && low != INT_MAX) atomicMin(&w->next[n], low);
        __syncthreads();
        const int cur = w->next[n];
        if (cur == INT_MAX) break;
        if (n == most) return false;
        if (key == cur) {
            *mine = n;
            w->slot[n] = cur;
            w->rank[n] = rank;
        }
        prev = cur;
    }
    if (tid == 0) {
        w->count = n;
        w->uneven = any_uneven;
    }
    if (tid < kWindow) w->index[tid] = (int8_t)*mine;
    __syncthreads();
    return true;
}

}  // namespace adapters

// Long inputs: true where the windows that suit it are done by a launch of k_adapter_tiles on the stream (*e: its error).
bool launch_adapter_tiles(const AdapterArgs &a, cudaStream_t s, cudaError_t *e);

}  // namespace muxq
