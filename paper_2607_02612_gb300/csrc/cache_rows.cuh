// What the kernels that write rows of a ragged batch into the paged cache share.
#pragma once

#include "cache.cuh"

namespace fz {

constexpr int kMostY = 65535;   // of a grid's height

// Whether sample i's slot is named by another sample too (all kThreads threads).  Every CTA reads all ids: 1 us for 256 samples, but
// the work grows with the square of the batch (1 to 65 tokens of 6 x 64 dims with and without ids: 1024 samples 21 and 20 us, 8192
// 197 and 163).
template <int kThreads>
__device__ __forceinline__ bool named_twice(const Ragged &in, int B, int i, int slot) {
    if (!in.ids) return false;
    bool twice = false;
    for (int j = threadIdx.x; j < B; j += kThreads) twice |= j != i && in.ids[j] == slot;
    return __syncthreads_or(twice);
}

// The lengths that no sample raises, where they go elsewhere (all threads; apart from the kernel, whose other CTAs fetch none of it).
template <int kThreads, typename P>
__device__ __noinline__ void copy_other_lengths(const P &p, int B) {
    __shared__ unsigned named[(FUSION_CACHE_MAX_BATCH + 32) / 32];
    const int tid = threadIdx.x, slots = p.c.max_batch;
    for (int w = tid; w < (slots + 31) / 32; w += kThreads) named[w] = 0u;
    __syncthreads();
    for (int j = tid; j < B; j += kThreads) {
        const int s = p.in.ids ? p.in.ids[j] : j;
        if (s >= 0 && s < slots) atomicOr(&named[s >> 5], 1u << (s & 31));
    }
    __syncthreads();
    for (int s = tid; s < slots; s += kThreads)
        if (!(named[s >> 5] >> (s & 31) & 1u)) p.lengths_out[s] = p.c.lengths[s];
}

}  // namespace fz
