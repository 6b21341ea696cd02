// Rows of a ragged batch go to the ends of their sequences in the paged cache: a copy, row by row, of keys, values,
// sizes and scores.  Bound by memory: every row is read once and written once.
//
// A CTA takes as many rows of one sample as give each thread kPer chunks of 16 bytes of K and of V, which it asks for before it
// looks at the sample's pages and ids, so that the checks cost no time of their own (after the checks: 256 samples of 100 to
// 197 tokens of 6 x 64 dims 23.8 us).  All CTAs of a sample read its length before the last of them to finish raises it (a
// counter per sample, zero between calls), where the length is raised in place.
#include "cache.cuh"

namespace fz {
namespace {

constexpr int kThreads = 256, kPer = 4;

// Whether sample i's slot is named by another sample too (all threads; the batch's ids are few).
__device__ bool named_twice(const Ragged &in, int B, int i, int slot) {
    if (!in.ids) return false;
    bool twice = false;
    for (int j = threadIdx.x; j < B; j += kThreads) twice |= j != i && in.ids[j] == slot;
    return __syncthreads_or(twice);
}

__global__ void __launch_bounds__(kThreads) k_cache_append(CacheAppendParams p, int rows_per_cta, int row_chunks, int head_chunks) {
    const int i = blockIdx.y, tid = threadIdx.x;
    const Cache &c = p.c;
    const int B = device_batch(p.in);
    if (i == p.in.max_batch) {   // the lengths that no sample raises, where they go elsewhere
        if (blockIdx.x > 0) return;
        __shared__ unsigned named[2048];
        if (B < 0 && tid == 0) raise_status(p.status, FUSION_DEV_BAD_BATCH);
        if (p.in_place) return;
        for (int w = tid; w < 2048; w += kThreads) named[w] = 0u;
        __syncthreads();
        for (int j = tid; j < B; j += kThreads) {
            const int s = p.in.ids ? p.in.ids[j] : j;
            if (s >= 0 && s < c.max_batch) atomicOr(&named[s >> 5], 1u << (s & 31));
        }
        __syncthreads();
        for (int s = tid; s < c.max_batch; s += kThreads)
            if (!(named[s >> 5] >> (s & 31) & 1u)) p.lengths_out[s] = c.lengths[s];
        return;
    }
    if (B < 0 || i >= B) return;
    const int slot = p.in.ids ? p.in.ids[i] : i;
    if (slot < 0 || slot >= c.max_batch) {
        if (blockIdx.x == 0 && tid == 0) raise_status(p.status, FUSION_DEV_BAD_IDS);
        return;
    }
    const int o0 = p.in.offsets[i], n = p.in.offsets[i + 1] - o0, at = c.lengths[slot];
    int bad = 0;
    if (o0 < 0 || n < 0 || n > p.in.max_tokens || (long long)o0 + n > p.in.max_rows) bad = FUSION_DEV_BAD_OFFSETS;
    else if (at < 0 || at > c.capacity || n > c.capacity - at) bad = FUSION_DEV_BAD_CACHE;
    const int r0 = blockIdx.x * rows_per_cta, r1 = bad ? r0 : min(n, r0 + rows_per_cta), chunks = (r1 - r0) * row_chunks;
    // chunk e of the CTA: row r0 + e / row_chunks, its (e % row_chunks)-th of all heads
    uint4 k[kPer], v[kPer];
    int row[kPer], ch[kPer];
    auto load = [&](int e0) {
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            const int e = e0 + x * kThreads + tid;
            row[x] = e / row_chunks;
            ch[x] = e - row[x] * row_chunks;
            if (e < chunks) {
                k[x] = ldg16(p.k + (size_t)(o0 + r0 + row[x]) * p.k_stride + (size_t)ch[x] * 16);
                v[x] = ldg16(p.v + (size_t)(o0 + r0 + row[x]) * p.v_stride + (size_t)ch[x] * 16);
            }
        }
    };
    load(0);
    const bool twice = named_twice(p.in, B, i, slot);
    if (twice) bad |= FUSION_DEV_BAD_IDS;
    if (!bad && n > 0) {
        bool wrong = false;
        for (int e = (at >> c.shift) + tid; e <= (at + n - 1) >> c.shift; e += kThreads)
            wrong |= (unsigned)c.table[(size_t)slot * c.max_pages + e] >= c.num_pages;
        if (__syncthreads_or(wrong)) bad = FUSION_DEV_BAD_CACHE;
    }
    if (bad) {   // nothing of this sample is written, and its slot's length stays (also where it is named twice)
        if (blockIdx.x == 0 && tid == 0) {
            raise_status(p.status, bad);
            if (!p.in_place) p.lengths_out[slot] = at;
        }
        return;
    }
    const unsigned low = (1u << c.shift) - 1u;
    for (int e0 = 0; e0 < chunks; e0 += kPer * kThreads) {
        if (e0 > 0) load(e0);   // (rows of more than kPer * kThreads chunks)
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            if (e0 + x * kThreads + tid >= chunks) break;
            const int pos = at + r0 + row[x], h = ch[x] / head_chunks, cc = ch[x] - h * head_chunks;
            unsigned page;
            cache_page(c, slot, pos, page);
            const size_t dst = ((size_t)(((page * (unsigned)c.kv_heads + h) << c.shift) + (pos & low)) * head_chunks + cc) * 16;
            *reinterpret_cast<uint4 *>(c.k + dst) = k[x];
            *reinterpret_cast<uint4 *>(c.v + dst) = v[x];
        }
    }
    for (int r = r0 + tid; r < r1; r += kThreads) {
        unsigned page;
        cache_page(c, slot, at + r, page);
        const size_t s = ((size_t)page << c.shift) + ((at + r) & low);
        if (c.sizes) c.sizes[s] = p.sizes ? p.sizes[o0 + r] : 1.0f;
        if (c.weights) c.weights[s] = p.scores ? p.scores[o0 + r] : 0.0f;
    }
    if (!p.in_place) {
        if (blockIdx.x == 0 && tid == 0) p.lengths_out[slot] = at + n;
        return;
    }
    __syncthreads();   // every thread of the CTA has read the length
    if (tid == 0) {
        if (gridDim.x > 1) {
            __threadfence();
            if (atomicAdd(&p.counters[i], 1) != (int)gridDim.x - 1) return;
            p.counters[i] = 0;
        }
        p.lengths_out[slot] = at + n;
    }
}

}  // namespace

cudaError_t launch_cache_append(int dtype, const CacheAppendParams &p, cudaStream_t s) {
    const int es = dtype == FUSION_BF16 ? 2 : 4, head_chunks = p.c.dim * es / 16, row_chunks = head_chunks * p.c.kv_heads;
    const int fit = kPer * kThreads / row_chunks, rows = fit > 1 ? fit : 1;
    k_cache_append<<<dim3((unsigned)ceil_div(p.in.max_tokens, rows), (unsigned)p.in.max_batch + 1), kThreads, 0, s>>>(
        p, rows, row_chunks, head_chunks);
    return cudaGetLastError();
}

}  // namespace fz
