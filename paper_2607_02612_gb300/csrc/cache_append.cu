// Rows of a ragged batch go to the ends of their sequences in the paged cache: a copy, row by row, of keys, values,
// sizes and scores.  Bound by memory: every row is read once and written once.
//
// A CTA takes as many rows of one sample as give each thread kPer chunks of 16 bytes of K and of V, all asked for at once after the
// sample's ids and pages have been checked (256 samples of 100 to 197 tokens of 6 x 64 dims 23.4 us, 74 % of the copy's rate; before
// the checks, in registers meanwhile, 23.9).  All CTAs of a sample read its length before the last of them to finish raises it (a
// counter per sample, zero between calls), where the length is raised in place.
#include "cache.cuh"

namespace fz {
namespace {

constexpr int kThreads = 256, kPer = 4;
constexpr int kMostY = 65535;   // of a grid's height

// Whether sample i's slot is named by another sample too (all threads).  Every CTA reads all ids: 1 us for 256 samples, but the work
// grows with the square of the batch (1 to 65 tokens of 6 x 64 dims with and without ids: 1024 samples 21 and 20 us, 8192 197 and 163).
__device__ bool named_twice(const Ragged &in, int B, int i, int slot) {
    if (!in.ids) return false;
    bool twice = false;
    for (int j = threadIdx.x; j < B; j += kThreads) twice |= j != i && in.ids[j] == slot;
    return __syncthreads_or(twice);
}

// The lengths that no sample raises, where they go elsewhere (all threads; apart from the kernel, whose other CTAs fetch none of it).
__device__ __noinline__ void copy_other_lengths(const CacheAppendParams &p, int B) {
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

// A row of CTAs per sample, and one more for the lengths while the grid has room for it.
__global__ void __launch_bounds__(kThreads, 4) k_cache_append(CacheAppendParams p, int row_chunks, int head_chunks) {
    const int i = blockIdx.y, tid = threadIdx.x;
    const Cache &c = p.c;
    wait_for_previous();
    const int B = device_batch(p.in);
    if (i == (int)gridDim.y - 1 && blockIdx.x == 0) {   // (with kMostY samples the last sample's first CTA too)
        if (B < 0 && tid == 0) raise_status(p.status, FUSION_DEV_BAD_BATCH);
        if (!p.in_place) copy_other_lengths(p, B);
    }
    if (B < 0 || i >= B) return;
    const int slot = p.in.ids ? p.in.ids[i] : i;
    if (slot < 0 || slot >= c.max_batch) {
        if (blockIdx.x == 0 && tid == 0) raise_status(p.status, FUSION_DEV_BAD_IDS);
        return;
    }
    const int o0 = p.in.offsets[i], n = p.in.offsets[i + 1] - o0, at = c.lengths[slot];
    const bool rows_ok = o0 >= 0 && n >= 0 && n <= p.in.max_tokens && (long long)o0 + n <= p.in.max_rows;
    // `side` rows side by side, a thread has the same chunk (of `width` threads' chunks) of kPer rows of the CTA
    const int width = min(row_chunks, kThreads), side = kThreads / width, r_mine = tid / width;
    const int r0 = blockIdx.x * side * kPer, r1 = rows_ok && r_mine < side ? min(n, r0 + side * kPer) : r0;
    // (plain loads: the kernel before may still write the rows while this one is resident, which the read-only path does not allow)
    uint4 k[kPer], v[kPer];
    auto load = [&](int ch) {
        const unsigned char *ks = p.k + (size_t)(o0 + r0 + r_mine) * p.k_stride + (size_t)ch * 16;
        const unsigned char *vs = p.v + (size_t)(o0 + r0 + r_mine) * p.v_stride + (size_t)ch * 16;
#pragma unroll
        for (int x = 0; x < kPer; ++x)
            if (r0 + r_mine + x * side < r1) {
                k[x] = *reinterpret_cast<const uint4 *>(ks + (size_t)(x * side) * p.k_stride);
                v[x] = *reinterpret_cast<const uint4 *>(vs + (size_t)(x * side) * p.v_stride);
            }
    };
    int bad = !rows_ok ? FUSION_DEV_BAD_OFFSETS : at < 0 || at > c.capacity || n > c.capacity - at ? FUSION_DEV_BAD_CACHE : 0;
    unsigned page[kPer];
    bool wrong = false;
    if (!bad) {
        const unsigned *pages = reinterpret_cast<const unsigned *>(c.table) + (size_t)slot * c.max_pages;
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            const int r = r0 + r_mine + x * side;
            page[x] = r < r1 ? pages[(at + r) >> c.shift] : 0u;
        }
        for (int e = (at >> c.shift) + tid; n > 0 && e <= (at + n - 1) >> c.shift; e += kThreads) wrong |= pages[e] >= c.num_pages;
    }
    if (named_twice(p.in, B, i, slot)) bad |= FUSION_DEV_BAD_IDS;
    if (__syncthreads_or(wrong)) bad |= FUSION_DEV_BAD_CACHE;
    if (bad) {   // nothing of this sample is written, and its slot's length stays (also where it is named twice)
        if (blockIdx.x == 0 && tid == 0) {
            raise_status(p.status, bad);
            if (!p.in_place) p.lengths_out[slot] = at;
        }
        return;
    }
    const unsigned low = (1u << c.shift) - 1u;
    for (int ch = tid % width; ch < row_chunks; ch += kThreads) {   // (once, unless a row has more than kThreads chunks)
        load(ch);
        const int h = ch / head_chunks, cc = ch - h * head_chunks;
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            const int r = r0 + r_mine + x * side;
            if (r >= r1) break;
            const size_t dst = ((size_t)(((page[x] * (unsigned)c.kv_heads + h) << c.shift) + ((at + r) & low)) * head_chunks + cc) * 16;
            *reinterpret_cast<uint4 *>(c.k + dst) = k[x];
            *reinterpret_cast<uint4 *>(c.v + dst) = v[x];
        }
    }
    for (int r = r0 + tid; r < min(n, r0 + side * kPer); r += kThreads) {
        unsigned pg;
        cache_page(c, slot, at + r, pg);
        const size_t s = ((size_t)pg << c.shift) + ((at + r) & low);
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
    const int rows = kPer * (row_chunks < kThreads ? kThreads / row_chunks : 1);
    // (samples of more rows than the cache has room for, or than there are, write nothing)
    long long most = p.in.max_tokens < p.c.capacity ? p.in.max_tokens : p.c.capacity;
    if (most > p.in.max_rows) most = p.in.max_rows;
    static_assert(FUSION_CACHE_MAX_BATCH <= kMostY, "a row of CTAs per sample");
    const dim3 grid((unsigned)(most > 0 ? (most + rows - 1) / rows : 1), (unsigned)(p.in.max_batch < kMostY ? p.in.max_batch + 1 : kMostY));
    return launch_after(k_cache_append, grid, kThreads, 0, 1, s, p, row_chunks, head_chunks);
}

}  // namespace fz
