// Eviction from the paged cache by accumulated attention weight.  A sequence of n tokens keeps m = min(budget, n): its
// first s = min(sinks, m), its last r = min(recent, m - s), and of the ones between the m - s - r of largest weight (ties:
// lowest position).  Kept rows move, in ascending position, to positions 0 .. m - 1.
//
// k_select, a CTA per sequence: a radix selection finds the smallest kept weight, eight bits of the ordered key per pass
// over the weights; one more pass in order writes the kept tokens' slots.  k_move, a CTA per (sequence, key head, K or V):
// rows in ascending position, a chunk read whole before it is written.  In place that is safe without a copy: position i
// receives a row from a position >= i, so a chunk's target holds no row that a later chunk reads.
#include "cache.cuh"

namespace fz {
namespace {

constexpr int kSelThreads = 512, kMoveThreads = 256;

__device__ __forceinline__ unsigned slot_of(const Cache &c, int b, int pos) {
    unsigned page;
    cache_page(c, b, pos, page);
    return (page << c.shift) + (unsigned)(pos & ((1 << c.shift) - 1));
}

__global__ void __launch_bounds__(kSelThreads) k_cache_select(CacheEvictParams p) {
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Cache &c = p.c;
    __shared__ int hist[256];
    __shared__ int s_digit, s_above;
    __shared__ int2 s_scan[kSelThreads / 32];
    const int n = cache_length(c, b), m = n < 0 ? 0 : min(max(p.budget[b], 0), n);
    const int first = min(p.sinks, m), last = min(p.recent, m - first), lo = first, hi = n - last, want = m - first - last;
    int bad = n < 0 ? FUSION_DEV_BAD_CACHE : 0;
    if (!bad) {   // every page that is read or written, every weight that is compared
        bool wrong = false, nan = false;
        for (int e = tid; e < (n + (1 << c.shift) - 1) >> c.shift; e += kSelThreads)
            wrong |= (unsigned)c.table[(size_t)b * c.max_pages + e] >= c.num_pages;
        const int pages_m = (m + (1 << c.shift) - 1) >> c.shift;
        wrong |= pages_m > p.pages_out;
        for (int e = tid; e < min(pages_m, p.pages_out); e += kSelThreads)
            wrong |= (unsigned)p.table_out[(size_t)b * p.pages_out + e] >= c.num_pages;
        if (__syncthreads_or(wrong)) bad = FUSION_DEV_BAD_CACHE;
        if (!bad && m < n) {
            for (int j = lo + tid; j < hi; j += kSelThreads) nan |= !isfinite(c.weights[slot_of(c, b, j)]);
            if (__syncthreads_or(nan)) bad = FUSION_DEV_NONFINITE;
        }
    }
    if (bad) {
        if (tid == 0) {
            raise_status(p.status, bad);
            p.plan[b] = make_int2(-1, 0);
            if (p.lengths_out != c.lengths) p.lengths_out[b] = 0;
        }
        return;
    }
    // the smallest kept key of the middle: `key` fixed from the top, `want` still to find among the keys that share it
    unsigned key = 0;
    int ties = want;   // kept tokens of exactly that key
    if (m < n && want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int e = tid; e < 256; e += kSelThreads) hist[e] = 0;
            __syncthreads();
            const unsigned mask = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
            for (int j = lo + tid; j < hi; j += kSelThreads) {
                const unsigned o = ordered_bits(c.weights[slot_of(c, b, j)]);
                if ((o & mask) == key) atomicAdd(&hist[o >> shift & 255u], 1);
            }
            __syncthreads();
            if (tid == 0) {
                int above = 0, d = 255;
                while (d > 0 && above + hist[d] < ties) above += hist[d--];
                s_digit = d;
                s_above = above;
            }
            __syncthreads();
            key |= (unsigned)s_digit << shift;
            ties -= s_above;
            __syncthreads();
        }
    }
    // the kept tokens in order; `moved`: the first whose position changes
    int2 run = make_int2(0, 0);   // kept keys above, keys equal, so far
    int moved = m;
    unsigned *keep = p.keep + (size_t)b * c.capacity;
    for (int j0 = 0; j0 < n; j0 += kSelThreads) {
        const int j = j0 + tid;
        unsigned slot = 0;
        bool above = false, equal = false;
        if (j < n) {
            slot = slot_of(c, b, j);
            if (m == n || j < lo || j >= hi) above = true;
            else if (want > 0) {
                const unsigned o = ordered_bits(c.weights[slot]);
                above = o > key;
                equal = o == key;
            }
        }
        const unsigned ba = __ballot_sync(0xFFFFFFFFu, above), be = __ballot_sync(0xFFFFFFFFu, equal), lt = (1u << lane) - 1u;
        if (lane == 0) s_scan[warp] = make_int2(__popc(ba), __popc(be));
        __syncthreads();
        int2 pre = run;
        for (int w = 0; w < kSelThreads / 32; ++w) {
            const int2 v = s_scan[w];
            if (w < warp) {
                pre.x += v.x;
                pre.y += v.y;
            }
            run.x += v.x;
            run.y += v.y;
        }
        const int a = pre.x + __popc(ba & lt), e = pre.y + __popc(be & lt);
        if (above || (equal && e < ties)) {
            const int i = a + min(e, ties);
            keep[i] = slot;
            if (p.keep_idx && i < p.keep_stride) p.keep_idx[(size_t)b * p.keep_stride + i] = j;
            if (i != j) moved = min(moved, i);
        }
        __syncthreads();
    }
    __shared__ int s_moved;
    if (tid == 0) s_moved = m;
    __syncthreads();
    if (moved < m) atomicMin(&s_moved, moved);
    __syncthreads();
    if (tid == 0) {
        p.plan[b] = make_int2(m, p.in_place ? s_moved : 0);
        p.lengths_out[b] = m;
    }
}

__global__ void __launch_bounds__(kMoveThreads) k_cache_move(CacheEvictParams p, int head_chunks) {
    const int b = blockIdx.y, job = blockIdx.x, tid = threadIdx.x;
    const Cache &c = p.c;
    const int2 plan = p.plan[b];
    const int m = plan.x;
    const unsigned *keep = p.keep + (size_t)b * c.capacity;
    auto target = [&](int i) {
        const unsigned page = (unsigned)p.table_out[(size_t)b * p.pages_out + (i >> c.shift)];
        return (page << c.shift) + (unsigned)(i & ((1 << c.shift) - 1));
    };
    if (job == 2 * c.kv_heads) {   // sizes and weights
        for (int i0 = plan.y; i0 < m; i0 += kMoveThreads) {
            const int i = i0 + tid;
            float z = 0.0f, w = 0.0f;
            if (i < m) {
                const unsigned src = keep[i];
                if (c.sizes) z = c.sizes[src];
                w = c.weights[src];
            }
            __syncthreads();
            if (i < m) {
                const unsigned dst = target(i);
                if (c.sizes) c.sizes[dst] = z;
                c.weights[dst] = w;
            }
            __syncthreads();
        }
        return;
    }
    unsigned char *pool = job < c.kv_heads ? c.k : c.v;
    const unsigned h = (unsigned)(job % c.kv_heads), low = (1u << c.shift) - 1u;
    auto row = [&](unsigned slot) { return ((size_t)((((slot >> c.shift) * (unsigned)c.kv_heads + h) << c.shift) + (slot & low)) * head_chunks) * 16; };
    constexpr int kPer = 4;
    const long long all = (long long)m * head_chunks;
    for (long long e0 = (long long)plan.y * head_chunks; e0 < all; e0 += kMoveThreads * kPer) {
        uint4 v[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const long long e = e0 + k * kMoveThreads + tid;
            if (e < all) v[k] = *reinterpret_cast<const uint4 *>(pool + row(keep[e / head_chunks]) + (e % head_chunks) * 16);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const long long e = e0 + k * kMoveThreads + tid;
            if (e < all) *reinterpret_cast<uint4 *>(pool + row(target((int)(e / head_chunks))) + (e % head_chunks) * 16) = v[k];
        }
        __syncthreads();
    }
}

}  // namespace

cudaError_t launch_cache_evict(int dtype, const CacheEvictParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    const int head_chunks = p.c.dim * (dtype == FUSION_BF16 ? 2 : 4) / 16;
    k_cache_select<<<(unsigned)p.c.max_batch, kSelThreads, 0, s>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    k_cache_move<<<dim3((unsigned)(2 * p.c.kv_heads + 1), (unsigned)p.c.max_batch), kMoveThreads, 0, s>>>(p, head_chunks);
    return cudaGetLastError();
}

}  // namespace fz
