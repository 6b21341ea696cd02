// Eviction from the paged cache by accumulated attention weight.  A sequence of n tokens keeps m = min(budget, n): its
// first s = min(sinks, m), its last r = min(recent, m - s), and of the ones between the m - s - r of largest weight (ties:
// lowest position).  Kept rows move, in ascending position, to positions 0 .. m - 1.
//
// k_cache_select, a CTA (or a cluster of them, for long sequences) per sequence: the ordered keys of the weights stay in shared
// memory, each warp's in a piece of its own; the smallest kept key is found from its 11 top bits down by three histograms (11
// bits spread weights, which share a few exponents, over enough bins that their atomics rarely meet; a pass whose bin is kept
// whole is the last).  Each warp then places its kept tokens behind those of the warps before it.  What bounds it is the chain
// of its phases and, of code that runs once, the fetching of its instructions, so all loops over keys are rolled (keys in
// registers and loops unrolled: 8 x 577 10.8 us, now 7.8; 157 x 34 11.4, now 8.8).  The CTAs of a cluster exchange sums of 32 bins,
// then read 32 bins of each other (all 2048 of each: 3000 cycles a pass).
//
// k_cache_move copies the rows.  Into other pages: any CTA any rows.  In place: a team of CTAs (a cluster) per (sequence, key
// head, K or V) takes the rows in ascending position, a step of them at a time, all read before any is written.  That is safe
// without a copy aside: position i receives a row from a position >= i, so no target of a step is read by a later step.  A step is
// load, barrier, store, one after the other (prompt of 32768 to 16384: 26.7 us, 40 % of DRAM's rate).
#include <atomic>

#include "cache.cuh"

namespace fz {
namespace {

constexpr int kHeld = 16;    // keys of a thread in shared memory, with their slots
constexpr int kAtOnce = 4;   // of them in flight
constexpr int kBins = 2048;  // of a histogram

__device__ __forceinline__ unsigned slot_of(const Cache &c, int b, int pos) {
    unsigned page;
    cache_page(c, b, pos, page);
    return (page << c.shift) + (unsigned)(pos & ((1 << c.shift) - 1));
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// Four numbers of every CTA of the cluster in each of its CTAs; two boxes in turn (par), so that one barrier does.
struct Exchange {
    int4 box[2][8];
};
template <int C>
__device__ __forceinline__ void exchange(Exchange &x, int &par, int rank, int4 v) {
    if constexpr (C == 1) {
        if (threadIdx.x == 0) x.box[par][0] = v;
        __syncthreads();
    } else {
        if (threadIdx.x < C) {
            const uint32_t mine = smem_addr(&x.box[par][rank]);
            uint32_t theirs;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(theirs) : "r"(mine), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(theirs), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
        }
        cluster_arrive();
        cluster_wait();
    }
    par ^= 1;
}

__device__ __forceinline__ int peer_load(const int *here, int k) {   // the number at the same place of CTA k of the cluster
    uint32_t theirs;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(theirs) : "r"(smem_addr(here)), "r"(k));
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(theirs) : "memory");
    return v;
}
__device__ __forceinline__ void peer_store(const int *here, int k, int v) {
    uint32_t theirs;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(theirs) : "r"(smem_addr(here)), "r"(k));
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(theirs), "r"(v) : "memory");
}
__device__ __forceinline__ void cp_async4(const void *dst, const void *src, bool read) {   // (zero if not read)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(read ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ int scan(int v, int lane) {   // inclusive, over the warp
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, v, s);
        if (lane >= s) v += u;
    }
    return v;
}

// C: CTAs of a sequence; each takes an equal part of the positions that are compared, each of its warps an equal part of those.
template <int C, int kSelThreads>
__global__ void __launch_bounds__(kSelThreads) k_cache_select(CacheEvictParams p) {
    constexpr int kSelWarps = kSelThreads / 32, kMine = kBins / kSelThreads, kCoarse = kBins / 32;   // bins of a thread; sums of 32 bins
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = C == 1 ? 0 : (int)cluster_rank();
    const Cache &c = p.c;
    extern __shared__ __align__(16) int sm[];   // a histogram for each pass (none is cleared that another CTA reads), keys, slots
    __shared__ Exchange box;
    __shared__ __align__(8) int s_coarse[3][C][kCoarse];
    __shared__ int2 s_count[kSelWarps];
    __shared__ int s_first;
    unsigned *keys = reinterpret_cast<unsigned *>(sm + 3 * kBins) + warp * kHeld * 32 + lane, *slots = keys + kHeld * kSelThreads;
    const int *pages = c.table + (size_t)b * c.max_pages;
    const unsigned low = (1u << c.shift) - 1u;
    wait_for_previous();
    int par = 0;
    // (one reading of the length and the budget for all, so that every CTA takes the same way whatever happens to them)
    const int n0 = cache_length(c, b), budget = p.budget[b];
#pragma unroll 2
    for (int e = tid; e < 3 * kBins / 4; e += kSelThreads) reinterpret_cast<int4 *>(sm)[e] = make_int4(0, 0, 0, 0);
    if constexpr (C > 1) {   // all CTAs of the cluster are here before one writes to another
        cluster_arrive();
        cluster_wait();
    }
    exchange<C>(box, par, rank, make_int4(n0, n0 < 0 ? 0 : min(max(budget, 0), n0), 0, 0));
    const int n = box.box[par ^ 1][0].x, m = box.box[par ^ 1][0].y;
    const int first = min(p.sinks, m), last = min(p.recent, m - first), lo = first, hi = n - last, want = m - first - last;
    const bool choose = m < n;                       // else every token stays
    const int middle = choose ? hi - lo : 0, per = (middle + C - 1) / C;
    const int at = lo + min(rank * per, middle), end = lo + min((rank + 1) * per, middle);
    const int rows = (end - at + kSelThreads - 1) / kSelThreads, held = min(rows, kHeld);
    const int j0 = at + warp * rows * 32 + lane, mine = min(end, at + (warp + 1) * rows * 32);   // this thread's positions, every 32nd to `mine`
    if (tid == 0) s_first = n;

    // ---- the pages that are read and written, the weights that are compared
    bool wrong = n < 0, nan = false;
    if (!wrong) {
        const int pages_n = (n + (1 << c.shift) - 1) >> c.shift, pages_m = (m + (1 << c.shift) - 1) >> c.shift;
        const int out_n = p.in_place ? 0 : min(pages_m, p.pages_out);
        const int *out = p.table_out + (size_t)b * p.pages_out;
        const unsigned page0 = tid < pages_n ? (unsigned)pages[tid] : 0u, out0 = tid < out_n ? (unsigned)out[tid] : 0u;
        for (int i0 = 0; i0 < held; i0 += kAtOnce) {
            unsigned page[kAtOnce];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) page[x] = (unsigned)pages[min(j0 + (i0 + x) * 32, n - 1) >> c.shift];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const int i = (i0 + x) * 32, j = j0 + i;
                const bool read = j < mine && page[x] < c.num_pages;
                const unsigned slot = read ? (page[x] << c.shift) + ((unsigned)j & low) : 0u;
                slots[i] = slot;
                cp_async4(keys + i, c.weights + slot, read);
            }
        }
        wrong = pages_m > p.pages_out || (tid < pages_n && page0 >= c.num_pages) || (tid < out_n && out0 >= c.num_pages);
        for (int e = tid + kSelThreads; e < pages_n; e += kSelThreads) wrong |= (unsigned)pages[e] >= c.num_pages;
        for (int e = tid + kSelThreads; e < out_n; e += kSelThreads) wrong |= (unsigned)out[e] >= c.num_pages;
        cp_async_wait();
        for (int i0 = 0; i0 < held; i0 += kAtOnce) {
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const int i = (i0 + x) * 32;
                const float w = __uint_as_float(keys[i]);
                nan |= want > 0 && !isfinite(w);                    // (zero where there is no position)
                keys[i] = j0 + i < mine ? ordered_bits(w) : 0u;   // (no finite weight has the key 0)
            }
        }
        for (int j = j0 + kHeld * 32; j < mine; j += 32) {
            unsigned page;
            if (cache_page(c, b, j, page)) nan |= want > 0 && !isfinite(c.weights[(page << c.shift) + ((unsigned)j & low)]);
        }
    }
    {
        int any = __syncthreads_or(wrong || nan), any_wrong = 0;
        if (any) any_wrong = __syncthreads_or(wrong);
        if constexpr (C > 1) {
            exchange<C>(box, par, rank, make_int4(any, any_wrong, 0, 0));
            for (int k = 0; k < C; ++k) {
                any |= box.box[par ^ 1][k].x;
                any_wrong |= box.box[par ^ 1][k].y;
            }
        }
        wrong = any_wrong != 0;
        nan = any != 0;
    }
    if (wrong || nan) {
        if (rank == 0 && tid == 0) {
            raise_status(p.status, wrong ? FUSION_DEV_BAD_CACHE : FUSION_DEV_NONFINITE);
            p.plan[b] = make_int2(-1, 0);
            if (p.lengths_out != c.lengths) p.lengths_out[b] = 0;
        }
        return;   // (after an exchange: nobody writes to a CTA's box any more)
    }
    // calls f(key, position, slot) for the thread's positions in turn, the warp's lanes together (key 0: no position)
    auto each = [&](auto f) {
        for (int i0 = 0; i0 < held; i0 += kAtOnce) {
            unsigned o[kAtOnce], slot[kAtOnce];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                o[x] = keys[(i0 + x) * 32];
                slot[x] = slots[(i0 + x) * 32];
            }
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) f(o[x], j0 + (i0 + x) * 32, slot[x]);
        }
        for (int i = kHeld; i < rows; ++i) {
            const int j = j0 + i * 32;
            const unsigned slot = j < mine ? slot_of(c, b, j) : 0u;
            f(j < mine ? ordered_bits(c.weights[slot]) : 0u, j, slot);
        }
    };

    // ---- T, the smallest kept key, from the top digit down; `left`: kept keys among those that share T's digits so far
    unsigned T = 0;
    int left = want;
    bool exact = want == 0;   // every key that shares T's digits is kept: no ties to break
#pragma unroll 1
    for (int pass = 0; choose && !exact && pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;   // 11, 11 and 10 bits
        const unsigned top = pass == 0 ? 0u : pass == 1 ? 0xFFFFFFFFu << 21 : 0xFFFFFFFFu << 10, digit = pass == 2 ? 1023u : 2047u;
        int *hist = sm + pass * kBins;
        each([&](unsigned o, int, unsigned) {
            if (o != 0u && (o & top) == T) atomicAdd(&hist[o >> shift & digit], 1);
        });
        __syncthreads();
        // sums of 32 bins, to all CTAs of the cluster
        int sum = 0;
#pragma unroll
        for (int x = 0; x < kMine; x += 2) {
            const int2 u = *reinterpret_cast<const int2 *>(&hist[tid * kMine + x]);
            sum += u.x + u.y;
        }
        constexpr int kSide = 32 / kMine;   // lanes of a sum
#pragma unroll
        for (int s = 1; s < kSide; s <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
        static_assert(C <= kSide, "a lane for every CTA of the cluster");
        int *coarse = s_coarse[pass][rank] + tid / kSide;
        if constexpr (C > 1) {
            if (tid % kSide < C) peer_store(coarse, tid % kSide, sum);
            cluster_arrive();
            cluster_wait();
        } else {
            if (tid % kSide == 0) *coarse = sum;
            __syncthreads();
        }
        // every warp finds the digit, from the largest down: among the sums, then among the bins of one
        int2 v = make_int2(0, 0);
        const int pair = kCoarse - 2 - 2 * lane;
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int2 u = *reinterpret_cast<const int2 *>(&s_coarse[pass][k][pair]);
            v.x += u.x;
            v.y += u.y;
        }
        int incl = scan(v.x + v.y, lane), before = incl - v.x - v.y;
        int here = __ffs(__ballot_sync(0xFFFFFFFFu, before < left && left <= incl)) - 1;
        const bool upper = before + v.y >= left;
        const int bins = __shfl_sync(0xFFFFFFFFu, upper ? pair + 1 : pair, here) * 32;
        left -= __shfl_sync(0xFFFFFFFFu, upper ? before : before + v.y, here);
        const int *bin = &hist[bins + 31 - lane];
        int cnt = 0;
        if constexpr (C > 1) {
#pragma unroll
            for (int k = 0; k < C; ++k) cnt += peer_load(bin, k);
        } else {
            cnt = *bin;
        }
        incl = scan(cnt, lane);
        here = __ffs(__ballot_sync(0xFFFFFFFFu, incl - cnt < left && left <= incl)) - 1;
        T |= (unsigned)(bins + 31 - here) << shift;
        left -= __shfl_sync(0xFFFFFFFFu, incl - cnt, here);
        exact = __shfl_sync(0xFFFFFFFFu, cnt, here) == left;
    }
    // kept: keys above the threshold, and the first `left` of those equal to it
    const unsigned above = want == 0 ? 0xFFFFFFFFu : exact ? T - 1u : T;
    const bool tied = choose && !exact;
    const int ties = tied ? left : 0;
    // ---- kept tokens and ties before this warp's
    int2 count = make_int2(0, 0);
    each([&](unsigned o, int, unsigned) {
        count.x += o > above;
        count.y += tied && o == above;
    });
    count = make_int2((int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)count.x), (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)count.y));
    if (lane == 0) s_count[warp] = count;
    __syncthreads();
    count = lane < kSelWarps ? s_count[lane] : make_int2(0, 0);
    int na = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)(lane < warp ? count.x : 0));
    int ne = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)(lane < warp ? count.y : 0));
    if constexpr (C > 1) {
        count.x = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)count.x);
        count.y = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)count.y);
        exchange<C>(box, par, rank, make_int4(count.x, count.y, 0, 0));
        for (int k = 0; k < rank; ++k) {
            na += box.box[par ^ 1][k].x;
            ne += box.box[par ^ 1][k].y;
        }
    }
    unsigned *keep = p.keep + (size_t)b * c.capacity;
    int *idx = p.keep_idx + (size_t)b * p.keep_stride;
    const int idx_n = p.keep_idx ? p.keep_stride : 0;
    auto put = [&](int i, int j, unsigned slot) {
        keep[i] = slot;
        if (i < idx_n) idx[i] = j;
    };
    // the first position that goes (where no weight is compared the first between, whatever its weight: a NaN of all ones has the key 0)
    int evicted = choose && want == 0 ? lo : n;
    const unsigned lt = (1u << lane) - 1u;
    na += first;
    each([&](unsigned o, int j, unsigned slot) {
        bool stays = o > above;
        const unsigned ba = __ballot_sync(0xFFFFFFFFu, stays);
        int i = na + __popc(ba & lt);
        na += __popc(ba);
        if (tied) {
            const unsigned be = __ballot_sync(0xFFFFFFFFu, o == above);
            const int before_e = ne + __popc(be & lt);
            stays |= o == above && before_e < ties;
            i += min(before_e, ties);
            ne += __popc(be);
        }
        evicted = stays || o == 0u ? evicted : min(evicted, j);
        if (stays) keep[i] = slot;
        if (stays && i < idx_n) idx[i] = j;
    });
    // ---- the tokens that stay anyway
    if (choose) {
        for (int i = rank * kSelThreads + tid; i < first; i += C * kSelThreads) put(i, i, slot_of(c, b, i));
        for (int i = rank * kSelThreads + tid; i < last; i += C * kSelThreads) put(m - last + i, n - last + i, slot_of(c, b, n - last + i));
    } else {
        for (int i = rank * kSelThreads + tid; i < m; i += C * kSelThreads) put(i, i, slot_of(c, b, i));
    }
    // ---- nothing before the first evicted position moves in place
    evicted = __reduce_min_sync(0xFFFFFFFFu, evicted);
    if (lane == 0 && evicted < n) atomicMin(&s_first, evicted);
    __syncthreads();
    evicted = s_first;
    if constexpr (C > 1) {   // (nor does a CTA leave whose histograms another reads)
        exchange<C>(box, par, rank, make_int4(evicted, 0, 0, 0));
        for (int k = 0; k < C; ++k) evicted = min(evicted, box.box[par ^ 1][k].x);
    }
    if (rank == 0 && tid == 0) {
        p.plan[b] = make_int2(m, p.in_place ? min(evicted, m) : 0);
        p.lengths_out[b] = m;
    }
}

constexpr int kMoveThreads = 512, kPer = 8;   // kPer units of a thread in flight
// `width` columns of a sequence's kept rows by a team of CTAs, a column being one of the 2 kv_heads * units units (16 bytes of keys
// and values, 4 of scales) of a token.  A thread has one column of rows `stride` apart.
template <bool kInPlace, typename U, typename Target>
__device__ __forceinline__ void move_columns(const CacheEvictParams &p, const int2 plan, const unsigned *keep, Target target,
                                             unsigned char *k, unsigned char *v, int units, int width, int group) {
    const int tid = threadIdx.x, team = gridDim.x, member = blockIdx.x, m = plan.x;
    const Cache &c = p.c;
    const unsigned low = (1u << c.shift) - 1u;
    const int stride = kMoveThreads / width, r0 = tid / width, step = stride * kPer, column = group * width + tid % width;
    const int h2 = column / units, unit = column - h2 * units;
    const bool idle = r0 >= stride || h2 >= 2 * c.kv_heads;
    unsigned char *pool = (h2 < c.kv_heads ? k : v) + unit * sizeof(U);
    const unsigned h = (unsigned)(h2 < c.kv_heads ? h2 : h2 - c.kv_heads);
    auto row = [&](unsigned slot) {
        return pool + (size_t)((((slot >> c.shift) * (unsigned)c.kv_heads + h) << c.shift) + (slot & low)) * units * sizeof(U);
    };
    U held[kPer];
    auto load = [&](int i0) {
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            const int i = i0 + r0 + x * stride;
            if (!idle && i < m) held[x] = *reinterpret_cast<const U *>(row(keep[i]));
        }
    };
    auto store = [&](int i0) {
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            const int i = i0 + r0 + x * stride;
            if (!idle && i < m) *reinterpret_cast<U *>(row(target(i))) = held[x];
        }
    };
    for (int s0 = plan.y; s0 < m; s0 += team * step) {   // (the same number of steps for every member)
        load(s0 + member * step);
        if (kInPlace) {
            cluster_arrive();
            cluster_wait();
        }
        store(s0 + member * step);
    }
}

// How the columns of one kind are dealt out: `width` of them a CTA, `groups` CTAs.
struct Columns {
    int units, width, groups;
};

// gridDim.x CTAs (in place: a cluster) per sequence and group of columns: the groups of keys and values, those of their scales, then
// one for sizes and weights.
template <bool kInPlace>
__global__ void __launch_bounds__(kMoveThreads, 2) k_cache_move(CacheEvictParams p, Columns rows, Columns scales) {
    const int b = blockIdx.z, tid = threadIdx.x, team = gridDim.x, member = blockIdx.x;
    const Cache &c = p.c;
    wait_for_previous();
    const int2 plan = p.plan[b];
    const int m = plan.x;
    const unsigned *keep = p.keep + (size_t)b * c.capacity;
    const unsigned low = (1u << c.shift) - 1u;
    auto target = [&](int i) {
        const unsigned page = (unsigned)p.table_out[(size_t)b * p.pages_out + (i >> c.shift)];
        return (page << c.shift) + ((unsigned)i & low);
    };
    if (blockIdx.y == gridDim.y - 1) {   // sizes and weights
        for (int i0 = plan.y + member * kMoveThreads; i0 - member * kMoveThreads < m; i0 += team * kMoveThreads) {
            const int i = i0 + tid;
            float z = 0.0f, w = 0.0f;
            if (i < m) {
                const unsigned src = keep[i];
                if (c.sizes) z = c.sizes[src];
                w = c.weights[src];
            }
            if (kInPlace) {
                cluster_arrive();
                cluster_wait();
            }
            if (i < m) {
                const unsigned dst = target(i);
                if (c.sizes) c.sizes[dst] = z;
                c.weights[dst] = w;
            }
        }
        return;
    }
    if ((int)blockIdx.y < rows.groups) move_columns<kInPlace, uint4>(p, plan, keep, target, c.k, c.v, rows.units, rows.width, blockIdx.y);
    else move_columns<kInPlace, uint32_t>(p, plan, keep, target, p.s.k, p.s.v, scales.units, scales.width, (int)blockIdx.y - rows.groups);
}

// Lets a kernel have `smem` bytes of dynamic shared memory, asked for once per device.
template <auto Kernel>
cudaError_t allow_smem(int smem) {
    constexpr int kDevices = 64;
    static std::atomic<bool> done[kDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < kDevices && done[dev].load(std::memory_order_acquire))) return e;
    e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && dev < kDevices) done[dev].store(true, std::memory_order_release);
    return e;
}
template <int C, int kSelThreads>
cudaError_t launch_select(const CacheEvictParams &p, cudaStream_t s) {
    constexpr int kSmem = (3 * kBins + 2 * kHeld * kSelThreads) * 4;
    const cudaError_t e = allow_smem<k_cache_select<C, kSelThreads>>(kSmem);
    if (e != cudaSuccess) return e;
    return launch_after(k_cache_select<C, kSelThreads>, dim3(C, (unsigned)p.c.max_batch), kSelThreads, (size_t)kSmem, C, s, p);
}

}  // namespace

cudaError_t launch_cache_evict(int row_bytes, const CacheEvictParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    const int head_chunks = row_bytes / 16;
    // Threads of a sequence, by the room of a row of the page table, since its length is known on the device alone (64 sequences of
    // 500 with room for 512, 4096, 32768, in place to half: 16.9, 17.8, 43.4 us).  Few where it is short, since every warp more has its
    // share of the phases (8 x 577: 256 threads 7.9 us, 512 8.1), more where each would have many keys (64 x 1900: 21.4 and 20.8;
    // 64 x 4000: 512 threads 34.2, 1024 32.4; 32 x 8192: 160.6 and 155.8), then clusters of up to 8 CTAs (8852: two of 1024 threads
    // 18.6, four of 512 18.8; 10973: 16.6 and 14.5; 32768: four of 1024 85.0, eight of 512 83.7).
    const int cap = p.c.capacity, k = kHeld;
    cudaError_t e = cap <= 64 * k     ? launch_select<1, 256>(p, s)
                    : cap <= 256 * k  ? launch_select<1, 512>(p, s)
                    : cap <= 512 * k  ? launch_select<1, 1024>(p, s)
                    : cap <= 1024 * k ? launch_select<4, 512>(p, s)
                    : cap <= 4096 * k ? launch_select<8, 512>(p, s)
                                      : launch_select<8, 1024>(p, s);
    if (e != cudaSuccess) return e;
    // Columns of a CTA: a head's, or more where the sequences are too short for a step of kPer rows by all threads (132 x 17 of 16
    // heads of 80 float32: 33 us with one head a CTA), or half of them (not below 128 bytes) where a team in place would leave SMs
    // idle.  Then enough CTAs to fill the GPU a few times, no more than a sequence has steps for.
    const long long most = p.in_place ? p.c.capacity : (long long)p.pages_out << p.c.shift;
    auto columns_of = [&](int units) {
        Columns k{units, units, 0};
        const int columns = 2 * p.c.kv_heads * units;
        while (k.width < kMoveThreads && k.width < columns && (long long)(kMoveThreads / k.width) * kPer > most) k.width *= 2;
        if (k.width > columns) k.width = columns;
        if (k.width > kMoveThreads) k.width = kMoveThreads;
        k.groups = (columns + k.width - 1) / k.width;
        return k;
    };
    Columns rows = columns_of(head_chunks), scales = p.s.k ? columns_of(p.s.bytes / 4) : Columns{1, 1, 0};
    auto team_of = [&] { return (p.in_place ? 608ll : 2432ll) / ((long long)(rows.groups + scales.groups + 1) * p.c.max_batch); };
    while (p.in_place && team_of() > 8 && rows.width <= head_chunks && rows.width >= 16 && rows.width % 2 == 0) {
        rows.width /= 2;
        rows.groups = (2 * p.c.kv_heads * head_chunks + rows.width - 1) / rows.width;
    }
    const int step = kMoveThreads / rows.width * kPer;
    const long long steps = (most + step - 1) / step;
    long long team = team_of();
    if (team > steps) team = steps;
    if (p.in_place) team = team >= 8 ? 8 : team >= 4 ? 4 : team >= 2 ? 2 : 1;
    if (team < 1) team = 1;
    const dim3 grid((unsigned)team, (unsigned)(rows.groups + scales.groups + 1), (unsigned)p.c.max_batch);
    return p.in_place ? launch_after(k_cache_move<true>, grid, kMoveThreads, 0, (int)team, s, p, rows, scales)
                      : launch_after(k_cache_move<false>, grid, kMoveThreads, 0, 1, s, p, rows, scales);
}

}  // namespace fz
