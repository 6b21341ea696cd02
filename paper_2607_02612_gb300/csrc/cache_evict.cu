// Eviction from the paged cache by accumulated attention weight.  A sequence of n tokens keeps m = min(budget, n): its
// first s = min(sinks, m), its last r = min(recent, m - s), and of the ones between the m - s - r of largest weight (ties:
// lowest position).  Kept rows move, in ascending position, to positions 0 .. m - 1.
//
// k_cache_select, a CTA (or a cluster of them, for long sequences) per sequence: the ordered keys of the weights stay in
// registers; the smallest kept key is found from its 11 top bits down by three histograms (11 bits spread weights, which share
// a few exponents, over enough bins that their atomics rarely meet; a pass whose bin is kept whole is the last).  One scan
// over the counts of all warps then places the kept tokens.
//
// k_cache_move copies the rows.  Into other pages: any CTA any rows.  In place: a team of CTAs (a cluster) per (sequence, key
// head, K or V) takes the rows in ascending position, a step of them at a time, all read before any is written.  That is safe
// without a copy aside: position i receives a row from a position >= i, so no target of a step is read by a later step, and
// the next step's rows are read while the team waits.
#include "cache.cuh"

namespace fz {
namespace {

constexpr int kKeys = 16;    // keys of a thread in registers
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

// Two numbers at the same place of CTA k of the cluster.
__device__ __forceinline__ int2 peer_pair(const int *here, int k) {
    uint32_t theirs;
    int2 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(theirs) : "r"(smem_addr(here)), "r"(k));
    asm volatile("ld.shared::cluster.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(theirs) : "memory");
    return v;
}

// C: CTAs of a sequence; each takes a run of the positions that are compared.
template <int C, int kSelThreads>
__global__ void __launch_bounds__(kSelThreads) k_cache_select(CacheEvictParams p) {
    constexpr int kSelWarps = kSelThreads / 32, kMine = kBins / kSelThreads;   // bins of a thread
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = C == 1 ? 0 : (int)cluster_rank();
    const Cache &c = p.c;
    __shared__ Exchange box;
    __shared__ __align__(16) int hist[kBins];
    __shared__ int s_warp[kSelWarps], s_digit[3];
    __shared__ int s_scan[kKeys * kSelWarps];
    __shared__ int s_first;
    wait_for_previous();
    int par = 0;
    if constexpr (C > 1) {   // all CTAs of the cluster are here before one writes to another
        cluster_arrive();
        cluster_wait();
    }
    // (one reading of the length and the budget for all, so that every CTA takes the same way whatever happens to them)
    const int n0 = cache_length(c, b);
    exchange<C>(box, par, rank, make_int4(n0, n0 < 0 ? 0 : min(max(p.budget[b], 0), n0), 0, 0));
    const int n = box.box[par ^ 1][0].x, m = box.box[par ^ 1][0].y;
    const int first = min(p.sinks, m), last = min(p.recent, m - first), lo = first, hi = n - last, want = m - first - last;
    const bool choose = m < n;                       // else every token stays
    // this CTA's run of [lo, hi): per positions from at on, kKeys * kSelThreads of them in registers
    const int middle = choose ? hi - lo : 0;
    const int per = C == 1 ? middle : ((middle + C - 1) / C + kSelThreads - 1) / kSelThreads * kSelThreads;
    const int at = lo + min(rank * per, middle), end = lo + min((rank + 1) * per, middle);
    auto key_at = [&](int j) { return ordered_bits(c.weights[slot_of(c, b, j)]); };

    // ---- the pages that are read and written, the weights that are compared
    bool wrong = n < 0, nan = false;
    unsigned key[kKeys];
    if (!wrong) {
        const int pages_n = (n + (1 << c.shift) - 1) >> c.shift, pages_m = (m + (1 << c.shift) - 1) >> c.shift;
        wrong = pages_m > p.pages_out;
        for (int e = tid; e < pages_n; e += kSelThreads) wrong |= (unsigned)c.table[(size_t)b * c.max_pages + e] >= c.num_pages;
        if (!p.in_place)
            for (int e = tid; e < min(pages_m, p.pages_out); e += kSelThreads)
                wrong |= (unsigned)p.table_out[(size_t)b * p.pages_out + e] >= c.num_pages;
        // (all pages, then all weights: no branch between the loads)
        const int top = max(end - 1, 0);   // (row b has a position 0)
#pragma unroll
        for (int i = 0; i < kKeys; ++i) key[i] = (unsigned)c.table[(size_t)b * c.max_pages + (min(at + i * kSelThreads + tid, top) >> c.shift)];
#pragma unroll
        for (int i = 0; i < kKeys; ++i)
            key[i] = __float_as_uint(c.weights[((key[i] < c.num_pages ? key[i] : 0u) << c.shift) +
                                               (unsigned)(min(at + i * kSelThreads + tid, top) & ((1 << c.shift) - 1))]);
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
            const bool here = at + i * kSelThreads + tid < end;
            nan |= here && want > 0 && !isfinite(__uint_as_float(key[i]));
            key[i] = here ? ordered_bits(__uint_as_float(key[i])) : 0u;   // (no finite weight has the key 0)
        }
        for (int j = at + kKeys * kSelThreads + tid; j < end; j += kSelThreads) {
            unsigned page;
            if (cache_page(c, b, j, page)) nan |= want > 0 && !isfinite(c.weights[(page << c.shift) + (unsigned)(j & ((1 << c.shift) - 1))]);
        }
    }
    for (int e = tid; e < kBins; e += kSelThreads) hist[e] = 0;
    {
        const int any_nan = __syncthreads_or(nan), any_wrong = __syncthreads_or(wrong);
        exchange<C>(box, par, rank, make_int4(any_nan, any_wrong, 0, 0));
        nan = wrong = false;
        for (int k = 0; k < C; ++k) {
            nan |= box.box[par ^ 1][k].x != 0;
            wrong |= box.box[par ^ 1][k].y != 0;
        }
    }
    if (wrong || nan) {
        if (rank == 0 && tid == 0) {
            raise_status(p.status, wrong ? FUSION_DEV_BAD_CACHE : FUSION_DEV_NONFINITE);
            p.plan[b] = make_int2(-1, 0);
            if (p.lengths_out != c.lengths) p.lengths_out[b] = 0;
        }
        return;   // (after an exchange: nobody writes to a CTA's box any more)
    }

    // ---- T, the smallest kept key, from the top digit down; `left`: kept keys among those that share T's digits so far
    unsigned T = 0;
    int left = want;
    bool exact = want == 0;   // every key that shares T's digits is kept: no ties to break
#pragma unroll 1
    for (int shift = 21; choose && !exact && shift >= 0; shift -= shift > 11 ? 11 : 10) {
        const unsigned width = shift > 0 ? 11u : 10u, top = shift == 21 ? 0u : 0xFFFFFFFFu << (shift + width);   // 11, 11 and 10 bits
#pragma unroll
        for (int i = 0; i < kKeys; ++i)
            if (key[i] != 0u && (key[i] & top) == T) atomicAdd(&hist[key[i] >> shift & (kBins - 1)], 1);
        for (int j = at + kKeys * kSelThreads + tid; j < end; j += kSelThreads) {
            const unsigned o = key_at(j);
            if ((o & top) == T) atomicAdd(&hist[o >> shift & (kBins - 1)], 1);
        }
        if constexpr (C > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
        // counts from the largest digit down, kMine a thread; the cluster's histograms are summed on the way
        const int low_bin = kBins - (tid + 1) * kMine;
        int v[kMine], incl = 0;
#pragma unroll
        for (int x = 0; x < kMine; x += 2) {
            int2 w = make_int2(0, 0);
            if constexpr (C > 1) {
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    const int2 u = peer_pair(&hist[low_bin + x], k);
                    w.x += u.x;
                    w.y += u.y;
                }
            } else {
                w = *reinterpret_cast<const int2 *>(&hist[low_bin + x]);
            }
            v[x] = w.x;
            v[x + 1] = w.y;
            incl += w.x + w.y;
        }
        const int mine = incl;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, incl, s);
            if (lane >= s) incl += u;
        }
        if (lane == 31) s_warp[warp] = incl;
        __syncthreads();
        {
            const int w = lane < kSelWarps ? s_warp[lane] : 0;
            incl += (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)(lane < warp ? w : 0));
        }
        int before = incl - mine;
        if (before < left && left <= incl) {   // one thread
            bool found = false;
#pragma unroll
            for (int x = kMine - 1; x >= 0; --x) {
                if (!found && before + v[x] >= left) {
                    found = true;
                    s_digit[0] = low_bin + x;
                    s_digit[1] = before;
                    s_digit[2] = v[x];
                }
                before += v[x];
            }
        }
        if constexpr (C > 1) {   // (nobody clears a histogram that another reads)
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
        T |= (unsigned)s_digit[0] << shift;
        left -= s_digit[1];
        exact = s_digit[2] == left;
        for (int e = tid; e < kBins; e += kSelThreads) hist[e] = 0;
        __syncthreads();
    }
    // kept: keys above the threshold, and the first `ties` of those equal to it
    const unsigned above = want == 0 ? 0xFFFFFFFFu : exact ? T - 1u : T;
    const bool tied = choose && !exact;
    // ---- per warp and row of kSelThreads positions: keys above (low half), keys equal (high half), kKeys rows at a time
    int total_a = 0, total_e = 0, evicted = n;   // evicted: the first position that goes
    const int rows = (end - at + kSelThreads - 1) / kSelThreads;
    auto count = [&](int i, unsigned o, bool here) {
        const unsigned ba = __ballot_sync(0xFFFFFFFFu, here && o > above), be = __ballot_sync(0xFFFFFFFFu, here && tied && o == above);
        if (lane == 0) s_scan[i * kSelWarps + warp] = __popc(ba) | __popc(be) << 16;
    };
    auto count_block = [&](int i0) {   // (rows that do not exist count nothing)
        if (i0 == 0) {
#pragma unroll
            for (int i = 0; i < kKeys; ++i) count(i, key[i], at + i * kSelThreads + tid < end);
        } else {
#pragma unroll 1
            for (int i = 0; i < kKeys; ++i) {
                const int j = at + (i0 + i) * kSelThreads + tid;
                count(i, j < end ? key_at(j) : 0u, j < end);
            }
        }
    };
    for (int i0 = 0; i0 < rows; i0 += kKeys) {
        count_block(i0);
        __syncthreads();
        int v = 0;
        for (int e = lane; e < kKeys * kSelWarps; e += 32) v += s_scan[e];   // (at most 16384 of each kind)
        v = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)v);
        total_a += v & 0xFFFF;
        total_e += (unsigned)v >> 16;
        if (rows > kKeys) __syncthreads();
    }
    int before_a = 0, before_e = 0, all_a = total_a;
    if constexpr (C > 1) {
        exchange<C>(box, par, rank, make_int4(total_a, total_e, 0, 0));
        all_a = 0;
        for (int k = 0; k < C; ++k) {
            const int4 o = box.box[par ^ 1][k];
            all_a += o.x;
            if (k < rank) {
                before_a += o.x;
                before_e += o.y;
            }
        }
    }
    const int ties = want - all_a;   // of the equal keys
    unsigned *keep = p.keep + (size_t)b * c.capacity;
    auto put = [&](int i, int j, unsigned slot) {
        keep[i] = slot;
        if (p.keep_idx && i < p.keep_stride) p.keep_idx[(size_t)b * p.keep_stride + i] = j;
    };
    for (int i0 = 0; i0 < rows; i0 += kKeys) {
        if (rows > kKeys) {   // (else the counts are still there)
            count_block(i0);
            __syncthreads();
        }
        // an exclusive scan of the counts: every warp for itself, kPart numbers a lane
        constexpr int kPart = kKeys * kSelWarps / 32;
        int mine = 0, part[kPart];
#pragma unroll
        for (int k = 0; k < kPart; ++k) {
            part[k] = mine;
            mine += s_scan[lane * kPart + k];
        }
        int incl = mine;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, incl, s);
            if (lane >= s) incl += v;
        }
        const int excl = incl - mine, block = __shfl_sync(0xFFFFFFFFu, incl, 31);
        // (the number of row i, warp w is the (i * kSelWarps + w)-th: lane 2 i + w / kPart, its (w % kPart)-th)
        int pre = excl;
#pragma unroll
        for (int k = 0; k < kPart; ++k)
            if (k == warp % kPart) pre += part[k];
        auto place = [&](int i, int j, unsigned o, unsigned slot) {
            const bool a = j < end && o > above, e = j < end && tied && o == above;
            const unsigned ba = __ballot_sync(0xFFFFFFFFu, a), be = __ballot_sync(0xFFFFFFFFu, e), lt = (1u << lane) - 1u;
            const int q = __shfl_sync(0xFFFFFFFFu, pre, 2 * i + warp / kPart);
            const int na = before_a + (q & 0xFFFF) + __popc(ba & lt), ne = before_e + (int)((unsigned)q >> 16) + __popc(be & lt);
            if (a || (e && ne < ties)) put(first + na + min(ne, ties), j, slot);
            else if (j < end) evicted = min(evicted, j);
        };
        if (i0 == 0) {
            unsigned slot[kKeys];
#pragma unroll
            for (int i = 0; i < kKeys; ++i) slot[i] = slot_of(c, b, min(at + i * kSelThreads + tid, max(end - 1, 0)));
#pragma unroll
            for (int i = 0; i < kKeys; ++i)
                if (i < rows) place(i, at + i * kSelThreads + tid, key[i], slot[i]);
        } else {
#pragma unroll 1
            for (int i = 0; i < kKeys && i0 + i < rows; ++i) {
                const int j = at + (i0 + i) * kSelThreads + tid;
                place(i, j, j < end ? key_at(j) : 0u, slot_of(c, b, min(j, end - 1)));
            }
        }
        before_a += block & 0xFFFF;
        before_e += (unsigned)block >> 16;
        __syncthreads();
    }
    // ---- the tokens that stay anyway
    if (choose) {
        for (int i = rank * kSelThreads + tid; i < first; i += C * kSelThreads) put(i, i, slot_of(c, b, i));
        for (int i = rank * kSelThreads + tid; i < last; i += C * kSelThreads) put(m - last + i, n - last + i, slot_of(c, b, n - last + i));
    } else {
        for (int i = rank * kSelThreads + tid; i < m; i += C * kSelThreads) put(i, i, slot_of(c, b, i));
    }
    // ---- nothing before the first evicted position moves in place
    if (tid == 0) s_first = n;
    __syncthreads();
    evicted = __reduce_min_sync(0xFFFFFFFFu, evicted);
    if (lane == 0 && evicted < n) atomicMin(&s_first, evicted);
    __syncthreads();
    evicted = s_first;
    exchange<C>(box, par, rank, make_int4(evicted, 0, 0, 0));
    if (rank == 0 && tid == 0) {
        for (int k = 0; k < C; ++k) evicted = min(evicted, box.box[par ^ 1][k].x);
        p.plan[b] = make_int2(m, p.in_place ? min(evicted, m) : 0);
        p.lengths_out[b] = m;
    }
}

constexpr int kMoveThreads = 512, kPer = 8;   // kPer 16-byte chunks of a thread in flight
// gridDim.x CTAs (in place: a cluster) per sequence and `width` columns, a column being one of the 2 kv_heads head_chunks chunks
// of a token's keys and values; the last group of columns: sizes and weights.  A thread has one column of rows `stride` apart.
template <bool kInPlace>
__global__ void __launch_bounds__(kMoveThreads, 2) k_cache_move(CacheEvictParams p, int head_chunks, int width) {
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
    const int stride = kMoveThreads / width, r0 = tid / width, step = stride * kPer, column = blockIdx.y * width + tid % width;
    const int h2 = column / head_chunks, chunk = column - h2 * head_chunks;
    const bool idle = r0 >= stride || h2 >= 2 * c.kv_heads;
    unsigned char *pool = (h2 < c.kv_heads ? c.k : c.v) + chunk * 16;
    const unsigned h = (unsigned)(h2 < c.kv_heads ? h2 : h2 - c.kv_heads);
    auto row = [&](unsigned slot) {
        return pool + (size_t)((((slot >> c.shift) * (unsigned)c.kv_heads + h) << c.shift) + (slot & low)) * head_chunks * 16;
    };
    uint4 v[kPer];
    auto load = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = i0 + r0 + k * stride;
            if (!idle && i < m) v[k] = *reinterpret_cast<const uint4 *>(row(keep[i]));
        }
    };
    auto store = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = i0 + r0 + k * stride;
            if (!idle && i < m) *reinterpret_cast<uint4 *>(row(target(i))) = v[k];
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

template <int C, int kSelThreads>
cudaError_t launch_select(const CacheEvictParams &p, cudaStream_t s) {
    return launch_after(k_cache_select<C, kSelThreads>, dim3(C, (unsigned)p.c.max_batch), kSelThreads, 0, C, s, p);
}

}  // namespace

cudaError_t launch_cache_evict(int dtype, const CacheEvictParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    const int head_chunks = p.c.dim * (dtype == FUSION_BF16 ? 2 : 4) / 16;
    // threads that hold a sequence's keys in registers: few where they do, since every warp more costs instructions (selection of
    // 8 x 577: 1024 threads 16.5 us, 256 threads 9.6), then clusters of up to 8 CTAs (32768: two of 1024 threads 29, four of 512 20)
    const int cap = p.c.capacity, k = kKeys;
    cudaError_t e = cap <= 256 * k    ? launch_select<1, 256>(p, s)
                    : cap <= 512 * k  ? launch_select<1, 512>(p, s)
                    : cap <= 1024 * k ? launch_select<2, 512>(p, s)
                    : cap <= 2048 * k ? launch_select<4, 512>(p, s)
                    : cap <= 4096 * k ? launch_select<8, 512>(p, s)
                                      : launch_select<8, 1024>(p, s);
    if (e != cudaSuccess) return e;
    // Columns of a CTA: a head's, or more where the sequences are too short for a step of kPer rows by all threads (132 x 17 of 16
    // heads of 80 float32: 33 us with one head a CTA), or half of them (not below 128 bytes) where a team in place would leave SMs
    // idle.  Then enough CTAs to fill the GPU a few times, no more than a sequence has steps for.
    const long long most = p.in_place ? p.c.capacity : (long long)p.pages_out << p.c.shift;
    const int columns = 2 * p.c.kv_heads * head_chunks;
    int width = head_chunks;
    while (width < kMoveThreads && width < columns && (long long)(kMoveThreads / width) * kPer > most) width *= 2;
    if (width > columns) width = columns;
    if (width > kMoveThreads) width = kMoveThreads;
    auto groups = [&] { return (columns + width - 1) / width; };
    auto team_of = [&] { return (p.in_place ? 608ll : 2432ll) / ((long long)(groups() + 1) * p.c.max_batch); };
    while (p.in_place && team_of() > 8 && width <= head_chunks && width >= 16 && width % 2 == 0) width /= 2;
    const int step = kMoveThreads / width * kPer;
    const long long steps = (most + step - 1) / step;
    long long team = team_of();
    if (team > steps) team = steps;
    if (p.in_place) team = team >= 8 ? 8 : team >= 4 ? 4 : team >= 2 ? 2 : 1;
    if (team < 1) team = 1;
    const dim3 grid((unsigned)team, (unsigned)(groups() + 1), (unsigned)p.c.max_batch);
    return p.in_place ? launch_after(k_cache_move<true>, grid, kMoveThreads, 0, (int)team, s, p, head_chunks, width)
                      : launch_after(k_cache_move<false>, grid, kMoveThreads, 0, 1, s, p, head_chunks, width);
}

}  // namespace fz
