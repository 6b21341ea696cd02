// Eviction from the paged cache by accumulated attention weight.  A sequence of n tokens keeps m = min(budget, n): its
// first s = min(sinks, m), its last r = min(recent, m - s), and of the ones between the m - s - r of largest weight (ties:
// lowest position).  Kept rows move, in ascending position, to positions 0 .. m - 1.
//
// k_cache_select, a CTA (or a cluster of them, for long sequences) per sequence: the ordered keys of the weights stay in
// registers, and the smallest kept key T is the largest T of which count(key >= T) is still the number wanted, two bits per
// step (three counts, one barrier).  Counting costs the same whatever the weights are; a histogram's atomics meet in a few
// bins, since attention weights share a few exponents (8 bits per pass: 43 us for 32 sequences of up to 8192, 103 us for one of
// 32768).  One scan over the counts of all warps then places the kept tokens.
//
// k_cache_move copies the rows.  Into other pages: any CTA any rows.  In place: a team of CTAs (a cluster) per (sequence, key
// head, K or V) takes the rows in ascending position, a step of them at a time, all read before any is written.  That is safe
// without a copy aside: position i receives a row from a position >= i, so no target of a step is read by a later step, and
// the next step's rows are read while the team waits.
#include "cache.cuh"

namespace fz {
namespace {

constexpr int kSelThreads = 1024, kSelWarps = kSelThreads / 32, kKeys = 16;   // keys of a thread in registers

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

// C: CTAs of a sequence; each takes a run of the positions that are compared.
template <int C>
__global__ void __launch_bounds__(kSelThreads) k_cache_select(CacheEvictParams p) {
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = C == 1 ? 0 : (int)cluster_rank();
    const Cache &c = p.c;
    __shared__ Exchange box;
    __shared__ int3 s_cnt[2][kSelWarps];
    __shared__ int s_scan[kKeys * kSelWarps];
    __shared__ int s_first;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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
    if (!wrong) {
        const int pages_n = (n + (1 << c.shift) - 1) >> c.shift, pages_m = (m + (1 << c.shift) - 1) >> c.shift;
        wrong = pages_m > p.pages_out;
        for (int e = tid; e < pages_n; e += kSelThreads) wrong |= (unsigned)c.table[(size_t)b * c.max_pages + e] >= c.num_pages;
        if (!p.in_place)
            for (int e = tid; e < min(pages_m, p.pages_out); e += kSelThreads)
                wrong |= (unsigned)p.table_out[(size_t)b * p.pages_out + e] >= c.num_pages;
    }
    wrong = __syncthreads_or(wrong);
    unsigned key[kKeys];
    if (!wrong) {
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
            const int j = at + i * kSelThreads + tid;
            float w = 0.0f;
            if (j < end) w = c.weights[slot_of(c, b, j)];
            nan |= !isfinite(w);
            key[i] = j < end ? ordered_bits(w) : 0u;   // (no finite weight has the key 0)
        }
        for (int j = at + kKeys * kSelThreads + tid; j < end; j += kSelThreads) nan |= !isfinite(c.weights[slot_of(c, b, j)]);
    }
    {
        const int any = __syncthreads_or(nan);
        exchange<C>(box, par, rank, make_int4(any, wrong, 0, 0));
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

    // ---- T: the largest with count(key >= T) >= want
    unsigned T = 0;
    bool exact = false;   // count(key >= T) == want: no ties to break
    int flip = 0;
    if (choose && want > 0) {
        for (int shift = 30; shift >= 0 && !exact; shift -= 2) {
            const unsigned t1 = T | 1u << shift, t2 = T | 2u << shift, t3 = T | 3u << shift;
            int n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
            for (int i = 0; i < kKeys; ++i) {
                if (at + i * kSelThreads >= end) break;
                n1 += key[i] >= t1;
                n2 += key[i] >= t2;
                n3 += key[i] >= t3;
            }
            for (int j = at + kKeys * kSelThreads + tid; j < end; j += kSelThreads) {
                const unsigned o = key_at(j);
                n1 += o >= t1;
                n2 += o >= t2;
                n3 += o >= t3;
            }
            n1 = __reduce_add_sync(0xFFFFFFFFu, n1);
            n2 = __reduce_add_sync(0xFFFFFFFFu, n2);
            n3 = __reduce_add_sync(0xFFFFFFFFu, n3);
            if (lane == 0) s_cnt[flip][warp] = make_int3(n1, n2, n3);
            __syncthreads();
            const int3 v = s_cnt[flip][lane];
            flip ^= 1;
            n1 = __reduce_add_sync(0xFFFFFFFFu, v.x);
            n2 = __reduce_add_sync(0xFFFFFFFFu, v.y);
            n3 = __reduce_add_sync(0xFFFFFFFFu, v.z);
            if constexpr (C > 1) {
                exchange<C>(box, par, rank, make_int4(n1, n2, n3, 0));
                n1 = n2 = n3 = 0;
                for (int k = 0; k < C; ++k) {
                    const int4 o = box.box[par ^ 1][k];
                    n1 += o.x;
                    n2 += o.y;
                    n3 += o.z;
                }
            }
            const int got = n3 >= want ? n3 : n2 >= want ? n2 : n1;
            T = n3 >= want ? t3 : n2 >= want ? t2 : n1 >= want ? t1 : T;
            exact = got == want;
        }
    }
    // kept: keys above the threshold, and the first `ties` of those equal to it
    const unsigned above = want == 0 ? 0xFFFFFFFFu : exact ? T - 1u : T;
    // ---- per warp and row of kSelThreads positions: keys above (low half), keys equal (high half); then a scan in order
    int total_a = 0, total_e = 0, evicted = n;   // evicted: the first position that goes
    const int rows = (end - at + kSelThreads - 1) / kSelThreads;
    auto key_of = [&](int i, int j) {   // beyond the registers: read again
        unsigned o = 0u;
        if (i < kKeys) {
#pragma unroll
            for (int k = 0; k < kKeys; ++k)
                if (k == i) o = key[k];
        } else if (j < end) {
            o = key_at(j);
        }
        return o;
    };
    // the kept tokens' slots; row blocks of kKeys rows, whose counts fit in shared memory; two passes where the ties' number
    // or the other CTAs' counts have to be known first
    auto count_block = [&](int i0) {
#pragma unroll 1
        for (int i = i0; i < min(rows, i0 + kKeys); ++i) {
            const unsigned o = key_of(i, at + i * kSelThreads + tid);
            const bool here = at + i * kSelThreads + tid < end;
            const unsigned ba = __ballot_sync(0xFFFFFFFFu, here && o > above), be = __ballot_sync(0xFFFFFFFFu, here && !exact && want > 0 && o == above);
            if (lane == 0) s_scan[(i - i0) * kSelWarps + warp] = __popc(ba) | __popc(be) << 16;
        }
        if (i0 + kKeys > rows)   // rows that do not exist
            for (int i = max(rows - i0, 0); i < kKeys; ++i)
                if (lane == 0) s_scan[i * kSelWarps + warp] = 0;
    };
    for (int i0 = 0; i0 < rows; i0 += kKeys) {
        count_block(i0);
        __syncthreads();
        int v = 0;
        for (int e = lane; e < kKeys * kSelWarps; e += 32) v += s_scan[e];   // (at most 16384 of each kind)
        v = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)v);
        total_a += v & 0xFFFF;
        total_e += (unsigned)v >> 16;
        __syncthreads();
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
    auto put = [&](int i, int j) {
        keep[i] = slot_of(c, b, j);
        if (p.keep_idx && i < p.keep_stride) p.keep_idx[(size_t)b * p.keep_stride + i] = j;
    };
    for (int i0 = 0; i0 < rows; i0 += kKeys) {
        if (rows > kKeys) {   // (else the counts are still there)
            count_block(i0);
            __syncthreads();
        }
        // an exclusive scan of the counts: every warp for itself, 16 numbers a lane
        int mine = 0, part[kKeys];
#pragma unroll
        for (int k = 0; k < kKeys; ++k) {
            part[k] = mine;
            mine += s_scan[lane * kKeys + k];
        }
        int incl = mine;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, incl, s);
            if (lane >= s) incl += v;
        }
        const int excl = incl - mine, block = __shfl_sync(0xFFFFFFFFu, incl, 31);
        // (the number of row i, warp w is the (i * kSelWarps + w)-th: lane 2 i + w / 16, its (w % 16)-th)
        int pre = excl;
#pragma unroll
        for (int k = 0; k < kKeys; ++k)
            if (k == (warp & 15)) pre += part[k];
#pragma unroll 1
        for (int i = i0; i < min(rows, i0 + kKeys); ++i) {
            const int j = at + i * kSelThreads + tid;
            const unsigned o = key_of(i, j);
            const bool a = j < end && o > above, e = j < end && !exact && want > 0 && o == above;
            const unsigned ba = __ballot_sync(0xFFFFFFFFu, a), be = __ballot_sync(0xFFFFFFFFu, e), lt = (1u << lane) - 1u;
            const int q = __shfl_sync(0xFFFFFFFFu, pre, 2 * (i - i0) + (warp >> 4));
            const int na = before_a + (q & 0xFFFF) + __popc(ba & lt), ne = before_e + ((unsigned)q >> 16) + __popc(be & lt);
            if (a || (e && ne < ties)) put(first + na + min(ne, ties), j);
            else if (j < end) evicted = min(evicted, j);
        }
        before_a += block & 0xFFFF;
        before_e += (unsigned)block >> 16;
        __syncthreads();
    }
    // ---- the tokens that stay anyway
    if (choose) {
        for (int i = rank * kSelThreads + tid; i < first; i += C * kSelThreads) put(i, i);
        for (int i = rank * kSelThreads + tid; i < last; i += C * kSelThreads) put(m - last + i, n - last + i);
    } else {
        for (int i = rank * kSelThreads + tid; i < m; i += C * kSelThreads) put(i, i);
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
// gridDim.x CTAs per (sequence, key head, K or V; the last job: sizes and weights); in place they are a cluster.
template <bool kInPlace>
__global__ void __launch_bounds__(kMoveThreads, 2) k_cache_move(CacheEvictParams p, int head_chunks) {
    const int b = blockIdx.z, job = blockIdx.y, tid = threadIdx.x, team = gridDim.x, member = blockIdx.x;
    const Cache &c = p.c;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int2 plan = p.plan[b];
    const int m = plan.x;
    const unsigned *keep = p.keep + (size_t)b * c.capacity;
    const unsigned low = (1u << c.shift) - 1u;
    auto target = [&](int i) {
        const unsigned page = (unsigned)p.table_out[(size_t)b * p.pages_out + (i >> c.shift)];
        return (page << c.shift) + ((unsigned)i & low);
    };
    if (job == 2 * c.kv_heads) {   // sizes and weights
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
    unsigned char *pool = job < c.kv_heads ? c.k : c.v;
    const unsigned h = (unsigned)(job < c.kv_heads ? job : job - c.kv_heads);
    auto row = [&](unsigned slot) {
        return pool + (size_t)((((slot >> c.shift) * (unsigned)c.kv_heads + h) << c.shift) + (slot & low)) * head_chunks * 16;
    };
    // rows of a step: as many whole rows as the CTA's chunks give; a thread has the same chunk of rows `stride` apart
    const int stride = kMoveThreads / head_chunks, chunk = tid % head_chunks, r0 = tid / head_chunks, step = stride * kPer;
    const bool idle = r0 >= stride;
    uint4 v[kPer];
    auto load = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = i0 + r0 + k * stride;
            if (!idle && i < m) v[k] = *reinterpret_cast<const uint4 *>(row(keep[i]) + chunk * 16);
        }
    };
    auto store = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = i0 + r0 + k * stride;
            if (!idle && i < m) *reinterpret_cast<uint4 *>(row(target(i)) + chunk * 16) = v[k];
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

template <int C>
cudaError_t launch_select(const CacheEvictParams &p, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(C, (unsigned)p.c.max_batch);
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = s;
    cudaLaunchAttribute a[1];
    a[0].id = cudaLaunchAttributeClusterDimension;
    a[0].val.clusterDim = {C, 1, 1};
    cfg.attrs = a;
    cfg.numAttrs = C > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_cache_select<C>, p);
}

}  // namespace

cudaError_t launch_cache_evict(int dtype, const CacheEvictParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    const int head_chunks = p.c.dim * (dtype == FUSION_BF16 ? 2 : 4) / 16;
    // as many CTAs as hold a sequence's keys in registers, up to 8
    const int need = ceil_div(p.c.capacity, kKeys * kSelThreads);
    cudaError_t e = need <= 1 ? launch_select<1>(p, s) : need <= 2 ? launch_select<2>(p, s) : need <= 4 ? launch_select<4>(p, s) : launch_select<8>(p, s);
    if (e != cudaSuccess) return e;
    // a team per (sequence, job): enough CTAs to fill the GPU a few times, no more than a sequence has steps for
    const int jobs = 2 * p.c.kv_heads + 1, step = kMoveThreads / head_chunks * kPer;
    const long long most = p.in_place ? p.c.capacity : (long long)p.pages_out << p.c.shift;
    long long team = (p.in_place ? 608ll : 2432ll) / ((long long)jobs * p.c.max_batch);
    const long long steps = (most + step - 1) / step;
    if (team > steps) team = steps;
    if (p.in_place) team = team >= 8 ? 8 : team >= 4 ? 4 : team >= 2 ? 2 : 1;
    if (team < 1) team = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)team, (unsigned)jobs, (unsigned)p.c.max_batch);
    cfg.blockDim = dim3(kMoveThreads);
    cfg.stream = s;
    cudaLaunchAttribute a[2];
    a[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a[0].val.programmaticStreamSerializationAllowed = 1;
    a[1].id = cudaLaunchAttributeClusterDimension;
    a[1].val.clusterDim = {(unsigned)team, 1, 1};
    cfg.attrs = a;
    cfg.numAttrs = p.in_place ? 2 : 1;
    return p.in_place ? cudaLaunchKernelEx(&cfg, k_cache_move<true>, p, head_chunks) : cudaLaunchKernelEx(&cfg, k_cache_move<false>, p, head_chunks);
}

}  // namespace fz
