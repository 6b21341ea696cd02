// What the attention kernels over the paged cache share: the batch cut into rounds of equal runs per CTA, the tokens of a
// round on their way into shared memory, and the join of runs that share a (sequence, key head).
#pragma once

#include <atomic>

#include "cache.cuh"

namespace fz {
namespace rounds {

constexpr int kMinRounds = 2;       // of a CTA: fewer and the join costs more than the split gains
constexpr int kAloneMost = 128, kAloneLeast = 256;   // visible tokens at most, (sequence, key head)s at least
constexpr float kLow = -3.0e38f;    // a maximum over nothing: finite, so that (-inf) - kLow is -inf
// Probabilities are 2^(x - shift) with a shift of at least the largest logit so far less kLag: up to 2^8, which costs no bits in
// float32 or bf16, and tiles whose maximum grows a little do not rescale (with 16 heads in a warp nearly every tile does).
constexpr float kLag = 8.0f;
constexpr float kNoPage = 3.0e38f;  // in the place of a log2 size (at most 128): the token's page id is out of range

__device__ __forceinline__ float ex2(float x) {   // 2^x, one MUFU instruction (2^-inf = 0)
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Log-sum-exp of a row (base 2) for the weights, of its maximum and sum.  No token with a part: +inf, so that 2^(x - lse) is 0 for
// logits of -inf.  Sum below zero, a bad page: kRefused, which no row has otherwise, and the same in all rows of the sequence.
constexpr float kRefused = -INFINITY;
__device__ __forceinline__ float log_sum(float maximum, float sum) {
    return sum < 0.0f ? kRefused : sum == 0.0f ? INFINITY : maximum + log2f(sum);
}
__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void *src, bool read) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(read ? 16 : 0) : "memory");
}
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where in the batch a round lies.
struct Place {
    int b, h, ch, u;       // sequence, key head, chunk of its query heads, round
    int n, vis, rounds;    // length, visible tokens, rounds of one key head
};
template <bool kEarly = false>
__device__ __forceinline__ void place_sequence(const CacheAttnParams &p, Place &s, int tokens, int b) {
    s.b = b;
    s.n = max(cache_length<kEarly>(p.c, b), 0);
    s.vis = visible(p, s.n);
    s.rounds = (s.vis + tokens - 1) / tokens;
}
template <bool kEarly = false>
__device__ __forceinline__ void place_next(const CacheAttnParams &p, Place &s, int tokens, int heads, int chunks) {
    if (++s.u < s.rounds) return;
    s.u = 0;
    if (++s.ch < chunks) return;
    s.ch = 0;
    if (++s.h < heads) return;
    s.h = 0;
    do {
        if (++s.b >= p.c.max_batch) {
            s.rounds = s.vis = 0;
            return;
        }
        place_sequence<kEarly>(p, s, tokens, s.b);
    } while (s.rounds == 0);
}

// The batch's rounds in `ctas` runs: the first `more` of len + 1 rounds, the others of len.  A boundary at most `snap` rounds
// inside a (sequence, key head) moves to its nearer end (its beginning first): a join costs more time than the few rounds that
// it would deal out.  (Rounds are counted in 32 bits: counts_fit.)
struct Run {
    unsigned total, len, more;
    unsigned r0, r1;   // this CTA's
    int ctas, snap;
    __device__ __forceinline__ void cut(unsigned rounds, int n) {
        total = rounds;
        ctas = n;
        len = total / (unsigned)n;
        more = total - len * (unsigned)n;
        r0 = begin(blockIdx.x);
        r1 = begin(blockIdx.x + 1);
        snap = len > 4 ? 4 : (int)len - 1;
    }
    __device__ __forceinline__ unsigned begin(unsigned k) const { return len * k + min(k, more); }
    __device__ __forceinline__ int of(unsigned x) const {   // the last run that begins at round x or before, boundaries not moved
        const unsigned big = more * (len + 1);
        return (int)(x < big ? x / (len + 1) : more + (x - big) / len);
    }
    // by how much a boundary moves that lies u rounds inside a (sequence, key head) of n rounds
    __device__ __forceinline__ int move(int u, int n) const { return u <= snap ? -u : n - u <= snap ? n - u : 0; }
    // the runs that share the (sequence, key head) of rounds [s0, s1): the first of them, and their number
    __device__ __forceinline__ int sharing(unsigned s0, unsigned s1, int &first) const {
        const int k0 = of(s0 + snap) + 1, k1 = of(s1 - snap - 1);   // the boundaries inside
        first = k0 - 1;
        return k1 - k0 + 2;
    }
};

// What a CTA needs to find its run.
template <int THREADS>
struct Finder {
    unsigned sums[THREADS / 32];   // rounds of the warps' sequences
    Place at[2];                   // of the run's first round and of the next run's
};
// This CTA's run and the place where it begins; false: it has none.  Every thread counts the rounds of a few sequences, the
// warps' sums go through shared memory, and the thread whose sequences hold a boundary looks it up (one barrier before and
// one after: 2.2 us with 64-bit scans by one thread, 1.2 now, 0.7 of them the reading of the lengths).  min_rounds: of a run.
// SNAP: the boundaries move to ends of (sequence, key head)s.  kEarly: called before the kernel's wait.
template <int THREADS, bool SNAP, bool kEarly>
__device__ __forceinline__ bool find_run(const CacheAttnParams &p, Finder<THREADS> &s, int tokens, int heads, int chunks, unsigned min_rounds,
                                         Run &run, Place &at) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned vheads = (unsigned)(heads * chunks);
    const int per = ceil_div(p.c.max_batch, THREADS), b0 = min(tid * per, p.c.max_batch), b1 = min(b0 + per, p.c.max_batch);
    unsigned mine = 0;
    for (int b = b0; b < b1; ++b) {
        place_sequence<kEarly>(p, at, tokens, b);
        mine += (unsigned)at.rounds * vheads;
    }
    const unsigned sum = __reduce_add_sync(0xFFFFFFFFu, mine);
    if (lane == 0) s.sums[warp] = sum;
    if (tid < 2) s.at[tid] = Place{};
    __syncthreads();
    unsigned total = 0, base = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const unsigned v = s.sums[w];
        total += v;
        if (w < warp) base += v;
    }
    const unsigned most = (total + min_rounds - 1) / min_rounds;
    const int ctas = (int)min(most, gridDim.x);
    if ((int)blockIdx.x >= ctas) return false;
    run.cut(total, ctas);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const unsigned x = k ? run.r1 : run.r0;
        if (x < base || x >= base + sum) continue;   // (warp-uniform)
        unsigned incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += v;
        }
        unsigned rem = x - base - (incl - mine);   // rounds of this thread's sequences before x (if it is one of theirs)
        if (x - base >= incl - mine && rem < mine) {
            for (int b = b0; b < b1; ++b) {
                if (per > 1) place_sequence<kEarly>(p, at, tokens, b);
                if (rem < (unsigned)at.rounds * vheads) break;
                rem -= (unsigned)at.rounds * vheads;
            }
            const unsigned vh = at.rounds > 0 ? rem / (unsigned)at.rounds : 0u;
            at.u = (int)(rem - vh * (unsigned)at.rounds);
            at.h = chunks == 1 ? (int)vh : (int)vh / chunks;
            at.ch = (int)vh - at.h * chunks;
            s.at[k] = at;
        }
    }
    __syncthreads();
    at = s.at[0];
    if (SNAP) {
        const int moved = run.move(at.u, at.rounds);
        if (run.r1 < total) run.r1 += run.move(s.at[1].u, s.at[1].rounds);
        run.r0 += moved;
        if (run.r0 >= run.r1) return false;
        if (moved < 0) at.u = 0;
        if (moved > 0) {
            at.u = at.rounds - 1;
            place_next<kEarly>(p, at, tokens, heads, chunks);
        }
    }
    return true;
}

// A token that a warp will load: its page (from the table, a round before its size) and place in it.
struct Token {
    unsigned page;
    int place;       // -1: no token here
    int h;
};

// Tokens of the rounds to come, a warp's share of TT per round: the page is read two rounds before the token's rows are
// asked for, the size one round before.  Rows without a token, or of size zero, arrive as zeros and weigh nothing (log2
// size -inf), whatever the cache holds there.
template <typename T, int DP, int TT, int W>
struct Stream {
    static constexpr int kRow = DP * (int)sizeof(T), kCpr = kRow / 16, kStage = 2 * TT * kRow, kRound = W * TT;
    Place ahead;             // of the next token to look up
    unsigned ahead_r, r1;
    Token t0, t1;            // t0's rows are asked for next (its size is here), then t1's
    float size0;

    __device__ __forceinline__ Token look_up(const CacheAttnParams &p, int chunks, int warp, int lane) {
        Token t{0u, -1, ahead.h};
        if (ahead_r < r1) {
            const int j = ahead.u * kRound + warp * TT + lane;
            if (lane < TT && j < ahead.vis) {
                const int pos = p.window && j >= p.sinks ? j + ahead.n - ahead.vis : j;
                t.place = cache_page(p.c, ahead.b, pos, t.page) ? pos & ((1 << p.c.shift) - 1) : -2;
            }
            ++ahead_r;
            place_next(p, ahead, kRound, p.c.kv_heads, chunks);
        }
        return t;
    }
    __device__ __forceinline__ float size_of(const CacheAttnParams &p, const Token &t) const {
        return t.place < 0 ? 0.0f : p.c.sizes ? p.c.sizes[((size_t)t.page << p.c.shift) + t.place] : 1.0f;
    }
    // Asks for a token's rows (K, then V, rows of kRow bytes with chunk c of row r at c ^ swizzle(r)).  swizzle is linear in the
    // bits of r, and a lane has the same chunk in every step, so a step costs one address for each pool and one exclusive or.
    template <typename Swizzle>
    __device__ __forceinline__ void ask(const CacheAttnParams &p, const Token &t, float size, int lane, unsigned char *stage, float *lsz,
                                        Swizzle swizzle) {
        const bool live = t.place >= 0 && size != 0.0f;
        const unsigned row = live ? ((t.page * (unsigned)p.c.kv_heads + (unsigned)t.h) << p.c.shift) + (unsigned)t.place : 0u;
        const unsigned lives = __ballot_sync(0xFFFFFFFFu, live), row_bytes = (unsigned)p.c.dim * (unsigned)sizeof(T);
        if (lane < TT) lsz[lane] = t.place == -2 ? kNoPage : live ? log2f(size) : -INFINITY;
        constexpr int kWide = kCpr < 32 ? 32 / kCpr : 1, kParts = kCpr > 32 ? kCpr / 32 : 1;   // rows of a step, steps of a row
        const int r_lane = lane / (32 / kWide);
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            const int cc = lane % (32 / kWide) + part * 32;
            const bool exists = (unsigned)cc * 16u < row_bytes;
            const unsigned mine = exists ? lives >> r_lane : 0u;
            const unsigned char *k = p.c.k + (exists ? cc : 0) * 16, *v = p.c.v + (exists ? cc : 0) * 16;
            const uint32_t dst = smem_addr(stage) + r_lane * kRow, at = (uint32_t)(cc ^ swizzle(r_lane)) * 16u;
#pragma unroll
            for (int e = 0; e < TT / kWide; ++e) {
                const size_t off = (size_t)__shfl_sync(0xFFFFFFFFu, row, e * kWide + r_lane) * row_bytes;
                const bool read = mine >> (e * kWide) & 1u;
                const uint32_t to = dst + e * kWide * kRow + (at ^ (uint32_t)(swizzle(e * kWide) * 16));
                cp_async16_zfill(to, k + off, read);
                cp_async16_zfill(to + TT * kRow, v + off, read);
            }
        }
        cp_async_commit();
    }
    // The next round's rows into `stage`.
    template <typename Swizzle>
    __device__ __forceinline__ void next(const CacheAttnParams &p, int chunks, int warp, int lane, unsigned char *stage, float *lsz, Swizzle swizzle) {
        ask(p, t0, size0, lane, stage, lsz, swizzle);
        t0 = t1;
        size0 = size_of(p, t0);
        t1 = look_up(p, chunks, warp, lane);
    }
    // The first S - 1 rounds' rows (all pages asked for at once, then all sizes).
    template <int S, typename Swizzle>
    __device__ __forceinline__ void begin(const CacheAttnParams &p, const Place &at, const Run &run, int chunks, int warp, int lane,
                                          unsigned char *stages, float *lsz, Swizzle swizzle) {
        ahead = at;
        ahead_r = run.r0;
        r1 = run.r1;
        Token t[S + 1];
        float size[S];
#pragma unroll
        for (int s = 0; s <= S; ++s) t[s] = look_up(p, chunks, warp, lane);
#pragma unroll
        for (int s = 0; s < S; ++s) size[s] = size_of(p, t[s]);
#pragma unroll
        for (int s = 0; s < S - 1; ++s) ask(p, t[s], size[s], lane, stages + s * kStage, lsz + s * TT, swizzle);
        t0 = t[S - 1];
        size0 = size[S - 1];
        t1 = t[S];
    }
};

// Zeros for sequences without tokens (a length out of range is told, its row left), dealt out over the grid.
template <typename T, int THREADS>
__device__ __forceinline__ void empty_sequences(const CacheAttnParams &p) {
    const int row = p.heads * p.c.dim * (int)sizeof(T) / 16, grid = (int)gridDim.x, lane = threadIdx.x & 31;
    for (long long b0 = blockIdx.x + (long long)(threadIdx.x >> 5) * 32 * grid; b0 < p.c.max_batch; b0 += (long long)THREADS * grid) {
        const long long b = b0 + (long long)lane * grid;   // a warp looks at 32 sequences at once
        const int n = b < p.c.max_batch ? cache_length(p.c, (int)b) : 1;
        if (n < 0) raise_status(p.status, FUSION_DEV_BAD_CACHE);
        for (unsigned none = __ballot_sync(0xFFFFFFFFu, n == 0); none; none &= none - 1u) {
            uint4 *o = reinterpret_cast<uint4 *>(p.out) + (size_t)(b0 + (long long)(__ffs(none) - 1) * grid) * row;
            for (int e = lane; e < row; e += 32) o[e] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// ---- the join of the runs that share a (sequence, key head) ------------------------------------------------------------
// Run k's result lies in slot 2 k + 1 where the (sequence, key head) begins in run k, else in slot 2 k: per query head a maximum
// and a sum (below zero: a bad page) and the output before the division.
constexpr int kJoinAtOnce = 16;     // in one step; more in two
constexpr int kJoinMost = 23;       // results joined at once: 23 * 23 covers kCacheMaxWide, and the rounds that short sequences have
template <int NQ> constexpr int kJoinScratch = (kJoinMost + 2) * NQ * 4;   // bytes

template <typename T> __device__ __forceinline__ void store4(T *dst, float4 v);
template <> __device__ __forceinline__ void store4<float>(float *dst, float4 v) { *reinterpret_cast<float4 *>(dst) = v; }
template <> __device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *dst, float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(dst) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

// Joins the results of runs k0, k0 + step, ... (n of them, n <= kJoinMost) in this order, into the output or into the first one's
// slot.  scratch: kJoinScratch<NQ> bytes of shared memory.
template <typename T, int NQ, int THREADS>
__device__ __forceinline__ void join_results(const CacheAttnParams &p, int c0, int k0, int step, int n, bool last, size_t head, int nq,
                                             float *scratch) {
    const int tid = threadIdx.x, dim = p.c.dim;
    float *weight = scratch, *sums = scratch + kJoinMost * NQ, *maxima = sums + NQ;
    auto slot = [&](int j) { return (size_t)2 * (k0 + j * step) + (k0 + j * step == c0); };
    if (tid < nq) {
        float2 ml[kJoinMost];
        float M = kLow, l = 0.0f;
        bool none = false;
#pragma unroll
        for (int j = 0; j < kJoinMost; ++j) ml[j] = j < n ? __ldcg(&p.part_ml[slot(j) * NQ + tid]) : make_float2(kLow, 0.0f);
#pragma unroll
        for (int j = 0; j < kJoinMost; ++j) {
            M = fmaxf(M, ml[j].x);
            none |= ml[j].y < 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kJoinMost; ++j)
            if (j < n) {
                const float f = ex2(ml[j].x - M);
                weight[j * NQ + tid] = f;
                l += ml[j].y * f;
            }
        sums[tid] = none ? -1.0f : l;
        maxima[tid] = none ? INFINITY : M;
    }
    __syncthreads();
    constexpr int kU = 4;   // columns of four in flight, for four results at a time
    const int all = nq * dim / 4;
    for (int e0 = tid; e0 < all; e0 += kU * THREADS) {
        float4 acc[kU];
        int q[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            acc[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            q[u] = min(e0 + u * THREADS, all - 1) * 4 / dim;
        }
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
            const float4 *src = reinterpret_cast<const float4 *>(p.part + slot(j) * NQ * dim);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const float4 v = __ldcg(src + min(e0 + u * THREADS, all - 1));
                const float f = weight[j * NQ + q[u]];
                acc[u] = make_float4(fmaf(v.x, f, acc[u].x), fmaf(v.y, f, acc[u].y), fmaf(v.z, f, acc[u].z), fmaf(v.w, f, acc[u].w));
            }
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int e = e0 + u * THREADS;
            if (e >= all) break;
            if (!last) {
                *reinterpret_cast<float4 *>(p.part + slot(0) * NQ * dim + (size_t)e * 4) = acc[u];
            } else if (sums[q[u]] >= 0.0f || sums[q[u]] != sums[q[u]]) {
                const float inv = 1.0f / sums[q[u]];
                store4(reinterpret_cast<T *>(p.out) + head * dim + (size_t)e * 4,
                       sums[q[u]] == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f)
                                          : make_float4(acc[u].x * inv, acc[u].y * inv, acc[u].z * inv, acc[u].w * inv));
            }
        }
    }
    if (tid < nq) {
        const float l = sums[tid];
        if (!last) p.part_ml[slot(0) * NQ + tid] = make_float2(maxima[tid], l);
        else if (p.logits) p.lse[head + tid] = log_sum(maxima[tid], l);
    }
}

// Whether this CTA is the last of n to come here (its writes before are seen by the last one).
__device__ __forceinline__ bool arrive_last(int *counter, int n, int &s_last) {
    __syncthreads();   // the CTA's writes come before thread 0's release, which passes them on
    if (threadIdx.x == 0) {
        int before;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
        s_last = before == n - 1;
        if (s_last) *counter = 0;
    }
    __syncthreads();
    return s_last;
}

// After a CTA has written its result of the (sequence, key head) of rounds [seg0, seg1): the last of the runs that share it
// joins their results.  More than kJoinAtOnce are joined in two steps, groups of about the square root of their number first,
// by the group's last: one CTA alone reads the results of 38 runs of 16 heads of 128 (300 KB) slower than two in turn a few each.
template <typename T, int NQ, int THREADS>
__device__ __forceinline__ void join_runs(const CacheAttnParams &p, const Run &run, unsigned seg0, unsigned seg1, size_t head, int nq,
                                          float *scratch, int &s_last) {
    int c0;
    const int n = run.sharing(seg0, seg1, c0);
    int size = n;   // of a group
    if (n > kJoinAtOnce)
        for (size = 3; size * size < n;) ++size;
    const int groups = (n + size - 1) / size, g = ((int)blockIdx.x - c0) / size, first = c0 + g * size, members = min(size, n - g * size);
    int *count1 = p.counters, *count2 = p.counters + 2 * kCacheMaxCtas;   // both by the slot of the first run
    if (members > 1 || groups == 1) {
        if (!arrive_last(&count1[2 * first + (first == c0)], members, s_last)) return;
        join_results<T, NQ, THREADS>(p, c0, first, 1, members, groups == 1, head, nq, scratch);
    }
    if (groups == 1) return;
    if (!arrive_last(&count2[2 * c0 + 1], groups, s_last)) return;
    join_results<T, NQ, THREADS>(p, c0, c0, size, groups, true, head, nq, scratch);
}

// Whether warps work alone (W = 1, CTAs of one warp) instead of four together.  Alone a warp needs no barrier, and sequences of
// a round or two leave no warp of a CTA idle (alone and together: 200 x 60 tokens of 8 heads 10.6 and 14.9 us, 181 x 87 of 16 heads
// 33.3 and 38.9); together they share longer ones (60 x 200 of 8 heads 16.8 and 13.8, 64 x 250 19.4 and 17.4).
inline bool warps_alone(const CacheAttnParams &p, int chunks) {
    return p.c.dim <= 128 && p.most <= kAloneMost && (long long)p.c.max_batch * p.c.kv_heads * chunks >= kAloneLeast;
}

// Whether the rounds of any batch that the host lets pass, of TT tokens for each of W warps, are fewer than 2^32.  A (sequence, part
// of a key head's query heads) has at most its places / round + 1 of them, and there are at most max_batch * heads; warps alone (TT
// down to 8) take calls of at most kAloneMost visible tokens only.
constexpr bool counts_fit(long long tt, long long w) {
    constexpr long long kHeads = (long long)FUSION_CACHE_MAX_BATCH * FUSION_CACHE_MAX_HEADS;
    return (w == 1 ? kHeads * ((kAloneMost + tt - 1) / tt) : kCacheMaxHeadTokens / (tt * w) + kHeads) < 1ll << 32;
}

// Host: as many CTAs as the GPU holds at once, or as there can be rounds.  What depends on the kernel and the device alone is
// asked once (asking costs the host 4 us a call).
template <auto Kernel, int THREADS>
cudaError_t resident_ctas(int smem, int &ctas) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    ctas = dev < kDevices ? known[dev].load(std::memory_order_acquire) : 0;
    if (ctas > 0) return cudaSuccess;
    int sms = 0, occ = 0;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, Kernel, THREADS, smem);
    if (e != cudaSuccess) return e;
    ctas = sms * (occ < 1 ? 1 : occ);
    if (dev < kDevices) known[dev].store(ctas, std::memory_order_release);
    return cudaSuccess;
}
template <auto Kernel, int W>
cudaError_t launch_rounds(int smem, const CacheAttnParams &p, int chunks, int tokens, cudaStream_t s) {
    int ctas = 0;
    const cudaError_t e = resident_ctas<Kernel, 32 * W>(smem, ctas);
    if (e != cudaSuccess) return e;
    const long long rounds = (long long)p.c.max_batch * p.c.kv_heads * chunks * ceil_div(p.most, tokens);
    constexpr int kMost = W == 1 ? kCacheMaxCtas : kCacheMaxWide;
    if (ctas > kMost) ctas = kMost;
    return launch_after(Kernel, dim3((unsigned)(ctas < rounds ? ctas : rounds)), 32 * W, (size_t)smem, 1, s, p, chunks);
}

}  // namespace rounds
}  // namespace fz
