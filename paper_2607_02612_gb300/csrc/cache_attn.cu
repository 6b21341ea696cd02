// Attention of one new token per sequence over the paged cache, and the accumulated attention weights.  For sequence
// b, query head a of key head h and the visible tokens j (the first `sinks` and the last `window`; all without a
// window), in base 2:
//   x_aj = scale2 q_a . k_hj + log2 s_j,   out_a = sum_j 2^(x_aj - m) v_hj / sum_j 2^(x_aj - m),   m = max_j x_aj,
//   weights_j += sum_a 2^(x_aj - lse_a),   lse_a = m + log2 sum_j 2^(x_aj - m).
//
// Work is cut into rounds: the next kWarps * TT visible tokens of one (sequence, key head).  Every CTA takes an equal
// run of the rounds of the whole batch, in the order (sequence, key head, token), whatever the sequences' lengths; a
// warp takes TT tokens of each round through stages of its own (cp.async) and keeps its own running maximum, sum and
// output.  Where a run ends with a (sequence, key head) the warps join in shared memory; a (sequence, key head) that
// several runs share leaves partial results, which the last of its CTAs to arrive joins in the order of the runs.
#include "cache.cuh"

namespace fz {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kMinRounds = 2;       // of a CTA: fewer and the join costs more than the split gains
constexpr float kLow = -3.0e38f;    // a maximum over nothing: finite, so that (-inf) - kLow is -inf
constexpr float kNoPage = 3.0e38f;  // in the place of a log2 size (at most 128): the token's page id is out of range

__device__ __forceinline__ float ex2(float x) {   // 2^x, one MUFU instruction (2^-inf = 0)
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void *src, bool read) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(read ? 16 : 0) : "memory");
}
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Visible tokens of a sequence of n tokens: the j-th is position j (j < sinks) or j + n - visible.
__device__ __forceinline__ int visible(const CacheAttnParams &p, int n) {
    return p.window ? min(n, p.window + p.sinks) : n;
}

// The batch's rounds (or tiles): every thread sums a run of sequences, a scan over the CTA gives the total; then the
// sequence of the rounds' number `first` is found by the thread whose run holds it.
template <int THREADS>
struct Batch {
    long long excl[THREADS / 32 + 1];
    long long total;
    int b;                // sequence of the first round
    long long rem;        // and the rounds of that sequence before it
};
__device__ __forceinline__ long long rounds_of(const CacheAttnParams &p, int b, int tokens, int heads) {
    const int n = cache_length(p.c, b);
    return n <= 0 ? 0 : (long long)((visible(p, n) + tokens - 1) / tokens) * heads;
}
template <int THREADS>
__device__ long long batch_total(const CacheAttnParams &p, Batch<THREADS> &s, int tokens, int heads, long long &mine, long long &before) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = ceil_div(p.c.max_batch, THREADS), b0 = min(tid * per, p.c.max_batch), b1 = min(b0 + per, p.c.max_batch);
    mine = 0;
    for (int b = b0; b < b1; ++b) mine += rounds_of(p, b, tokens, heads);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) s.excl[warp] = incl;
    __syncthreads();
    if (tid == 0) {
        long long t = 0;
        for (int w = 0; w < THREADS / 32; ++w) {
            const long long v = s.excl[w];
            s.excl[w] = t;
            t += v;
        }
        s.total = t;
    }
    __syncthreads();
    before = s.excl[warp] + incl - mine;
    return s.total;
}
template <int THREADS>
__device__ void batch_find(const CacheAttnParams &p, Batch<THREADS> &s, int tokens, int heads, long long mine, long long before, long long first) {
    if (first >= before && first < before + mine) {
        const int per = ceil_div(p.c.max_batch, THREADS);
        long long at = before;
        for (int b = threadIdx.x * per;; ++b) {
            const long long r = rounds_of(p, b, tokens, heads);
            if (first < at + r) {
                s.b = b;
                s.rem = first - at;
                break;
            }
            at += r;
        }
    }
    __syncthreads();
}

// Where in the batch a round lies.
struct Place {
    int b, vh, u;          // sequence, key head (times query chunk), round
    int n, vis, rounds;    // length, visible tokens, rounds of one key head
};
__device__ __forceinline__ void place_sequence(const CacheAttnParams &p, Place &s, int tokens) {
    s.n = max(cache_length(p.c, s.b), 0);
    s.vis = visible(p, s.n);
    s.rounds = (s.vis + tokens - 1) / tokens;
}
__device__ __forceinline__ void place_next(const CacheAttnParams &p, Place &s, int tokens, int vheads) {
    if (++s.u < s.rounds) return;
    s.u = 0;
    if (++s.vh < vheads) return;
    s.vh = 0;
    do {
        if (++s.b >= p.c.max_batch) {
            s.rounds = s.vis = 0;
            return;
        }
        place_sequence(p, s, tokens);
    } while (s.rounds == 0);
}

// A token that a warp will load: its page (from the table, a round before its size) and place in it.
struct Token {
    unsigned page;
    int place;       // -1: no token here
    int vh;
};

// The CTA's shared memory: per warp and stage TT rows of K, TT rows of V; then the tokens' log2 sizes, the queries, the
// warps' joined output.
template <typename T, int DP, int NQ, int TT, int S>
struct Layout {
    static constexpr int kRow = DP * (int)sizeof(T);
    static constexpr int kStage = 2 * TT * kRow;
    static constexpr int kJoinQ = NQ < 4 ? NQ : 4;        // query heads joined at a time
    static constexpr int kJoinPitch = DP + 4;
    static constexpr int kStages = kWarps * S * kStage;
    static constexpr int kLsz = kStages;                  // float [kWarps][S][TT]
    static constexpr int kP = kLsz + kWarps * S * TT * 4; // float [kWarps][TT][NQ]
    static constexpr int kQ = kP + kWarps * TT * NQ * 4;  // float [2][NQ][DP]
    static constexpr int kJoin = kQ + 2 * NQ * DP * 4;    // float [kWarps][kJoinQ][kJoinPitch]
    static constexpr int kTotal = kJoin + kWarps * kJoinQ * kJoinPitch * 4;
};

template <typename T, int DP, int NQ, int TT, int S>
__global__ void __launch_bounds__(kThreads) k_cache_attn(CacheAttnParams p, int chunks) {
    using L = Layout<T, DP, NQ, TT, S>;
    constexpr int kRound = kWarps * TT, kCpr = L::kRow / 16, kPer = 16 / (int)sizeof(T), kD = DP / 32;
    extern __shared__ __align__(128) unsigned char sm[];
    __shared__ Batch<kThreads> batch;
    __shared__ float s_m[kWarps][NQ], s_l[kWarps][NQ];
    __shared__ int s_bad, s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Cache &c = p.c;
    const int vheads = c.kv_heads * chunks, es = (int)sizeof(T);

    // sequences without tokens: zeros (and a length out of range is told)
    for (int b = blockIdx.x; b < c.max_batch; b += gridDim.x) {
        const int n = cache_length(c, b);
        if (n > 0) continue;
        if (n < 0) {
            if (tid == 0) raise_status(p.status, FUSION_DEV_BAD_CACHE);
            continue;
        }
        uint4 *o = reinterpret_cast<uint4 *>(p.out) + (size_t)b * p.heads * c.dim * es / 16;
        for (int e = tid; e < p.heads * c.dim * es / 16; e += kThreads) o[e] = make_uint4(0u, 0u, 0u, 0u);
    }

    long long mine, before;
    const long long total = batch_total(p, batch, kRound, vheads, mine, before);
    const long long most = (total + kMinRounds - 1) / kMinRounds;
    const int ctas = most < (long long)gridDim.x ? (int)most : (int)gridDim.x;   // that take part
    if ((int)blockIdx.x >= ctas) return;
    const long long r0 = total * blockIdx.x / ctas, r1 = total * (blockIdx.x + 1) / ctas;
    batch_find(p, batch, kRound, vheads, mine, before, r0);
    Place at;
    at.b = batch.b;
    place_sequence(p, at, kRound);
    at.vh = (int)(batch.rem / at.rounds);
    at.u = (int)(batch.rem % at.rounds);
    Place ahead = at;          // of the token that load_token takes next
    long long ahead_r = r0;

    unsigned char *stages = sm + warp * S * L::kStage;
    float *lsz = reinterpret_cast<float *>(sm + L::kLsz) + warp * S * TT;
    float *pw = reinterpret_cast<float *>(sm + L::kP) + warp * TT * NQ;
    float *qs = reinterpret_cast<float *>(sm + L::kQ);
    float *join = reinterpret_cast<float *>(sm + L::kJoin);
    const int row_chunks = c.dim * es / 16;   // 16-byte chunks of a row that exist

    // the page of this lane's token of the round `ahead`, then the next round
    bool bad = false;
    auto load_token = [&]() {
        Token t;
        t.place = -1;
        t.page = 0;
        t.vh = ahead.vh;
        if (ahead_r < r1) {
            const int j = ahead.u * kRound + warp * TT + lane;
            if (lane < TT && j < ahead.vis) {
                const int pos = p.window && j >= p.sinks ? j + ahead.n - ahead.vis : j;
                if (cache_page(c, ahead.b, pos, t.page)) t.place = pos & ((1 << c.shift) - 1);
                else t.place = -2;
            }
            ++ahead_r;
            place_next(p, ahead, kRound, vheads);
        }
        return t;
    };
    auto load_size = [&](const Token &t) {
        return t.place < 0 ? 0.0f : c.sizes ? c.sizes[((size_t)t.page << c.shift) + t.place] : 1.0f;
    };
    // the rows of a round into a stage; rows without a token (or of size zero) are zeros and weigh nothing
    auto issue = [&](const Token &t, float size, int st) {
        const unsigned row = ((t.page * (unsigned)c.kv_heads + (unsigned)(t.vh / chunks)) << c.shift) + (unsigned)t.place;
        const unsigned live = __ballot_sync(0xFFFFFFFFu, t.place >= 0 && size != 0.0f);
        if (lane < TT) lsz[st * TT + lane] = t.place == -2 ? kNoPage : t.place >= 0 && size != 0.0f ? log2f(size) : -INFINITY;
        unsigned char *ks = stages + st * L::kStage, *vs = ks + TT * L::kRow;
#pragma unroll
        for (int e = 0; e < TT * kCpr / 32; ++e) {
            const int x = e * 32 + lane, r = x / kCpr, cc = x % kCpr;
            const unsigned rr = __shfl_sync(0xFFFFFFFFu, row, r);
            const bool read = (live >> r & 1u) && cc < row_chunks;
            const size_t off = read ? ((size_t)rr * row_chunks + cc) * 16 : 0;
            const int sw = (r * kCpr + (cc ^ (((r & 1) << 2 | (r >> 1 & 3)) & (kCpr - 1)))) * 16;
            cp_async16_zfill(smem_addr(ks + sw), c.k + off, read);
            cp_async16_zfill(smem_addr(vs + sw), c.v + off, read);
        }
    };
    // the scaled queries of a (sequence, key head) as float32
    auto load_q = [&](int b, int vh, float *dst) {
        const int h = vh / chunks, ch = vh % chunks;
        for (int e = tid; e < NQ * DP; e += kThreads) {
            const int q = e / DP, d = e % DP, a = ch * NQ + q;
            dst[e] = a < p.group && d < c.dim
                         ? Elem<T>::to_f(reinterpret_cast<const T *>(p.q)[(size_t)b * p.q_stride + (size_t)(h * p.group + a) * c.dim + d]) * p.scale2
                         : 0.0f;
        }
    };

    Token t0 = load_token(), t1;
#pragma unroll
    for (int s = 0; s < S - 1; ++s) {
        t1 = load_token();
        issue(t0, load_size(t0), s);
        cp_async_commit();
        t0 = t1;
    }
    t1 = load_token();
    float size0 = load_size(t0);
    load_q(at.b, at.vh, qs);
    if (tid == 0) s_bad = 0;
    __syncthreads();

    float m[NQ], l[NQ], o[NQ][kD];
    auto reset = [&]() {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            m[q] = kLow;
            l[q] = 0.0f;
#pragma unroll
            for (int d = 0; d < kD; ++d) o[q][d] = 0.0f;
        }
    };
    reset();
    int st = 0, qpar = 0;
    long long seg0 = r0 - at.u;   // first round of the (sequence, key head)
    for (long long r = r0; r < r1; ++r) {
        // ---- loads: rows of round r + S - 1, size of the one after, page of the one after that
        __syncwarp();
        issue(t0, size0, st == 0 ? S - 1 : st - 1);
        cp_async_commit();
        t0 = t1;
        size0 = load_size(t0);
        t1 = load_token();
        cp_async_wait<S - 1>();
        __syncwarp();

        // ---- logits: four lanes per token, eight tokens at a time
        const unsigned char *ks = stages + st * L::kStage, *vs = ks + TT * L::kRow;
        const float *q0 = qs + qpar * NQ * DP, *lz = lsz + st * TT;
        const int j0 = at.u * kRound + warp * TT, cnt = min(TT, at.vis - j0);
        const int h = at.vh / chunks, ch = at.vh % chunks, nq = min(NQ, p.group - ch * NQ);
        const int head0 = h * p.group + ch * NQ;
        if (cnt > 0) {
            float x[TT / 8][NQ];
            const int quad = lane & 3;
#pragma unroll
            for (int k = 0; k < TT / 8; ++k) {
                const int row = 8 * k + (lane >> 2), sw = (row & 1) << 2 | (row >> 1 & 3);
#pragma unroll
                for (int q = 0; q < NQ; ++q) x[k][q] = 0.0f;
#pragma unroll
                for (int i = 0; i < kCpr / 4; ++i) {
                    const int cc = 4 * i + quad;
                    float kv[kPer];
                    chunk_to_f(*reinterpret_cast<const uint4 *>(ks + (row * kCpr + (cc ^ (sw & (kCpr - 1)))) * 16), kv);
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int e = 0; e < kPer; e += 4) {
                            const float4 qv = *reinterpret_cast<const float4 *>(q0 + q * DP + cc * kPer + e);
                            x[k][q] = fmaf(kv[e], qv.x, fmaf(kv[e + 1], qv.y, fmaf(kv[e + 2], qv.z, fmaf(kv[e + 3], qv.w, x[k][q]))));
                        }
                }
                const float z = lz[row];
                bad |= z == kNoPage;
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    x[k][q] += __shfl_xor_sync(0xFFFFFFFFu, x[k][q], 1);
                    x[k][q] += __shfl_xor_sync(0xFFFFFFFFu, x[k][q], 2);
                    x[k][q] = z == -INFINITY || z == kNoPage ? -INFINITY : x[k][q] + z;
                }
                if (p.logits && quad == 0 && row < cnt)
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
                        if (q < nq) p.logits[((size_t)at.b * p.heads + head0 + q) * p.lstride + j0 + row] = x[k][q];
            }
            // ---- softmax with a running maximum
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                float mx = x[0][q];
#pragma unroll
                for (int k = 1; k < TT / 8; ++k) mx = fmaxf(mx, x[k][q]);
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, s));
                const float mn = fmaxf(m[q], mx), f = ex2(m[q] - mn);
                m[q] = mn;
                l[q] *= f;
#pragma unroll
                for (int d = 0; d < kD; ++d) o[q][d] *= f;
#pragma unroll
                for (int k = 0; k < TT / 8; ++k) {
                    const float pr = ex2(x[k][q] - mn);
                    l[q] += pr;
                    if ((lane & 3) == 0) pw[(8 * k + (lane >> 2)) * NQ + q] = pr;
                }
            }
            __syncwarp();
            // ---- o += p v: every lane has kD dims
#pragma unroll 4
            for (int row = 0; row < TT; ++row) {
                const int sw = (row & 1) << 2 | (row >> 1 & 3), cc = lane * kD / kPer;
                float v[kD];
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    const int cd = cc + d / kPer;
                    v[d] = Elem<T>::to_f(reinterpret_cast<const T *>(vs + (row * kCpr + (cd ^ (sw & (kCpr - 1)))) * 16)[(lane * kD + d) % kPer]);
                }
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const float pr = pw[row * NQ + q];
#pragma unroll
                    for (int d = 0; d < kD; ++d) o[q][d] = fmaf(pr, v[d], o[q][d]);
                }
            }
        }

        // ---- the end of a (sequence, key head), or of the run: the warps' results together
        if (at.u + 1 == at.rounds || r + 1 == r1) {
            Place next = at;
            place_next(p, next, kRound, vheads);
            if (r + 1 < r1) load_q(next.b, next.vh, qs + (qpar ^ 1) * NQ * DP);
            if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(&s_bad, 1);
            bad = false;
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) l[q] += __shfl_xor_sync(0xFFFFFFFFu, l[q], s);
                if (lane == 0) {
                    s_m[warp][q] = m[q];
                    s_l[warp][q] = l[q];
                }
            }
            __syncthreads();
            const bool whole = seg0 >= r0 && seg0 + at.rounds <= r1;
            const int slot = 2 * blockIdx.x + (seg0 >= r0 ? 1 : 0);   // of a partial result
            const bool seg_bad = s_bad != 0;
#pragma unroll
            for (int q1 = 0; q1 < NQ; q1 += L::kJoinQ) {
#pragma unroll
                for (int q = q1; q < q1 + L::kJoinQ; ++q) {
                    float M = s_m[0][q];
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) M = fmaxf(M, s_m[w][q]);
                    const float f = ex2(m[q] - M);
#pragma unroll
                    for (int d = 0; d < kD; ++d) join[(warp * L::kJoinQ + q - q1) * L::kJoinPitch + lane * kD + d] = o[q][d] * f;
                }
                __syncthreads();
                for (int e = tid; e < L::kJoinQ * DP; e += kThreads) {
                    const int q = q1 + e / DP, d = e % DP;
                    if (q >= nq || d >= c.dim) continue;
                    float M = s_m[0][q], sum = 0.0f, ls = 0.0f;
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) M = fmaxf(M, s_m[w][q]);
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        ls += s_l[w][q] * ex2(s_m[w][q] - M);
                        sum += join[(w * L::kJoinQ + q - q1) * L::kJoinPitch + d];
                    }
                    if (whole) {
                        if (!seg_bad)
                            reinterpret_cast<T *>(p.out)[((size_t)at.b * p.heads + head0 + q) * c.dim + d] = (T)(ls == 0.0f ? 0.0f : sum / ls);
                        if (d == 0 && p.logits)
                            p.lse[(size_t)at.b * p.heads + head0 + q] = seg_bad || ls == 0.0f ? INFINITY : M + log2f(ls);
                    } else {
                        p.part[((size_t)slot * NQ + q) * c.dim + d] = sum;
                        if (d == 0) p.part_ml[(size_t)slot * NQ + q] = make_float2(seg_bad ? INFINITY : M, seg_bad ? -1.0f : ls);
                    }
                }
                __syncthreads();
            }
            if (seg_bad && tid == 0) raise_status(p.status, FUSION_DEV_BAD_CACHE);
            if (!whole) {
                // the runs c0 .. c1 share it: the last one to arrive joins their results in order
                auto run_of = [&](long long x) { return (int)(((x + 1) * ctas + total - 1) / total) - 1; };
                const int c0 = run_of(seg0), c1 = run_of(seg0 + at.rounds - 1);
                __threadfence();
                __syncthreads();
                if (tid == 0) {
                    s_last = atomicAdd(&p.counters[c0], 1) == c1 - c0;
                    if (s_last) p.counters[c0] = 0;
                    __threadfence();
                }
                __syncthreads();
                if (s_last) {
                    for (int e = tid; e < nq * c.dim; e += kThreads) {
                        const int q = e / c.dim, d = e % c.dim;
                        float M = kLow, sum = 0.0f, ls = 0.0f;
                        bool none = false;
                        for (int k = c0; k <= c1; ++k) {
                            const size_t ps = ((size_t)2 * k + (k == c0)) * NQ + q;
                            const float2 ml = __ldcg(&p.part_ml[ps]);
                            if (ml.y < 0.0f) {
                                none = true;
                                break;
                            }
                            const float mn = fmaxf(M, ml.x), f0 = ex2(M - mn), f1 = ex2(ml.x - mn);
                            sum = sum * f0 + __ldcg(&p.part[ps * c.dim + d]) * f1;
                            ls = ls * f0 + ml.y * f1;
                            M = mn;
                        }
                        if (!none)
                            reinterpret_cast<T *>(p.out)[((size_t)at.b * p.heads + head0 + q) * c.dim + d] = (T)(ls == 0.0f ? 0.0f : sum / ls);
                        if (d == 0 && p.logits) p.lse[(size_t)at.b * p.heads + head0 + q] = none || ls == 0.0f ? INFINITY : M + log2f(ls);
                    }
                }
            }
            if (tid == 0) s_bad = 0;
            __syncthreads();
            reset();
            qpar ^= 1;
            seg0 = r + 1;
        }
        place_next(p, at, kRound, vheads);
        if (++st == S) st = 0;
    }
    cp_async_wait<0>();
}

// weights_j += sum over the query heads of 2^(x - lse): a thread per visible token, the heads in order.
constexpr int kWeightThreads = 256;
__global__ void __launch_bounds__(kWeightThreads) k_cache_weights(CacheAttnParams p) {
    __shared__ Batch<kWeightThreads> batch;
    const Cache &c = p.c;
    long long mine, before;
    const long long total = batch_total(p, batch, kWeightThreads, 1, mine, before);
    const long long r0 = total * blockIdx.x / gridDim.x, r1 = total * (blockIdx.x + 1) / gridDim.x;
    if (r0 >= r1) return;
    batch_find(p, batch, kWeightThreads, 1, mine, before, r0);
    Place at;
    at.b = batch.b;
    place_sequence(p, at, kWeightThreads);
    at.vh = 0;
    at.u = (int)batch.rem;
    for (long long r = r0; r < r1; ++r) {
        const int j = at.u * kWeightThreads + threadIdx.x;
        unsigned page;
        const int pos = p.window && j >= p.sinks ? j + at.n - at.vis : j;
        if (j < at.vis && cache_page(c, at.b, pos, page)) {
            const float *x = p.logits + (size_t)at.b * p.heads * p.lstride + j, *lse = p.lse + (size_t)at.b * p.heads;
            float w = 0.0f;
#pragma unroll 8
            for (int h = 0; h < p.heads; ++h) w += ex2(x[h * p.lstride] - lse[h]);
            float *dst = c.weights + ((size_t)page << c.shift) + (pos & ((1 << c.shift) - 1));
            *dst += w;
        }
        place_next(p, at, kWeightThreads, 1);
    }
}

template <typename T, int DP, int NQ, int TT, int S>
cudaError_t launch(const CacheAttnParams &p, cudaStream_t s) {
    using L = Layout<T, DP, NQ, TT, S>;
    int dev = 0, sms = 0, occ = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_cache_attn<T, DP, NQ, TT, S>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, k_cache_attn<T, DP, NQ, TT, S>, kThreads, L::kTotal);
    if (e != cudaSuccess) return e;
    const int chunks = ceil_div(p.group, NQ);
    const long long rounds = (long long)p.c.max_batch * p.c.kv_heads * chunks * ceil_div(p.most, kWarps * TT);
    long long ctas = (long long)sms * (occ < 1 ? 1 : occ);
    if (ctas > kCacheMaxCtas) ctas = kCacheMaxCtas;
    if (ctas > rounds) ctas = rounds;
    k_cache_attn<T, DP, NQ, TT, S><<<(unsigned)(ctas < 1 ? 1 : ctas), kThreads, L::kTotal, s>>>(p, chunks);
    return cudaGetLastError();
}
template <typename T, int NQ>
cudaError_t launch_dim(const CacheAttnParams &p, cudaStream_t s) {
    constexpr int k = 4 / (int)sizeof(T);
    if (p.c.dim <= 64) return launch<T, 64, NQ, 16 * k, 3>(p, s);
    if (p.c.dim <= 128) return launch<T, 128, NQ, 8 * k, 3>(p, s);
    return launch<T, 256, NQ, 8, 3>(p, s);
}

}  // namespace

cudaError_t launch_cache_attention(int dtype, const CacheAttnParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    cudaError_t e;
    if (dtype == FUSION_BF16)
        e = p.group == 1 ? launch_dim<__nv_bfloat16, 1>(p, s) : p.group <= 4 ? launch_dim<__nv_bfloat16, 4>(p, s) : launch_dim<__nv_bfloat16, 8>(p, s);
    else
        e = p.group == 1 ? launch_dim<float, 1>(p, s) : p.group <= 4 ? launch_dim<float, 4>(p, s) : launch_dim<float, 8>(p, s);
    if (e != cudaSuccess || !p.logits) return e;
    const long long tiles = (long long)p.c.max_batch * ceil_div(p.most, kWeightThreads);
    k_cache_weights<<<(unsigned)(tiles < 1216 ? tiles : 1216), kWeightThreads, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace fz
