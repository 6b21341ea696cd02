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
#include "cache_rounds.cuh"

namespace fz {
namespace {

using namespace rounds;

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
    static constexpr int kJoinBytes = kWarps * kJoinQ * kJoinPitch * 4;
    static constexpr int kTotal = kJoin + (kJoinBytes > kJoinScratch<NQ> ? kJoinBytes : kJoinScratch<NQ>);   // (or the join of the runs)
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
    const int vheads = c.kv_heads * chunks;
    if (p.logits) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Run run;
    Place at;
    if (!find_run(p, batch, kRound, vheads, run, at)) {
        empty_sequences<T>(p);
        return;
    }
    const long long r0 = run.r0, r1 = run.r1;

    unsigned char *stages = sm + warp * S * L::kStage;
    float *lsz = reinterpret_cast<float *>(sm + L::kLsz) + warp * S * TT;
    float *pw = reinterpret_cast<float *>(sm + L::kP) + warp * TT * NQ;
    float *qs = reinterpret_cast<float *>(sm + L::kQ);
    float *join = reinterpret_cast<float *>(sm + L::kJoin);
    auto swizzle = [](int r) { return ((r & 1) << 2 | (r >> 1 & 3)) & (kCpr - 1); };
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

    Stream<T, DP, TT> in;
    in.template begin<S>(p, at, run, chunks, vheads, warp, lane, stages, lsz, swizzle);
    empty_sequences<T>(p);
    load_q(at.b, at.vh, qs);
    if (tid == 0) s_bad = 0;
    __syncthreads();
    bool bad = false;

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
        __syncwarp();
        const int next_st = st == 0 ? S - 1 : st - 1;
        in.next(p, chunks, vheads, warp, lane, stages + next_st * L::kStage, lsz + next_st * TT, swizzle);
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
                const int row = 8 * k + (lane >> 2), sw = swizzle(row);
#pragma unroll
                for (int q = 0; q < NQ; ++q) x[k][q] = 0.0f;
#pragma unroll
                for (int i = 0; i < kCpr / 4; ++i) {
                    const int cc = 4 * i + quad;
                    float kv[kPer];
                    chunk_to_f(*reinterpret_cast<const uint4 *>(ks + (row * kCpr + (cc ^ sw)) * 16), kv);
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
                const int sw = swizzle(row), cc = lane * kD / kPer;
                float v[kD];
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    const int cd = cc + d / kPer;
                    v[d] = Elem<T>::to_f(reinterpret_cast<const T *>(vs + (row * kCpr + (cd ^ sw)) * 16)[(lane * kD + d) % kPer]);
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
                join_runs<T, NQ>(p, run, seg0, seg0 + at.rounds, (size_t)at.b * p.heads + head0, nq, join, s_last);
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

// weights_j += sum over the query heads of 2^(x - lse): tiles of 128 visible tokens, four to a lane, the heads dealt out to
// the CTA's warps; the warps' sums are added in order.  A programmatic dependent of the attention kernel: it finds its tokens
// meanwhile.  (A thread per token and all heads in turn took 14 us for 64 x 4096 tokens of 32 heads.)
constexpr int kWeightThreads = 256, kWeightTile = 128, kWeightCtas = 608;
__global__ void __launch_bounds__(kWeightThreads) k_cache_weights(CacheAttnParams p) {
    constexpr int kW = kWeightThreads / 32;
    __shared__ Batch<kWeightThreads> batch;
    __shared__ __align__(16) float part[kW][kWeightTile];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Cache &c = p.c;
    long long mine, before;
    const long long total = batch_total(p, batch, kWeightTile, 1, mine, before);
    Run run;
    run.cut(total, (int)gridDim.x);
    if (run.r0 >= run.r1) return;
    batch_find(p, batch, kWeightTile, 1, mine, before, run.r0, -1);
    Place at;
    at.b = batch.b[0];
    place_sequence(p, at, kWeightTile);
    at.vh = 0;
    at.u = (int)batch.rem[0];
    for (long long r = run.r0; r < run.r1; ++r) {
        const int j0 = at.u * kWeightTile, j = j0 + tid;   // the token that this thread updates
        unsigned page = 0;
        const int pos = p.window && j >= p.sinks ? j + at.n - at.vis : j;
        const bool here = tid < kWeightTile && j < at.vis && cache_page(c, at.b, pos, page);
        float *dst = c.weights + ((size_t)page << c.shift) + (pos & ((1 << c.shift) - 1));
        if (r == run.r0) asm volatile("griddepcontrol.wait;" ::: "memory");
        const float old = here ? *dst : 0.0f;
        float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (j0 + 4 * lane < at.vis) {   // (up to three logits past the sequence are there, and not used)
            const float *x = p.logits + (size_t)at.b * p.heads * p.lstride + j0 + 4 * lane, *lse = p.lse + (size_t)at.b * p.heads;
#pragma unroll 4
            for (int h = warp; h < p.heads; h += kW) {
                const float4 v = __ldcg(reinterpret_cast<const float4 *>(x + h * p.lstride));
                const float s = lse[h];
                w.x += ex2(v.x - s);
                w.y += ex2(v.y - s);
                w.z += ex2(v.z - s);
                w.w += ex2(v.w - s);
            }
        }
        *reinterpret_cast<float4 *>(&part[warp][4 * lane]) = w;
        __syncthreads();
        if (here) {
            float sum = part[0][tid];
#pragma unroll
            for (int k = 1; k < kW; ++k) sum += part[k][tid];
            *dst = old + sum;
        }
        __syncthreads();
        place_next(p, at, kWeightTile, 1);
    }
}

template <int DP, int NQ, int TT, int S>
cudaError_t launch(const CacheAttnParams &p, cudaStream_t s) {
    using L = Layout<float, DP, NQ, TT, S>;
    return launch_rounds<k_cache_attn<float, DP, NQ, TT, S>>(L::kTotal, p, ceil_div(p.group, NQ), kWarps * TT, s);
}
template <int NQ>
cudaError_t launch_dim(const CacheAttnParams &p, cudaStream_t s) {
    if (p.c.dim <= 64) return launch<64, NQ, 16, 3>(p, s);
    if (p.c.dim <= 128) return launch<128, NQ, 8, 3>(p, s);
    return launch<256, NQ, 8, 3>(p, s);
}

}  // namespace

cudaError_t launch_cache_attention(int dtype, const CacheAttnParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    const cudaError_t e = dtype == FUSION_BF16 ? launch_cache_attention_bf16(p, s)
                          : p.group == 1       ? launch_dim<1>(p, s)
                          : p.group <= 4       ? launch_dim<4>(p, s)
                                               : launch_dim<8>(p, s);
    if (e != cudaSuccess || !p.logits) return e;
    const long long tiles = (long long)p.c.max_batch * ceil_div(p.most, kWeightTile);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles < kWeightCtas ? tiles : kWeightCtas));
    cfg.blockDim = dim3(kWeightThreads);
    cfg.stream = s;
    cudaLaunchAttribute a[1];
    a[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = a;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_cache_weights, p);
}

}  // namespace fz
