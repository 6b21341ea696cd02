// Attention of one new token per sequence over the paged cache, and the accumulated attention weights.  For sequence
// b, query head a of key head h and the visible tokens j (the first `sinks` and the last `window`; all without a
// window), in base 2:
//   x_aj = scale2 q_a . k_hj + log2 s_j,   out_a = sum_j 2^(x_aj - m) v_hj / sum_j 2^(x_aj - m),   m = max_j x_aj,
//   weights_j += sum_a 2^(x_aj - lse_a),   lse_a = m + log2 sum_j 2^(x_aj - m).
//
// Work is cut into rounds: the next TT visible tokens per warp of a CTA of one (sequence, key head).  Every CTA takes an equal
// run of the rounds of the whole batch, in the order (sequence, key head, token), whatever the sequences' lengths; a
// warp takes TT tokens of each round through stages of its own (cp.async) and keeps its own running maximum, sum and
// output.  Where a run ends with a (sequence, key head) the warps join in shared memory; a (sequence, key head) that
// several runs share leaves partial results, which the last of its CTAs to arrive joins in the order of the runs.
#include "cache_rounds.cuh"

namespace fz {
namespace {

using namespace rounds;

// The CTA's shared memory: per warp and stage TT rows of K, TT rows of V; the tokens' log2 sizes; their probabilities, each
// twice (a packed multiplication's operand); then the queries or, at the end of a (sequence, key head), the warps' outputs.
template <int DP, int NQ, int TT, int S, int W>
struct Layout {
    static constexpr int kRow = DP * 4, kStage = 2 * TT * kRow;
    static constexpr int kJoinQ = NQ < 2 ? NQ : 2;        // query heads joined at a time
    static constexpr int kPitch = DP + 4;
    static constexpr int kLsz = W * S * kStage;          // float [W][S][TT]
    static constexpr int kP = kLsz + W * S * TT * 4;     // float2 [W][TT][NQ]
    static constexpr int kShared = kP + W * TT * NQ * 8;
    static constexpr int kQBytes = NQ * kRow, kJoinBytes = W * kJoinQ * kPitch * 4, kScratch = kJoinScratch<NQ>;
    static constexpr int kTotal = kShared + (kQBytes > kJoinBytes ? kQBytes > kScratch ? kQBytes : kScratch
                                             : kJoinBytes > kScratch ? kJoinBytes : kScratch);
};

// W: warps of a CTA.
template <int DP, int NQ, int TT, int S, int W>
__global__ void __launch_bounds__(32 * W, W == 1 ? 12 : S == 2 ? 3 : 1) k_cache_attn_f32(CacheAttnParams p, int chunks) {
    using L = Layout<DP, NQ, TT, S, W>;
    constexpr int kWarps = W, kThreads = 32 * W;
    constexpr int kRound = kWarps * TT, kCpr = L::kRow / 16;
    // What bounds groups of four heads and more is not memory but the reading of operands from shared memory, so a lane's products
    // are blocked: for q k four lanes per token, a lane has kMt tokens and kHeads heads (eight heads: two halves side by side, 4 x 4
    // or 2 x 4 a lane; with 32 x 4096 of 8 heads of 64, 128, 256 dims: 65.4, 67.4, 83.6 us with all eight in a lane, 62.1, 60.1, 72.3 so).
    // Then each lane of the four gets the sums of kMine heads, so that a softmax is computed once (in all four: 72.4 for 64 dims).
    constexpr int kSides = NQ == 8 ? 2 : 1, kHeads = NQ / kSides, kRows = 8 / kSides, kMt = TT / kRows;
    constexpr int kMine = kHeads < 4 ? kHeads : kHeads / 4;   // heads whose softmax a lane holds
    // For p v a lane has kV chunks of four dims of every kGroups-th row (two with eight heads of 64 dims: spills, 71.1).
    constexpr int kV = NQ == 8 && DP < 256 ? 1 : 2, kLanes = DP / (4 * kV), kGroups = 32 / kLanes;
    extern __shared__ __align__(128) unsigned char sm[];
    __shared__ Finder<kThreads> finder;
    __shared__ float s_m[kWarps][NQ], s_l[kWarps][NQ];
    __shared__ int s_bad, s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int quad = lane & 3, row0 = lane >> 2 & (kRows - 1), h0 = kSides == 1 ? 0 : (lane >> 4) * kHeads;
    const int my0 = h0 + (kHeads < 4 ? 0 : quad * kMine);
    const Cache &c = p.c;
    wait_for_previous();
    Run run;
    Place at;
    if (!find_run<kThreads, true, false>(p, finder, kRound, c.kv_heads, chunks, kMinRounds, run, at)) {
        empty_sequences<float, kThreads>(p);
        return;
    }
    const unsigned r0 = run.r0, r1 = run.r1;

    unsigned char *stages = sm + warp * S * L::kStage;
    float *lsz = reinterpret_cast<float *>(sm + L::kLsz) + warp * S * TT;
    float2 *pw = reinterpret_cast<float2 *>(sm + L::kP) + warp * TT * NQ;
    float *qs = reinterpret_cast<float *>(sm + L::kShared), *join = qs;
    // (two tokens' chunks at the same place of their rows lie in different halves of the banks)
    auto swizzle = [](int r) { return (r & 1) << 2 | (r >> 1 & 3); };
    // the scaled queries of a (sequence, key head): read ahead into registers, then written to shared memory
    constexpr int kQPer = (NQ * DP / 4 + kThreads - 1) / kThreads;
    float4 qv[kQPer];
    auto read_q = [&](int b, int h, int ch) {
        const float *src = reinterpret_cast<const float *>(p.q) + (size_t)b * p.q_stride + (size_t)(h * p.group + ch * NQ) * c.dim;
#pragma unroll
        for (int k = 0; k < kQPer; ++k) {
            const int e = tid + k * kThreads, q = e / (DP / 4), d = e % (DP / 4) * 4;
            qv[k] = q < min(NQ, p.group - ch * NQ) && d < c.dim ? *reinterpret_cast<const float4 *>(src + (size_t)q * c.dim + d)
                                                                : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    };
    auto write_q = [&]() {
#pragma unroll
        for (int k = 0; k < kQPer; ++k) {
            const int e = tid + k * kThreads;
            if (e < NQ * DP / 4)
                reinterpret_cast<float4 *>(qs)[e] = make_float4(qv[k].x * p.scale2, qv[k].y * p.scale2, qv[k].z * p.scale2, qv[k].w * p.scale2);
        }
    };
    // those of the (sequence, key head) after the one of round r, if this run has it
    auto read_next_q = [&](unsigned r) {
        if (r + at.rounds - at.u >= r1) return;
        Place next = at;
        next.u = at.rounds - 1;
        place_next(p, next, kRound, c.kv_heads, chunks);
        read_q(next.b, next.h, next.ch);
    };
    read_q(at.b, at.h, at.ch);
    Stream<float, DP, TT, W> in;
    in.template begin<S>(p, at, run, chunks, warp, lane, stages, lsz, swizzle);
    write_q();
    empty_sequences<float, kThreads>(p);
    if (tid == 0) s_bad = 0;
    __syncthreads();

    bool bad = false;
    float m[kMine], l[kMine];
    float2 o[NQ][2 * kV];
    auto begin_head = [&]() {
#pragma unroll
        for (int e = 0; e < kMine; ++e) {
            m[e] = kLow;
            l[e] = 0.0f;
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
            for (int d = 0; d < 2 * kV; ++d) o[q][d] = make_float2(0.0f, 0.0f);
    };
    begin_head();
    int st = 0;
    unsigned seg0 = r0 - at.u;   // first round of the (sequence, key head)
    for (unsigned r = r0;; ++r) {
        if (r == r0 || at.u == 0) read_next_q(r);
        __syncwarp();
        const int next_st = st == 0 ? S - 1 : st - 1;
        in.next(p, chunks, warp, lane, stages + next_st * L::kStage, lsz + next_st * TT, swizzle);
        cp_async_wait<S - 1>();
        __syncwarp();

        const unsigned char *ks = stages + st * L::kStage, *vs = ks + TT * L::kRow;
        const float *lz = lsz + st * TT;
        const int j0 = at.u * kRound + warp * TT, cnt = min(TT, at.vis - j0);
        const int nq = min(NQ, p.group - at.ch * NQ), head0 = at.h * p.group + at.ch * NQ;
        if (cnt > 0) {
            // ---- logits
            float2 acc[kMt][kHeads];
#pragma unroll
            for (int k = 0; k < kMt; ++k)
#pragma unroll
                for (int q = 0; q < kHeads; ++q) acc[k][q] = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < kCpr / 4; ++i) {
                const int cc = 4 * i + quad;
                float4 kv[kMt];
#pragma unroll
                for (int k = 0; k < kMt; ++k)
                    kv[k] = *reinterpret_cast<const float4 *>(ks + ((kRows * k + row0) * kCpr + (cc ^ swizzle(kRows * k + row0))) * 16);
#pragma unroll
                for (int q = 0; q < kHeads; ++q) {
                    const float4 qq = *reinterpret_cast<const float4 *>(qs + (h0 + q) * DP + cc * 4);
#pragma unroll
                    for (int k = 0; k < kMt; ++k) {
                        acc[k][q] = __ffma2_rn(make_float2(kv[k].x, kv[k].y), make_float2(qq.x, qq.y), acc[k][q]);
                        acc[k][q] = __ffma2_rn(make_float2(kv[k].z, kv[k].w), make_float2(qq.z, qq.w), acc[k][q]);
                    }
                }
            }
            // the four lanes' sums of a token, each to the lane that holds its head (all in every lane below four heads)
            float x[kMt][kMine];
#pragma unroll
            for (int k = 0; k < kMt; ++k) {
                if constexpr (kHeads < 4) {
#pragma unroll
                    for (int q = 0; q < kHeads; ++q) {
                        x[k][q] = acc[k][q].x + acc[k][q].y;
                        x[k][q] += __shfl_xor_sync(0xFFFFFFFFu, x[k][q], 1);
                        x[k][q] += __shfl_xor_sync(0xFFFFFFFFu, x[k][q], 2);
                    }
                } else {
                    float half[kHeads / 2];
#pragma unroll
                    for (int q = 0; q < kHeads / 2; ++q) {
                        const float lo = acc[k][q].x + acc[k][q].y, hi = acc[k][q + kHeads / 2].x + acc[k][q + kHeads / 2].y;
                        half[q] = (quad & 2 ? hi : lo) + __shfl_xor_sync(0xFFFFFFFFu, quad & 2 ? lo : hi, 2);
                    }
#pragma unroll
                    for (int e = 0; e < kMine; ++e)
                        x[k][e] = (quad & 1 ? half[e + kMine] : half[e]) + __shfl_xor_sync(0xFFFFFFFFu, quad & 1 ? half[e] : half[e + kMine], 1);
                }
                const float z = lz[kRows * k + row0];
                const bool off = z == -INFINITY || z == kNoPage;
                bad |= z == kNoPage;
#pragma unroll
                for (int e = 0; e < kMine; ++e) x[k][e] = off ? -INFINITY : x[k][e] + z;
                if (p.logits && (kHeads >= 4 || quad == 0) && kRows * k + row0 < cnt) {
                    float *dst = p.logits + ((size_t)at.b * p.heads + head0 + my0) * p.lstride + j0 + kRows * k + row0;
#pragma unroll
                    for (int e = 0; e < kMine; ++e)
                        if (my0 + e < nq) dst[e * p.lstride] = x[k][e];
                }
            }
            // ---- the running shift: where a logit exceeds it by more than kLag, it becomes the maximum, and the output and the sums follow
            bool grows = false;
            float mx[kMine];
#pragma unroll
            for (int e = 0; e < kMine; ++e) {
                mx[e] = m[e];
#pragma unroll
                for (int k = 0; k < kMt; ++k) mx[e] = fmaxf(mx[e], x[k][e]);
                grows |= mx[e] > m[e] + kLag;
            }
            if (__any_sync(0xFFFFFFFFu, grows)) {
                float f[kMine];
#pragma unroll
                for (int e = 0; e < kMine; ++e) {
#pragma unroll
                    for (int s = 4; s < 4 * kRows; s <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xFFFFFFFFu, mx[e], s));
                    f[e] = ex2(m[e] - mx[e]);
                    m[e] = mx[e];
                    l[e] *= f[e];
                }
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const float fq = kHeads < 4 ? f[q % kMine] : __shfl_sync(0xFFFFFFFFu, f[q % kMine], q / kHeads * 16 + q % kHeads / kMine);
#pragma unroll
                    for (int d = 0; d < 2 * kV; ++d) o[q][d] = __fmul2_rn(o[q][d], make_float2(fq, fq));
                }
            }
#pragma unroll
            for (int k = 0; k < kMt; ++k) {
                float pr[kMine];
#pragma unroll
                for (int e = 0; e < kMine; ++e) {
                    pr[e] = ex2(x[k][e] - m[e]);
                    l[e] += pr[e];
                }
                if (kHeads >= 4 || quad == 0) {
#pragma unroll
                    for (int e = 0; e < kMine; ++e) pw[(kRows * k + row0) * NQ + my0 + e] = make_float2(pr[e], pr[e]);
                }
            }
            __syncwarp();
            // ---- o += p v
#pragma unroll 4
            for (int i = 0; i < TT / kGroups; ++i) {
                const int row = i * kGroups + lane / kLanes;
                float4 v[kV];
#pragma unroll
                for (int d = 0; d < kV; ++d)
                    v[d] = *reinterpret_cast<const float4 *>(vs + (row * kCpr + ((lane % kLanes + d * kLanes) ^ swizzle(row))) * 16);
                float2 pr[NQ];
                if constexpr (NQ == 1) {
                    pr[0] = pw[row];
                } else {
#pragma unroll
                    for (int q = 0; q < NQ; q += 2) {
                        const float4 two = *reinterpret_cast<const float4 *>(&pw[row * NQ + q]);
                        pr[q] = make_float2(two.x, two.y);
                        pr[q + 1] = make_float2(two.z, two.w);
                    }
                }
#pragma unroll
                for (int q = 0; q < NQ; ++q)
#pragma unroll
                    for (int d = 0; d < kV; ++d) {
                        o[q][2 * d] = __ffma2_rn(pr[q], make_float2(v[d].x, v[d].y), o[q][2 * d]);
                        o[q][2 * d + 1] = __ffma2_rn(pr[q], make_float2(v[d].z, v[d].w), o[q][2 * d + 1]);
                    }
            }
        }

        // ---- the end of a (sequence, key head), or of the run: the warps' results together
        if (at.u + 1 == at.rounds || r + 1 == r1) {
            if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(&s_bad, 1);
            bad = false;
#pragma unroll
            for (int e = 0; e < kMine; ++e) {
#pragma unroll
                for (int s = 4; s < 4 * kRows; s <<= 1) l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], s);
                if (row0 == 0 && (kHeads >= 4 || quad == 0)) {
                    s_m[warp][my0 + e] = m[e];
                    s_l[warp][my0 + e] = l[e];
                }
            }
            __syncthreads();   // (and every warp is past its products with the queries)
            const bool whole = seg0 >= r0 && seg0 + at.rounds <= r1, seg_bad = s_bad != 0;
            const size_t head = (size_t)at.b * p.heads + head0, slot = (size_t)(2 * blockIdx.x + (seg0 >= r0 ? 1 : 0)) * NQ;   // of a partial result
#pragma unroll
            for (int q1 = 0; q1 < NQ; q1 += L::kJoinQ) {
#pragma unroll
                for (int q = q1; q < q1 + L::kJoinQ; ++q) {
                    float M = s_m[0][q];
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) M = fmaxf(M, s_m[w][q]);
                    const float f = ex2(s_m[warp][q] - M);
                    // the groups' sums: of the lanes with the same columns each ends with its share of them
                    float v[4 * kV];
#pragma unroll
                    for (int d = 0; d < 2 * kV; ++d) {
                        v[2 * d] = o[q][d].x * f;
                        v[2 * d + 1] = o[q][d].y * f;
                    }
                    constexpr int kShare = 4 * kV / kGroups;
                    int col = 0;   // of the lane's columns
#pragma unroll
                    for (int s = 16, n = 2 * kV; s >= kLanes; s >>= 1, n >>= 1) {
                        const bool upper = lane & s;
                        col += upper ? n : 0;
#pragma unroll
                        for (int i = 0; i < n; ++i) v[i] = (upper ? v[i + n] : v[i]) + __shfl_xor_sync(0xFFFFFFFFu, upper ? v[i] : v[i + n], s);
                    }
                    float *dst = join + (warp * L::kJoinQ + q - q1) * L::kPitch + lane % kLanes * 4 + col / 4 * kLanes * 4 + col % 4;
                    if constexpr (kShare == 2) {
                        *reinterpret_cast<float2 *>(dst) = make_float2(v[0], v[1]);
                    } else {
#pragma unroll
                        for (int d = 0; d < kShare / 4; ++d)
                            *reinterpret_cast<float4 *>(dst + d * kLanes * 4) = make_float4(v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]);
                    }
                }
                __syncthreads();
                for (int e = tid; e < L::kJoinQ * DP / 4; e += kThreads) {
                    const int qq = e / (DP / 4), q = q1 + qq, d = e % (DP / 4) * 4;
                    if (q >= nq || d >= c.dim) continue;
                    float M = s_m[0][q], ls = 0.0f;
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) M = fmaxf(M, s_m[w][q]);
                    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        ls += s_l[w][q] * ex2(s_m[w][q] - M);
                        const float4 v = *reinterpret_cast<const float4 *>(join + (w * L::kJoinQ + qq) * L::kPitch + d);
                        sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
                    }
                    if (whole) {
                        const float inv = 1.0f / ls;
                        if (!seg_bad)
                            store4(reinterpret_cast<float *>(p.out) + (head + q) * c.dim + d,
                                   ls == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
                        if (d == 0 && p.logits) p.lse[head + q] = log_sum(M, seg_bad ? -1.0f : ls);
                    } else {
                        *reinterpret_cast<float4 *>(p.part + (slot + q) * c.dim + d) = sum;
                        if (d == 0) p.part_ml[slot + q] = make_float2(seg_bad ? INFINITY : M, seg_bad ? -1.0f : ls);
                    }
                }
                __syncthreads();
            }
            if (tid == 0) {
                if (seg_bad) raise_status(p.status, FUSION_DEV_BAD_CACHE);
                s_bad = 0;
            }
            if (!whole) {
                join_runs<float, NQ, kThreads>(p, run, seg0, seg0 + at.rounds, head, nq, join, s_last);
                __syncthreads();
            }
            if (r + 1 == r1) break;
            write_q();
            __syncthreads();
            begin_head();
            seg0 = r + 1;
        }
        place_next(p, at, kRound, c.kv_heads, chunks);
        if (++st == S) st = 0;
    }
    cp_async_wait<0>();   // (of rounds past the run: nothing but zeros)
}

// weights_j += sum over the query heads of 2^(x - lse): tiles of 128 visible tokens, four to a lane, the heads dealt out to
// the CTA's warps; the warps' sums are added in order.  A programmatic dependent of the attention kernel: it finds its tokens
// meanwhile.  (A thread per token and all heads in turn took 14 us for 64 x 4096 tokens of 32 heads.)
constexpr int kWeightThreads = 256, kWeightTile = 128, kWeightCtas = 608;
__global__ void __launch_bounds__(kWeightThreads) k_cache_weights(CacheAttnParams p) {
    constexpr int kW = kWeightThreads / 32;
    __shared__ Finder<kWeightThreads> finder;
    __shared__ __align__(16) float part[kW][kWeightTile];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Cache &c = p.c;
    Run run;
    Place at;
    const bool works = find_run<kWeightThreads, false, true>(p, finder, kWeightTile, 1, 1, 1u, run, at);
    // the token that this thread updates, and its place in its page (-1: none)
    int j0 = 0, place = -1;
    unsigned page = 0;
    auto look_up = [&]() {
        j0 = at.u * kWeightTile;
        const int j = j0 + tid, pos = p.window && j >= p.sinks ? j + at.n - at.vis : j;
        place = tid < kWeightTile && j < at.vis && cache_page<true>(c, at.b, pos, page) ? pos & ((1 << c.shift) - 1) : -1;
    };
    // (lengths and pages are complete in the L2 cache, from where they are read: wait_for_previous)
    if (works) look_up();
    wait_for_previous();
    for (unsigned r = run.r0; works && r < run.r1; ++r) {
        if (r > run.r0) look_up();
        const bool here = place >= 0;
        float *dst = c.weights + ((size_t)page << c.shift) + place;
        const float old = here ? *dst : 0.0f, first = p.lse[(size_t)at.b * p.heads];
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
            if (first != kRefused) *dst = old + sum;   // (another sequence may hold a refused one's pages by now)
        }
        __syncthreads();
        place_next(p, at, kWeightTile, 1, 1);
    }
}

template <int DP, int NQ, int TT, int S>
cudaError_t launch(const CacheAttnParams &p, cudaStream_t s) {
    static_assert(counts_fit(TT, 4) && (DP > 128 || counts_fit(TT, 1)), "rounds are counted in 32 bits");
    const int chunks = ceil_div(p.group, NQ);
    if constexpr (DP <= 128)
        if (warps_alone(p, chunks)) return launch_rounds<k_cache_attn_f32<DP, NQ, TT, S, 1>, 1>(Layout<DP, NQ, TT, S, 1>::kTotal, p, chunks, TT, s);
    return launch_rounds<k_cache_attn_f32<DP, NQ, TT, S, 4>, 4>(Layout<DP, NQ, TT, S, 4>::kTotal, p, chunks, 4 * TT, s);
}
template <int NQ>
cudaError_t launch_dim(const CacheAttnParams &p, cudaStream_t s) {
    if (p.c.dim <= 64) return launch<64, NQ, 16, 2>(p, s);
    if (p.c.dim <= 128) return launch<128, NQ, 8, 2>(p, s);
    return launch<256, NQ, 8, 3>(p, s);
}

}  // namespace

cudaError_t launch_cache_attention(int dtype, const CacheAttnParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    const cudaError_t e = dtype == FUSION_BF16 ? launch_cache_attention_bf16(p, s)
                          : p.group == 1       ? launch_dim<1>(p, s)
                          : p.group <= 4       ? launch_dim<4>(p, s)
                                               : launch_dim<8>(p, s);
    return e != cudaSuccess || !p.logits ? e : launch_cache_weights(p, s);
}

cudaError_t launch_cache_weights(const CacheAttnParams &p, cudaStream_t s) {
    const long long tiles = (long long)p.c.max_batch * ceil_div(p.most, kWeightTile);
    return launch_after(k_cache_weights, dim3((unsigned)(tiles < kWeightCtas ? tiles : kWeightCtas)), kWeightThreads, 0, 1, s, p);
}

}  // namespace fz
