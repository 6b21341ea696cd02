// bf16 attention of one new token per sequence over the paged cache (the formulas and the cut into rounds: cache_attn.cu),
// both products on the warp's matrix instruction m16n8k16.
//
// The tokens are the M rows and the query heads of a key head the N columns, so that a group of up to eight heads fills the
// instruction's smallest N: S^T = K Q^T (A: 16 tokens x 16 dims of K as it lies, B: the queries), then O^T += V^T P^T (A: 16
// dims x 16 tokens, V's rows read transposed, B: the probabilities, whose accumulator layout becomes the operand's by one 8 x 8
// transposition per 8 tokens).  A probability is the sum of two bf16 terms there, p and what its rounding lost, so that the
// products keep 16 bits of it: one term alone made the error against 64 bits 1.3 times that of the output's own rounding, and
// the second product costs nothing while memory is the bound (64 x 4096: 101.7 and 100.8 us).  A lane's accumulators of both products belong to the same two heads, so the running maximum
// and the rescaling need no exchange but the maximum over a column's tokens.
//
// What bounds it: memory.  A token's K and V of one key head, 4 dim bytes, give 4 dim group flops: for a group of 8, 8 flops
// per byte where tensor cores break even near 280, so tcgen05's 128-row tiles would be idle all the same, with a round trip
// through tensor memory between the products.
#include "cache_rounds.cuh"

namespace fz {
namespace {

using namespace rounds;

__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {   // an 8 x 8 matrix of b16, a row per four lanes
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Shared memory of a CTA: per warp S stages of TT rows of K and of V; the tokens' log2 sizes; then the queries, or, at the end of
// a (sequence, key head), the warps' outputs on their way to each other, kTiles steps of 16 dims at a time.
template <int DP, int NT, int TT, int S, int W>
struct Layout {
    static constexpr int kNq = 8 * NT, kRow = 2 * DP, kStage = 2 * TT * kRow;
    static constexpr int kTiles = 2, kPitch = 16 * kTiles + 4;   // (pitches of 4 mod 16: no bank conflicts)
    static constexpr int kLsz = W * S * kStage;
    static constexpr int kShared = kLsz + W * S * TT * 4;
    static constexpr int kQBytes = kNq * kRow, kJoinBytes = W * kNq * kPitch * 4, kScratch = kJoinScratch<kNq>;
    static constexpr int kTotal = kShared + (kQBytes > kJoinBytes ? kQBytes > kScratch ? kQBytes : kScratch
                                             : kJoinBytes > kScratch ? kJoinBytes : kScratch);
};

// W: warps of a CTA.
template <int DP, int NT, int TT, int S, int W>
__global__ void __launch_bounds__(32 * W, W == 1 ? 12 : S == 2 ? 3 : 1) k_cache_attn_mma(CacheAttnParams p, int chunks) {
    using L = Layout<DP, NT, TT, S, W>;
    constexpr int kWarps = W, kThreads = 32 * W;
    constexpr int kNq = L::kNq, kRound = kWarps * TT, kRow = L::kRow, kKs = DP / 16, kMt = TT / 16;
    constexpr int kQPer = (kNq * DP / 8 + kThreads - 1) / kThreads;   // 16-byte chunks of the queries per thread
    constexpr bool kQRegs = NT * DP <= 128;     // the queries' fragments stay in registers
    constexpr bool kQEarly = NT == 1;           // the next queries are asked for as soon as these are in use
    extern __shared__ __align__(128) unsigned char sm[];
    __shared__ Finder<kThreads> finder;
    __shared__ float s_m[kWarps][kNq], s_l[kWarps][kNq];
    __shared__ int s_bad, s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const Cache &c = p.c;
    wait_for_previous();
    Run run;
    Place at;
    if (!find_run<kThreads, true, false>(p, finder, kRound, c.kv_heads, chunks, kMinRounds, run, at)) {
        empty_sequences<__nv_bfloat16, kThreads>(p);
        return;
    }
    const unsigned r0 = run.r0, r1 = run.r1;

    unsigned char *stages = sm + warp * S * L::kStage, *qs = sm + L::kShared;
    float *lsz = reinterpret_cast<float *>(sm + L::kLsz) + warp * S * TT;
    float *join = reinterpret_cast<float *>(sm + L::kShared);
    auto swizzle = [](int r) { return r & 7; };

    // the queries of a (sequence, key head): read ahead into registers, then written to shared memory
    uint4 qv[kQPer];
    auto read_q = [&](int b, int h, int ch) {
        const __nv_bfloat16 *src = reinterpret_cast<const __nv_bfloat16 *>(p.q) + (size_t)b * p.q_stride + (size_t)(h * p.group + ch * kNq) * c.dim;
#pragma unroll
        for (int k = 0; k < kQPer; ++k) {
            const int e = tid + k * kThreads, q = e / (DP / 8), cc = e % (DP / 8);
            qv[k] = q < min(kNq, p.group - ch * kNq) && cc * 8 < c.dim ? *reinterpret_cast<const uint4 *>(src + (size_t)q * c.dim + cc * 8)
                                                                     : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    auto write_q = [&]() {
#pragma unroll
        for (int k = 0; k < kQPer; ++k) {
            const int e = tid + k * kThreads, q = e / (DP / 8), cc = e % (DP / 8);
            if (q < kNq) *reinterpret_cast<uint4 *>(qs + q * kRow + ((cc ^ (q & 7)) << 4)) = qv[k];
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
    Stream<__nv_bfloat16, DP, TT, W> in;
    in.template begin<S>(p, at, run, chunks, warp, lane, stages, lsz, swizzle);
    write_q();
    empty_sequences<__nv_bfloat16, kThreads>(p);
    if (tid == 0) s_bad = 0;
    __syncthreads();

    float m[NT][2], l[NT][2], o[kKs][NT][4];
    uint32_t qf[kQRegs ? kKs : 1][NT][2];
    bool bad = false;
    auto q_fragments = [&](int ks2, int n, uint32_t (&r)[4]) {   // of two steps of 16 dims
        ldsm_x4(smem_addr(qs) + (8 * n + (lane & 7)) * kRow + (((4 * ks2 + (lane >> 3)) ^ (lane & 7)) << 4), r[0], r[1], r[2], r[3]);
    };
    auto begin_head = [&]() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n][0] = m[n][1] = kLow;
            l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int k = 0; k < kKs; ++k) o[k][n][0] = o[k][n][1] = o[k][n][2] = o[k][n][3] = 0.0f;
            if constexpr (kQRegs) {
#pragma unroll
                for (int k = 0; k < kKs; k += 2) {
                    uint32_t r[4];
                    q_fragments(k / 2, n, r);
                    qf[k][n][0] = r[0];
                    qf[k][n][1] = r[1];
                    qf[k + 1][n][0] = r[2];
                    qf[k + 1][n][1] = r[3];
                }
            }
        }
    };
    begin_head();
    int st = 0;
    unsigned seg0 = r0 - at.u;   // first round of the (sequence, key head)
    for (unsigned r = r0;; ++r) {
        if (kQEarly && (r == r0 || at.u == 0)) read_next_q(r);
        __syncwarp();
        const int next_st = st == 0 ? S - 1 : st - 1;
        in.next(p, chunks, warp, lane, stages + next_st * L::kStage, lsz + next_st * TT, swizzle);
        cp_async_wait<S - 1>();
        __syncwarp();

        const uint32_t ks = smem_addr(stages + st * L::kStage), vs = ks + TT * kRow;
        const float *lz = lsz + st * TT;
        const int j0 = at.u * kRound + warp * TT;
        const int nq = min(kNq, p.group - at.ch * kNq), head0 = at.h * p.group + at.ch * kNq;
        if (j0 < at.vis) {
            // ---- S^T = K Q^T
            float x[kMt][NT][4];
#pragma unroll
            for (int i = 0; i < kMt; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) x[i][n][0] = x[i][n][1] = x[i][n][2] = x[i][n][3] = 0.0f;
#pragma unroll
            for (int k = 0; k < kKs; k += 2) {
                uint32_t b[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if constexpr (kQRegs) {
                        b[n][0] = qf[k][n][0];
                        b[n][1] = qf[k][n][1];
                        b[n][2] = qf[k + 1][n][0];
                        b[n][3] = qf[k + 1][n][1];
                    } else {
                        q_fragments(k / 2, n, b[n]);
                    }
                }
#pragma unroll
                for (int i = 0; i < kMt; ++i)
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        uint32_t a[4];
                        ldsm_x4(ks + (16 * i + (lane & 15)) * kRow + (((2 * (k + kk) + (lane >> 4)) ^ (lane & 7)) << 4), a[0], a[1], a[2], a[3]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma_bf16_16816(x[i][n], a, b[n][2 * kk], b[n][2 * kk + 1]);
                    }
            }
            // ---- logits in base 2; a masked token's are -inf
#pragma unroll
            for (int i = 0; i < kMt; ++i) {
                const float z0 = lz[16 * i + g], z1 = lz[16 * i + 8 + g];
                const bool off0 = z0 == -INFINITY || z0 == kNoPage, off1 = z1 == -INFINITY || z1 == kNoPage;
                bad |= z0 == kNoPage || z1 == kNoPage;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    x[i][n][0] = off0 ? -INFINITY : fmaf(x[i][n][0], p.scale2, z0);
                    x[i][n][1] = off0 ? -INFINITY : fmaf(x[i][n][1], p.scale2, z0);
                    x[i][n][2] = off1 ? -INFINITY : fmaf(x[i][n][2], p.scale2, z1);
                    x[i][n][3] = off1 ? -INFINITY : fmaf(x[i][n][3], p.scale2, z1);
                }
                if (p.logits) {
                    float *dst = p.logits + ((size_t)at.b * p.heads + head0) * p.lstride + j0 + 16 * i + g;
                    const bool in0 = j0 + 16 * i + g < at.vis, in1 = j0 + 16 * i + 8 + g < at.vis;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (8 * n + 2 * t + e < nq) {
                                if (in0) dst[(8 * n + 2 * t + e) * p.lstride] = x[i][n][e];
                                if (in1) dst[(8 * n + 2 * t + e) * p.lstride + 8] = x[i][n][2 + e];
                            }
                }
            }
            // ---- the running shift: where a logit exceeds it by more than kLag, it becomes the maximum, and O and the sums follow
            float mx[NT][2];
            bool grows = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    mx[n][e] = m[n][e];
#pragma unroll
                    for (int i = 0; i < kMt; ++i) mx[n][e] = fmaxf(mx[n][e], fmaxf(x[i][n][e], x[i][n][2 + e]));
                    grows |= mx[n][e] > m[n][e] + kLag;
                }
            if (__any_sync(0xFFFFFFFFu, grows)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int s = 4; s < 32; s <<= 1) mx[n][e] = fmaxf(mx[n][e], __shfl_xor_sync(0xFFFFFFFFu, mx[n][e], s));
                        const float f = ex2(m[n][e] - mx[n][e]);
                        m[n][e] = mx[n][e];
                        l[n][e] *= f;
#pragma unroll
                        for (int k = 0; k < kKs; ++k) {
                            o[k][n][e] *= f;
                            o[k][n][2 + e] *= f;
                        }
                    }
            }
            // ---- O^T += V^T P^T
#pragma unroll
            for (int i = 0; i < kMt; ++i) {
                uint32_t b[NT][2], b_lo[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float p0 = ex2(x[i][n][0] - m[n][0]), p1 = ex2(x[i][n][1] - m[n][1]);
                    const float p2 = ex2(x[i][n][2] - m[n][0]), p3 = ex2(x[i][n][3] - m[n][1]);
                    l[n][0] += p0 + p2;
                    l[n][1] += p1 + p3;
                    const uint32_t h0 = pack(p0, p1), h1 = pack(p2, p3);
                    b[n][0] = transpose8(h0);
                    b[n][1] = transpose8(h1);
                    b_lo[n][0] = transpose8(pack(p0 - __uint_as_float(h0 << 16), p1 - __uint_as_float(h0 & 0xFFFF0000u)));
                    b_lo[n][1] = transpose8(pack(p2 - __uint_as_float(h1 << 16), p3 - __uint_as_float(h1 & 0xFFFF0000u)));
                }
#pragma unroll
                for (int k = 0; k < kKs; ++k) {
                    uint32_t a[4];
                    ldsm_x4_t(vs + (16 * i + (lane & 7) + ((lane >> 4) << 3)) * kRow + (((2 * k + (lane >> 3 & 1)) ^ (lane & 7)) << 4), a);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_bf16_16816(o[k][n], a, b[n][0], b[n][1]);
                        mma_bf16_16816(o[k][n], a, b_lo[n][0], b_lo[n][1]);
                    }
                }
            }
        }

        // ---- the end of a (sequence, key head), or of the run: the warps' results together
        if (at.u + 1 == at.rounds || r + 1 == r1) {
            if (!kQEarly) read_next_q(r);
            if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(&s_bad, 1);
            bad = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int s = 4; s < 32; s <<= 1) l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, l[n][e], s);
                    if (g == 0) {
                        s_m[warp][8 * n + 2 * t + e] = m[n][e];
                        s_l[warp][8 * n + 2 * t + e] = l[n][e];
                    }
                }
            __syncthreads();   // (and every warp is past its products with the queries)
            const bool whole = seg0 >= r0 && seg0 + at.rounds <= r1, seg_bad = s_bad != 0;
            const size_t head = (size_t)at.b * p.heads + head0, slot = (size_t)(2 * blockIdx.x + (seg0 >= r0 ? 1 : 0)) * kNq;   // of a partial result
            float f[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float M = s_m[0][8 * n + 2 * t + e];
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) M = fmaxf(M, s_m[w][8 * n + 2 * t + e]);
                    f[n][e] = ex2(m[n][e] - M);
                }
            // a thread joins four dims of one head (kMine of them) per step
            constexpr int kMine = (kNq * 4 * L::kTiles + kThreads - 1) / kThreads;
            float sums[kMine];
#pragma unroll
            for (int x = 0; x < kMine; ++x) {
                const int q = min((x * kThreads + tid) / (4 * L::kTiles), kNq - 1);
                float M = s_m[0][q], ls = 0.0f;
#pragma unroll
                for (int w = 1; w < kWarps; ++w) M = fmaxf(M, s_m[w][q]);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) ls += s_l[w][q] * ex2(s_m[w][q] - M);
                sums[x] = ls;
                const int e = x * kThreads + tid;
                if (e < 4 * L::kTiles * nq && e % (4 * L::kTiles) == 0) {
                    if (!whole) p.part_ml[slot + q] = make_float2(seg_bad ? INFINITY : M, seg_bad ? -1.0f : ls);
                    else if (p.logits) p.lse[head + q] = log_sum(M, seg_bad ? -1.0f : ls);
                }
            }
#pragma unroll
            for (int k1 = 0; k1 < kKs; k1 += L::kTiles) {
                float *dst = join + (warp * kNq + 2 * t) * L::kPitch + g;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (8 * n + 2 * t >= nq) break;
#pragma unroll
                    for (int k = 0; k < L::kTiles; ++k) {
                        float *to = dst + 8 * n * L::kPitch + 16 * k;
                        to[0] = o[k1 + k][n][0] * f[n][0];
                        to[L::kPitch] = o[k1 + k][n][1] * f[n][1];
                        to[8] = o[k1 + k][n][2] * f[n][0];
                        to[L::kPitch + 8] = o[k1 + k][n][3] * f[n][1];
                    }
                }
                __syncthreads();
#pragma unroll
                for (int x = 0; x < kMine; ++x) {
                    const int e = x * kThreads + tid, q = e / (4 * L::kTiles), d0 = e % (4 * L::kTiles) * 4, d = 16 * k1 + d0;
                    if (q >= nq || d >= c.dim) continue;
                    float4 sum = *reinterpret_cast<const float4 *>(join + q * L::kPitch + d0);
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) {
                        const float4 v = *reinterpret_cast<const float4 *>(join + (w * kNq + q) * L::kPitch + d0);
                        sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
                    }
                    const float inv = 1.0f / sums[x];
                    if (!whole)
                        *reinterpret_cast<float4 *>(p.part + (slot + q) * c.dim + d) = sum;
                    else if (!seg_bad)
                        store4(reinterpret_cast<__nv_bfloat16 *>(p.out) + (head + q) * c.dim + d,
                               sums[x] == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
                }
                __syncthreads();
            }
            if (tid == 0) {
                if (seg_bad) raise_status(p.status, FUSION_DEV_BAD_CACHE);
                s_bad = 0;
            }
            if (!whole) {
                join_runs<__nv_bfloat16, kNq, kThreads>(p, run, seg0, seg0 + at.rounds, head, nq, join, s_last);
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

template <int DP, int NT, int TT, int S>
cudaError_t launch(const CacheAttnParams &p, cudaStream_t s) {
    static_assert(counts_fit(TT, 4) && (DP > 128 || counts_fit(TT, 1)), "rounds are counted in 32 bits");
    const int chunks = ceil_div(p.group, 8 * NT);
    if constexpr (DP <= 128)
        if (warps_alone(p, chunks)) return launch_rounds<k_cache_attn_mma<DP, NT, TT, S, 1>, 1>(Layout<DP, NT, TT, S, 1>::kTotal, p, chunks, TT, s);
    return launch_rounds<k_cache_attn_mma<DP, NT, TT, S, 4>, 4>(Layout<DP, NT, TT, S, 4>::kTotal, p, chunks, 4 * TT, s);
}
template <int NT>
cudaError_t launch_dim(const CacheAttnParams &p, cudaStream_t s) {
    // (two stages let three CTAs share an SM, which hides more than a third stage: 64 x 4096 with weights 112 -> 103 us)
    if (p.c.dim <= 64) return launch<64, NT, 32, 2>(p, s);
    if (p.c.dim <= 128) return launch<128, NT, 16, 2>(p, s);
    return launch<256, NT, 16, 3>(p, s);
}

}  // namespace

cudaError_t launch_cache_attention_bf16(const CacheAttnParams &p, cudaStream_t s) {
    // groups beyond 16 heads go in parts of 16, the later ones reading K and V from the L2 cache: 32 heads a warp leave it 255
    // registers and two CTAs per SM (8 x 8192 with one key head of 32 query heads 22.9 us, in two parts 19.8)
    return p.group <= 8 ? launch_dim<1>(p, s) : launch_dim<2>(p, s);
}

}  // namespace fz
