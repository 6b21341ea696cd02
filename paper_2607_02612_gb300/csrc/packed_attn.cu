// Attention of one new token per sequence over the paged cache in 4 bits (the formulas and the cut into rounds: cache_attn.cu, the
// numbers: fp4.cuh), both products on the warp's matrix instruction m16n8k16 with float16 operands and float32 sums.
//
// As in bf16 the tokens are the M rows and the query heads the N columns: S^T = K Q^T, then O^T += V^T P^T.  What differs is how the
// operands come about.  Codes and scales lie in shared memory as in the cache; a lane reads words of eight codes and makes its
// own fragments: the conversion gives two dims of one token, which is what K's fragment needs, and a product with their scale.
// V's fragment pairs the same dim of two tokens, so two tokens' words are interleaved by halves of a byte first.  Which
// dims and tokens a fragment's rows and columns stand for is free as long as both operands agree:
//   K: lane (g, t) has dims t DP/4 .. (t + 1) DP/4 - 1 of a row, and reads the same dims of head g's query, straight from memory;
//   V: lane (g, t) has words g, g + 8, ..., of its four tokens, so its sums are of 8 dims in a row;
//   tokens: row i of a tile is token order(i), so that the lanes' reads of both spread over the banks.
// Values of the cache are exact in float16.  A query is not, so it enters times a power of two that brings its largest dim to
// 2^14 .. 2^15 (float32 queries as the sum of two float16).  Probabilities are 2^(x - shift), at most 2^(kLag + kUp) = 2^15: kUp
// keeps the small ones out of float16's subnormal numbers.  One float16 term (two for float32): its 11 bits lie 3 below the output's.
// Against probabilities in float32, 3 to 10 % of a bf16 output's numbers are rounded to a neighbour, and its error against 64 bits grows by 0.1
// to 0.6 % (1.3e-3 to 1.7e-3 of it).  Two terms take both away (at most 0.5 % of the numbers differ) and cost time: 64 x 4096 with weights
// 55.5 and 59.2 us, 4 x 65537 71.5 and 78.0, 113 x 21188 of 64 / 4 heads of 32 221 and 248; calls of up to 25 us at most 1 us.
//
// What bounds it: memory (9/8 dim bytes of a token and key head) and the issue of instructions (8 for eight codes of K, 11 of V, and a
// round's own) together: 64 sequences of up to 4096, 32 / 8 heads of 128, 47 us for 152 MB, which memory alone would give in 22; as
// many tokens again cost 32.  14 us do not depend on the tokens: the run is found after 2, its first round here after 5, the joins take 4.
// A round is 32 tokens of a warp (or 64: launch), asked for one round ahead (two rounds ahead 48 us), three CTAs per SM (four, of 128 registers,
// 48.5).
#include <float.h>

#include "cache_rounds.cuh"
#include "fp4.cuh"

namespace fz {
namespace {

using namespace rounds;

constexpr float kUp = 7.0f;
constexpr int kSnap = 1;      // rounds, of 128 tokens (256 up to 64 dims of bf16), or of 32 where warps are alone
// Rounds that the end of a (sequence, key head) counts for, one in which the warps join (64 x 4096 with weights 61 us without it, 56 so)
// and nothing else is done.  A warp alone joins nothing (200 x 60: 9.7 and 8.2).
template <int W> constexpr int kTail = W == 1 ? 0 : 1;

__device__ __forceinline__ uint32_t transpose8(uint32_t v) {   // an 8 x 8 matrix of b16, a row per four lanes
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// d += A B, B the sum of kTerms terms.  With two, for float32 results, the lower term comes first and the sum is added by itself: the
// matrix instruction cuts its sums off instead of rounding them (16 x 577 float32: off by 6.3e-7 of the result when it adds to d).
template <int kTerms, typename B>
__device__ __forceinline__ void products(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, B b) {
    if constexpr (kTerms == 1) {
        mma_f16_16816(d, a0, a1, a2, a3, b(0, 0), b(0, 1));
    } else {
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int term = kTerms - 1; term >= 0; --term) mma_f16_16816(s, a0, a1, a2, a3, b(term, 0), b(term, 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] += s[e];
    }
}
// BYTES from src, or zeros.  (A predicate, not a number of bytes to read, which would cost instructions at every copy.)
template <int BYTES> __device__ __forceinline__ void copy_or_zero(uint32_t dst, unsigned long long src, bool read) {
    if constexpr (BYTES == 16)
        asm volatile("{ .reg .pred p; setp.eq.u32 p, %2, 0; cp.async.cg.shared.global [%0], [%1], 16, p; }" ::"r"(dst), "l"(src), "r"((int)read) : "memory");
    else
        asm volatile("{ .reg .pred p; setp.eq.u32 p, %2, 0; cp.async.ca.shared.global [%0], [%1], %3, p; }" ::"r"(dst), "l"(src), "r"((int)read), "n"(BYTES)
                     : "memory");
}
// base + a b, in one instruction
__device__ __forceinline__ unsigned long long at_row(const unsigned char *base, unsigned a, unsigned b) {
    unsigned long long r;
    asm("mad.wide.u32 %0, %1, %2, %3;" : "=l"(r) : "r"(a), "r"(b), "l"(base));
    return r;
}
// The bits of a where m has ones, those of b elsewhere.
__device__ __forceinline__ uint32_t pick_bits(uint32_t a, uint32_t b, uint32_t m) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xE4;" : "=r"(r) : "r"(a), "r"(b), "r"(m));
    return r;
}

// The token of row i of a tile's half, and the place of 16-byte chunk c of row r: c ^ swizzle(r), linear in the bits of r.  A row of
// codes is a quarter, a half or all of the banks wide; tokens and places are such that eight lanes that read K (two rows of
// a half, 16 bytes each; four rows of a quarter) and all lanes that read V (a word of eight lanes of every other row) meet no bank twice.
template <int DP> __device__ __forceinline__ int order(int i) {
    if constexpr (DP == 64) {
        const int high = i >> 2, two = (i & 1) << 1 | (i >> 1 & 1);
        return high << 2 | (two ^ (high << 1));              // 0 2 1 3 6 4 7 5
    } else {
        return i & 1 ? 4 + (i >> 1 ^ 1) : i >> 1;            // 0 5 1 4 2 7 3 6
    }
}
template <int DP> __device__ __forceinline__ int swizzle(int r) {
    return DP == 64 ? 0 : DP == 128 ? r & 2 : (r & 3) << 1 | (r >> 2 & 1);
}

// Shared memory of a CTA: per warp S stages of TT rows of K's and of V's codes and of their scales; the tokens' log2 sizes; the
// queries of this (sequence, key head) and the next; the warps' outputs on their way to each other, at the end of a (sequence, key head),
// kJoinDims dims at a time.
template <typename T, int DP, int NT, int S, int W, int TT>
struct Layout {
    static constexpr int kNq = 8 * NT, kRow = DP / 2, kScales = DP / 16, kStage = 2 * TT * (kRow + kScales);
    static constexpr int kQPitch = DP * (int)sizeof(T) + 16, kQ = kNq * kQPitch;
    static constexpr int kJoinDims = DP < 128 ? DP : 128, kPitch = kJoinDims + 8;
    static constexpr int kLsz = W * S * kStage;
    static constexpr int kQueries = kLsz + W * S * TT * 4;
    static constexpr int kJoin = kQueries + 2 * kQ;
    static constexpr int kJoinBytes = W * kNq * kPitch * 4, kScratch = kJoinScratch<kNq>;
    static constexpr int kTotal = kJoin + (kJoinBytes > kScratch ? kJoinBytes : kScratch);
};

// The tokens of the rounds to come, kPer to a lane (rounds::Stream with rows in 4 bits).
template <int DP, int W, int TT>
struct PackedStream {
    static constexpr int kRow = DP / 2, kScales = DP / 16, kCpr = kRow / 16, kStage = 2 * TT * (kRow + kScales), kRound = W * TT, kPer = TT / 32;
    Place ahead;             // of the next round to look up
    unsigned ahead_r, r1;
    Token t0[kPer], t1[kPer];   // t0's rows are asked for next (their sizes are here), then t1's
    float size0[kPer];
    unsigned plain;          // a bit per stage: all of its tokens are there, of size 1

    __device__ __forceinline__ void look_up(const PackedAttnParams &p, int chunks, int warp, int lane, Token (&t)[kPer]) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) t[i] = Token{0u, -1, ahead.h};
        if (ahead_r < r1) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int j = ahead.u * kRound + warp * TT + i * 32 + lane;
                if (j < ahead.vis) {
                    const int pos = p.window && j >= p.sinks ? j + ahead.n - ahead.vis : j;
                    t[i].place = cache_page(p.c, ahead.b, pos, t[i].page) ? pos & ((1 << p.c.shift) - 1) : -2;
                }
            }
            ++ahead_r;
            place_next<false, kTail<W>>(p, ahead, kRound, p.c.kv_heads, chunks);
        }
    }
    __device__ __forceinline__ void sizes_of(const PackedAttnParams &p, const Token (&t)[kPer], float (&size)[kPer]) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            size[i] = t[i].place < 0 ? 0.0f : p.c.sizes ? p.c.sizes[((size_t)t[i].page << p.c.shift) + t[i].place] : 1.0f;
    }
    // Asks for the rows of a round's tokens, and notes their log2 sizes unless all are 0.
    __device__ __forceinline__ void ask(const PackedAttnParams &p, const Token (&t)[kPer], const float (&size)[kPer], int lane, int st,
                                        unsigned char *stages, float *lsz) {
        const unsigned row_bytes = (unsigned)p.c.dim / 2;
        unsigned row[kPer], lives[kPer];
        bool live[kPer], one = true;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            live[i] = t[i].place >= 0 && size[i] != 0.0f;
            one = one && live[i] && size[i] == 1.0f;
            row[i] = live[i] ? ((t[i].page * (unsigned)p.c.kv_heads + (unsigned)t[i].h) << p.c.shift) + (unsigned)t[i].place : 0u;
            lives[i] = __ballot_sync(0xFFFFFFFFu, live[i]);
        }
        const bool all_plain = __all_sync(0xFFFFFFFFu, one);
        plain = (plain & ~(1u << st)) | (unsigned)all_plain << st;
        if (!all_plain) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                lsz[st * TT + i * 32 + lane] = t[i].place == -2 ? kNoPage : live[i] ? log2f(size[i]) : -INFINITY;
        }
        constexpr int kWide = 32 / kCpr;   // rows of a step
        const int r_lane = lane / kCpr, cc = lane % kCpr;
        const bool exists = (unsigned)cc * 16u < row_bytes;
        const unsigned char *k = p.c.k + (exists ? cc : 0) * 16, *v = p.c.v + (exists ? cc : 0) * 16;
        const uint32_t stage = smem_addr(stages) + st * kStage, dst = stage + r_lane * kRow, at = (uint32_t)(cc ^ swizzle<DP>(r_lane)) * 16u;
#pragma unroll
        for (int e = 0; e < TT / kWide; ++e) {
            const int i = e * kWide / 32, r = e * kWide % 32;
            const unsigned theirs = __shfl_sync(0xFFFFFFFFu, row[i], r + r_lane);
            const bool read = exists && (lives[i] >> r_lane >> r & 1u);
            const uint32_t to = dst + e * kWide * kRow + (at ^ (uint32_t)(swizzle<DP>(e * kWide) * 16));
            copy_or_zero<16>(to, at_row(k, theirs, row_bytes), read);
            copy_or_zero<16>(to + TT * kRow, at_row(v, theirs, row_bytes), read);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t ks = stage + 2 * TT * kRow + (i * 32 + lane) * kScales, vs = ks + TT * kScales;
            const unsigned long long kz = at_row(p.s.k, row[i], (unsigned)p.s.bytes), vz = at_row(p.s.v, row[i], (unsigned)p.s.bytes);
            if constexpr (kScales <= 8) {
                copy_or_zero<kScales>(ks, kz, live[i]);
                copy_or_zero<kScales>(vs, vz, live[i]);
            } else {   // rows of 12 or 16 bytes
#pragma unroll
                for (int e = 0; e < kScales; e += 4) {
                    const bool read = live[i] && e < p.s.bytes;
                    copy_or_zero<4>(ks + e, kz + (read ? e : 0), read);
                    copy_or_zero<4>(vs + e, vz + (read ? e : 0), read);
                }
            }
        }
        cp_async_commit();
    }
    __device__ __forceinline__ void next(const PackedAttnParams &p, int chunks, int warp, int lane, int st, unsigned char *stages, float *lsz) {
        ask(p, t0, size0, lane, st, stages, lsz);
#pragma unroll
        for (int i = 0; i < kPer; ++i) t0[i] = t1[i];
        sizes_of(p, t0, size0);
        look_up(p, chunks, warp, lane, t1);
    }
    // The first S - 1 rounds' rows (all pages asked for at once, then all sizes).
    template <int S>
    __device__ __forceinline__ void begin(const PackedAttnParams &p, const Place &at, const Run &run, int chunks, int warp, int lane,
                                          unsigned char *stages, float *lsz) {
        ahead = at;
        ahead_r = run.r0;
        r1 = run.r1;
        plain = 0u;
        Token t[S + 1][kPer];
        float size[S][kPer];
#pragma unroll
        for (int s = 0; s <= S; ++s) look_up(p, chunks, warp, lane, t[s]);
#pragma unroll
        for (int s = 0; s < S; ++s) sizes_of(p, t[s], size[s]);
#pragma unroll
        for (int s = 0; s < S - 1; ++s) ask(p, t[s], size[s], lane, s, stages, lsz);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            t0[i] = t[S - 1][i];
            size0[i] = size[S - 1][i];
            t1[i] = t[S][i];
        }
    }
};

template <int N> __device__ __forceinline__ void load_words(const unsigned char *src, uint32_t (&w)[N]) {   // aligned to their size, or 16
    if constexpr (N == 1) {
        w[0] = *reinterpret_cast<const uint32_t *>(src);
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2 *>(src);
        w[0] = v.x, w[1] = v.y;
    } else {
        static_assert(N == 4, "up to 16 bytes");
        const uint4 v = *reinterpret_cast<const uint4 *>(src);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
}
// Two numbers of a row.
__device__ __forceinline__ float2 load2(const __nv_bfloat16 *src, int i) {
    const uint32_t w = reinterpret_cast<const uint32_t *>(src)[i];
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 load2(const float *src, int i) { return reinterpret_cast<const float2 *>(src)[i]; }

// T: type of queries and output.  W: warps of a CTA.  TT: tokens of a warp and round.
template <typename T, int DP, int NT, int S, int W, int TT>
__global__ void __launch_bounds__(32 * W, W == 1 ? 12 : DP <= 128 && NT == 1 ? 3 : 2) k_packed_attn(PackedAttnParams p, int chunks) {
    using L = Layout<T, DP, NT, S, W, TT>;
    constexpr int kThreads = 32 * W, kTerms = sizeof(T) == 4 ? 2 : 1;
    constexpr int kNq = L::kNq, kRound = W * TT, kRow = L::kRow, kScales = L::kScales, kKs = DP / 16, kMt = TT / 16;
    constexpr int kKw = DP / 32, kVw = DP / 64;   // words of a K row and of a V row that a lane has
    extern __shared__ __align__(128) unsigned char sm[];
    __shared__ Finder<kThreads> finder;
    __shared__ float s_m[W][kNq], s_l[W][kNq];
    __shared__ int s_bad, s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const Cache &c = p.c;

    unsigned char *stages = sm + warp * S * L::kStage;
    float *lsz = reinterpret_cast<float *>(sm + L::kLsz) + warp * S * TT;
    float *join = reinterpret_cast<float *>(sm + L::kJoin);
    PackedStream<DP, W, TT> in;
    wait_for_previous();
    Run run;
    Place at;
    if (!find_run<kThreads, true, false, kSnap, kTail<W>>(p, finder, kRound, c.kv_heads, chunks, kMinRounds, run, at)) {
        empty_sequences<T, kThreads>(p);
        return;
    }
    const unsigned r0 = run.r0, r1 = run.r1;

    // asks for the queries of a (sequence, key head), into one of two places in turn (with the next group of copies)
    int q_at = 0;
    auto ask_q = [&](const Place &s, int where) {
        const int heads = min(kNq, p.group - s.ch * kNq);
        const unsigned char *src = reinterpret_cast<const unsigned char *>(
            reinterpret_cast<const T *>(p.q) + (size_t)s.b * p.q_stride + (size_t)(s.h * p.group + s.ch * kNq) * c.dim);
        constexpr int kChunks = DP * (int)sizeof(T) / 16;
        const int row = c.dim * (int)sizeof(T);
        for (int e = tid; e < kNq * kChunks; e += kThreads) {
            const int q = e / kChunks, cc = e % kChunks * 16;
            const bool read = q < heads && cc < row;
            copy_or_zero<16>(smem_addr(sm + L::kQueries + where * L::kQ + q * L::kQPitch + cc),
                             reinterpret_cast<unsigned long long>(src + (read ? (size_t)q * row + cc : 0)), read);
        }
    };
    // those of the (sequence, key head) after this one, if this run has it
    auto ask_next_q = [&](unsigned r) {
        if (r + at.rounds - at.u >= r1) return;
        Place next = at;
        next.u = at.rounds - 1;
        place_next<false, kTail<W>>(p, next, kRound, c.kv_heads, chunks);
        ask_q(next, q_at ^ 1);
    };
    ask_q(at, q_at);
    cp_async_commit();
    in.template begin<S>(p, at, run, chunks, warp, lane, stages, lsz);
    empty_sequences<T, kThreads>(p);
    if (tid == 0) s_bad = 0;
    cp_async_wait<S - 1>();   // (all but the first rounds)
    __syncthreads();

    // scales behind the last dim: zero for K, whose dims are summed, whatever the cache holds there (V's give sums of their own)
    uint32_t k_mask = 0u;
#pragma unroll
    for (int i = 0; i < kVw; ++i)
        if ((t * kVw + i) * 16 < c.dim) k_mask |= 0xFFu << (8 * i);
    const uint32_t v_pick = (uint32_t)(g / 2) | (uint32_t)(4 + g / 2) << 4;   // a byte of each of two words

    float m[NT][2], l[NT][2], factor[NT][2], o[kKs][NT][4];
    uint32_t qf[kTerms][kKs][NT][2];
    bool bad = false;
    auto begin_head = [&]() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const T *src = reinterpret_cast<const T *>(sm + L::kQueries + q_at * L::kQ + (8 * n + g) * L::kQPitch) + t * (DP / 4);
            float2 q[2 * kKs];
            uint32_t top = 0u;
#pragma unroll
            for (int i = 0; i < 2 * kKs; ++i) {
                q[i] = load2(src, i);
                top = max(top, max(__float_as_uint(q[i].x) & 0x7FFFFFFFu, __float_as_uint(q[i].y) & 0x7FFFFFFFu));
            }
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            // the largest dim to 2^14 .. 2^15, small ones by way of 2^64 times it, so that no factor is out of range
            const bool low = top < 64u << 23;
            const float lift = low ? 0x1p64f : 1.0f;
            top = __float_as_uint(__uint_as_float(top) * lift);
            const int up = min(14 + 127 - (int)(top >> 23), 113);   // (113: a query of zeros)
            const float f = __int_as_float((127 + up) << 23);
#pragma unroll
            for (int i = 0; i < 2 * kKs; ++i) {
                const float x = q[i].x * lift * f, y = q[i].y * lift * f;
                const uint32_t h = pack_half(x, y);
                qf[0][i / 2][n][i & 1] = h;
                if constexpr (kTerms == 2) qf[kTerms - 1][i / 2][n][i & 1] = pack_half(x - half_low(h), y - half_high(h));
            }
            float back = p.scale2 * __int_as_float((127 - up) << 23) * (low ? 0x1p-64f : 1.0f);
            back = fminf(fmaxf(back, -FLT_MAX), FLT_MAX);   // (infinity times 0 is NaN)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                factor[n][e] = __shfl_sync(0xFFFFFFFFu, back, (2 * t + e) * 4);
                m[n][e] = kLow;
                l[n][e] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kKs; ++k) o[k][n][0] = o[k][n][1] = o[k][n][2] = o[k][n][3] = 0.0f;
        }
    };
    begin_head();
    int st = 0;
    unsigned seg0 = r0 - at.u;   // first round of the (sequence, key head)
    for (unsigned r = r0;; ++r) {
        if (r == r0 || at.u == 0) ask_next_q(r);
        __syncwarp();
        in.next(p, chunks, warp, lane, st == 0 ? S - 1 : st - 1, stages, lsz);
        cp_async_wait<S - 1>();
        __syncwarp();

        const bool plain = in.plain >> st & 1u;
        const int nq = min(kNq, p.group - at.ch * kNq), head0 = at.h * p.group + at.ch * kNq;
        const unsigned char *ks = stages + st * L::kStage, *vs = ks + TT * kRow, *kz = vs + TT * kRow, *vz = kz + TT * kScales;
        const float *lz = lsz + st * TT;
        const int j0 = at.u * kRound + warp * TT;
        if (j0 < at.vis) {
            // ---- S^T = K Q^T
            float x[kMt][NT][4];
#pragma unroll
            for (int i = 0; i < kMt; ++i) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][n][e] = 0.0f;
                uint32_t sc[2][kVw];
                const unsigned char *from[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = 16 * i + 8 * h + order<DP>(g);
                    from[h] = ks + row * kRow;
                    const unsigned char *scales = kz + row * kScales + t * kVw;
                    if constexpr (DP == 64) {
                        sc[h][0] = scales_to_half((*scales & k_mask) * 0x0101u);
                    } else if constexpr (DP == 128) {
                        const uint32_t two = scales_to_half(*reinterpret_cast<const unsigned short *>(scales) & k_mask);
                        sc[h][0] = __byte_perm(two, two, 0x1010);
                        sc[h][1] = __byte_perm(two, two, 0x3232);
                    } else {
                        const uint32_t four = *reinterpret_cast<const uint32_t *>(scales) & k_mask;
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t two = scales_to_half(four >> (16 * j));
                            sc[h][2 * j] = __byte_perm(two, two, 0x1010);
                            sc[h][2 * j + 1] = __byte_perm(two, two, 0x3232);
                        }
                    }
                }
                constexpr int kAtOnce = DP == 64 ? 2 : 4;   // words of a load
#pragma unroll
                for (int j0w = 0; j0w < kKw; j0w += kAtOnce) {
                    uint32_t kw[2][kAtOnce];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int chunk = DP == 64 ? 0 : DP == 128 ? t : 2 * t + j0w / 4;
                        load_words<kAtOnce>(from[h] + (DP == 64 ? 8 * t : (chunk ^ swizzle<DP>(order<DP>(g))) << 4), kw[h]);
                    }
#pragma unroll
                    for (int jj = 0; jj < kAtOnce; ++jj) {
                        const int j = j0w + jj;
                        uint32_t a[2][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            codes_to_half(kw[h][jj], a[h]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) a[h][e] = mul_half2(a[h][e], sc[h][j / 2]);
                        }
#pragma unroll
                        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
                                products<kTerms>(x[i][n], a[0][2 * kk], a[1][2 * kk], a[0][2 * kk + 1], a[1][2 * kk + 1],
                                                 [&](int term, int e) { return qf[term][2 * j + kk][n][e]; });
                    }
                }
            }
            // ---- logits in base 2; a masked token's are -inf
            if (plain) {
#pragma unroll
                for (int i = 0; i < kMt; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[i][n][e] *= factor[n][e & 1];
            } else {
#pragma unroll
                for (int i = 0; i < kMt; ++i) {
                    const float z0 = lz[16 * i + order<DP>(g)], z1 = lz[16 * i + order<DP>(g) + 8];
                    const bool off0 = z0 == -INFINITY || z0 == kNoPage, off1 = z1 == -INFINITY || z1 == kNoPage;
                    bad |= z0 == kNoPage || z1 == kNoPage;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            x[i][n][e] = off0 ? -INFINITY : fmaf(x[i][n][e], factor[n][e], z0);
                            x[i][n][2 + e] = off1 ? -INFINITY : fmaf(x[i][n][2 + e], factor[n][e], z1);
                        }
                }
            }
            if (p.logits) {
                float *dst = p.logits + ((size_t)at.b * p.heads + head0 + 2 * t) * p.lstride + (j0 + order<DP>(g));
                const int left = at.vis - j0 - order<DP>(g);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (8 * n + 2 * t + e < nq) {
                            float *to = dst + (8 * n + e) * p.lstride;
#pragma unroll
                            for (int i = 0; i < kMt; ++i) {
                                if (16 * i < left) to[16 * i] = x[i][n][e];
                                if (16 * i + 8 < left) to[16 * i + 8] = x[i][n][2 + e];
                            }
                        }
            }
            // ---- the running shift: kUp below the largest logit when it was set; where a logit exceeds that by kLag, it moves, and O
            // and the sums follow
            float mx[NT][2];
            bool grows = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    mx[n][e] = fmaxf(x[0][n][e], x[0][n][2 + e]);
#pragma unroll
                    for (int i = 1; i < kMt; ++i) mx[n][e] = fmaxf(mx[n][e], fmaxf(x[i][n][e], x[i][n][2 + e]));
                    grows |= mx[n][e] > m[n][e] + (kUp + kLag);
                }
            if (__any_sync(0xFFFFFFFFu, grows)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int s = 4; s < 32; s <<= 1) mx[n][e] = fmaxf(mx[n][e], __shfl_xor_sync(0xFFFFFFFFu, mx[n][e], s));
                        const float to = fmaxf(m[n][e], mx[n][e] - kUp), f = ex2(m[n][e] - to);
                        m[n][e] = to;
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
                uint32_t b[kTerms][NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float p0 = ex2(x[i][n][0] - m[n][0]), p1 = ex2(x[i][n][1] - m[n][1]);
                    const float p2 = ex2(x[i][n][2] - m[n][0]), p3 = ex2(x[i][n][3] - m[n][1]);
                    l[n][0] += p0 + p2;
                    l[n][1] += p1 + p3;
                    const uint32_t h0 = pack_half(p0, p1), h1 = pack_half(p2, p3);
                    b[0][n][0] = transpose8(h0);
                    b[0][n][1] = transpose8(h1);
                    if constexpr (kTerms == 2) {
                        b[kTerms - 1][n][0] = transpose8(pack_half(p0 - half_low(h0), p1 - half_high(h0)));
                        b[kTerms - 1][n][1] = transpose8(pack_half(p2 - half_low(h1), p3 - half_high(h1)));
                    }
                }
                uint32_t sz[4][kVw];
#pragma unroll
                for (int j = 0; j < 4; ++j) load_words<kVw>(vz + (16 * i + 8 * (j >> 1) + order<DP>(2 * t + (j & 1))) * kScales, sz[j]);
#pragma unroll
                for (int w = 0; w < kVw; ++w) {
                    uint32_t vw[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int token = order<DP>(2 * t + (j & 1));
                        vw[j] = *reinterpret_cast<const uint32_t *>(vs + (16 * i + 8 * (j >> 1) + token) * kRow + (((g / 4 + 2 * w) ^ swizzle<DP>(token)) << 4) +
                                                                    (g & 3) * 4);
                    }
                    uint32_t a[4][4];   // fragment registers of four steps of 16 dims
#pragma unroll
                    for (int pair = 0; pair < 2; ++pair) {
                        const uint32_t u = vw[2 * pair], v = vw[2 * pair + 1];
                        const uint32_t s = scales_to_half(__byte_perm(sz[2 * pair][w], sz[2 * pair + 1][w], v_pick));
                        codes_to_half(pick_bits(u, v * 16u, 0x0F0F0F0Fu), a[2 * pair]);      // even dims
                        codes_to_half(pick_bits(u >> 4, v, 0x0F0F0F0Fu), a[2 * pair + 1]);   // odd dims
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            a[2 * pair][e] = mul_half2(a[2 * pair][e], s);
                            a[2 * pair + 1][e] = mul_half2(a[2 * pair + 1][e], s);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            products<kTerms>(o[4 * w + e][n], a[0][e], a[1][e], a[2][e], a[3][e], [&](int term, int i) { return b[term][n][i]; });
                }
            }
        }

        // ---- the end of a (sequence, key head), or of the run: the warps' results together
        if (at.u + 1 == at.rounds || r + 1 == r1) {
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
            __syncthreads();
            const bool whole = seg0 >= r0 && seg0 + at.rounds <= r1, seg_bad = s_bad != 0;
            const size_t head = (size_t)at.b * p.heads + head0, slot = (size_t)(2 * blockIdx.x + (seg0 >= r0 ? 1 : 0)) * kNq;   // of a partial result
            float f[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float M = s_m[0][8 * n + 2 * t + e];
#pragma unroll
                    for (int w = 1; w < W; ++w) M = fmaxf(M, s_m[w][8 * n + 2 * t + e]);
                    f[n][e] = ex2(m[n][e] - M);
                }
            // a thread joins four dims of kMine heads per step of kJoinDims dims
            constexpr int kAcross = L::kJoinDims / 4, kMine = (kNq * kAcross + kThreads - 1) / kThreads;
#pragma unroll
            for (int w0 = 0; w0 < kVw; w0 += L::kJoinDims / 64) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (8 * n + 2 * t + e >= nq) break;
                        float *to = join + (warp * kNq + 8 * n + 2 * t + e) * L::kPitch + 8 * g;
#pragma unroll
                        for (int k = 0; k < L::kJoinDims / 16; k += 2)
                            *reinterpret_cast<float4 *>(to + k / 4 * 64 + 2 * (k % 4)) =
                                make_float4(o[4 * w0 + k][n][e] * f[n][e], o[4 * w0 + k][n][2 + e] * f[n][e],
                                            o[4 * w0 + k + 1][n][e] * f[n][e], o[4 * w0 + k + 1][n][2 + e] * f[n][e]);
                    }
                __syncthreads();
#pragma unroll
                for (int y = 0; y < kMine; ++y) {
                    const int e = y * kThreads + tid, q = e / kAcross, d0 = e % kAcross * 4, d = 64 * w0 + d0;
                    if (q >= nq || d >= c.dim) continue;
                    float M = s_m[0][q], ls = 0.0f;
#pragma unroll
                    for (int w = 1; w < W; ++w) M = fmaxf(M, s_m[w][q]);
                    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        ls += s_l[w][q] * ex2(s_m[w][q] - M);
                        const float4 v = *reinterpret_cast<const float4 *>(join + (w * kNq + q) * L::kPitch + d0);
                        sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
                    }
                    const float inv = 1.0f / ls;
                    if (!whole)
                        *reinterpret_cast<float4 *>(p.part + (slot + q) * c.dim + d) = sum;
                    else if (!seg_bad)
                        store4(reinterpret_cast<T *>(p.out) + (head + q) * c.dim + d,
                               ls == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
                    if (d == 0) {
                        if (!whole) p.part_ml[slot + q] = make_float2(seg_bad ? INFINITY : M, seg_bad ? -1.0f : ls);
                        else if (p.logits) p.lse[head + q] = log_sum(M, seg_bad ? -1.0f : ls);
                    }
                }
                __syncthreads();
            }
            if (tid == 0) {
                if (seg_bad) raise_status(p.status, FUSION_DEV_BAD_CACHE);
                s_bad = 0;
            }
            if (!whole) {
                join_runs<T, kNq, kThreads>(p, run, seg0, seg0 + at.rounds, head, nq, join, s_last);
                __syncthreads();
            }
            if (r + 1 == r1) break;
            const int had = at.u;
            const bool first = seg0 < r0 && r - r0 < (unsigned)S;   // (the run began inside)
            place_next<false, kTail<W>>(p, at, kRound, c.kv_heads, chunks);
            if (had + 1 < S || first) cp_async_wait<0>();   // the next queries were asked for fewer rounds ago than wait() waits for
            q_at ^= 1;
            __syncthreads();
            begin_head();
            seg0 = r + 1;
        } else {
            place_next<false, kTail<W>>(p, at, kRound, c.kv_heads, chunks);
        }
        if (++st == S) st = 0;
    }
    cp_async_wait<0>();   // (of rounds past the run: nothing but zeros)
}

template <typename T, int DP, int NT, int S, int W, int TT>
cudaError_t launch_warps(const PackedAttnParams &p, int chunks, cudaStream_t s) {
    static_assert(counts_fit(TT, W, kTail<W>), "rounds are counted in 32 bits");
    return launch_rounds<k_packed_attn<T, DP, NT, S, W, TT>, W>(Layout<T, DP, NT, S, W, TT>::kTotal, p, chunks, W * TT, s);
}
template <typename T, int DP, int NT>
cudaError_t launch(const PackedAttnParams &p, cudaStream_t s) {
    // Rounds of 64 tokens a warp where as many bytes as 32 of 128 dims are in flight then, that is up to 64 dims (bf16, 38 sequences of up to
    // 25130, 48 / 3 heads: 59.7 us with 32, now 47.9; 53 of up to 25537, 32 / 8 heads of 32: 197 and 157; 145 of up to 2435, 24 / 6 heads,
    // weights: 48.1 and 43.8), but not for float32, which the products bound (16 x 577 13.2 and 13.8, 13 x 10469 27.5 and 26.9), nor alone.
    constexpr int kStages = 2, kTokens = DP == 64 && sizeof(T) == 2 ? 64 : 32;
    const int chunks = ceil_div(p.group, 8 * NT);
    if constexpr (DP <= 128)
        if (warps_alone(p, chunks)) return launch_warps<T, DP, NT, kStages, 1, 32>(p, chunks, s);
    return launch_warps<T, DP, NT, kStages, 4, kTokens>(p, chunks, s);
}
template <typename T, int NT>
cudaError_t launch_dim(const PackedAttnParams &p, cudaStream_t s) {
    if (p.c.dim <= 64) return launch<T, 64, NT>(p, s);
    if (p.c.dim <= 128) return launch<T, 128, NT>(p, s);
    return launch<T, 256, NT>(p, s);
}

}  // namespace

cudaError_t launch_packed_attention(int dtype, const PackedAttnParams &p, cudaStream_t s) {
    if (p.c.max_batch == 0) return cudaSuccess;
    const cudaError_t e = dtype == FUSION_BF16 ? (p.group <= 8 ? launch_dim<__nv_bfloat16, 1>(p, s) : launch_dim<__nv_bfloat16, 2>(p, s))
                                               : launch_dim<float, 1>(p, s);
    return e != cudaSuccess || !p.logits ? e : launch_cache_weights(p, s);
}

}  // namespace fz
