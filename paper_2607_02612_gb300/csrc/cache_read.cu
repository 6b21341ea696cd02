// Rows of cached sequences back into a ragged batch: a copy, or the values of a cache in 4 bits (a code's times its group's
// scale, exact in bf16 and in float32: fp4.cuh).  Bound by memory: every row is read once and written once.
//
// A CTA takes as many rows of one sample as give each thread kPer pieces of K and of V, all asked for at once; a piece of a packed row
// is what gives 32 bytes, which go out in one store (48000 rows of 8 x 128 bf16: 42 us, 88 % of the copy's rate; in pieces of 16 bytes 51).
#include "cache_rows.cuh"
#include "fp4.cuh"

namespace fz {
namespace {

constexpr int kThreads = 256, kPer = 4;

__device__ __forceinline__ uint32_t to_bf16(uint32_t h) {   // two float16 whose values bf16 holds
    const __nv_bfloat162 v = __floats2bfloat162_rn(half_low(h), half_high(h));
    return *reinterpret_cast<const uint32_t *>(&v);
}

// What a thread reads at a time, kBytes of a row: 16 codes as bf16, 8 as float32, 16 bytes as they are.
template <typename T> struct Piece;
template <> struct Piece<__nv_bfloat16> { using Held = uint2; static constexpr int kBytes = 32; };
template <> struct Piece<float> { using Held = uint32_t; static constexpr int kBytes = 32; };
template <> struct Piece<uint4> { using Held = uint4; static constexpr int kBytes = 16; };
// 32 bytes at once, or in two halves where they are not aligned to that.
__device__ __forceinline__ void store32(unsigned char *to, const uint32_t (&v)[8], bool aligned) {
    if (aligned) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                     "r"(v[5]), "r"(v[6]), "r"(v[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4 *>(to)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4 *>(to)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}
__device__ __forceinline__ void values_of(uint32_t codes, uint32_t scale, uint32_t (&v)[4]) {   // of eight codes
    codes_to_half(codes, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul_half2(v[i], scale);
}
__device__ __forceinline__ void put(unsigned char *to, uint2 codes, uint32_t scale, bool aligned) {   // as bf16
    const uint32_t s = scales_to_half(scale * 0x0101u);
    uint32_t a[4], b[4];
    values_of(codes.x, s, a);
    values_of(codes.y, s, b);
    const uint32_t v[8] = {to_bf16(a[0]), to_bf16(a[1]), to_bf16(a[2]), to_bf16(a[3]), to_bf16(b[0]), to_bf16(b[1]), to_bf16(b[2]), to_bf16(b[3])};
    store32(to, v, aligned);
}
__device__ __forceinline__ void put(unsigned char *to, uint32_t codes, uint32_t scale, bool aligned) {   // as float32
    uint32_t a[4], v[8];
    values_of(codes, scales_to_half(scale * 0x0101u), a);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __float_as_uint(half_low(a[i]));
        v[2 * i + 1] = __float_as_uint(half_high(a[i]));
    }
    store32(to, v, aligned);
}
__device__ __forceinline__ void put(unsigned char *to, uint4 v, uint32_t, bool) { *reinterpret_cast<uint4 *>(to) = v; }

// T: the type of a cache in 4 bits' values; uint4: a copy of pieces of 16 bytes.  pieces: of a head's row.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) k_cache_read(CacheReadParams p, int row_pieces, int pieces) {
    constexpr bool kFour = sizeof(T) != 16;
    using Held = typename Piece<T>::Held;
    constexpr int kBytes = Piece<T>::kBytes;
    const int i = blockIdx.y, tid = threadIdx.x;
    const Cache &c = p.c;
    wait_for_previous();
    const int B = device_batch(p.in);
    if (B < 0 || i >= B) {
        if (B < 0 && i == 0 && blockIdx.x == 0 && tid == 0) raise_status(p.status, FUSION_DEV_BAD_BATCH);
        return;
    }
    const int slot = p.in.ids ? p.in.ids[i] : i;
    const bool id_ok = slot >= 0 && slot < c.max_batch;
    const int o0 = p.in.offsets[i], n = p.in.offsets[i + 1] - o0, at = p.starts ? p.starts[i] : 0, held = id_ok ? cache_length(c, slot) : -1;
    const bool rows_ok = o0 >= 0 && n >= 0 && n <= p.in.max_tokens && (long long)o0 + n <= p.in.max_rows;
    int bad = !id_ok ? FUSION_DEV_BAD_IDS : !rows_ok ? FUSION_DEV_BAD_OFFSETS : at < 0 || held < 0 || at > held || n > held - at ? FUSION_DEV_BAD_CACHE : 0;
    // `side` rows side by side, a thread has the same piece (of `width` threads' pieces) of kPer rows of the CTA
    const int width = min(row_pieces, kThreads), side = kThreads / width, r_mine = tid / width;
    const int r0 = blockIdx.x * side * kPer;
    const unsigned *pages = reinterpret_cast<const unsigned *>(c.table) + (size_t)(id_ok ? slot : 0) * c.max_pages;
    bool wrong = false;
    unsigned page[kPer];
    int r1 = r0;
    if (!bad) {
        r1 = r_mine < side ? min(n, r0 + side * kPer) : r0;
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            const int r = r0 + r_mine + x * side;
            page[x] = r < r1 ? pages[(at + r) >> c.shift] : 0u;
        }
        for (int e = (at >> c.shift) + tid; n > 0 && e <= (at + n - 1) >> c.shift; e += kThreads) wrong |= pages[e] >= c.num_pages;
    }
    if (__syncthreads_or(wrong)) bad |= FUSION_DEV_BAD_CACHE;
    if (bad) {
        if (blockIdx.x == 0 && tid == 0) raise_status(p.status, bad);
        return;
    }
    const unsigned low = (1u << c.shift) - 1u;
    const bool aligned = ((reinterpret_cast<uintptr_t>(p.k_out) | reinterpret_cast<uintptr_t>(p.v_out)) & 31u) == 0;
    for (int ch = tid % width; ch < row_pieces; ch += kThreads) {   // (once, unless a row has more than kThreads pieces)
        const int h = ch / pieces, cc = ch - h * pieces;
        auto held_row = [&](int x) {
            return (size_t)(((page[x] * (unsigned)c.kv_heads + h) << c.shift) + ((unsigned)(at + r0 + r_mine + x * side) & low));
        };
        auto given = [&](int x) { return ((size_t)(o0 + r0 + r_mine + x * side) * row_pieces + ch); };
        Held k[kPer], v[kPer];
        uint32_t ks[kPer], vs[kPer];
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            if (r0 + r_mine + x * side >= r1) break;
            const size_t row = held_row(x), from = row * pieces + cc, scale = row * p.s.bytes + cc * (int)sizeof(Held) / 8;
            if (p.k_out) {
                k[x] = reinterpret_cast<const Held *>(c.k)[from];
                if (kFour) ks[x] = p.s.k[scale];
            }
            if (p.v_out) {
                v[x] = reinterpret_cast<const Held *>(c.v)[from];
                if (kFour) vs[x] = p.s.v[scale];
            }
        }
#pragma unroll
        for (int x = 0; x < kPer; ++x) {
            if (r0 + r_mine + x * side >= r1) break;
            const size_t to = given(x) * kBytes;
            if (p.k_out) put(p.k_out + to, k[x], ks[x], aligned);
            if (p.v_out) put(p.v_out + to, v[x], vs[x], aligned);
        }
    }
    for (int r = r0 + tid; r < min(n, r0 + side * kPer); r += kThreads) {
        unsigned pg;
        if (!cache_page(c, slot, at + r, pg)) continue;   // (checked)
        const size_t s = ((size_t)pg << c.shift) + ((unsigned)(at + r) & low);
        if (p.sizes_out) p.sizes_out[o0 + r] = c.sizes ? c.sizes[s] : 1.0f;
        if (p.weights_out) p.weights_out[o0 + r] = c.weights ? c.weights[s] : 0.0f;
    }
}

template <typename T> cudaError_t launch(const CacheReadParams &p, int pieces, cudaStream_t s) {
    const int row_pieces = pieces * p.c.kv_heads, rows = kPer * (row_pieces < kThreads ? kThreads / row_pieces : 1);
    long long most = p.in.max_tokens < p.c.capacity ? p.in.max_tokens : p.c.capacity;   // (a sample of more rows is refused)
    if (most > p.in.max_rows) most = p.in.max_rows;
    if (p.in.max_batch == 0) return cudaSuccess;
    static_assert(FUSION_CACHE_MAX_BATCH <= kMostY, "a row of CTAs per sample");
    const dim3 grid((unsigned)(most > 0 ? (most + rows - 1) / rows : 1), (unsigned)p.in.max_batch);
    return launch_after(k_cache_read<T>, grid, kThreads, 0, 1, s, p, row_pieces, pieces);
}

}  // namespace

cudaError_t launch_cache_read(int dtype, const CacheReadParams &p, cudaStream_t s) {
    if (!p.s.k) return launch<uint4>(p, p.c.dim * (dtype == FUSION_BF16 ? 2 : 4) / 16, s);
    return dtype == FUSION_BF16 ? launch<__nv_bfloat16>(p, p.c.dim / 16, s) : launch<float>(p, p.c.dim / 8, s);
}

}  // namespace fz
