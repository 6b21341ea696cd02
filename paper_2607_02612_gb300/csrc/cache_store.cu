// Rows of a ragged batch go to the ends of their sequences in the paged cache, with more than a copy on the way: keys (and the
// queries of the same rows) rotated by their positions, or keys and values rounded to 4 bits, or both.  In a pair (a, b) of dims
// with the cosine c and sine s of the row's position and the pair's frequency:
//   a' = fl(a c) - fl(b s),   b' = fl(b c) + fl(a s);
// 4 bits: fp4.cuh.  Bound by memory: every row is read once and written once, a row of the table is read once per row and
// comes mostly from the caches.
//
// A thread has one unit of a row, two segments of S dims (8, or a group of 16 in 4 bits) that a rotation by halves turns with
// one another, and in turn that unit of several heads of keys, queries and values, kPer of them asked for at once: the cosines
// and sines stay in registers.  Units lie next to each other in the lanes, then heads, then rows.
#include "cache_rows.cuh"
#include "fp4.cuh"

namespace fz {
namespace {

constexpr int kThreads = 256;
constexpr int kBadShift = 16;   // a sample's counter: its CTAs that are done, and from this bit on those with a bad position
constexpr int kMostX = 2432;    // CTAs of a sample, at most (four waves of four on each of 152 SMs)
static_assert(kMostX < 1 << kBadShift, "a sample's CTAs are counted below the bad ones");

enum Pairs { kNone, kHalves, kAdjacent };
// Heads of a thread in flight: as many as registers hold without spills.
template <typename T, bool kFour> constexpr int per_thread() { return kFour ? (sizeof(T) == 2 ? 2 : 1) : (sizeof(T) == 2 ? 4 : 2); }

template <typename T> __device__ __forceinline__ void to_float(const uint4 &w, float *x);
template <> __device__ __forceinline__ void to_float<float>(const uint4 &w, float *x) {
    x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y), x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
}
template <> __device__ __forceinline__ void to_float<__nv_bfloat16>(const uint4 &w, float *x) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
}
template <typename T> __device__ __forceinline__ uint4 from_float(const float *x);
template <> __device__ __forceinline__ uint4 from_float<float>(const float *x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <> __device__ __forceinline__ uint4 from_float<__nv_bfloat16>(const float *x) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        v[i] = *reinterpret_cast<const uint32_t *>(&p);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Two segments of S numbers, as they lie in memory.
template <typename T, int S>
struct Unit {
    static constexpr int kChunk = 16 / (int)sizeof(T), kChunks = S / kChunk;   // numbers of 16 bytes; 16 bytes of a segment
    uint4 w[2][kChunks];
    __device__ __forceinline__ void load(const T *a, const T *b, bool second) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            w[0][i] = reinterpret_cast<const uint4 *>(a)[i];
            if (second) w[1][i] = reinterpret_cast<const uint4 *>(b)[i];
        }
    }
    __device__ __forceinline__ void store(T *a, T *b, bool second) const {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            reinterpret_cast<uint4 *>(a)[i] = w[0][i];
            if (second) reinterpret_cast<uint4 *>(b)[i] = w[1][i];
        }
    }
    __device__ __forceinline__ void floats(int s, float (&x)[S]) const {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) to_float<T>(w[s][i], x + i * kChunk);
    }
    __device__ __forceinline__ void set(int s, const float (&x)[S]) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) w[s][i] = from_float<T>(x + i * kChunk);
    }
};

// Cosines and sines of a unit's S pairs.
template <int S>
struct Angles {
    float c[S], s[S];
    __device__ __forceinline__ void load(const float *row, int half, int pair) {
#pragma unroll
        for (int i = 0; i < S; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(row + pair + i), w = *reinterpret_cast<const float4 *>(row + half + pair + i);
            c[i] = v.x, c[i + 1] = v.y, c[i + 2] = v.z, c[i + 3] = v.w;
            s[i] = w.x, s[i + 1] = w.y, s[i + 2] = w.z, s[i + 3] = w.w;
        }
    }
    static __device__ __forceinline__ void turn(float &a, float &b, float c, float s) {
        const float x = __fadd_rn(__fmul_rn(a, c), -__fmul_rn(b, s));
        b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
        a = x;
    }
    template <int P> __device__ __forceinline__ void turn(float (&a)[S], float (&b)[S]) const {
        if constexpr (P == kHalves) {
#pragma unroll
            for (int i = 0; i < S; ++i) turn(a[i], b[i], c[i], s[i]);
        } else {
#pragma unroll
            for (int i = 0; i < S / 2; ++i) turn(a[2 * i], a[2 * i + 1], c[i], s[i]);
#pragma unroll
            for (int i = 0; i < S / 2; ++i) turn(b[2 * i], b[2 * i + 1], c[S / 2 + i], s[S / 2 + i]);
        }
    }
};

// Rows of CTAs as in k_cache_append: one per sample, and one more for the lengths while the grid has room for it.  `lanes`:
// threads that share the heads of a unit.
template <typename T, bool kFour, int P>
__global__ void __launch_bounds__(kThreads, 2) k_cache_store(CacheStoreParams p, int units, int lanes) {
    constexpr int S = kFour ? 16 : 8, kPer = per_thread<T, kFour>();
    const int i = blockIdx.y, tid = threadIdx.x;
    const Cache &c = p.c;
    wait_for_previous();
    const int B = device_batch(p.in);
    if (i == (int)gridDim.y - 1 && blockIdx.x == 0) {
        if (B < 0 && tid == 0) raise_status(p.status, FUSION_DEV_BAD_BATCH);
        if (!p.in_place) copy_other_lengths<kThreads>(p, B);
    }
    if (B < 0 || i >= B) return;
    const int slot = p.in.ids ? p.in.ids[i] : i;
    if (slot < 0 || slot >= c.max_batch) {
        if (blockIdx.x == 0 && tid == 0) raise_status(p.status, FUSION_DEV_BAD_IDS);
        return;
    }
    const int o0 = p.in.offsets[i], n = p.in.offsets[i + 1] - o0, at = c.lengths[slot];
    const bool rows_ok = o0 >= 0 && n >= 0 && n <= p.in.max_tokens && (long long)o0 + n <= p.in.max_rows;
    int bad = !rows_ok ? FUSION_DEV_BAD_OFFSETS : at < 0 || at > c.capacity || n > c.capacity - at ? FUSION_DEV_BAD_CACHE : 0;
    const unsigned *pages = reinterpret_cast<const unsigned *>(c.table) + (size_t)slot * c.max_pages;
    bool wrong = false;
    if (!bad)
        for (int e = (at >> c.shift) + tid; n > 0 && e <= (at + n - 1) >> c.shift; e += kThreads) wrong |= pages[e] >= c.num_pages;
    if (named_twice<kThreads>(p.in, B, i, slot)) bad |= FUSION_DEV_BAD_IDS;
    if (__syncthreads_or(wrong)) bad |= FUSION_DEV_BAD_CACHE;
    if (bad) {   // nothing of this sample is written, and its slot's length stays (also where it is named twice)
        if (blockIdx.x == 0 && tid == 0) {
            raise_status(p.status, bad);
            if (!p.in_place) p.lengths_out[slot] = at;
        }
        return;
    }
    // this thread's unit: its dims, whether they are rotated, and its first head
    const int per_row = units * lanes, side = kThreads / per_row, mine = tid / per_row, u = tid % units, lane = tid / units % lanes;
    const int turning = p.turned / (2 * S);   // units that a rotation turns, the first ones
    const bool turned = P != kNone && u < turning;
    const int plain_a = 2 * S * u;
    const int a = P == kHalves ? (u < turning ? S * u : p.turned + 2 * S * (u - turning)) : plain_a;
    const int b = P == kHalves && u < turning ? a + p.turned / 2 : a + S;
    const bool second = b < c.dim, plain_second = plain_a + S < c.dim;   // (of 8 dims, a row's last unit may have one segment)
    const int heads = p.q ? p.heads : 0, all = 2 * c.kv_heads + heads;   // keys, queries, values
    const unsigned low = (1u << c.shift) - 1u;
    bool bad_position = false;
    for (int r0 = blockIdx.x * side; r0 < n; r0 += gridDim.x * side) {
        const int r = r0 + mine;
        if (mine >= side || r >= n) continue;
        unsigned page;
        if (!cache_page(c, slot, at + r, page)) continue;   // (checked)
        const unsigned place = (unsigned)(at + r) & low;
        const size_t row = (size_t)(o0 + r);
        Angles<S> w;
        if constexpr (P != kNone) {
            const unsigned pos = (unsigned)(p.positions ? p.positions[row] : at + r);
            if (pos >= (unsigned)p.table_rows) {
                bad_position = true;
                continue;
            }
            if (turned) w.load(p.table + (size_t)pos * p.turned, p.turned / 2, S * u);
        }
        for (int x0 = lane; x0 < all; x0 += lanes * kPer) {
            Unit<T, S> v[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int x = x0 + k * lanes;
                if (x >= all) break;
                const bool value = x >= c.kv_heads + heads;
                const unsigned char *base = x < c.kv_heads ? p.k + row * p.k_stride
                                            : value        ? p.v + row * p.v_stride
                                                           : p.q + row * p.q_stride;
                const int h = x < c.kv_heads ? x : value ? x - c.kv_heads - heads : x - c.kv_heads;
                const T *src = reinterpret_cast<const T *>(base) + (size_t)h * c.dim;
                if (value) v[k].load(src + plain_a, src + plain_a + S, plain_second);
                else v[k].load(src + a, src + b, second);
            }
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int x = x0 + k * lanes;
                if (x >= all) break;
                const bool value = x >= c.kv_heads + heads, query = !value && x >= c.kv_heads;
                const int h = x < c.kv_heads ? x : value ? x - c.kv_heads - heads : x - c.kv_heads;
                const int da = value ? plain_a : a, db = value ? plain_a + S : b;
                const bool two = value ? plain_second : second;
                if (!kFour || query) {
                    if constexpr (P != kNone)
                        if (turned && !value) {
                            float xa[S], xb[S];
                            v[k].floats(0, xa);
                            v[k].floats(1, xb);
                            w.template turn<P>(xa, xb);
                            v[k].set(0, xa);
                            v[k].set(1, xb);
                        }
                    unsigned char *pool = value ? c.v : c.k;
                    T *dst = query ? reinterpret_cast<T *>(p.q_out) + (row * heads + h) * c.dim
                                   : reinterpret_cast<T *>(pool) + (size_t)(((page * (unsigned)c.kv_heads + h) << c.shift) + place) * c.dim;
                    v[k].store(dst + da, dst + db, two);
                } else if constexpr (kFour) {
                    float xa[S], xb[S];
                    v[k].floats(0, xa);
                    v[k].floats(1, xb);
                    if constexpr (P != kNone)
                        if (turned && !value) w.template turn<P>(xa, xb);
                    const size_t to = (size_t)(((page * (unsigned)c.kv_heads + h) << c.shift) + place);
                    unsigned char *codes = (value ? c.v : c.k) + to * (c.dim / 2), *scales = (value ? p.s.v : p.s.k) + to * p.s.bytes;
                    uint32_t sa, sb;
                    const uint2 ca = quantise(xa, sa), cb = quantise(xb, sb);
                    *reinterpret_cast<uint2 *>(codes + da / 2) = ca;
                    *reinterpret_cast<uint2 *>(codes + db / 2) = cb;
                    scales[da / 16] = (unsigned char)sa;
                    scales[db / 16] = (unsigned char)sb;
                    if (u == 0)   // (the bytes behind the last scale)
                        for (int e = c.dim / 16; e < p.s.bytes; ++e) scales[e] = 0;
                }
            }
        }
        if (u == 0 && lane == 0) {
            const size_t s = ((size_t)page << c.shift) + place;
            if (c.sizes) c.sizes[s] = p.sizes ? p.sizes[row] : 1.0f;
            if (c.weights) c.weights[s] = p.scores ? p.scores[row] : 0.0f;
        }
    }
    // every CTA of the sample has read its length before the last one raises it
    const bool any = __syncthreads_or(bad_position);
    if (tid == 0) {
        int others = 0;
        if (gridDim.x > 1) {
            __threadfence();
            const int before = atomicAdd(&p.counters[i], 1 + (any ? 1 << kBadShift : 0));
            if ((before & ((1 << kBadShift) - 1)) != (int)gridDim.x - 1) return;
            p.counters[i] = 0;
            others = before >> kBadShift;
        }
        const bool none = any || others > 0;
        if (none) raise_status(p.status, FUSION_DEV_BAD_POSITION);
        if (!none || !p.in_place) p.lengths_out[slot] = none ? at : at + n;
    }
}

template <typename T, bool kFour, int P>
cudaError_t launch(const CacheStoreParams &p, cudaStream_t s) {
    constexpr int S = kFour ? 16 : 8, kPer = per_thread<T, kFour>();
    const int units = ceil_div(p.c.dim, 2 * S), all = 2 * p.c.kv_heads + (p.q ? p.heads : 0);
    int lanes = ceil_div(all, kPer);
    if (lanes > kThreads / units) lanes = kThreads / units;
    const int rows = kThreads / (units * lanes);
    // (samples of more rows than the cache has room for, or than there are, write nothing)
    long long most = p.in.max_tokens < p.c.capacity ? p.in.max_tokens : p.c.capacity;
    if (most > p.in.max_rows) most = p.in.max_rows;
    long long x = most > 0 ? (most + rows - 1) / rows : 1;
    if (x > kMostX) x = kMostX;
    static_assert(FUSION_CACHE_MAX_BATCH <= kMostY, "a row of CTAs per sample");
    const dim3 grid((unsigned)x, (unsigned)(p.in.max_batch < kMostY ? p.in.max_batch + 1 : kMostY));
    return launch_after(k_cache_store<T, kFour, P>, grid, kThreads, 0, 1, s, p, units, lanes);
}
template <typename T, bool kFour>
cudaError_t launch_pairs(int pairs, const CacheStoreParams &p, cudaStream_t s) {
    if constexpr (kFour)
        if (p.turned == 0) return launch<T, kFour, kNone>(p, s);
    return pairs == FUSION_PAIRS_HALVES ? launch<T, kFour, kHalves>(p, s) : launch<T, kFour, kAdjacent>(p, s);
}

}  // namespace

cudaError_t launch_cache_store(int dtype, int pairs, const CacheStoreParams &p, cudaStream_t s) {
    if (dtype == FUSION_BF16) return p.s.k ? launch_pairs<__nv_bfloat16, true>(pairs, p, s) : launch_pairs<__nv_bfloat16, false>(pairs, p, s);
    return p.s.k ? launch_pairs<float, true>(pairs, p, s) : launch_pairs<float, false>(pairs, p, s);
}

}  // namespace fz
